"""The block that answers requests, and the block behind its norm: what they are made of and what they refuse (no GPU needed)."""
import pytest

from paper_2504_03871_amd import binding as B

torch = pytest.importorskip("torch")

SIZES = dict(T=64, d_model=64, d_ff=128, d_shared=192, E=8, k=2)


def source(**kw):
    from paper_2504_03871_amd.block import SharedExpertMoE
    return SharedExpertMoE(**{**SIZES, **kw}, score=B.make_score(B.SCORE_SIGMOID), device="cpu")


def served(monkeypatch, src=None, T=16, **kw):
    """A ServedBlock whose weights stay as they are: without a GPU nothing is quantised."""
    from paper_2504_03871_amd.block import ServedBlock
    monkeypatch.setattr(B, "moe_quant_weight", lambda *a, **k: None)
    src = source() if src is None else src
    return ServedBlock(src, torch.ones(SIZES["d_model"], dtype=torch.bfloat16), T, **kw)


@pytest.mark.parametrize("T", [1, 64, 500])
def test_the_training_batch_s_capacity_is_no_limit_on_requests(monkeypatch, T):
    src = source(capacity=3)
    assert served(monkeypatch, src, T).cfg.capacity <= 0          # unlimited
    assert served(monkeypatch, src, T, capacity=9).cfg.capacity == 9


def test_the_residual_stream_may_be_of_full_precision(monkeypatch):
    assert served(monkeypatch).h.dtype == torch.bfloat16
    s = served(monkeypatch, stream=B.DTYPE_F32)
    assert s.h.dtype == torch.float32 and s.norm.stream == B.DTYPE_F32 and s.norm.dtype == B.DTYPE_BF16 and s.out.dtype == torch.bfloat16
