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


def norm_calls(monkeypatch):
    """Nothing may be launched: what the norm is called with."""
    calls = []
    for name in ("moe_norm_fwd", "moe_norm_bwd"):
        monkeypatch.setattr(B, name, lambda *a, **k: calls.append(a))
    from paper_2504_03871_amd.block import SharedExpertMoE
    monkeypatch.setattr(SharedExpertMoE, "forward", lambda self: None)
    monkeypatch.setattr(SharedExpertMoE, "backward", lambda self, accumulate=0: None)
    return calls


def wrong(T, d, dtype, other):
    """Tensors that are not [T, d] of dtype, without gaps, on this device."""
    return [torch.empty(T, d, dtype=other), torch.empty(T - 1, d, dtype=dtype), torch.empty(T, d + 8, dtype=dtype), torch.empty(T * d, dtype=dtype),
            torch.empty(T, 2 * d, dtype=dtype)[:, ::2], torch.empty(d, T, dtype=dtype).T, torch.empty(T, d, dtype=dtype, device="meta")]


@pytest.mark.parametrize("stream", [None, B.DTYPE_F32])
def test_operands_that_are_not_the_block_s_rows_are_refused(monkeypatch, stream):
    from paper_2504_03871_amd.block import NormedBlock
    T, d, half = SIZES["T"], SIZES["d_model"], torch.bfloat16
    st, not_st = (half, torch.float32) if stream is None else (torch.float32, half)
    calls = norm_calls(monkeypatch)
    n, s = NormedBlock(source(), stream=stream), served(monkeypatch, T=T, stream=stream)
    branch, res = torch.empty(T, d, dtype=half), torch.empty(T, d, dtype=st)
    for b in (n, s):
        for t in wrong(T, d, half, torch.float16) + [None]:
            with pytest.raises(ValueError, match="branch"):
                b.forward(t, res)
        for t in wrong(T, d, st, not_st):
            with pytest.raises(ValueError, match="residual"):
                b.forward(branch, t)
    for t in wrong(T, d, st, not_st):
        with pytest.raises(ValueError, match="d_h"):
            n.backward(t)
    assert not calls
    n.forward(branch)
    n.forward(branch, res)
    n.backward()
    n.backward(res)
    n.forward(branch.view(2, T // 2, d), res.view(4, 2, T // 8, d))      # sequences of a batch
    assert len(calls) == 5


def test_gamma_is_a_row_of_the_block_s_type(monkeypatch):
    from paper_2504_03871_amd.block import ServedBlock
    src = source()
    served(monkeypatch, src)
    for g in (torch.ones(SIZES["d_model"]), torch.ones(SIZES["d_model"] + 1, dtype=torch.bfloat16), torch.ones(2, SIZES["d_model"], dtype=torch.bfloat16),
              torch.ones(2 * SIZES["d_model"], dtype=torch.bfloat16)[::2], None):
        with pytest.raises(ValueError, match="gamma"):
            ServedBlock(src, g, 4)


@pytest.mark.parametrize("p", [-0.1, 1.0, float("nan"), 2.0])
def test_a_probability_that_is_none_is_refused(p):
    from paper_2504_03871_amd.block import NormedBlock
    with pytest.raises(ValueError, match="0 <= p < 1"):
        NormedBlock(source(), p=p)
