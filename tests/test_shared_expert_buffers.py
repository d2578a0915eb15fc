"""Buffers of the block with a shared expert: what 8-bit checkpoints let several blocks share, and what is refused (no GPU needed)."""
import pytest

from paper_2504_03871_amd import binding as B

torch = pytest.importorskip("torch")

SIZES = dict(T=64, d_model=64, d_ff=128, d_shared=192, E=8, k=2)


def block(fmt=B.PACK_NONE, **kw):
    from paper_2504_03871_amd.block import SharedExpertMoE
    return SharedExpertMoE(**{**SIZES, **kw}, score=B.make_score(B.SCORE_SIGMOID), fmt=fmt, device="cpu")


def buffers(blk):
    """{address: bytes} of every buffer that a block and its layer hold."""
    out = {}
    for owner in (blk, blk.moe):
        for v in vars(owner).values():
            for t in v if isinstance(v, (list, tuple)) else [v]:
                if isinstance(t, torch.Tensor):
                    out[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
    return out


@pytest.mark.parametrize("fmt", [B.PACK_E4M3, B.PACK_I8])
def test_checkpoints_take_less_memory_than_the_planes(fmt):
    plain = sum(buffers(block()).values())
    first = block(fmt)
    second = block(fmt, saved=first.moe.saved, pre=first.pre)
    shared = buffers(first)
    own = sum(n for at, n in buffers(second).items() if at not in shared)
    A, planes = SIZES["T"] * SIZES["k"], 3
    kept = 2 * (planes * A * SIZES["d_ff"] + 2 * SIZES["T"] * SIZES["d_shared"])               # bf16 planes of both experts
    codes = 33 * (2 * A * SIZES["d_ff"] + 2 * SIZES["T"] * SIZES["d_shared"]) // 32
    assert own == plain - kept + codes


def test_shared_buffers_are_checked():
    donor = block(B.PACK_I8)
    ok = dict(saved=donor.moe.saved, pre=donor.pre)
    block(B.PACK_E4M3, **ok)
    for name in ok:                                   # kept as they are until the backward: another block's forward would overwrite them
        with pytest.raises(ValueError):
            block(**{name: ok[name]})
    for saved in (donor.moe.saved[:-1], donor.moe.saved.view(torch.bfloat16), torch.cat([donor.moe.saved] * 2)[::2]):
        with pytest.raises(ValueError):
            block(B.PACK_I8, saved=saved)
    for pre in (donor.pre[:1], [donor.pre[0], None], [p[:-1] for p in donor.pre], [p.float() for p in donor.pre],
                [torch.empty(SIZES["T"], 2 * SIZES["d_shared"], dtype=torch.bfloat16)[:, ::2] for _ in range(2)], [donor.pre[0]] * 2):
        with pytest.raises(ValueError):
            block(B.PACK_I8, pre=pre)
    block(B.PACK_I8, saved=torch.empty(donor.moe.saved.numel() + 256, dtype=torch.uint8))      # larger is fine
