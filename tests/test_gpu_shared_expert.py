"""The block with scored routing, a shared expert and 8-bit checkpoints against a 64-bit computation of its formulas."""
import numpy as np
import pytest

from oracle import operators_oracle as O
from paper_2504_03871_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def make(T, d, f, fs, E, k, dtype, act, fmt, seed=0):
    from paper_2504_03871_amd.block import SharedExpertMoE
    blk = SharedExpertMoE(T, d, f, fs, E, k, B.make_score(B.SCORE_SIGMOID, 4, 2, 2, 1, 1.5), dtype=dtype, act=act, fmt=fmt)
    r = np.random.default_rng(seed)
    m = blk.moe
    for t, std in ((m.x, 1), (m.Wr, d ** -0.5), (m.W1, d ** -0.5), (m.W1b, d ** -0.5), (m.W2, f ** -0.5), (m.d_out, 1), (blk.Wg, d ** -0.5),
                   (blk.Wu, d ** -0.5), (blk.Wd, fs ** -0.5)):
        if t is not None:
            t.copy_(torch.as_tensor(r.normal(0, std, tuple(t.shape))).to(t.dtype))
    blk.balance.copy_(torch.as_tensor(np.round(r.normal(0, 20, E)) * 1e-3))
    return blk


def reference(blk, act):
    """Outputs and gradients in 64 bits at the choice that was made (checked against the oracle's for the same logits)."""
    m = blk.moe
    f = lambda t: t.detach().double().cpu()  # noqa: E731
    idx = m.topk_idx.long().cpu()
    ridx, _ = O.route(m.logits.cpu().numpy(), "sigmoid", idx.shape[1], blk.balance.cpu().numpy(), 4, 2, 2, 1, 1.5)
    assert np.array_equal(idx.numpy(), ridx)
    leaf = {n: f(t).requires_grad_(True) for n, t in (("x", m.x), ("Wr", m.Wr), ("W1", m.W1), ("W2", m.W2), ("Wg", blk.Wg), ("Wu", blk.Wu), ("Wd", blk.Wd))}
    W1b = f(m.W1b).requires_grad_(True) if m.W1b is not None else None
    x = leaf["x"]
    s = torch.sigmoid(x @ leaf["Wr"]).gather(1, idx)
    w = 1.5 * s / s.sum(dim=1, keepdim=True)
    out = torch.nn.functional.silu(x @ leaf["Wg"]) * (x @ leaf["Wu"]) @ leaf["Wd"]
    for e in range(m.E):
        t, j = (idx == e).nonzero(as_tuple=True)
        a = x[t] @ leaf["W1"][e]
        h = torch.nn.functional.silu(a) * (x[t] @ W1b[e]) if act == B.ACT_SWIGLU else torch.nn.functional.gelu(a)
        out = out.index_add(0, t, w[t, j, None] * (h @ leaf["W2"][e]))
    out.backward(f(m.d_out))
    got = {"out": (m.out, out), "dx": (m.dx, x.grad), "dWr": (m.dWr, leaf["Wr"].grad), "dW1": (m.dW1, leaf["W1"].grad), "dW2": (m.dW2, leaf["W2"].grad),
           "dWg": (blk.dWg, leaf["Wg"].grad), "dWu": (blk.dWu, leaf["Wu"].grad), "dWd": (blk.dWd, leaf["Wd"].grad)}
    if W1b is not None:
        got["dW1b"] = (m.dW1b, W1b.grad)
    return {n: float(((f(a) - b).norm() / b.norm()).detach()) for n, (a, b) in got.items()}


# A chain of at most eight fp32 products and sums of up to 512 terms: sqrt(512) roundings of 2^-24 each, times eight, is 1e-5.  bf16: at
# most eight roundings of 2^-9 rms on the way to any output (pre-activations, h, y, dy, dz, dx_perm and the sums of two paths).
EXACT = {B.DTYPE_F32: 1e-5, B.DTYPE_BF16: 8 * 2.0 ** -9}


@pytest.mark.parametrize("act", [B.ACT_GELU, B.ACT_SWIGLU])
@pytest.mark.parametrize("dtype", [B.DTYPE_F32, B.DTYPE_BF16])
def test_block_against_64_bits(dtype, act):
    blk = make(200, 128, 192, 320, 16, 4, dtype, act, B.PACK_NONE)
    blk.step()
    for name, err in reference(blk, act).items():
        assert err <= EXACT[dtype], (name, err)


@pytest.mark.parametrize("fmt,step", [(B.PACK_I8, 2.0 ** -7), (B.PACK_E4M3, 2.0 ** -4)])
def test_block_with_checkpoints_in_8_bits(fmt, step):
    """The forward is that without checkpoints, bit by bit; a gradient is off by what a rounding of the pre-activations does: at most
    `step` of a block's largest value (64ths of up to twice it) or of the value (e4m3), through slopes of at most 1.2 and their
    change, in two factors."""
    plain = make(200, 128, 192, 320, 16, 4, B.DTYPE_BF16, B.ACT_SWIGLU, B.PACK_NONE)
    plain.step()
    blk = make(200, 128, 192, 320, 16, 4, B.DTYPE_BF16, B.ACT_SWIGLU, fmt)
    blk.forward()
    assert torch.equal(blk.moe.out, plain.moe.out)
    blk.moe.saved.fill_(255)          # what lies in the shared buffers does not matter until the backward
    for p in blk.pre:
        p.fill_(float("nan"))
    blk.backward()
    for name, err in reference(blk, B.ACT_SWIGLU).items():
        assert err <= EXACT[B.DTYPE_BF16] + 2 * 1.2 * step, (name, err)
    once = {n: getattr(o, n).clone() for o, n in ((blk, "dWg"), (blk, "dWd"), (blk.moe, "dW1"), (blk.moe, "dWr"))}
    blk.backward(accumulate=1)        # a second backward adds the same again: doubling is exact but for one rounding of the sum
    for name, g in once.items():
        now = getattr(blk if hasattr(blk, name) else blk.moe, name)
        assert torch.all((now - 2 * g).abs() <= 2.0 ** -22 * g.abs().max()), name


def test_balance_update_evens_out_the_load():
    blk = make(512, 64, 64, 64, 16, 2, B.DTYPE_BF16, B.ACT_GELU, B.PACK_NONE)
    blk.moe.Wr.mul_(0.2)
    blk.balance.zero_()
    blk.balance[:3] = 0.2             # three experts drawn towards
    spread = []
    for _ in range(60):
        blk.forward()
        spread.append(int(blk.moe.counts.max() - blk.moe.counts.min()))
        blk.update_balance(0.01)
    assert min(spread[-10:]) < spread[0] // 2


@pytest.mark.parametrize("fmt", [B.PACK_I8, B.PACK_E4M3])
def test_blocks_that_share_their_planes(fmt):
    """Two blocks one after the other, backward in reverse, in one set of planes: the bits of blocks with planes of their own."""
    from paper_2504_03871_amd.block import SharedExpertMoE
    args = (200, 128, 192, 320, 16, 4, B.DTYPE_BF16, B.ACT_SWIGLU, fmt)
    alone = [make(*args, seed=s) for s in (1, 2)]
    shared = [make(*args, seed=1), make(*args, seed=2)]
    again = SharedExpertMoE(200, 128, 192, 320, 16, 4, shared[1].score, act=B.ACT_SWIGLU, fmt=fmt, saved=shared[0].moe.saved, pre=shared[0].pre)
    for name in ("x", "Wr", "W1", "W1b", "W2", "d_out"):
        getattr(again.moe, name).copy_(getattr(shared[1].moe, name))
    for name in ("Wg", "Wu", "Wd", "balance"):
        getattr(again, name).copy_(getattr(shared[1], name))
    shared[1] = again
    for blk in alone:
        blk.step()
    for blk in shared:
        blk.forward()
    for blk in reversed(shared):
        blk.backward()
    for a, b in zip(alone, shared):
        for name in ("out", "dx", "dW1", "dW1b", "dW2", "dWr"):
            assert torch.equal(getattr(a.moe, name), getattr(b.moe, name)), name
        for name in ("dWg", "dWu", "dWd"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
