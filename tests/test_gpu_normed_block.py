"""Blocks behind their norm, in training and in 8 bits for inference, against a 64-bit computation of their formulas."""
import numpy as np
import pytest

from oracle import norm8_oracle as N
from oracle import operators_oracle as O
from paper_2504_03871_amd import binding as B
from tests.test_gpu_shared_expert import EXACT, make

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

T, D, F, FS, E, K = 200, 128, 192, 320, 16, 4
EPS = 1e-6


def f64(t):
    return t.detach().double().cpu()


def normed(dtype, stream=None, p=0.0, layer=0, seed=0):
    from paper_2504_03871_amd.block import NormedBlock
    n = NormedBlock(make(T, D, F, FS, E, K, dtype, B.ACT_SWIGLU, B.PACK_NONE, seed=seed), stream=stream, p=p, seed=77, layer=layer, eps=EPS)
    n.gamma.copy_(torch.as_tensor(1 + 0.2 * np.random.default_rng(seed + 9).normal(size=D)))
    return n


def block_of(x, leaf, idx):
    """The block's formulas in 64 bits at a given choice of experts."""
    s = torch.sigmoid(x @ leaf["Wr"]).gather(1, idx)
    w = 1.5 * s / s.sum(dim=1, keepdim=True)
    out = torch.nn.functional.silu(x @ leaf["Wg"]) * (x @ leaf["Wu"]) @ leaf["Wd"]
    for e in range(E):
        t, j = (idx == e).nonzero(as_tuple=True)
        h = torch.nn.functional.silu(x[t] @ leaf["W1"][e]) * (x[t] @ leaf["W1b"][e])
        out = out.index_add(0, t, w[t, j, None] * (h @ leaf["W2"][e]))
    return out


def leaves(blk):
    m = blk.moe
    return {n: f64(t).requires_grad_(True) for n, t in (("Wr", m.Wr), ("W1", m.W1), ("W1b", m.W1b), ("W2", m.W2), ("Wg", blk.Wg), ("Wu", blk.Wu), ("Wd", blk.Wd))}


@pytest.mark.parametrize("dtype, stream, p", [(B.DTYPE_F32, None, 0.0), (B.DTYPE_F32, None, 0.3), (B.DTYPE_BF16, None, 0.0), (B.DTYPE_BF16, B.DTYPE_F32, 0.2)])
def test_two_blocks_forward_and_backward(dtype, stream, p):
    """h1 = x + 0, out1 = block1(norm(h1)), h2 = h1 + dropout(out1), out2 = block2(norm(h2)); the loss takes h2 and out2."""
    a, b = normed(dtype, stream, 0.0, 0, 1), normed(dtype, stream, p, 1, 2)
    r = np.random.default_rng(3)
    td, st = a.block.moe.tdtype, a.h.dtype
    x = torch.as_tensor(r.normal(size=(T, D))).to(td).cuda()
    d_h2 = torch.as_tensor(r.normal(size=(T, D))).to(st).cuda()
    b.step.fill_(5)
    out1, h1 = a.forward(x)
    out2, h2 = b.forward(out1, h1)
    d_out1, d_h1 = b.backward(d_h2)
    a.block.moe.d_out.copy_(d_out1)
    d_x, d_x_stream = a.backward(d_h1)
    got = {"out2": out2, "h2": h2, "d_x": d_x, "d_x_stream": d_x_stream, "dgamma1": a.dgamma, "dgamma2": b.dgamma}
    # 64 bits
    lx = f64(x).requires_grad_(True)
    mask = torch.from_numpy(N.drop_mask(T, D, p, 77, (1 << 32) + 5))
    la, lb, g1, g2 = leaves(a.block), leaves(b.block), f64(a.gamma).requires_grad_(True), f64(b.gamma).requires_grad_(True)
    rms = lambda h, g: g * h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + EPS)  # noqa: E731
    w1 = block_of(rms(lx, g1), la, a.block.moe.topk_idx.long().cpu())
    wh2 = lx + w1 * mask
    w2 = block_of(rms(wh2, g2), lb, b.block.moe.topk_idx.long().cpu())
    ((w2 * f64(b.block.moe.d_out)).sum() + (wh2 * f64(d_h2)).sum()).backward()
    want = {"out2": w2, "h2": wh2, "d_x": lx.grad, "d_x_stream": lx.grad, "dgamma1": g1.grad, "dgamma2": g2.grad}
    for blk, leaf, tag in ((a.block, la, "1"), (b.block, lb, "2")):
        for name, t in (("Wr", blk.moe.dWr), ("W1", blk.moe.dW1), ("W1b", blk.moe.dW1b), ("W2", blk.moe.dW2), ("Wg", blk.dWg), ("Wu", blk.dWu), ("Wd", blk.dWd)):
            got["d" + name + tag], want["d" + name + tag] = t, leaf[name].grad
    for name in want:
        err = float(((f64(got[name]) - want[name]).norm() / want[name].norm()).detach())
        # two blocks one behind the other, a norm in front of each: twice one block's, and an eighth for the norms
        assert err <= 2.25 * EXACT[dtype], (name, err)


def test_a_captured_step_has_its_own_mask_on_every_replay():
    n = normed(B.DTYPE_BF16, B.DTYPE_F32, 0.25)
    r = np.random.default_rng(0)
    x, res = torch.as_tensor(r.normal(size=(T, D))).bfloat16().cuda(), torch.as_tensor(r.normal(size=(T, D))).float().cuda()
    d_h = torch.as_tensor(r.normal(size=(T, D))).float().cuda()
    keep = [n.h, n.block.moe.out, n.d_branch, n.dh, n.dgamma]

    def step():
        n.step.add_(1)
        n.forward(x, res)
        n.backward(d_h)
    want = []
    for _ in range(4):
        step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in keep])
    assert not torch.equal(want[0][0], want[1][0])
    n.step.zero_()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    n.step.zero_()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(keep, w):
            assert torch.equal(a, b)
        torch.zeros(1000, device="cuda").sum()       # eager work in between


@pytest.mark.parametrize("T8", [1, 7, 40, 200])
@pytest.mark.parametrize("dtype", [B.DTYPE_BF16, B.DTYPE_F16])
def test_block_in_8_bits(dtype, T8):
    from paper_2504_03871_amd.block import ServedBlock
    n = normed(dtype)
    m = n.block.moe
    s = ServedBlock(n.block, n.gamma, T8, eps=EPS)
    r = np.random.default_rng(1)
    x, res = (torch.as_tensor(r.normal(size=(T8, D))).to(m.tdtype).cuda() for _ in range(2))
    out, h = s.forward(x, res)
    idx = s.topk_idx.long().cpu()
    ridx, _ = O.route(s.logits.cpu().numpy(), "sigmoid", K, s.balance.cpu().numpy(), 4, 2, 2, 1, 1.5)
    assert np.array_equal(idx.numpy(), ridx)
    # the definition in 64 bits, from h as it is stored; what is stored in between has the storage type
    y = N.norm_fwd(f64(h).numpy(), f64(n.gamma).numpy(), EPS)[0]
    q, qs = N.quant_rows(y.astype(np.float32))
    weight = lambda W: (lambda c, sc: (c.T.astype(np.float64), sc.astype(np.float64)))(*N.quant_rows(np.ascontiguousarray(f64(W).float().numpy().T)))  # noqa: E731
    store = lambda v: torch.from_numpy(v).to(m.tdtype).double().numpy()  # noqa: E731

    def ffn(q, qs, up, gate, down):
        (wg, sg), (wu, su), (wd, sd) = weight(up), weight(gate), weight(down)
        hid = N.linear8(q, qs, [wg, wu], [sg, su], [None, None], "swiglu", None)[0]
        c, cs = N.quant_rows(store(hid).astype(np.float32))
        return N.linear8(c, cs, [wd], [sd], [None], "none", None)[0]
    want = ffn(q, qs, n.block.Wg, n.block.Wu, n.block.Wd)
    w = f64(s.topk_w).numpy()
    for e in range(E):
        t, j = np.nonzero(idx.numpy() == e)
        if t.size:
            np.add.at(want, t, w[t, j][:, None] * ffn(q[t], qs[t], m.W1[e], m.W1b[e], m.W2[e]))
    err = np.linalg.norm(f64(out).numpy() - want) / np.linalg.norm(want)
    # y_perm, the routed sum and out are rounded, and hidden once more where its last bit falls otherwise: four roundings of the type; a code
    # that falls otherwise with it moves its row by a 127th of its largest value over the root of its length
    assert err <= 4 * torch.finfo(m.tdtype).eps / 2 + 1e-3, err
    # and the block without quantising is what it stands for: codes are good to half a 127th of a row's largest value, about 3 of its
    # standard deviations here, over the square root of three: 0.7 % of a product's terms, twice for both operands, in three products
    m.x[:T8] = s.y
    m.x[T8:] = 0
    n.block.forward()
    full = f64(m.out[:T8]).numpy()
    assert np.linalg.norm(f64(out).numpy() - full) <= 0.06 * np.linalg.norm(full)


def test_block_in_8_bits_captured():
    from paper_2504_03871_amd.block import ServedBlock
    n = normed(B.DTYPE_BF16)
    s = ServedBlock(n.block, n.gamma, 5, eps=EPS)
    r = np.random.default_rng(1)
    xs = [torch.as_tensor(r.normal(size=(5, D))).bfloat16().cuda() for _ in range(3)]
    want = [s.forward(x, xs[0])[0].clone() for x in xs]
    x = xs[0].clone()
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        s.forward(x, xs[0])
    for v, w in zip(xs, want):
        x.copy_(v)
        s.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.out, w)


def test_full_precision_has_no_8_bit_experts():
    from paper_2504_03871_amd.block import ServedBlock
    n = normed(B.DTYPE_F32)
    with pytest.raises(ValueError):
        ServedBlock(n.block, n.gamma, 4)
