"""Scored routing, activations in 8 bits and dense products with an epilogue on the GPU, against the 64-bit oracle."""
import math

import numpy as np
import pytest

from oracle import operators_oracle as O
from paper_2504_03871_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DT = {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16}
FMT = {"e4m3": B.PACK_E4M3, "i8": B.PACK_I8}
U = 2.0 ** -24           # rounding to fp32, half a step
F32_MAX = float(np.finfo(np.float32).max)


def half_step(dtype):
    return torch.finfo(TD[dtype]).eps / 2


def dev(a, dtype=torch.float32):
    return torch.as_tensor(np.asarray(a)).to(dtype).to(DEV)


def f64(t):
    return t.detach().double().cpu().numpy()


# ---- scored routing ------------------------------------------------------------------------------------------------

def route_inputs(T, E, seed, kind):
    """Logits as they come, and at the places where a choice can go wrong."""
    r = np.random.default_rng(seed)
    l = r.normal(0, 1.5, (T, E))
    if kind == "masked":
        l[r.random((T, E)) < 0.4] = -np.inf
        l[::3] = -np.inf                                    # rows with nothing left
    elif kind == "odd":
        l[r.random((T, E)) < 0.1] = np.nan
        l[r.random((T, E)) < 0.1] = np.inf
        l[r.random((T, E)) < 0.1] = -F32_MAX                # the type's lowest value takes part
        l[1::4] = np.nan
    elif kind == "ties":
        l = r.integers(-2, 3, (T, E)).astype(np.float64)
        l[::2] = 0.25
    elif kind == "tiny":
        l = l - 100.0                                       # sigmoids of 1e-44: only their ratios are left
    elif kind == "wide":
        l = l * 20.0
    return l.astype(np.float32)


SHAPES = [  # T, E, k, groups, top_groups, rank
    (1, 1, 1, 1, 1, 1), (1, 256, 8, 8, 4, 2), (17, 8, 2, 1, 1, 1), (5, 12, 3, 4, 2, 2), (33, 16, 8, 16, 8, 1), (100, 33, 5, 1, 1, 1),
    (64, 64, 6, 8, 3, 1), (31, 72, 8, 3, 1, 2), (48, 160, 8, 8, 3, 2), (16, 255, 4, 5, 2, 2), (70, 256, 8, 8, 4, 2), (15, 128, 1, 16, 1, 2),
]


def run_route(l, kind, k, balance, groups, top, rank, renorm, scale):
    T, E = l.shape
    cfg = B.make_cfg(T, 64, 64, E, k)
    sc = B.make_score(B.SCORE_SOFTMAX if kind == "softmax" else B.SCORE_SIGMOID, groups, top, rank, renorm, scale)
    lg = dev(l)
    idx = torch.full((T, k), -7, dtype=torch.int32, device=DEV)
    w = torch.full((T, k), 7.0, device=DEV)
    B.moe_route_scored(cfg, sc, None, None, None, None if balance is None else dev(balance), lg, None, idx, w)
    dw = dev(np.random.default_rng(9).normal(0, 1, (T, k)))
    dl = torch.full((T, E), 7.0, device=DEV)
    B.moe_route_scored_bwd(cfg, sc, None, None, lg, idx, dw, dl, None, None)
    return idx.cpu().numpy(), f64(w), f64(dw), f64(dl)


def check_route(l, kind, k, balance, groups, top, rank, renorm, scale):
    idx, w, dw, dl = run_route(l, kind, k, balance, groups, top, rank, renorm, scale)
    ridx, rw = O.route(l, kind, k, balance, groups, top, rank, renorm, scale)
    assert np.array_equal(idx, ridx)
    # A weight is a quotient of exponentials of l - top: each is good to 2^-24 of its argument (rounded once) and three units
    # in the last place (half-steps: six), the sum of up to 256 of them to eight rounding errors of its pairwise order and one per
    # term of a lane, the quotient and the scale to one each
    lf = np.where(np.isfinite(l), l.astype(np.float64), 0.0)
    reach = np.abs(np.where(np.abs(lf) < 1e30, lf, 0.0)).max(axis=1, keepdims=True) * 2
    rel = (reach + 6 + 24 + 2) * U
    tiny = 2.0 ** -120
    assert np.all(np.abs(w - rw) <= rel * np.abs(rw) + tiny)
    rdl = O.route_bwd(l, kind, ridx, dw, renorm, scale)
    s, _ = O.scores(l, kind)
    p = np.zeros_like(s)
    for t in range(len(l)):
        for j, e in enumerate(ridx[t]):
            if e >= 0:
                p[t, e] = abs(rw[t, j])
    most = np.abs(dw).max(axis=1, keepdims=True)
    size = 2 * most * (p + (abs(scale) * s if kind == "softmax" and not renorm else 0))
    assert np.all(np.abs(dl - rdl) <= (2 * rel + 16 * U) * size + tiny), np.abs(dl - rdl).max()


@pytest.mark.parametrize("inputs", ["plain", "masked", "odd", "ties", "tiny", "wide"])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_scored_routing(shape, kind, inputs):
    T, E, k, groups, top, rank = shape
    l = route_inputs(T, E, sum(shape), inputs)
    r = np.random.default_rng(E)
    bal = (np.round(r.normal(0, 30, E)) * 0.001).astype(np.float32)
    for renorm, scale, balance in ((1, 1.0, None), (0, 2.5, bal), (1, 2.5, bal), (0, 1.0, None)):
        check_route(l, kind, k, balance, groups, top, rank, renorm, scale)


def test_keys_closer_than_single_precision_resolves():
    """Scores plus bias that differ by less than an fp32 step, in both orders of the expert ids, and in the scores of groups."""
    E = 32
    base = 0.3
    l = np.full((64, E), -4.0, np.float32)
    bal = np.zeros(E, np.float32)
    bal[:16] = np.float32(0.25)
    for t in range(64):
        a, b = t % 16, 16 + (t * 7) % 16
        l[t, a] = base + t * 1e-3
        # the logit whose sigmoid lies a quarter above: the nearest fp32 numbers around it give keys 1e-8 apart
        v = 1 / (1 + math.exp(-float(l[t, a]))) + 0.25
        x = np.float32(math.log(v / (1 - v)))
        l[t, b] = np.nextafter(x, np.float32(9)) if t % 2 else np.nextafter(x, np.float32(-9))
    for groups, rank in ((1, 1), (2, 1), (2, 2), (4, 2)):
        check_route(l, "sigmoid", 1, bal, groups, 1, rank, 0, 1.0)
        check_route(l, "sigmoid", 4, bal, groups, groups, rank, 1, 1.0)


def test_balance_of_minus_infinity_closes_an_expert():
    l = route_inputs(20, 24, 3, "plain")
    bal = np.zeros(24, np.float32)
    bal[::2] = -np.inf
    check_route(l, "sigmoid", 8, bal, 3, 2, 2, 1, 1.0)
    bal[:] = -np.inf
    idx, w, _, dl = run_route(l, "softmax", 3, bal, 1, 1, 1, 1, 1.0)
    assert (idx == -1).all() and (w == 0).all() and (dl == 0).all()


def test_routing_gradient_against_differences():
    """d sum(w dw) / d l by central differences of the oracle's weights at a fixed choice, in 64 bits."""
    for kind, renorm, scale in (("softmax", 1, 2.0), ("softmax", 0, 1.0), ("sigmoid", 1, 1.5), ("sigmoid", 0, 1.0)):
        l = route_inputs(6, 20, 5, "plain")
        idx, _, dw, dl = run_route(l, kind, 4, None, 1, 1, 1, renorm, scale)
        h = 1e-4
        for t in range(6):
            for e in range(20):
                two = []
                for sign in (1, -1):
                    m = l.astype(np.float64)[t:t + 1].copy()
                    m[0, e] += sign * h
                    s, ll = O.scores(m, kind)
                    two.append((O.weights(ll[0], s[0], idx[t], kind, renorm) * scale * dw[t]).sum())
                # differences: h^2 / 6 of a third derivative that is at most about 4 scale sum |dw|; kernel: fp32
                size = abs(scale) * np.abs(dw[t]).sum()
                assert abs((two[0] - two[1]) / (2 * h) - dl[t, e]) <= size * (h * h + 40 * U)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,d,E,k", [(1, 64, 8, 2), (77, 192, 40, 4), (300, 1024, 256, 8)])
def test_scored_routing_from_the_gate_product(dtype, T, d, E, k):
    """The whole gate: product, choice, and the gradients of x and Wr for sparse and dense logit gradients."""
    r = np.random.default_rng(T)
    x, Wr = dev(r.normal(0, 1, (T, d)), TD[dtype]), dev(r.normal(0, d ** -0.5, (d, E)))
    bias = dev(r.normal(0, 0.3, E))
    cfg = B.make_cfg(T, d, 64, E, k, DT[dtype])
    ws = torch.empty(B.moe_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    for kind, renorm in ((B.SCORE_SIGMOID, 1), (B.SCORE_SOFTMAX, 0)):
        sc = B.make_score(kind, 1, 1, 1, renorm, 1.0)
        logits, idx, w = torch.empty(T, E, device=DEV), torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
        B.moe_route_scored(cfg, sc, x, Wr, bias, None, None, logits, idx, w, ws)
        ref = f64(x) @ f64(Wr) + f64(bias)
        size = np.abs(f64(x)) @ np.abs(f64(Wr)) + 1
        term = 2.0 ** -17 if dtype != "f32" else 0.0          # the weight as two bf16 terms
        assert np.all(np.abs(f64(logits) - ref) <= (8 * math.sqrt(d) * U + term) * size)
        name = "sigmoid" if kind == B.SCORE_SIGMOID else "softmax"
        ridx, rw = O.route(logits.cpu().numpy(), name, k, renorm=renorm)
        assert np.array_equal(idx.cpu().numpy(), ridx)
        assert np.allclose(f64(w), rw, rtol=60 * U, atol=0)
        dw = dev(r.normal(0, 1, (T, k)))
        dl, dWr, dx = torch.empty(T, E, device=DEV), dev(np.ones((d, E))), dev(r.normal(0, 1, (T, d)), TD[dtype])
        before = f64(dx)
        B.moe_route_scored_bwd(cfg, sc, x, Wr, logits, idx, dw, dl, dWr, dx, ws, accumulate=1)
        g = f64(dl)
        rdl = O.route_bwd(logits.cpu().numpy(), name, ridx, f64(dw), renorm)
        assert np.abs(g - rdl).max() <= 100 * U * max(1.0, np.abs(rdl).max())
        want, size = f64(x).T @ g + 1, np.abs(f64(x)).T @ np.abs(g) + 1
        assert np.all(np.abs(f64(dWr) - want) <= (8 * math.sqrt(T) * U + term) * size)
        want, size = before + g @ f64(Wr).T, np.abs(before) + np.abs(g) @ np.abs(f64(Wr)).T
        # 2^-25: half the step of fp16's subnormal numbers
        assert np.all(np.abs(f64(dx) - want) <= half_step(dtype) * np.abs(want) + 8 * math.sqrt(E) * U * size + 2.0 ** -25)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,d,E,k,bias", [(1, 4096, 256, 8, True), (4, 64, 36, 3, False), (9, 1088, 100, 8, True), (3, 2880, 8, 2, False),
                                          (256, 1024, 256, 8, True), (2, 64, 4, 1, True), (513, 128, 64, 6, False)])
def test_scored_routing_of_few_tokens(dtype, T, d, E, k, bias):
    """Product and choice for decode batches and on both sides of the line between the two products."""
    r = np.random.default_rng(T + d)
    x, Wr, b = dev(r.normal(0, 1, (T, d)), TD[dtype]), dev(r.normal(0, d ** -0.5, (d, E))), dev(r.normal(0, 0.3, E)) if bias else None
    cfg, sc = B.make_cfg(T, d, 64, E, k, DT[dtype]), B.make_score(B.SCORE_SIGMOID, 1, 1, 1, 1, 2.5)
    ws = torch.empty(B.moe_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    logits, idx, w = torch.full((T, E), 7.0, device=DEV), torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    B.moe_route_scored(cfg, sc, x, Wr, b, None, None, logits, idx, w, ws)
    ref = f64(x) @ f64(Wr) + (f64(b) if bias else 0)
    size = np.abs(f64(x)) @ np.abs(f64(Wr)) + 1
    term = 2.0 ** -17 if dtype != "f32" else 0.0   # the weight as two 16-bit terms, where the matrix cores take it
    assert np.all(np.abs(f64(logits) - ref) <= (8 * math.sqrt(d) * U + term) * size)
    ridx, rw = O.route(logits.cpu().numpy(), "sigmoid", k, renorm=1, scale=2.5)
    assert np.array_equal(idx.cpu().numpy(), ridx)
    assert np.allclose(f64(w), rw, rtol=60 * U, atol=0)


@pytest.mark.parametrize("kind,renorm", [(B.SCORE_SIGMOID, 1), (B.SCORE_SIGMOID, 0), (B.SCORE_SOFTMAX, 0)])
@pytest.mark.parametrize("T,d,E,k", [(33, 68, 3, 1), (5, 516, 17, 8), (64, 260, 33, 3), (1, 4, 2, 2)])
def test_scored_input_gradient_odd_sizes(T, d, E, k, kind, renorm):
    """dx += d_logits Wr^T in fp32 where no tile of tokens, columns or experts is whole; a token without experts adds nothing."""
    r = np.random.default_rng(100 * T + E)
    lg = r.normal(0, 1, (T, E)).astype(np.float32)
    if T > 1:
        lg[T // 2] = -np.inf
    logits, Wr = dev(lg), dev(r.normal(0, 1, (d, E)))
    cfg, sc = B.make_cfg(T, d, 64, E, k, DT["f32"]), B.make_score(kind, 1, 1, 1, renorm, 1.5)
    ws = torch.empty(B.moe_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    idx, w = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    B.moe_route_scored(cfg, sc, None, None, None, None, logits, None, idx, w, ws)
    dw, dl, dx = dev(r.normal(0, 1, (T, k))), torch.empty(T, E, device=DEV), dev(r.normal(0, 1, (T, d)))
    before = f64(dx)
    B.moe_route_scored_bwd(cfg, sc, None, Wr, logits, idx, dw, dl, None, dx, ws)
    g = f64(dl)
    want, size = before + g @ f64(Wr).T, np.abs(before) + np.abs(g) @ np.abs(f64(Wr)).T
    # fp32 sums of at most E + 1 terms
    assert np.all(np.abs(f64(dx) - want) <= (E + 2) * U * size)
    if T > 1:
        assert np.array_equal(f64(dx)[T // 2], before[T // 2])


def test_empty_slots_travel_through_the_layer():
    """Tokens without an expert: dropped by dispatch, nothing in the output, no gradient."""
    from paper_2504_03871_amd.layer import MoELayer
    T, d, f, E, k = 40, 64, 128, 8, 4
    L = MoELayer(T, d, f, E, k)
    r = np.random.default_rng(0)
    for t, std in ((L.x, 1), (L.Wr, 0.1), (L.W1, 0.05), (L.W2, 0.05), (L.d_out, 1)):
        t.copy_(dev(r.normal(0, std, tuple(t.shape))))
    lg = route_inputs(T, E, 1, "masked")
    L.logits.copy_(dev(lg))
    sc = B.make_score(B.SCORE_SIGMOID, 1, 1, 1, 1, 1.0)
    B.moe_route_scored(L.cfg, sc, None, None, None, None, L.logits, None, L.topk_idx, L.topk_w)
    L.dispatch(); L.ffn_fwd(); L.combine(); L.combine_bwd()
    B.moe_route_scored_bwd(L.cfg, sc, None, None, L.logits, L.topk_idx, L.d_topk_w, L.d_logits, None, None)
    idx = L.topk_idx.cpu().numpy()
    assert (idx[::3] == -1).all() and (idx == -1).sum() > 40
    assert int(L.counts.sum()) == (idx >= 0).sum()
    assert (f64(L.out)[::3] == 0).all() and (f64(L.d_logits)[::3] == 0).all() and (f64(L.d_topk_w)[idx == -1] == 0).all()


# ---- 8 bits ----------------------------------------------------------------------------------------------------------

def pack_inputs(rows, width, dtype, seed):
    r = np.random.default_rng(seed)
    v = r.normal(0, 1, (rows, width)) * np.exp(r.normal(0, 3, (rows, 1)))
    t = torch.as_tensor(v).to(TD[dtype])
    if rows >= 8:
        big = torch.finfo(TD[dtype]).max
        small = torch.finfo(TD[dtype]).tiny * torch.finfo(TD[dtype]).eps
        t[1] = 0
        t[2, ::3] = big
        t[3, 0] = -big
        t[4] = small * torch.arange(width, dtype=torch.float64).to(TD[dtype])       # subnormal numbers
        t[5, width // 2] = math.inf
        t[6, width - 1] = math.nan
        t[7] = torch.linspace(-2, 2, width)                                         # many ties of both grids
    return t


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width,pitch", [(1, 1, 1), (9, 4, 4), (8, 31, 40), (12, 33, 33), (10, 64, 64), (16, 516, 516), (20, 200, 264), (40, 1024, 1024)])
def test_pack_and_unpack(rows, width, pitch, dtype, fmt):
    v = pack_inputs(rows, width, dtype, rows + width)
    src = torch.full((rows, pitch), 77.0, dtype=TD[dtype])
    src[:, :width] = v
    src = src.to(DEV)
    n = B.moe_pack8_bytes(rows, width)
    codes, scales = (torch.full((m + 64,), 0xAB, dtype=torch.uint8, device=DEV) for m in n)
    B.moe_pack8(DT[dtype], FMT[fmt], rows, width, pitch, src, codes, scales)
    rc, rs, rv = O.pack(v.double().numpy(), fmt)
    assert np.array_equal(scales[:n[1]].cpu().numpy().reshape(rs.shape), rs)
    got = codes[:n[0]].cpu().numpy().reshape(rc.shape)
    known = np.repeat(rs != 255, 32, axis=1)
    assert np.array_equal(got[known], rc[known])
    assert (codes[n[0]:] == 0xAB).all() and (scales[n[1]:] == 0xAB).all()
    out = torch.full((rows, pitch), 77.0, dtype=TD[dtype], device=DEV)
    B.moe_unpack8(DT[dtype], FMT[fmt], rows, width, pitch, codes, scales, out)
    most = torch.finfo(TD[dtype]).max
    want = torch.as_tensor(np.clip(rv, -most, most)).to(TD[dtype])
    back = out.cpu()
    assert torch.equal(back[:, :width].isnan(), want.isnan())
    assert torch.equal(torch.nan_to_num(back[:, :width].float()), torch.nan_to_num(want.float()))
    assert (back[:, width:] == 77.0).all()


def test_pack_of_every_bf16_number():
    """Each bf16 number in a block of its own with a second value that fixes the scale, and alone."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = torch.zeros(65536, 32, dtype=torch.bfloat16)
    v[:, 0] = bits
    v[:, 5] = bits * 0.37
    v[:, 9] = -bits * 0.011
    for fmt in FMT:
        codes, scales = (torch.empty(m, dtype=torch.uint8, device=DEV) for m in B.moe_pack8_bytes(65536, 32))
        B.moe_pack8(B.DTYPE_BF16, FMT[fmt], 65536, 32, 32, v.to(DEV), codes, scales)
        rc, rs, _ = O.pack(v.double().numpy(), fmt)
        assert np.array_equal(scales.cpu().numpy().reshape(rs.shape), rs)
        ok = np.repeat(rs != 255, 32, axis=1)
        assert np.array_equal(codes.cpu().numpy().reshape(rc.shape)[ok], rc[ok])


def test_pack_beyond_32_bit_offsets():
    rows, width = 66000, 65536
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("memory")
    src = torch.zeros(rows, width, dtype=torch.bfloat16, device=DEV)
    tail = pack_inputs(8, width, "bf16", 5)
    src[-8:] = tail.to(DEV)
    codes, scales = (torch.empty(m, dtype=torch.uint8, device=DEV) for m in B.moe_pack8_bytes(rows, width))
    B.moe_pack8(B.DTYPE_BF16, B.PACK_I8, rows, width, width, src, codes, scales)
    src.fill_(5.0)
    B.moe_unpack8(B.DTYPE_BF16, B.PACK_I8, rows, width, width, codes, scales, src)
    _, _, rv = O.pack(tail.double().numpy(), "i8")
    most = torch.finfo(torch.bfloat16).max
    want = torch.as_tensor(np.clip(rv, -most, most)).to(torch.bfloat16)
    assert torch.equal(torch.nan_to_num(src[-8:].cpu().float()), torch.nan_to_num(want.float()))
    assert int((src[:-8] != 0).sum()) == 0


@pytest.mark.parametrize("sliced", [False, True])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("dtype,f", [("f32", 100), ("bf16", 192), ("f16", 64)])
def test_saved_planes(dtype, f, act, sliced):
    T, E, k = 37, 6, 2
    A, mats = T * k, 2 if act == "swiglu" else 1
    cfg = B.make_cfg(T, 64, f, E, k, DT[dtype], B.ACT_SWIGLU if act == "swiglu" else B.ACT_GELU)
    kept = np.array([20, 0, 7, 30, 0, 11])                    # 68 of 74 rows in use
    offsets = np.concatenate([[0], np.cumsum(kept)])
    lo, hi = ([3, 0, 5, 0, 0, 9], [15, 4, 2, 99, 1, 11]) if sliced else (None, None)
    live = np.zeros(A, bool)
    for e in range(E):
        a, b = (min(max(lo[e], 0), kept[e]), min(max(hi[e], 0), kept[e])) if sliced else (0, kept[e])
        live[offsets[e] + a:offsets[e] + max(a, b)] = True
    r = np.random.default_rng(f)
    pre = dev(r.normal(0, 2, (mats, A, f)), TD[dtype])
    pre[:, torch.as_tensor(~live).to(DEV)] = math.nan         # rows that may not be read
    i32 = lambda a: None if a is None else dev(a, torch.int32)  # noqa: E731
    for fmt in FMT:
        codes, scales = (torch.full((m,), 0xAB, dtype=torch.uint8, device=DEV) for m in B.moe_saved_pack8_bytes(cfg))
        args = (i32(offsets), i32(kept), i32(lo), i32(hi))
        B.moe_saved_pack8(cfg, FMT[fmt], pre, *args, codes, scales)
        out = torch.full((mats + 1, A, f), 77.0, dtype=TD[dtype], device=DEV)
        B.moe_saved_restore8(cfg, FMT[fmt], codes, scales, *args, out)
        dead = torch.as_tensor(~live).to(DEV)
        nb = -(-f // 32)
        assert (codes.view(mats, A, nb * 32)[:, dead] == 0xAB).all() and (scales.view(mats, A, nb)[:, dead] == 0xAB).all()
        assert (out[:, dead] == 77.0).all()
        z = [O.pack(f64(pre[m])[live], fmt)[2] for m in range(mats)]
        for m in range(mats):
            assert np.array_equal(f64(out[m])[live], z[m])
        h = O.act(z, act)
        slack = 4e-7 * np.abs(z[0]) * (np.abs(z[1]) if mats == 2 else 1)   # Phi to 3e-7; sigmoid to a few units in the last place
        assert np.all(np.abs(f64(out[-1])[live] - h) <= half_step(dtype) * np.abs(h) + slack + 2.0 ** -25)


# ---- dense products --------------------------------------------------------------------------------------------------

def linear_case(T, d, n, dtype, act, bias=True, residual=True, seed=0):
    r = np.random.default_rng(seed + T + d + n)
    mats = 2 if act == "swiglu" else 1
    new = lambda *s, std=1.0: dev(r.normal(0, std, s), TD[dtype])  # noqa: E731
    return dict(T=T, d=d, n=n, dtype=dtype, act=act, mats=mats, x=new(T, d), W=[new(d, n, std=d ** -0.5) for _ in range(mats)],
                b=[new(n, std=0.3) for _ in range(mats)] if bias else [None, None][:mats], r=new(T, n) if residual else None, dy=new(T, n),
                pre=[new(T, n, std=1.2) for _ in range(mats)], add=new(T, d))


def two(v):
    return (list(v) + [None, None])[:2]


ACTS = {"none": B.ACT_NONE, "gelu": B.ACT_GELU, "swiglu": B.ACT_SWIGLU}


def run_fwd(c, keep=True, y=None, stream=None):
    lin = B.make_linear(c["T"], c["d"], c["n"], DT[c["dtype"]], ACTS[c["act"]])
    ws = torch.empty(max(16, B.moe_linear_workspace_bytes(lin)), dtype=torch.uint8, device=DEV)
    y = torch.full((c["T"], c["n"]), 77.0, dtype=TD[c["dtype"]], device=DEV) if y is None else y
    pre = [torch.full_like(y, 77.0) for _ in range(c["mats"])] if keep and c["act"] != "none" else []
    B.moe_linear_fwd(lin, c["x"], *two(c["W"]), *two(c["b"]), c["r"], *two(pre), y, ws, stream=stream)
    return y, pre


def check_fwd(c):
    y, pre = run_fwd(c)
    x, W = f64(c["x"]), [f64(w) for w in c["W"]]
    z = [x @ w + (0 if b is None else f64(b)) for w, b in zip(W, c["b"])]
    # fp32 sums of K exact products in an order of the kernel's choosing: a random walk of at most K roundings of the running
    # sum, 6 sigma; the running sum is at most the sum of magnitudes
    err = [6 * math.sqrt(c["d"]) * U * (np.abs(x) @ np.abs(w) + 1) for w in W]
    hs = half_step(c["dtype"])
    for p, zz, e in zip(pre, z, err):
        assert np.all(np.abs(f64(p) - zz) <= hs * np.abs(zz) + e + 2.0 ** -25)
    want = O.act(z, c["act"])
    slopes = O.act_slopes(z, c["act"])
    slack = sum((np.abs(s) + e) * e for s, e in zip(slopes, err)) + 8e-7 * np.abs(z[0]) * (np.abs(z[-1]) if c["mats"] == 2 else 1)
    want = want + (0 if c["r"] is None else f64(c["r"]))
    assert np.all(np.abs(f64(y) - want) <= hs * np.abs(want) + slack + 2.0 ** -25), np.abs(f64(y) - want).max()
    return y


def run_bwd(c, grad="f32", fmt=None, accumulate=0, add=True, skip=(), fill=77.0):
    lin = B.make_linear(c["T"], c["d"], c["n"], DT[c["dtype"]], ACTS[c["act"]], pre=FMT[fmt] if fmt else B.PACK_NONE, grad=DT[grad])
    ws = torch.empty(max(16, B.moe_linear_workspace_bytes(lin)), dtype=torch.uint8, device=DEV)
    new = lambda *s, t=TD[grad]: torch.full(s, fill, dtype=t, device=DEV)  # noqa: E731
    dx = None if "dx" in skip else new(c["T"], c["d"], t=TD[c["dtype"]])
    dW = [] if "dW" in skip else [new(c["d"], c["n"]) for _ in range(c["mats"])]
    db = [] if "db" in skip else [new(c["n"]) for _ in range(c["mats"])]
    pre, sc = (c["pre"], []) if c["act"] != "none" else ([], [])
    if fmt:
        packed = []
        for p in pre:
            q = [torch.empty(m, dtype=torch.uint8, device=DEV) for m in B.moe_pack8_bytes(c["T"], c["n"])]
            B.moe_pack8(DT[c["dtype"]], FMT[fmt], c["T"], c["n"], c["n"], p, *q)
            packed.append(q)
        pre, sc = [q[0] for q in packed], [q[1] for q in packed]
    B.moe_linear_bwd(lin, c["dy"], c["x"], *two(c["W"]), *two(pre), *two(sc), c["add"] if add else None, dx, *two(dW), *two(db), accumulate, ws)
    return dx, dW, db


def check_bwd(c, grad="f32", fmt=None, accumulate=0, add=True):
    dx, dW, db = run_bwd(c, grad, fmt, accumulate, add, fill=0.5 if accumulate else 77.0)
    old = 0.5 if accumulate else 0.0
    pre = [f64(p) for p in c["pre"]]
    if fmt:
        pre = [O.pack(p, fmt)[2] for p in pre]
    dy, x = f64(c["dy"]), f64(c["x"])
    dz = [dy * s for s in O.act_slopes(pre, c["act"])] if c["act"] != "none" else [dy]
    hs, hg = half_step(c["dtype"]), half_step(grad)
    # dz: the slope to 1e-6 (rational approximation, fast reciprocal), then one rounding to the storage type; the products' sums
    # carry the independent roundings of dz (6 sigma) and of fp32 accumulation as in the forward
    fuzz = 1e-6 if c["act"] != "none" else 0.0
    round_dz = hs if c["act"] != "none" else 0.0
    mag = np.abs(dy) * (1 + sum(np.abs(p) for p in pre)) if c["act"] != "none" else np.abs(dy)
    want = sum(g @ f64(w).T for g, w in zip(dz, c["W"])) + (f64(c["add"]) if add else 0)
    walk = sum(np.sqrt((g ** 2) @ (f64(w).T ** 2)) for g, w in zip(dz, c["W"]))
    sums = sum(np.abs(g) @ np.abs(f64(w)).T + fuzz / U * 0 for g, w in zip(dz, c["W"]))
    slope = sum(mag @ np.abs(f64(w)).T for w in c["W"]) * fuzz
    tol = hs * np.abs(want) + 6 * round_dz * walk + 6 * math.sqrt(2 * c["n"]) * U * (sums + 1) + slope + 2.0 ** -25
    assert np.all(np.abs(f64(dx) - want) <= tol), ("dx", np.abs(f64(dx) - want).max())
    for m, g in enumerate(dz):
        want = x.T @ g + old
        tol = hg * np.abs(want) + 6 * round_dz * np.sqrt((x.T ** 2) @ (g ** 2)) + 6 * math.sqrt(c["T"] + 16) * U * (np.abs(x).T @ np.abs(g) + 1) + \
            np.abs(x).T @ mag * fuzz
        assert np.all(np.abs(f64(dW[m]) - want) <= tol), ("dW", np.abs(f64(dW[m]) - want).max())
        want = g.sum(axis=0) + old
        tol = hg * np.abs(want) + 6 * math.sqrt(c["T"] + 16) * U * (np.abs(g).sum(axis=0) + 1) + fuzz * mag.sum(axis=0)
        assert np.all(np.abs(f64(db[m]) - want) <= tol), ("db", np.abs(f64(db[m]) - want).max())


SIZES = [("bf16", 1, 64, 64), ("bf16", 1, 1024, 192), ("f16", 7, 2048, 320), ("bf16", 33, 512, 1088), ("f16", 64, 256, 64), ("bf16", 65, 192, 448),
         ("bf16", 161, 1024, 512), ("f16", 300, 2880, 320), ("bf16", 513, 256, 2048), ("bf16", 700, 2048, 256), ("f16", 1025, 64, 832),
         ("f32", 1, 4, 4), ("f32", 3, 100, 36), ("f32", 70, 516, 132), ("f32", 257, 68, 1540), ("f32", 1000, 256, 512)]


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("dtype,T,d,n", SIZES)
def test_linear_forward(dtype, T, d, n, act):
    check_fwd(linear_case(T, d, n, dtype, act))
    check_fwd(linear_case(T, d, n, dtype, act, bias=False, residual=False))


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("dtype,T,d,n", SIZES)
def test_linear_backward(dtype, T, d, n, act):
    c = linear_case(T, d, n, dtype, act)
    check_bwd(c)
    check_bwd(c, grad=dtype, add=False)
    check_bwd(c, accumulate=1)


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("dtype,T,d,n", [("bf16", 5, 64, 64), ("f16", 300, 128, 448), ("f32", 70, 64, 100)])
def test_linear_backward_from_packed_pre_activations(dtype, T, d, n, act, fmt):
    check_bwd(linear_case(T, d, n, dtype, act), fmt=fmt)


# One size at least for every tile shape of the products and of the weight gradient, whole rounds of tiles, a rest and K parts.  T, d, n of
# the forward; dx has d columns over n, or over 2 n where two products are chained.
LARGE = [("bf16", 8192, 1024, 4096, "none"), ("bf16", 8191, 4096, 1024, "none"), ("f16", 4000, 2048, 4160, "swiglu"), ("bf16", 2300, 1088, 1984, "swiglu"),
         ("bf16", 1024, 4096, 1024, "none"), ("f16", 600, 8192, 320, "swiglu"), ("bf16", 3001, 2880, 1088, "gelu"), ("bf16", 48, 14336, 512, "none"),
         ("bf16", 20000, 512, 768, "none"), ("f32", 2048, 1024, 516, "swiglu"), ("f32", 150, 2048, 260, "none")]


@pytest.mark.parametrize("dtype,T,d,n,act", LARGE)
def test_linear_large(dtype, T, d, n, act):
    """Every element against products in 64 bits on the device; tolerances as above."""
    c = linear_case(T, d, n, dtype, act)
    y, _ = run_fwd(c, keep=False)
    hs = half_step(dtype)
    x, W = c["x"].double(), [w.double() for w in c["W"]]
    z = [x @ w + b.double() for w, b in zip(W, c["b"])]
    err = [6 * math.sqrt(d) * U * (x.abs() @ w.abs() + 1) for w in W]
    if act == "none":
        want, slack = z[0], err[0]
    elif act == "gelu":
        want, slack = torch.nn.functional.gelu(z[0]), 1.2 * err[0] + 8e-7 * z[0].abs()
    else:
        sg = torch.sigmoid(z[0])
        want = z[0] * sg * z[1]
        slack = 1.2 * z[1].abs() * err[0] + z[0].abs() * err[1] + 2 * err[0] * err[1] + 8e-7 * z[0].abs() * z[1].abs()
    want = want + c["r"].double()
    assert ((y.double() - want).abs() <= hs * want.abs() + slack + 2.0 ** -25).all()
    del z, err, want, slack, y
    for grad in {"f32", dtype}:
        dx, dW, db = run_bwd(c, grad=grad)
        pre, dy = [p.double() for p in c["pre"]], c["dy"].double()
        if act == "none":
            dz = [dy]
        elif act == "gelu":
            dz = [dy * (0.5 * torch.erfc(-pre[0] / math.sqrt(2)) + pre[0] * torch.exp(-0.5 * pre[0] ** 2) / math.sqrt(2 * math.pi))]
        else:
            sg = torch.sigmoid(pre[0])
            dz = [dy * pre[1] * sg * (1 + pre[0] * (1 - sg)), dy * pre[0] * sg]
        fuzz, rdz = (0.0, 0.0) if act == "none" else (1e-6, hs)
        mag = dy.abs() * (1 + sum(p.abs() for p in pre))
        want = sum(g @ w.t() for g, w in zip(dz, W)) + c["add"].double()
        walk = sum((g ** 2 @ (w.t() ** 2)).sqrt() for g, w in zip(dz, W))
        sums = sum(g.abs() @ w.t().abs() for g, w in zip(dz, W)) + 1
        slope = fuzz * sum(mag @ w.t().abs() for w in W)
        assert ((dx.double() - want).abs() <= hs * want.abs() + 6 * rdz * walk + 6 * math.sqrt(2 * n) * U * sums + slope + 2.0 ** -25).all()
        hg = half_step(grad)
        for m, g in enumerate(dz):
            want = x.t() @ g
            tol = hg * want.abs() + 6 * rdz * ((x.t() ** 2) @ (g ** 2)).sqrt() + 6 * math.sqrt(T + 16) * U * (x.t().abs() @ g.abs() + 1) + fuzz * (x.t().abs() @ mag)
            assert ((dW[m].double() - want).abs() <= tol).all()
            want = g.sum(dim=0)
            tol = hg * want.abs() + 6 * math.sqrt(T + 16) * U * (g.abs().sum(dim=0) + 1) + fuzz * mag.sum(dim=0)
            assert ((db[m].double() - want).abs() <= tol).all()


def test_linear_long_token_axis():
    """Weight gradients over many tokens, in segments: few tiles, a token count that no segment divides."""
    for dtype, T, d, n in (("bf16", 9001, 64, 128), ("f32", 4099, 64, 68)):
        c = linear_case(T, d, n, dtype, "gelu")
        check_bwd(c)
        check_bwd(c, accumulate=1)


def test_linear_outputs_may_be_skipped():
    c = linear_case(130, 128, 192, "bf16", "swiglu")
    full = run_bwd(c)
    for skip in (("dx",), ("dW",), ("db",), ("dx", "db"), ("dW", "db"), ("dx", "dW")):
        part = run_bwd(c, skip=skip)
        for name, a, b in zip(("dx", "dW", "db"), part, full):
            if name in skip:
                continue
            for u, v in zip(a if isinstance(a, list) else [a], b if isinstance(b, list) else [b]):
                assert torch.equal(u, v), (skip, name)


def test_linear_residual_in_place():
    """The residual may be the output itself, and dx_add dx itself."""
    for dtype, T, d, n in (("bf16", 20, 1024, 256), ("bf16", 300, 2048, 256), ("bf16", 600, 64, 256), ("f32", 70, 64, 100)):
        c = linear_case(T, d, n, dtype, "none")
        apart, _ = run_fwd(c)
        y = c["r"].clone()
        run_fwd({**c, "r": y}, y=y)
        assert torch.equal(apart, y)


def test_linear_non_finite_values_stay_in_their_rows():
    c = linear_case(200, 128, 128, "bf16", "gelu")
    clean, _ = run_fwd(c)
    c["x"][17] = math.nan
    c["x"][150, 3] = math.inf
    y, _ = run_fwd(c)
    rest = [i for i in range(200) if i not in (17, 150)]
    assert torch.equal(y[rest], clean[rest])
    assert y[17].isnan().all() and not torch.isfinite(y[150]).all()


def test_linear_without_tokens():
    for accumulate, want in ((0, 0.0), (1, 7.0)):
        c = dict(T=0, d=64, n=128, dtype="bf16", act="gelu", mats=1, x=torch.empty(0, 64, dtype=torch.bfloat16, device=DEV))
        c.update(W=[dev(np.ones((64, 128)), torch.bfloat16)], b=[None], r=None, dy=torch.empty(0, 128, dtype=torch.bfloat16, device=DEV),
                 pre=[torch.empty(0, 128, dtype=torch.bfloat16, device=DEV)], add=None)
        run_fwd(c)
        _, dW, db = run_bwd(c, accumulate=accumulate, fill=7.0)
        assert (dW[0] == want).all() and (db[0] == want).all()


def test_linear_gradient_against_differences():
    """Directional derivatives of sum(dy y) by central differences of the fp32 forward."""
    for act in ("gelu", "swiglu"):
        c = linear_case(40, 32, 48, "f32", act, residual=False)
        y, pre = run_fwd(c)
        dx, dW, db = run_bwd({**c, "pre": pre}, add=False)
        r = np.random.default_rng(2)
        h = 2.0 ** -6

        def loss(**change):
            yy, _ = run_fwd({**c, **change})
            return float((f64(yy) * f64(c["dy"])).sum())
        # truncation: h^2 / 6 of a third derivative of order one per unit direction; rounding: |y| 2^-24 sqrt(outputs) / h
        for name, grads in (("x", [dx]), ("W", dW), ("b", db)):
            for i, g in enumerate(grads):
                v = torch.as_tensor(r.normal(0, 1, tuple(g.shape))).to(torch.float32).to(DEV)
                v = v / v.norm()
                moved = []
                for s in (h, -h):
                    t = (c["x"] if name == "x" else c[name][i]) + s * v
                    moved.append(loss(**({"x": t} if name == "x" else {name: [t if j == i else o for j, o in enumerate(c[name])]})))
                want = (moved[0] - moved[1]) / (2 * h)
                noise = 16 * U * float(np.linalg.norm(f64(y) * f64(c["dy"]))) * math.sqrt(32) / h
                assert abs(want - float((f64(g) * f64(v)).sum())) <= h * h * float(np.linalg.norm(f64(c["dy"]))) + noise, (act, name)


def test_linear_beyond_32_bit_offsets():
    T, d, n = (1 << 19) + 3, 64, 8256        # 4.3e9 outputs
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("memory")
    x = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV)
    r = np.random.default_rng(0)
    tail = dev(r.normal(0, 1, (5, d)), torch.bfloat16)
    x[-5:] = tail
    W = dev(r.normal(0, 0.1, (d, n)), torch.bfloat16)
    lin = B.make_linear(T, d, n)
    ws = torch.empty(max(16, B.moe_linear_workspace_bytes(lin)), dtype=torch.uint8, device=DEV)
    y = torch.full((T, n), 7.0, dtype=torch.bfloat16, device=DEV)
    B.moe_linear_fwd(lin, x, W, None, None, None, None, None, None, y, ws)
    want = f64(tail) @ f64(W)
    assert np.all(np.abs(f64(y[-5:]) - want) <= 2.0 ** -8 * np.abs(want) + 1e-5)
    assert int((y[:-5] != 0).sum()) == 0
    dW = torch.empty(d, n, device=DEV)
    y[:-5] = 1.0
    B.moe_linear_bwd(lin, y, x, W, None, None, None, None, None, None, None, dW, None, None, None, 0, ws)
    want = f64(tail).T @ f64(y[-5:])
    assert np.abs(f64(dW) - want).max() <= 1e-5 * np.abs(want).max()


def test_operators_on_a_stream_and_in_a_graph():
    """On a side stream, and captured: every replay gives the eager bits, with eager calls between the replays."""
    c = linear_case(300, 2048, 256, "bf16", "gelu")
    lin = B.make_linear(300, 2048, 256, B.DTYPE_BF16, B.ACT_GELU)
    ws = torch.empty(B.moe_linear_workspace_bytes(lin), dtype=torch.uint8, device=DEV)
    y, z, dx = torch.empty_like(c["dy"]), torch.empty_like(c["dy"]), torch.empty_like(c["x"])
    dW, db = torch.empty(2048, 256, device=DEV), torch.empty(256, device=DEV)
    lg = dev(route_inputs(300, 256, 1, "plain"))
    cfg, sc = B.make_cfg(300, 64, 64, 256, 8), B.make_score(B.SCORE_SIGMOID, 8, 4, 2, 1, 2.5)
    idx, w, dl = torch.empty(300, 8, dtype=torch.int32, device=DEV), torch.empty(300, 8, device=DEV), torch.empty(300, 256, device=DEV)
    bal = dev(np.linspace(-0.05, 0.05, 256))
    codes, scales = (torch.empty(m, dtype=torch.uint8, device=DEV) for m in B.moe_pack8_bytes(300, 256))

    def step():
        B.moe_route_scored(cfg, sc, None, None, None, bal, lg, None, idx, w)
        B.moe_route_scored_bwd(cfg, sc, None, None, lg, idx, w, dl, None, None)
        B.moe_linear_fwd(lin, c["x"], c["W"][0], None, c["b"][0], None, c["r"], z, None, y, ws)
        B.moe_pack8(B.DTYPE_BF16, B.PACK_E4M3, 300, 256, 256, z, codes, scales)
        B.moe_unpack8(B.DTYPE_BF16, B.PACK_E4M3, 300, 256, 256, codes, scales, z)
        B.moe_linear_bwd(lin, c["dy"], c["x"], c["W"][0], None, z, None, None, None, None, dx, dW, None, db, None, 0, ws)

    outs = (idx, w, dl, y, z, dx, dW, db, codes, scales)
    step()
    torch.cuda.synchronize()
    eager = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            o.zero_()
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


def test_tensors_must_be_contiguous():
    c = linear_case(64, 64, 128, "bf16", "none")
    with pytest.raises(ValueError):
        run_fwd({**c, "x": torch.empty(64, 64, dtype=torch.bfloat16, device=DEV).t()})
    big = torch.zeros(8, 64, dtype=torch.bfloat16, device=DEV)
    codes, scales = (torch.empty(m, dtype=torch.uint8, device=DEV) for m in B.moe_pack8_bytes(8, 40))
    B.moe_pack8(B.DTYPE_BF16, B.PACK_I8, 8, 40, 64, big[:, :40], codes, scales)          # a view of rows that are 64 apart
    with pytest.raises(ValueError):
        B.moe_pack8(B.DTYPE_BF16, B.PACK_I8, 8, 40, 40, big[:, :40], codes, scales)      # the pitch says something else


# ---- choices among keys of zero, next to it and beyond the finite numbers -------------------------------------------

def zero_rows(E, seed):
    """Rows whose open logits are all zero, of either sign, or a few steps of 2^-149 from it: all experts, runs of 16, scattered ones."""
    r = np.random.default_rng(seed)
    rows = []
    for sign in (0.0, -0.0):
        rows.append(np.full(E, sign))
        for first in range(0, E, 16):
            row = np.full(E, -np.inf)
            row[first:first + 16] = sign
            rows.append(row)
    for share in (0.1, 0.5, 1.0):
        row = np.where(r.random(E) < 0.5, 0.0, -0.0)
        rows.append(np.where(r.random(E) < share, row, -np.inf))
        row = r.integers(-20, 21, E) * 2.0 ** -149
        rows.append(np.where(r.random(E) < share, row, -np.inf))
    return np.array(rows, dtype=np.float32)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [3, 16, 17, 18, 19, 33, 36, 39, 64, 72, 129, 144, 256])
def test_equal_logits_of_zero(E, kind):
    """Equal logits by ascending expert, whatever their size: a router whose weights start at zero, tokens of zeros."""
    l = zero_rows(E, E)
    for k in sorted({1, min(4, E), min(7, E), min(8, E)}):
        check_route(l, kind, k, None, 1, 1, 1, 1, 1.0)
    for groups in (2, 3, 4, 8, 16):
        if E % groups == 0 and E // groups >= 2:
            top = (groups + 1) // 2
            for rank in (1, 2):
                check_route(l, kind, min(8, E // groups * top), None, groups, top, rank, 1, 1.0)


@pytest.mark.parametrize("E,groups", [(18, 1), (36, 4), (64, 8), (144, 3), (256, 8)])
def test_sigmoid_scores_below_the_smallest_fp32_number(E, groups):
    """Scores that single precision rounds to zero, with a balance of zeros and summed up in groups: equal ones by ascending expert,
    different ones by their double precision scores (but for scores that are zero there too)."""
    r = np.random.default_rng(E)
    l = np.concatenate([np.full((4, E), -100.0), np.full((4, E), -800.0), r.uniform(-140, -86, (24, E)), r.choice([-90.0, -95.0, -800.0, -900.0], (24, E))])
    l[r.random(l.shape) < 0.2] = -np.inf
    l[0], l[4] = -100.0, -800.0
    for rank in (1, 2):
        for balance in (np.zeros(E, np.float32), None) if groups > 1 and rank == 2 else (np.zeros(E, np.float32),):
            top = (groups + 1) // 2
            for k in (1, min(8, E // groups * top)):
                check_route(l.astype(np.float32), "sigmoid", k, balance, groups, top, rank, 1, 1.0)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_finite_masks_and_logits_of_any_size(kind):
    """Experts closed by a large finite number instead of minus infinity: open ones first, then closed ones by ascending expert."""
    r = np.random.default_rng(7)
    for E, k, groups, top in ((64, 6, 1, 1), (256, 8, 8, 4), (40, 8, 1, 1)):
        l = route_inputs(60, E, E, "plain")
        l[:20][r.random((20, E)) < 0.97] = -1e9
        l[20:40][r.random((20, E)) < 0.3] = -F32_MAX
        l[40:, ::3] = np.nextafter(np.float32(0.5), np.float32(1))      # neighbours in single precision, and equal ones
        l[40:, 1::3] = 0.5
        l[50:, 2::3] = np.nextafter(np.float32(0.5), np.float32(0))
        idx = run_route(l, kind, k, None, groups, top, 1, 1, 1.0)[0]
        assert np.array_equal(idx, O.route(l, kind, k, None, groups, top, 1, 1, 1.0)[0])


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,groups,top,rank", [(64, 4, 1, 1, 1), (256, 8, 1, 1, 1), (64, 6, 8, 3, 2), (36, 3, 4, 2, 2), (64, 4, 4, 1, 1), (40, 8, 5, 3, 2)])
def test_balance_of_any_size(E, k, groups, top, rank, kind):
    """Plus infinity counts as the largest number: such experts come first, by ascending expert, and a group whose others are closed
    still scores minus infinity in a sum of two.  Finite numbers up to the largest."""
    r = np.random.default_rng(E + k)
    for trial in range(12):
        l = route_inputs(40, E, trial, "masked" if trial % 2 else "plain")
        bal = np.where(r.random(E) < 0.5, 0.01, -0.02).astype(np.float32)
        bal[r.choice(E, max(2, E // 8), replace=False)] = np.inf if trial % 3 else F32_MAX
        if trial % 3 != 1:  # else no finite number is large
            bal[r.choice(E, 2, replace=False)] = -F32_MAX
        if trial % 4 == 3:
            bal[r.choice(E, E // 3, replace=False)] = -np.inf
        if trial >= 8:      # the first group: one expert that can be chosen, with a balance of plus infinity
            size = E // groups
            l[:, :size], bal[0] = -np.inf, np.inf
            l[:, 0] = 0.5
        idx, w, _, _ = run_route(l, kind, k, bal, groups, top, rank, 1, 1.0)
        ridx, rw = O.route(l, kind, k, np.minimum(bal, np.float32(F32_MAX)), groups, top, rank, 1, 1.0)
        assert np.array_equal(idx, ridx), trial
        assert np.allclose(w, rw, rtol=100 * U, atol=0)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_order_where_scores_round_to_the_same_number(kind):
    """Without a balance the logits order the experts, with one (of zeros too) the double precision keys, equal ones by expert."""
    T, E, k = 48, 64, 6
    r = np.random.default_rng(4)
    l = (r.normal(0, 1, (T, E)) + (60 if kind == "sigmoid" else -900)).astype(np.float32)   # sigmoids of exactly 1, softmax scores of exactly 0
    if kind == "softmax":
        l[:, 5] = 0.0
    by_logit = np.argsort(-l, axis=1, kind="stable")[:, :k]
    by_score = np.tile(np.arange(k), (T, 1))
    if kind == "softmax":
        by_score[:, 0], by_score[:, 1:] = 5, np.arange(k - 1)
    for groups, top in ((1, 1), (4, 4)):
        for rank in (1, 2):
            logits_decide = groups == 1 or rank == 1
            assert np.array_equal(run_route(l, kind, k, None, groups, top, rank, 1, 1.0)[0], by_logit if logits_decide else by_score)
            assert np.array_equal(run_route(l, kind, k, np.zeros(E, np.float32), groups, top, rank, 1, 1.0)[0], by_score)


def test_pack_scales_at_the_largest_element():
    """The scale doubles where the largest magnitude would saturate: above 448 (e4m3), from 127.5 64ths on (which would round to 128)."""
    for fmt, most, up in (("e4m3", 448.0, np.nextafter(np.float32(448), np.float32(500))), ("i8", np.nextafter(np.float32(127.5 / 64), np.float32(0)), 127.5 / 64)):
        v = torch.zeros(2, 32, device=DEV)
        v[0, 3], v[1, 3] = float(most), float(up)
        codes, scales = (torch.empty(m, dtype=torch.uint8, device=DEV) for m in B.moe_pack8_bytes(2, 32))
        B.moe_pack8(B.DTYPE_F32, FMT[fmt], 2, 32, 32, v, codes, scales)
        assert scales.tolist() == [127, 128]
        assert codes.view(2, 32)[:, 3].tolist() == ([0x7e, 0x76] if fmt == "e4m3" else [127, 64])


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_unpack_of_every_code(dtype, fmt):
    """Codes from elsewhere too: e4m3's two NaN codes, which pack never writes, -128 64ths, every code under scales of any size."""
    scales = torch.tensor([0, 1, 60, 118, 127, 135, 200, 246, 254, 255], dtype=torch.uint8)
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).repeat(len(scales), 1)
    n = B.moe_pack8_bytes(len(scales), 256)
    assert n == (codes.numel(), len(scales) * 8)
    out = torch.empty(len(scales), 256, dtype=TD[dtype], device=DEV)
    B.moe_unpack8(DT[dtype], FMT[fmt], len(scales), 256, 256, codes.to(DEV), scales.repeat_interleave(8).to(DEV), out)
    value = codes.view(torch.int8).double() / 64
    if fmt == "e4m3":
        a = codes.long() & 127
        m, e = (a & 7).double(), (a >> 3).double()
        value = torch.where(a < 8, m * 2.0 ** -9, (8 + m) * torch.exp2(e - 10)) * torch.where(codes > 127, -1.0, 1.0)
        value = torch.where(a == 127, math.nan, value)
    most = torch.finfo(TD[dtype]).max
    want = torch.clamp(value * torch.exp2(scales.double() - 127)[:, None], -most, most)
    want[scales == 255] = math.nan
    got = out.cpu()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(torch.nan_to_num(got.double()), torch.nan_to_num(want.to(TD[dtype]).double()))


@pytest.mark.parametrize("dtype,T,d,n,act", [("bf16", 16, 4096, 256, "gelu"), ("f16", 300, 2048, 320, "swiglu"), ("bf16", 700, 256, 512, "none"),
                                             ("f32", 70, 1024, 132, "swiglu"), ("f32", 300, 64, 100, "gelu")])
def test_linear_forward_in_its_own_workspace(dtype, T, d, n, act):
    c = linear_case(T, d, n, dtype, act)
    whole, _ = run_fwd(c, keep=False)
    lin = B.make_linear(T, d, n, DT[dtype], ACTS[act])
    need = B.moe_linear_fwd_workspace_bytes(lin)
    ws = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device=DEV)
    y = torch.full_like(whole, 77.0)
    B.moe_linear_fwd(lin, c["x"], *two(c["W"]), *two(c["b"]), c["r"], None, None, y, ws, ws_bytes=need)
    assert torch.equal(y, whole) and (ws[need:] == 0xAB).all()


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("dtype,T,d,n,with_dw", [
    ("bf16", 300, 256, 2048, True), ("f16", 64, 128, 1024, True),       # both gradients in one launch, K parts
    ("bf16", 300, 512, 4096, False), ("f16", 33, 256, 8192, False),     # dx alone, K parts
    ("bf16", 4100, 1024, 512, True), ("f16", 2300, 2048, 1088, True),   # large tiles, whole and in parts
    ("f32", 70, 132, 1024, True), ("f32", 300, 64, 2048, False), ("f32", 900, 516, 100, True)])
def test_linear_input_gradient_in_place(dtype, T, d, n, with_dw, act):
    """dx_add may be dx itself: the bits of a sum with dx_add apart."""
    c = linear_case(T, d, n, dtype, act)
    lin = B.make_linear(T, d, n, DT[dtype], ACTS[act])
    ws = torch.empty(B.moe_linear_workspace_bytes(lin), dtype=torch.uint8, device=DEV)
    pre = two(c["pre"] if act != "none" else [])
    dW = [torch.empty(d, n, device=DEV) for _ in range(c["mats"])] if with_dw else []

    def dx_of(add, dx):
        B.moe_linear_bwd(lin, c["dy"], c["x"], *two(c["W"]), *pre, None, None, add, dx, *two(dW), None, None, 0, ws)
        return dx
    apart = dx_of(c["add"], torch.full_like(c["x"], 77.0))
    without = dx_of(None, torch.full_like(c["x"], 77.0))
    assert not torch.equal(apart, without)
    mine = c["add"].clone()
    assert torch.equal(dx_of(mine, mine), apart)
