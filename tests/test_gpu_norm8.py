"""The norm with its residual, dropout and products in 8-bit integers on the GPU, against the 64-bit oracle."""
import numpy as np
import pytest

from oracle import norm8_oracle as O
from paper_2504_03871_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DEV = "cuda:0"
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DT = {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16}
ACT = {"none": B.ACT_NONE, "gelu": B.ACT_GELU, "swiglu": B.ACT_SWIGLU}
U = 2.0 ** -24           # rounding to fp32, half a step


def half_step(dtype):
    return torch.finfo(TD[dtype]).eps / 2


def least(dtype):
    """Half of the smallest number's step: what a rounding of values next to zero is off by."""
    return torch.finfo(TD[dtype]).smallest_normal * torch.finfo(TD[dtype]).eps / 2


def dev(a, dtype="f32"):
    return torch.as_tensor(np.asarray(a)).to(TD[dtype]).to(DEV)


def f64(t):
    return t.detach().double().cpu().numpy()


def empty(*shape, dtype="f32", fill=12288.0):
    return torch.full(shape, fill, dtype=TD[dtype], device=DEV)


def near(name, got, want, tol):
    got = f64(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape, (name, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.nanmax(np.where(bad, np.abs(got - want) / tol, 0))))


# ---- dropout -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows, width, p, res", [(1, 1, 0.5, False), (3, 7, 0.1, True), (5, 8, 0.0, True), (17, 65, 0.3, False), (300, 517, 0.5, False),
                                                  (64, 1024, 0.999999, True), (2, 16383, 0.2, True), (700, 4096, 0.1, True)])
def test_dropout(dtype, rows, width, p, res):
    r = np.random.default_rng(rows + width)
    x, q = dev(r.normal(size=(rows, width)), dtype), dev(r.normal(size=(rows, width)), dtype)
    seed, offset = (1 << 63) + 12345, (7 << 40) + rows
    y = empty(rows, width, dtype=dtype)
    B.moe_dropout(DT[dtype], rows, width, B.make_drop(p, seed, offset), x, q if res else None, y)
    v = f64(x) * O.drop_mask(rows, width, p, seed, offset)
    want = v + f64(q) if res else v
    # the scale's rounding, the product's, the sum's, the result's
    near("y", y, want, 2 * U * np.abs(v) + (U + half_step(dtype)) * np.abs(want) * (1 + 4 * U) + U * np.abs(v) + least(dtype))
    if not res:
        assert np.array_equal(f64(y) == 0, v == 0)


def test_dropout_replaces_what_is_no_number_and_works_in_place():
    x = torch.full((8, 64), float("nan"), device=DEV)
    x[4:] = float("inf")
    m = O.drop_mask(8, 64, 0.5, 1, 2)
    B.moe_dropout(B.DTYPE_F32, 8, 64, B.make_drop(0.5, 1, 2), x, None, x)
    got = f64(x)
    assert (got[m == 0] == 0).all() and np.isnan(got[:4][m[:4] > 0]).all() and np.isinf(got[4:][m[4:] > 0]).all()
    a, q = dev(np.ones((8, 64))), dev(np.full((8, 64), 3.0))
    B.moe_dropout(B.DTYPE_F32, 8, 64, B.make_drop(0.5, 1, 2), a, q, q)
    assert np.array_equal(f64(q), 3 + m)


def test_dropout_step_on_the_device_gives_every_replay_its_mask():
    x, y, step = dev(np.ones((33, 100))), empty(33, 100), torch.zeros(1, dtype=torch.int64, device=DEV)
    drop = B.make_drop(0.25, 99, 1000, step)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        B.moe_dropout(B.DTYPE_F32, 33, 100, drop, x, None, y)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step.add_(1)
        B.moe_dropout(B.DTYPE_F32, 33, 100, drop, x, None, y)
    for i in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        near("y", y, O.drop_mask(33, 100, 0.25, 99, 1000 + i), 4 * U)
        B.moe_dropout(B.DTYPE_F32, 33, 100, B.make_drop(0.25, 99, 1), x, None, empty(33, 100))   # eager work in between
        torch.cuda.synchronize()


# ---- norm ----------------------------------------------------------------------------------------------------------

def norm_tolerance(d):
    """Relative error of a row's mean square in fp32, and of what is made of it: every thread adds up to 32 squares one after the other,
    six exchanges and eight waves on top, each rounding at most U; half of that in the root, and a few for the root, the
    quotient and the two products.  (At most 64 U in all.)"""
    return (32 + 6 + 8 + 2) / 2 * U + 8 * U


NORM = [  # T, d
    (1, 1), (3, 7), (5, 8), (2, 64), (4, 100), (1, 500), (3, 512), (9, 516), (2, 1000), (3, 1024), (2, 1091), (5, 2048), (3, 3000), (3, 4096), (1, 4100),
    (2, 4099), (2, 8192), (1, 8200), (1, 16384), (2, 16383), (300, 72), (77, 24), (1024, 513), (1025, 1000), (1100, 100), (1500, 1091), (2048, 264), (2049, 264), (2100, 520), (2500, 1091), (2200, 63),
]
KINDS = [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]


def norm_case(T, d, dtype, stream, seed):
    r = np.random.default_rng(seed)
    size = np.exp(r.normal(0, 1, (T, 1)))
    return (dev(r.normal(size=(T, d)) * size, dtype), dev(r.normal(size=(T, d)) * size, stream), dev(1 + 0.3 * r.normal(size=d), dtype),
            dev(r.normal(size=(T, d)), dtype), dev(r.normal(size=(T, d)), stream))


@pytest.mark.parametrize("dtype, stream", KINDS)
@pytest.mark.parametrize("T, d", NORM)
def test_norm_forward_and_backward(T, d, dtype, stream):
    eps = 1e-5
    for p, res, gam in ((0.0, True, True), (0.2, True, True), (0.1, False, True), (0.0, False, False)):
        x, q, g, dy, add = norm_case(T, d, dtype, stream, T + d)
        norm = B.make_norm(T, d, DT[dtype], DT[stream], eps=eps)
        drop = B.make_drop(p, 5, 6) if p else None
        m = O.drop_mask(T, d, p, 5, 6)
        h, rstd, y, dh, dx, dg = empty(T, d, dtype=stream), empty(T), empty(T, d, dtype=dtype), empty(T, d, dtype=stream), empty(T, d, dtype=dtype), empty(d)
        codes, scales = torch.full((T, d), 99, dtype=torch.int8, device=DEV), empty(T)
        B.moe_norm_fwd(norm, drop, x, q if res else None, g if gam else None, h, rstd, y, codes, scales)
        v = f64(x) * m
        want = v + f64(q) if res else v
        near("h", h, want, 3 * U * np.abs(v) + (U + half_step(stream)) * (1 + 4 * U) * np.abs(want) + least(stream))
        hs, gs = f64(h), f64(g) if gam else np.ones(d)   # the norm is that of h as it is stored
        wy, wr = O.norm_fwd(hs, gs, eps)
        tol = norm_tolerance(d)
        near("rstd", rstd, wr, tol * wr)
        near("y", y, wy, (tol + half_step(dtype)) * (1 + tol) * np.abs(wy) + least(dtype))
        # codes of y before its rounding: half a step of a whole number, and y's own error
        ws = np.abs(wy).max(axis=1) / 127
        near("scales", scales, np.maximum(ws, 2.0 ** -100 / 127), (tol + 4 * U) * ws + U * 2.0 ** -100)
        near("codes", codes.double() * scales.double()[:, None], wy, (0.5 + 127 * (2 * tol + 6 * U)) * np.maximum(ws, 2.0 ** -100)[:, None])
        y2 = empty(T, d, dtype=dtype)
        B.moe_norm_fwd(norm, drop, x, q if res else None, g if gam else None, None, None, y2, None, None)   # nothing kept: the same y
        assert torch.equal(y, y2)
        c2, s2 = torch.zeros_like(codes), empty(T)
        B.moe_norm_fwd(norm, drop, x, q if res else None, g if gam else None, None, None, None, c2, s2)
        assert torch.equal(codes, c2) and torch.equal(scales, s2)

        ws_ = torch.empty(B.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device=DEV)
        B.moe_norm_bwd(norm, drop, dy, h, g if gam else None, rstd, add if res else None, dh, dx, dg, 0, ws_)
        wa = f64(add) if res else np.zeros((T, d))
        wdh, wdg = O.norm_bwd(f64(dy), hs, gs, eps, wa)
        u, a = hs * wr[:, None], gs * f64(dy)
        # the sum of products with terms of either sign: the error goes by the sum of their sizes
        size = wr[:, None] * (np.abs(a) + np.abs(u) * np.abs(a * u).mean(axis=1, keepdims=True)) + np.abs(wa)
        near("dh", dh, wdh, 2 * tol * size + 8 * U * size + half_step(stream) * np.abs(wdh) + least(stream))
        near("dx", dx, wdh * m, (2 * tol * size + 10 * U * size) * m + half_step(dtype) * np.abs(wdh * m) + least(dtype))
        near("dgamma", dg, wdg, (tol + (T + 40) * U) * np.abs(f64(dy) * u).sum(axis=0) + 1e-30)
        dg2 = dg.clone()
        B.moe_norm_bwd(norm, drop, dy, h, g if gam else None, rstd, add if res else None, None, None, dg2, 1, ws_)   # added to
        near("dgamma twice", dg2, 2 * f64(dg), 2 * U * np.abs(f64(dg)) + 1e-30)
        if not res:
            continue
        B.moe_norm_bwd(norm, drop, dy, h, g, rstd, add, add, None, None, 0, None)                        # in place
        assert torch.equal(add, dh)
        r2 = q.clone()
        B.moe_norm_fwd(norm, drop, x, r2, g if gam else None, r2, None, y2, None, None)                   # h over the residual
        assert torch.equal(r2, h) and torch.equal(y2, y)


@pytest.mark.parametrize("T, d", [(3, 64), (700, 1091), (2048, 520), (3000, 256)])
@pytest.mark.parametrize("dtype, stream", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_norm_backward_in_place_with_the_gradient_of_gamma(T, d, dtype, stream):
    """dx over dy and dh over dh_add, dh over h, and dh over dy where the types are one: the gradients of the same call with places of its own."""
    x, h, g, dy, add = norm_case(T, d, dtype, stream, 5)
    norm, drop = B.make_norm(T, d, DT[dtype], DT[stream]), B.make_drop(0.25, 3)
    rstd, y = empty(T), empty(T, d, dtype=dtype)
    B.moe_norm_fwd(norm, None, h if dtype == stream else h.to(TD[dtype]), None, g, None, rstd, y, None, None)
    dh, dx, dg, ws = empty(T, d, dtype=stream), empty(T, d, dtype=dtype), empty(d), torch.empty(B.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device=DEV)
    B.moe_norm_bwd(norm, drop, dy, h, g, rstd, add, dh, dx, dg, 0, ws)
    sums = (norm_tolerance(d) + (T + 40) * U) * (dy.double().abs() * (h.double() * rstd.double()[:, None]).abs()).sum(dim=0) + 1e-30
    for places in ("dx over dy, dh over dh_add", "dh over h", "dh over dy"):
        if places == "dh over dy" and dtype != stream:
            continue
        dy2, h2, add2, dg2 = dy.clone(), h.clone(), add.clone(), empty(d)
        to_h, to_x = {"dx over dy, dh over dh_add": (add2, dy2), "dh over h": (h2, empty(T, d, dtype=dtype)), "dh over dy": (dy2, empty(T, d, dtype=dtype))}[places]
        B.moe_norm_bwd(norm, drop, dy2, h2, g, rstd, add2, to_h, to_x, dg2, 0, ws)
        assert torch.equal(to_h, dh) and torch.equal(to_x, dx), places
        assert bool(((dg2.double() - dg.double()).abs() <= 2 * sums).all()), places     # another order of the sum


def test_norm_gradient_against_differences_of_its_forward():
    T, d, eps = 6, 40, 1e-3
    x, q, g, dy, add = norm_case(T, d, "f32", "f32", 3)
    norm, drop = B.make_norm(T, d, B.DTYPE_F32, eps=eps), B.make_drop(0.3, 8, 9)
    h, rstd, y, dh, dx, dg = (empty(T, d), empty(T), empty(T, d), empty(T, d), empty(T, d), empty(d))
    run = lambda x, q, g: B.moe_norm_fwd(norm, drop, x, q, g, h, rstd, y, None, None)  # noqa: E731
    loss = lambda: float((y.double() * dy.double()).sum() + (h.double() * add.double()).sum())  # noqa: E731
    run(x, q, g)
    B.moe_norm_bwd(norm, drop, dy, h, g, rstd, add, dh, dx, dg, 0, torch.empty(B.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device=DEV))
    r, t = np.random.default_rng(4), 2.0 ** -7
    for _ in range(4):
        vx, vq, vg = dev(r.normal(size=(T, d))), dev(r.normal(size=(T, d))), dev(r.normal(size=d))
        run(x + t * vx, q + t * vq, g + t * vg)
        up = loss()
        run(x - t * vx, q - t * vq, g - t * vg)
        num = (up - loss()) / (2 * t)
        want = float((dx.double() * vx.double()).sum() + (dh.double() * vq.double()).sum() + (dg.double() * vg.double()).sum())
        size = float((dx.double() * vx.double()).abs().sum() + (dh.double() * vq.double()).abs().sum())
        # t^2 times third derivatives of a function of size one, and 2 T d fp32 roundings over t
        assert abs(num - want) < (8 * t * t + 2 * T * d * U / t) * size, (num, want, size)


def test_norm_rows_that_hold_zeros_or_no_numbers_and_what_lies_behind_the_last():
    T, d = 4, 136
    x = torch.zeros((T, d), dtype=torch.bfloat16, device=DEV)
    x[1, 5], x[2, 7] = float("nan"), float("inf")
    x[3] = 2.0
    norm = B.make_norm(T, d, B.DTYPE_BF16, eps=1e-6)
    y, codes, scales = empty(T + 1, d, dtype="bf16"), torch.full((T + 1, d), 99, dtype=torch.int8, device=DEV), empty(T + 1)
    B.moe_norm_fwd(norm, None, x, None, None, None, None, y, codes, scales)
    got = f64(y)
    assert (got[0] == 0).all() and np.isnan(got[1]).all() and np.isnan(got[2][7]) and (got[3] == 1).all()
    assert (got[T] == 12288).all() and (codes[T] == 99).all() and float(scales[T]) == 12288
    assert not codes[:3].any() and torch.isnan(scales[1:3]).all() and (codes[3] == 127).all()
    for n in (B.make_norm(0, d, B.DTYPE_BF16),):
        B.moe_norm_fwd(n, None, None, None, None, None, None, None, None, None)
        dg = empty(d)
        B.moe_norm_bwd(n, None, None, None, None, None, None, None, None, dg, 1, None)
        assert (dg == 12288).all()
        B.moe_norm_bwd(n, None, None, None, None, None, None, None, None, dg, 0, None)
        assert (dg == 0).all()


@pytest.mark.parametrize("T, d", [(5000, 256), (700, 1536)])
def test_norm_backward_of_many_rows_is_the_same_every_time_and_in_a_graph(T, d):
    x, q, g, dy, add = norm_case(T, d, "bf16", "f32", 1)
    norm, drop = B.make_norm(T, d, B.DTYPE_BF16, B.DTYPE_F32, grad=B.DTYPE_BF16), B.make_drop(0.1, 1)
    h, rstd, y, dh, dx = empty(T, d), empty(T), empty(T, d, dtype="bf16"), empty(T, d), empty(T, d, dtype="bf16")
    dg = empty(d, dtype="bf16")
    ws = torch.empty(B.moe_norm_bwd_workspace_bytes(norm), dtype=torch.uint8, device=DEV)

    def run():
        B.moe_norm_fwd(norm, drop, x, q, g, h, rstd, y, None, None)
        B.moe_norm_bwd(norm, drop, dy, h, g, rstd, add, dh, dx, dg, 0, ws)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in (h, y, dh, dx, dg)]
    hs, u = f64(h), None
    u = hs * (1 / np.sqrt((hs * hs).mean(axis=1) + 1e-6))[:, None]
    wdg = (f64(dy) * u).sum(axis=0)
    near("dgamma", dg, wdg, (norm_tolerance(d) + 64 * U) * np.abs(f64(dy) * u).sum(axis=0) + half_step("bf16") * np.abs(wdg))
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run()
    for _ in range(3):
        for t in (h, y, dh, dx, dg, ws):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((h, y, dh, dx, dg), want):
            assert torch.equal(t, w)


# ---- quantising ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows, width, pitch", [(1, 1, 1), (3, 7, 9), (9, 64, 64), (5, 100, 104), (4, 1024, 1024), (2, 2048, 2052), (3, 3001, 3001), (2, 4096, 4096),
                                                 (3, 8192, 8192), (2, 14336, 14336), (2, 32768, 32768), (1, 65536, 65536), (2, 40001, 40008), (257, 320, 320)])
def test_quantised_rows(dtype, rows, width, pitch):
    r = np.random.default_rng(width)
    v = r.normal(size=(rows, width)) * np.exp(r.normal(0, 3, (rows, 1)))
    if rows > 2:
        v[0], v[1, width // 2], v[2, 0] = 0, np.nan, -np.inf
    src = torch.full((rows, pitch), float("nan"), dtype=TD[dtype], device=DEV)
    src[:, :width] = dev(v, dtype)
    codes, scales = torch.full((rows * width + 16,), 99, dtype=torch.int8, device=DEV), empty(rows + 1)
    B.moe_quant_rows(DT[dtype], rows, width, pitch, src[:, :width], codes, scales)
    wq, wsc = O.quant_rows(src[:, :width].float().cpu().numpy())
    assert np.array_equal(codes[:rows * width].cpu().numpy().reshape(rows, width), wq)
    assert np.array_equal(scales[:rows].cpu().numpy(), wsc, equal_nan=True)
    assert (codes[rows * width:] == 99).all() and float(scales[rows]) == 12288


def test_quantised_rows_next_to_the_ends_of_fp32():
    v = np.array([[3.4028234e38, -1, 1e38], [1e-45, -1e-45, 0], [2.0 ** -100, 2.0 ** -101, -(2.0 ** -107)], [1.5 * 2.0 ** -101, 0, 1e-38]], dtype=np.float32)
    codes, scales = torch.empty((4, 3), dtype=torch.int8, device=DEV), empty(4)
    B.moe_quant_rows(B.DTYPE_F32, 4, 3, 3, torch.from_numpy(v).to(DEV), codes, scales)
    wq, wsc = O.quant_rows(v)
    assert np.array_equal(codes.cpu().numpy(), wq) and np.array_equal(scales.cpu().numpy(), wsc)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n, K, N", [(1, 64, 64), (3, 128, 192), (1, 1088, 64), (2, 64, 640)])
def test_quantised_weights(dtype, n, K, N):
    r = np.random.default_rng(K + N)
    w = r.normal(size=(n, K, N)) * np.exp(r.normal(0, 1, (n, 1, N)))
    w[0, :, 3] = 0
    w[-1, 5, N - 1] = np.inf
    W = dev(w, dtype)
    codes, scales = torch.empty(n * K * N, dtype=torch.int8, device=DEV), empty(n, N)
    B.moe_quant_weight(DT[dtype], n, K, N, W, codes, scales)
    for i in range(n):
        wq, wsc = O.quant_weight(W[i].float().cpu().numpy())
        assert np.array_equal(codes.view(n, -1)[i].cpu().numpy(), wq), i
        assert np.array_equal(scales[i].cpu().numpy(), wsc, equal_nan=True)


# ---- products in 8 bits --------------------------------------------------------------------------------------------

def codes(r, *shape):
    return r.integers(-128, 128, shape).astype(np.int8)


def laid(c):
    return torch.from_numpy(O.lay_weight(c)).to(DEV)


def linear8(T, K, N, dtype, act, x, xs, w, ws, b=(None, None), res=None, y=None):
    lin = B.make_linear8(T, K, N, DT[dtype], ACT[act])
    y = empty(T, N, dtype=dtype) if y is None else y
    space = torch.full((B.moe_linear8_workspace_bytes(lin),), 77, dtype=torch.uint8, device=DEV)
    two = lambda v: (list(v) + [None])[:2]  # noqa: E731
    w, ws, b = two(w), two(ws), two(b)
    B.moe_linear8_fwd(lin, x, xs, w[0], ws[0], w[1], ws[1], b[0], b[1], res, y, space)
    return y


def linear8_tolerance(y, size, res, dtype):
    """fp32: a sum's conversion, the scales' product, theirs with the sum, the bias, the activation (erfc, exp, a quotient: up to 8 U)
    and the residual, every one U of the sizes that go in; 16 bits: activations good to 1e-6 of those, and the result's rounding."""
    size = size + (0 if res is None else np.abs(res))
    return (20 * U if dtype == "f32" else 2e-6) * size + half_step(dtype) * np.abs(y) + least(dtype)


SHAPES = [  # T, K, N
    (1, 64, 64), (1, 4096, 128), (2, 128, 192), (7, 192, 64), (15, 320, 128), (16, 64, 64), (17, 128, 128), (33, 448, 64), (48, 256, 320), (64, 1024, 64),
    (3, 16384, 64), (40, 8192, 128), (65, 64, 64), (100, 192, 128), (128, 128, 256), (129, 576, 320), (300, 1088, 192), (513, 320, 1088), (1000, 128, 64), (700, 256, 2048),
]


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T, K, N", SHAPES)
def test_products(T, K, N, dtype, act):
    r = np.random.default_rng(T + K + N)
    mats = 2 if act == "swiglu" else 1
    x, w = codes(r, T, K), [codes(r, K, N) for _ in range(mats)]
    unit = 1.0 / (74.0 * 74.0 * K ** 0.5)      # sums of random codes have this size: z of about one
    xs = np.float32(np.exp(r.normal(0, 0.5, T)))
    ws = [np.float32(unit * np.exp(r.normal(0, 0.5, N))) for _ in range(mats)]
    full = (T + N) % 3 != 0
    b = [dev(r.normal(size=N), dtype) if full else None for _ in range(mats)]
    res = dev(r.normal(size=(T, N)), dtype) if full else None
    dx, dxs, dw, dws = torch.from_numpy(x).to(DEV), dev(xs), [laid(v) for v in w], [dev(v) for v in ws]
    y = linear8(T, K, N, dtype, act, dx, dxs, dw, dws, b, res, empty(T + 1, N, dtype=dtype))
    want, size = O.linear8(x, xs, w, ws, [None if v is None else f64(v) for v in b], act, None if res is None else f64(res))
    near("y", y[:T], want, linear8_tolerance(want, size, None if res is None else f64(res), dtype))
    assert (y[T] == 12288).all()
    if full:
        linear8(T, K, N, dtype, act, dx, dxs, dw, dws, b, res, res)      # the residual's own place
        assert torch.equal(res, y[:T])


def test_a_tile_of_every_shape():
    """Sizes at which each of the tile shapes is chosen, whole and partly filled."""
    for T, K, N in ((2048, 256, 4096), (2047, 192, 4032), (8192, 128, 1024), (1500, 1024, 576), (1500, 2880, 2048), (1413, 2752, 1984), (4000, 2112, 2048)):
        r = np.random.default_rng(T)
        x, w = codes(r, T, K), codes(r, K, N)
        xs, ws = np.float32(r.random(T) + 0.5), np.float32(r.random(N) + 0.5) / K
        for dtype in ("bf16", "f32"):
            y = linear8(T, K, N, dtype, "none", torch.from_numpy(x).to(DEV), dev(xs), [laid(w)], [dev(ws)])
            want = (torch.from_numpy(x).to(DEV).double() @ torch.from_numpy(w).to(DEV).double()).cpu().numpy() * xs.astype(np.float64)[:, None] * ws.astype(np.float64)
            near("y", y, want, 4 * U * np.abs(want) + half_step(dtype) * np.abs(want))
            res = dev(r.normal(size=(T, N)), dtype)
            y = linear8(T, K, N, dtype, "none", torch.from_numpy(x).to(DEV), dev(xs), [laid(w)], [dev(ws)], res=res)
            want_r = want + f64(res)
            near("y", y, want_r, 5 * U * (np.abs(want) + np.abs(f64(res))) + half_step(dtype) * np.abs(want_r))


def test_the_longest_sums_are_exact():
    K, N = B.MAX_ROW, 64
    for T in (1, 65):
        x, w = np.full((T, K), -128, np.int8), np.full((K, N), -128, np.int8)
        w[:, 1] = 127
        w[::2, 2] = 127
        y = linear8(T, K, N, "f32", "none", torch.from_numpy(x).to(DEV), dev(np.ones(T)), [laid(w)], [dev(np.ones(N))])
        got = f64(y)
        assert (got[:, 0] == 2.0 ** 30).all() and (got[:, 1] == -128.0 * 127 * K).all() and (got[:, 2] == 64.0 * K).all()


@pytest.mark.parametrize("act", ["gelu", "swiglu"])
def test_a_row_has_the_same_bits_whatever_stands_beside_it(act):
    r = np.random.default_rng(5)
    T, K, N = 700, 704, 512
    x, w = codes(r, T, K), [codes(r, K, N) for _ in range(2 if act == "swiglu" else 1)]
    xs, ws = dev(r.random(T) + 0.5), [dev((r.random(N) + 0.5) / 1e5) for _ in w]
    dx, dw, res = torch.from_numpy(x).to(DEV), [laid(v) for v in w], dev(r.normal(size=(T, N)), "bf16")
    y = linear8(T, K, N, "bf16", act, dx, xs, dw, ws, res=res)
    for n in (1, 16, 20, 40, 64, 65, 128, 300):
        assert torch.equal(linear8(n, K, N, "bf16", act, dx[:n], xs[:n], dw, ws, res=res[:n].contiguous()), y[:n]), n


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_every_kernel_gives_a_row_the_same_bits(dtype, act):
    """Two million results, by strips, by tiles of every size and by K parts: sums just beside a border of fp16, zeros of both signs."""
    r = np.random.default_rng(6)
    T, K, N = 512, 1088, 4096
    x, w = torch.from_numpy(codes(r, T, K)).to(DEV), [torch.randint(-127, 128, (K * N,), dtype=torch.int8, device=DEV) for _ in range(2 if act == "swiglu" else 1)]
    x[5] = 0
    xs, ws = dev(r.random(T) + 0.5), [dev((r.random(N) + 0.5) * 10.0 ** r.uniform(-7, -4, N)) for _ in w]
    bits = lambda y: y.view(torch.int32 if dtype == "f32" else torch.int16)  # noqa: E731
    y = linear8(T, K, N, dtype, act, x, xs, w, ws)
    for n in (16, 32, 64, 128, 256):
        parts = torch.cat([linear8(n, K, N, dtype, act, x[i:i + n].contiguous(), xs[i:i + n].contiguous(), w, ws) for i in range(0, T, n)])
        assert torch.equal(bits(parts), bits(y)), n
    # many rows, in the other tiles, the widest last
    for n in (380, 700, 1000, 1500, 2000, 8 * T):
        rows = torch.arange(n, device=DEV) % T
        assert torch.equal(bits(linear8(n, K, N, dtype, act, x[rows], xs[rows], w, ws)), bits(y)[rows]), n


def test_a_token_that_is_no_number_stays_one():
    x, xs = torch.ones((3, 64), dtype=torch.int8, device=DEV), dev([1.0, float("nan"), 2.0])
    y = linear8(3, 64, 64, "bf16", "none", x, xs, [laid(np.ones((64, 64), np.int8))], [dev(np.ones(64))])
    assert torch.isnan(y[1]).all() and (y[0] == 64).all() and (y[2] == 128).all()


# ---- experts -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("T, E, k, d, f, cap, sliced", [(1, 1, 1, 64, 64, 0, False), (4, 16, 2, 128, 192, 0, False), (9, 256, 8, 64, 128, 0, True), (100, 4, 2, 192, 128, 40, False),
                                                         (300, 3, 2, 128, 320, 0, True), (600, 2, 1, 64, 64, 0, False), (1500, 5, 2, 192, 192, 600, True), (2000, 3, 2, 64, 128, 0, False),
                                                         (2100, 2, 2, 2048, 2048, 0, True)])
def test_experts_are_the_dense_products_of_their_rows(T, E, k, d, f, cap, sliced, act, dtype):
    r = np.random.default_rng(T + E)
    idx = np.stack([r.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    if T > 100:
        idx[r.random((T, k)) < 0.02] = -1                  # dropped assignments
    check_experts(r, idx, T, E, k, d, f, cap, sliced, act, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act", ["gelu", "swiglu"])
@pytest.mark.parametrize("f", [64, 576, 2048, 2112])
def test_one_expert_of_many_has_all_tokens(f, act, dtype):
    """Groups of sixteen rows of it and one of nine, beside experts of one row and of none, in rows up to and beyond those that the second
    product quantises by itself."""
    T, E, k = 57, 20, 2
    r = np.random.default_rng(f)
    idx = np.stack([np.full(T, 3), np.where(np.arange(T) < 9, np.arange(T) + 7, -1)], axis=1).astype(np.int32)
    check_experts(r, idx, T, E, k, 128, f, 0, False, act, dtype)


def check_experts(r, idx, T, E, k, d, f, cap, sliced, act, dtype):
    mats = 2 if act == "swiglu" else 1
    cfg = B.make_cfg(T, d, f, E, k, DT[dtype], ACT[act], cap)
    i32 = lambda n: torch.full((n,), -7, dtype=torch.int32, device=DEV)  # noqa: E731
    counts, kept, offsets, row_of, src_of = i32(E), i32(E), i32(E + 1), i32(T * k), i32(T * k)
    lo = hi = None
    if sliced:
        lo, hi = (torch.from_numpy(r.integers(a, b, E).astype(np.int32)).to(DEV) for a, b in ((-2, T // 3 + 2), (0, 2 * T)))
    ws = torch.empty(max(B.moe_workspace_bytes(cfg), B.moe_expert_ffn8_workspace_bytes(cfg)), dtype=torch.uint8, device=DEV)
    x = torch.from_numpy(codes(r, T, d)).to(DEV)
    xs = dev(r.random(T) + 0.5)
    w1 = [np.stack([codes(r, d, f) for _ in range(E)]) for _ in range(mats)]
    w2 = np.stack([codes(r, f, d) for _ in range(E)])
    lay = lambda w: torch.stack([laid(v) for v in w])  # noqa: E731
    s1, s2 = [dev((r.random((E, f)) + 0.5) / (5000 * d ** 0.5)) for _ in range(mats)], dev((r.random((E, d)) + 0.5) / (5000 * f ** 0.5))
    l1, l2 = [lay(w) for w in w1], lay(w2)
    B.moe_dispatch(cfg, None, torch.from_numpy(idx).to(DEV), lo, hi, counts, kept, offsets, row_of, src_of, None, ws)
    y = empty(T * k, d, dtype=dtype)
    two = lambda v: (list(v) + [None])[:2]  # noqa: E731
    B.moe_expert_ffn_fwd8(cfg, x, xs, l1[0], s1[0], two(l1)[1], two(s1)[1], l2, s2, src_of, offsets, kept, lo, hi, y, ws)
    want = empty(T * k, d, dtype=dtype)
    off, kp, src = offsets.cpu().numpy(), kept.cpu().numpy(), src_of.cpu().numpy()
    for e in range(E):
        a, b = 0, int(kp[e])
        if sliced:
            a, b = (min(max(int(v[e]), 0), int(kp[e])) for v in (lo, hi))
        n = b - a
        if n <= 0:
            continue
        rows = slice(off[e] + a, off[e] + b)
        tok = torch.from_numpy(src[rows] // k).to(DEV).long()
        h = linear8(n, d, f, dtype, act, x[tok].contiguous(), xs[tok].contiguous(), [l[e] for l in l1], [s[e].contiguous() for s in s1])
        hc, hs = torch.empty((n, f), dtype=torch.int8, device=DEV), empty(n)
        B.moe_quant_rows(DT[dtype], n, f, f, h, hc, hs)
        want[rows] = linear8(n, f, d, dtype, "none", hc, hs, [l2[e]], [s2[e].contiguous()])
    assert torch.equal(y, want)


# ---- beyond 32 bits ------------------------------------------------------------------------------------------------

def test_matrices_of_more_than_2_to_the_32_elements():
    """The last rows of matrices past 2^32 elements are those of the same rows by themselves."""
    rows, width = (1 << 18) + 3, 16384
    x = torch.full((rows, width), 0.5, dtype=torch.bfloat16, device=DEV)
    r = np.random.default_rng(0)
    tail = dev(r.normal(size=(3, width)), "bf16")
    x[-3:] = tail
    norm, y = B.make_norm(rows, width, B.DTYPE_BF16), torch.empty_like(x)
    B.moe_norm_fwd(norm, None, x, None, None, None, None, y, None, None)
    y3 = empty(3, width, dtype="bf16")
    B.moe_norm_fwd(B.make_norm(3, width, B.DTYPE_BF16), None, tail, None, None, None, None, y3, None, None)
    assert torch.equal(y[-3:], y3) and bool((y[1 << 17] == 1).all())
    B.moe_dropout(B.DTYPE_BF16, rows, width, B.make_drop(0.5, 3, 4), x, None, y)
    m = O.drop_mask(3, width, 0.5, 3, 4, first_row=rows - 3)
    assert np.array_equal(f64(y[-3:]), f64(tail) * m)
    q, s, q3, s3 = torch.empty((rows, width), dtype=torch.int8, device=DEV), empty(rows), torch.empty((3, width), dtype=torch.int8, device=DEV), empty(3)
    B.moe_quant_rows(B.DTYPE_BF16, rows, width, width, x, q, s)
    B.moe_quant_rows(B.DTYPE_BF16, 3, width, width, tail, q3, s3)
    assert torch.equal(q[-3:], q3) and torch.equal(s[-3:], s3)
    del x
    # a product with that many results, and rows of A past 2^32 bytes
    w, ws = codes(r, width, 64), dev(r.random(64))
    lw = [laid(w)]
    y = linear8(rows, width, 64, "bf16", "none", q, s, lw, [ws])
    assert torch.equal(y[-3:], linear8(3, width, 64, "bf16", "none", q3, s3, lw, [ws]))
    del q, y
    T, N = (1 << 18) + 5, 16384
    xs, w = codes(r, T, 64), codes(r, 64, N)
    dx, sx, lw, ws = torch.from_numpy(xs).to(DEV), dev(r.random(T)), [laid(w)], dev(r.random(N))
    y = linear8(T, 64, N, "bf16", "none", dx, sx, lw, [ws])
    assert torch.equal(y[-5:], linear8(5, 64, N, "bf16", "none", dx[-5:].contiguous(), sx[-5:].contiguous(), lw, [ws]))


@pytest.mark.parametrize("T", [3, 20, 50, 900])
def test_weights_of_more_than_the_caches_hold(T):
    """Their first columns' results, and single experts', are those of the same weights by themselves."""
    torch.manual_seed(T)
    K, N, n = 8192, 45056, 2048                       # 369 MB, requested as streaming data, and 17 MB
    any8 = lambda *s: torch.randint(-127, 128, s, dtype=torch.int8, device=DEV)  # noqa: E731
    x, xs, w, ws = any8(T, K), torch.rand(T, device=DEV), any8(N * K), torch.rand(N, device=DEV) / 5000
    y = linear8(T, K, N, "bf16", "none", x, xs, [w], [ws])
    assert torch.equal(y[:, :n], linear8(T, K, n, "bf16", "none", x, xs, [w[:n * K].clone()], [ws[:n].clone()]))
    for act in ("swiglu", "gelu"):
        E, k, d, f = 64, 2, 2048, 1024
        if act == "gelu":
            f = 1536                                  # 403 MB either way
        cfg = B.make_cfg(T, d, f, E, k, B.DTYPE_BF16, ACT[act])
        idx = torch.rand(T, E, device=DEV).topk(k).indices.int().contiguous()
        i32 = lambda m: torch.empty(m, dtype=torch.int32, device=DEV)  # noqa: E731
        counts, kept, offsets, row_of, src_of = i32(E), i32(E), i32(E + 1), i32(T * k), i32(T * k)
        room = torch.empty(max(B.moe_workspace_bytes(cfg), B.moe_expert_ffn8_workspace_bytes(cfg)), dtype=torch.uint8, device=DEV)
        B.moe_dispatch(cfg, None, idx, None, None, counts, kept, offsets, row_of, src_of, None, room)
        w1 = [any8(E, d * f) for _ in range(2 if act == "swiglu" else 1)]
        s1, w2, s2 = [torch.rand(E, f, device=DEV) / 20000 for _ in w1], any8(E, f * d), torch.rand(E, d, device=DEV) / 20000
        y = empty(T * k, d, dtype="bf16")
        B.moe_expert_ffn_fwd8(cfg, x[:, :d].contiguous(), xs, w1[0], s1[0], w1[1] if len(w1) > 1 else None, s1[1] if len(w1) > 1 else None, w2, s2, src_of, offsets, kept, None, None, y, room)
        off = offsets.tolist()
        for e in range(E):
            n_rows = off[e + 1] - off[e]
            if n_rows == 0:
                continue
            tok = (src_of[off[e]:off[e + 1]] // k).long()
            h = linear8(n_rows, d, f, "bf16", act, x[tok, :d].contiguous(), xs[tok].contiguous(), [v[e].clone() for v in w1], [v[e].clone() for v in s1])
            hc, hs = torch.empty((n_rows, f), dtype=torch.int8, device=DEV), empty(n_rows)
            B.moe_quant_rows(B.DTYPE_BF16, n_rows, f, f, h, hc, hs)
            assert torch.equal(y[off[e]:off[e + 1]], linear8(n_rows, f, d, "bf16", "none", hc, hs, [w2[e].clone()], [s2[e].clone()])), e


def test_calls_on_two_streams_at_once():
    """Calls with buffers of their own do not see each other."""
    r = np.random.default_rng(7)
    T, K, N = 100, 8192, 256
    x, w = codes(r, T, K), codes(r, K, N)
    xs, ws = dev(r.random(T) / K), dev(r.random(N))
    dx, lw = torch.from_numpy(x).to(DEV), [laid(w)]
    want = linear8(T, K, N, "bf16", "none", dx, xs, lw, [ws])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(linear8(T, K, N, "bf16", "none", dx, xs, lw, [ws]))
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g, want)
