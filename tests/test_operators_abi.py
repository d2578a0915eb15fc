"""Argument checks of scored routing, 8-bit activations and dense products: refused before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2504_03871_amd import binding as B

P, Q = 0x10000, 0x10008       # aligned / misaligned addresses that are never dereferenced
S = ctypes.c_void_p(0)


def refused(code, fn, *a, **kw):
    with pytest.raises(B.MoeError) as ei:
        fn(*a, **kw)
    assert ei.value.code == code, (ei.value, code)


def score(**kw):
    return B.make_score(**{**dict(score=B.SCORE_SIGMOID, groups=4, top_groups=2, group_rank=2, renorm=1, scale=1.0), **kw})


def test_scored_routing_refusals():
    cfg = B.make_cfg(8, 64, 128, 16, 4)
    fwd = lambda sc, c=cfg, x=None, logits=P, idx=P, ws=None, **kw: B.moe_route_scored(c, sc, x, None, None, None, logits, None, idx, P, ws, stream=S, **kw)  # noqa: E731
    for bad in (dict(groups=0), dict(groups=3), dict(groups=17), dict(top_groups=0), dict(top_groups=5), dict(group_rank=0), dict(group_rank=3),
                dict(groups=16, top_groups=16), dict(groups=8, top_groups=1), dict(scale=float("nan")), dict(scale=float("inf"))):
        refused(-2, fwd, score(**bad))
    refused(-3, fwd, score(score=2))
    refused(-1, fwd, score(), logits=None)                     # neither logits nor x
    refused(-1, fwd, score(), idx=None)
    refused(-5, fwd, score(), idx=Q)
    refused(-5, fwd, score(), logits=Q)
    refused(-7, fwd, score(), ws=P, ws_bytes=16)
    refused(-2, fwd, score(), c=B.make_cfg(8, 64, 128, 16, 17))
    bwd = lambda **kw: B.moe_route_scored_bwd(cfg, score(), *[kw.get(n, d) for n, d in (  # noqa: E731
        ("x", None), ("Wr", None), ("logits", P), ("idx", P), ("dw", P), ("dl", P), ("dWr", None), ("dx", None), ("ws", None))], stream=S)
    for missing in ("logits", "idx", "dw", "dl"):
        refused(-1, bwd, **{missing: None})
    refused(-1, bwd, dWr=P, ws=P)            # the weight gradient needs x
    refused(-1, bwd, dWr=P, x=P)             # and a workspace
    refused(-1, bwd, dx=P, ws=P)             # the input gradient needs Wr
    refused(-5, bwd, dl=Q)


def test_pack8_refusals_and_sizes():
    assert B.moe_pack8_bytes(3, 33) == (3 * 64, 3 * 2)
    assert B.moe_pack8_bytes(0, 1) == (0, 0)
    assert B.moe_pack8_bytes(1 << 30, 64) == (1 << 36, 1 << 31)
    for rows, width in ((-1, 4), (4, 0), (1 << 40, 64)):
        refused(-2, B.moe_pack8_bytes, rows, width)
    pack = lambda dt=B.DTYPE_BF16, fmt=B.PACK_I8, rows=4, width=40, pitch=40, src=P, codes=P, sc=P: B.moe_pack8(dt, fmt, rows, width, pitch, src, codes, sc, stream=S)  # noqa: E731
    unpack = lambda dt=B.DTYPE_BF16, fmt=B.PACK_I8, rows=4, width=40, pitch=40, dst=P, codes=P, sc=P: B.moe_unpack8(dt, fmt, rows, width, pitch, codes, sc, dst, stream=S)  # noqa: E731
    for f in (pack, unpack):
        refused(-3, f, dt=3)
        refused(-3, f, fmt=B.PACK_NONE)
        refused(-3, f, fmt=3)
        refused(-2, f, pitch=39)
        refused(-2, f, rows=-1)
        refused(-1, f, codes=None)
        refused(-1, f, sc=None)
        refused(-5, f, codes=Q)
        f(rows=0, codes=None)                # nothing to do
    refused(-1, pack, src=None)
    refused(-5, pack, src=Q)
    refused(-1, unpack, dst=None)


def test_saved8_refusals_and_sizes():
    cfg = B.make_cfg(8, 64, 128, 4, 2)
    assert B.moe_saved_pack8_bytes(cfg) == (16 * 128, 16 * 4)
    assert B.moe_saved_pack8_bytes(B.make_cfg(8, 64, 100, 4, 2, B.DTYPE_F32, B.ACT_SWIGLU)) == (2 * 16 * 128, 2 * 16 * 4)
    for f in (lambda fmt=B.PACK_I8, a=P, o=P, lo=None, c=P: B.moe_saved_pack8(cfg, fmt, a, o, P, lo, None, c, P, stream=S),
              lambda fmt=B.PACK_I8, a=P, o=P, lo=None, c=P: B.moe_saved_restore8(cfg, fmt, c, P, o, P, lo, None, a, stream=S)):
        refused(-3, f, fmt=0)
        refused(-4, f, lo=P)
        refused(-1, f, o=None)
        refused(-1, f, a=None)
        refused(-5, f, c=Q)


def test_linear_refusals():
    ok = dict(T=8, d_in=64, d_out=128, dtype=B.DTYPE_BF16, act=B.ACT_GELU)
    assert B.moe_linear_workspace_bytes(B.make_linear(**ok)) > 0
    for bad in (dict(T=-1), dict(T=(1 << 24) + 1), dict(d_in=72), dict(d_out=100), dict(d_in=0), dict(d_in=32768, d_out=32768)):
        refused(-2, B.moe_linear_workspace_bytes, B.make_linear(**{**ok, **bad}))
    for bad in (dict(dtype=3), dict(act=3), dict(pre=3), dict(grad=B.DTYPE_F16)):
        refused(-3, B.moe_linear_workspace_bytes, B.make_linear(**{**ok, **bad}))
    B.moe_linear_workspace_bytes(B.make_linear(**{**ok, "dtype": B.DTYPE_F32, "d_in": 68, "d_out": 100}))
    big = 1 << 40

    def fwd(act=B.ACT_GELU, x=P, W=P, Wb=None, b=None, bb=None, r=None, pre=None, preb=None, y=P, ws=P, n=big):
        B.moe_linear_fwd(B.make_linear(**{**ok, "act": act}), x, W, Wb, b, bb, r, pre, preb, y, ws, stream=S, ws_bytes=n)
    for missing in ("x", "W", "y", "ws"):
        refused(-1, fwd, **{missing: None})
    refused(-7, fwd, n=16)
    refused(-3, fwd, Wb=P)                                   # a second matrix without SwiGLU
    refused(-3, fwd, bb=P)
    refused(-3, fwd, act=B.ACT_NONE, pre=P)                  # nothing to keep
    refused(-1, fwd, act=B.ACT_SWIGLU)                       # SwiGLU without its second matrix
    refused(-1, fwd, act=B.ACT_SWIGLU, Wb=P, pre=P)          # one pre-activation plane of two
    for odd in ("x", "W", "b", "r", "pre", "y", "ws"):
        refused(-5, fwd, **{odd: Q})

    def bwd(act=B.ACT_GELU, pk=B.PACK_NONE, grad=B.DTYPE_F32, dy=P, x=P, W=P, Wb=None, pre=P, preb=None, sc=None, scb=None, add=None, dx=P, dW=P,
            dWb=None, db=P, dbb=None, acc=0, ws=P, n=big):
        B.moe_linear_bwd(B.make_linear(**{**ok, "act": act}, pre=pk, grad=grad), dy, x, W, Wb, pre, preb, sc, scb, add, dx, dW, dWb, db, dbb, acc, ws,
                         stream=S, ws_bytes=n)
    for missing in ("dy", "x", "W", "pre", "ws"):
        refused(-1, bwd, **{missing: None})
    refused(-1, bwd, pk=B.PACK_I8)                           # packed without scales
    refused(-1, bwd, act=B.ACT_SWIGLU, Wb=P, preb=P, dbb=P)  # one weight gradient of two
    refused(-1, bwd, act=B.ACT_SWIGLU, preb=P, dWb=P, dbb=P)
    refused(-3, bwd, dWb=P)
    refused(-3, bwd, grad=B.DTYPE_BF16, acc=1)               # sums over calls are kept in fp32
    refused(-7, bwd, n=16)
    for odd in ("dy", "x", "pre", "add", "dx", "dW", "db"):
        refused(-5, bwd, **{odd: Q})


def test_linear_workspace_covers_every_cut():
    """The plan's regions for sizes around its lines: sizes grow with T and no call asks for more than a few times its tensors."""
    for dtype in (B.DTYPE_BF16, B.DTYPE_F32):
        for act in (B.ACT_NONE, B.ACT_GELU, B.ACT_SWIGLU):
            for T in (1, 63, 64, 65, 160, 161, 511, 512, 513, 4096, 100000):
                n = B.moe_linear_workspace_bytes(B.make_linear(T, 256, 512, dtype, act))
                assert 0 < n < (1 << 30) + 16 * T * 512 * 4, (T, n)


def test_linear_widths_keep_a_tile_below_32_bits():
    """256 rows of 2^20 16-bit values are half a GiB; twice as wide a row and its tile's gradient sums would need offsets past 2^31."""
    for dtype, d in ((B.DTYPE_BF16, 64), (B.DTYPE_F32, 4)):
        wide = 1 << 20
        assert B.moe_linear_workspace_bytes(B.make_linear(256, d, wide, dtype, B.ACT_GELU)) > 0
        assert B.moe_linear_workspace_bytes(B.make_linear(256, wide, d, dtype, B.ACT_GELU)) > 0
        refused(-2, B.moe_linear_workspace_bytes, B.make_linear(256, d, wide + 64, dtype, B.ACT_GELU))
        refused(-2, B.moe_linear_workspace_bytes, B.make_linear(256, wide + 64, d, dtype, B.ACT_GELU))


def test_linear_forward_needs_its_own_workspace_only():
    """Inference brings room for the sums of K parts, none for gradients: 1.9 GB of dz at 32768 x 14336 SwiGLU are the backward's."""
    lin = B.make_linear(32768, 4096, 14336, B.DTYPE_BF16, B.ACT_SWIGLU)
    assert B.moe_linear_workspace_bytes(lin) > 2 * 32768 * 14336 * 2
    assert B.moe_linear_fwd_workspace_bytes(lin) < 256 << 20
    for dtype in (B.DTYPE_F32, B.DTYPE_BF16, B.DTYPE_F16):
        for act in (B.ACT_NONE, B.ACT_GELU, B.ACT_SWIGLU):
            for T, d, n in ((0, 64, 64), (1, 64, 64), (1, 4096, 1024), (64, 2048, 256), (300, 1024, 192), (4096, 256, 512), (100000, 64, 128)):
                lin = B.make_linear(T, d, n, dtype, act)
                need, both = B.moe_linear_fwd_workspace_bytes(lin), B.moe_linear_workspace_bytes(lin)
                assert need % 256 == 0 and (need >= 256 or T == 0) and need <= both
                if T == 0:
                    continue
                Wb = P if act == B.ACT_SWIGLU else None
                refused(-7, B.moe_linear_fwd, lin, P, P, Wb, None, None, None, None, None, P, P, stream=S, ws_bytes=need - 1)
                refused(-7, B.moe_linear_bwd, lin, P, P, P, Wb, P, Wb, None, None, None, P, P, Wb, P, Wb, 0, P, stream=S, ws_bytes=both - 1)


def test_packed_matrices_are_as_large_as_the_call_says():
    """A tensor with fewer rows, narrower ones or smaller elements than `rows`, `pitch` and `dtype` say would be read past its end."""
    torch = pytest.importorskip("torch")
    whole = torch.zeros(8, 64, dtype=torch.bfloat16)
    for t, rows, width, pitch, dt in ((whole[:, :40].contiguous(), 8, 40, 64, B.DTYPE_BF16), (whole, 9, 64, 64, B.DTYPE_BF16), (whole[:, :40], 9, 40, 64, B.DTYPE_BF16),
                                      (whole, 8, 64, 64, B.DTYPE_F32), (whole.view(-1)[:500], 8, 60, 64, B.DTYPE_BF16), (whole[:, :40], 8, 40, 64, B.DTYPE_F32)):
        with pytest.raises(ValueError):
            B.moe_pack8(dt, B.PACK_I8, rows, width, pitch, t, P, P, stream=S)
        with pytest.raises(ValueError):
            B.moe_unpack8(dt, B.PACK_I8, rows, width, pitch, P, P, t, stream=S)
    for t, rows, width, pitch in ((whole, 8, 64, 64), (whole[:, :40], 8, 40, 64), (whole[:, :40], 3, 40, 64), (whole, 8, 40, 64), (whole.view(-1)[:488], 8, 40, 64)):
        assert B._rows_ptr(t, B.DTYPE_BF16, rows, width, pitch) == whole.data_ptr()
