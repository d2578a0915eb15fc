"""Argument checks of the norm, dropout and the products in 8 bits: refused before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2504_03871_amd import binding as B

P, Q = 0x10000, 0x10008       # aligned / misaligned addresses that are never dereferenced
S = ctypes.c_void_p(0)
BIG = 1 << 40


def refused(code, fn, *a, **kw):
    with pytest.raises(B.MoeError) as ei:
        fn(*a, **kw)
    assert ei.value.code == code, (ei.value, code)


def test_dropout_refusals():
    def call(dt=B.DTYPE_BF16, rows=4, width=8, drop=B.make_drop(0.1, 1), x=P, r=None, y=P):
        B.moe_dropout(dt, rows, width, drop, x, r, y, stream=S)
    refused(-3, call, dt=3)
    refused(-1, call, drop=None)
    for p in (-0.1, 1.0, float("nan"), 2.0):
        refused(-2, call, drop=B.make_drop(p, 1))
    refused(-5, call, drop=B.make_drop(0.1, 1, 0, 0x10004))
    for bad in (dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=(1 << 20) + 1), dict(rows=1 << 30, width=64)):
        refused(-2, call, **bad)
    refused(-1, call, x=None)
    refused(-1, call, y=None)
    for odd in ("x", "r", "y"):
        refused(-5, call, **{odd: Q})
    call(rows=0, x=None, y=None)


def test_drop_step_must_lie_on_the_gpu():
    import torch
    with pytest.raises(ValueError):
        B.make_drop(0.1, 1, 0, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        B.make_drop(0.1, 1, 0, torch.zeros(1, dtype=torch.int32))


OK = dict(T=8, d=64, dtype=B.DTYPE_BF16)


def test_norm_refusals():
    assert B.moe_norm_bwd_workspace_bytes(B.make_norm(**OK)) >= 64 * 4
    for bad in (dict(T=-1), dict(T=(1 << 24) + 1), dict(d=0), dict(d=B.MAX_NORM + 1), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=-1.0)):
        refused(-2, B.moe_norm_bwd_workspace_bytes, B.make_norm(**{**OK, **bad}))
    for bad in (dict(dtype=3), dict(stream=B.DTYPE_F16), dict(grad=B.DTYPE_F16), dict(dtype=B.DTYPE_F32, stream=B.DTYPE_BF16)):
        refused(-3, B.moe_norm_bwd_workspace_bytes, B.make_norm(**{**OK, **bad}))

    def fwd(drop=None, x=P, r=P, g=P, h=P, rs=P, y=2 * P, c=None, s=None, **kw):
        B.moe_norm_fwd(B.make_norm(**{**OK, **kw}), drop, x, r, g, h, rs, y, c, s, stream=S)
    refused(-1, fwd, x=None)
    refused(-1, fwd, y=None)
    refused(-1, fwd, c=P)
    refused(-1, fwd, s=P)
    refused(-2, fwd, drop=B.make_drop(1.0, 1))
    refused(-8, fwd, y=P)
    for odd in ("x", "r", "g", "h", "rs", "y"):
        refused(-5, fwd, **{odd: Q})
    refused(-5, fwd, c=Q, s=P)
    fwd(T=0, x=None, y=None)

    def bwd(drop=None, dy=P, h=P, g=P, rs=P, add=None, dh=P, dx=None, dg=P, acc=0, ws=P, n=BIG, **kw):
        B.moe_norm_bwd(B.make_norm(**{**OK, **kw}), drop, dy, h, g, rs, add, dh, dx, dg, acc, ws, stream=S, ws_bytes=n)
    for missing in ("dy", "h", "rs", "ws"):
        refused(-1, bwd, **{missing: None})
    refused(-7, bwd, n=16)
    refused(-8, bwd, dx=P)
    refused(-3, bwd, grad=B.DTYPE_BF16, acc=1)
    refused(-2, bwd, drop=B.make_drop(-1, 1))
    for odd in ("dy", "h", "g", "rs", "add", "dh", "dx", "dg", "ws"):
        refused(-5, bwd, **{odd: Q})
    bwd(dh=None, dg=None, ws=None)        # nothing asked for


def test_norm_workspace_is_a_row_for_each_block():
    for d in (1, 7, 64, 516, 1024, 4096, 8192, 16384, 16383):
        last = 0
        for T in (1, 3, 100, 1000, 5000, 100000, 1 << 24):
            n = B.moe_norm_bwd_workspace_bytes(B.make_norm(T, d))
            assert last <= n <= 1024 * d * 4 + 256 and n >= min(T, 4) // 4 * d * 4
            last = n


def test_quantising_refusals():
    def rows(dt=B.DTYPE_BF16, n=4, width=40, pitch=40, src=P, c=P, s=P):
        B.moe_quant_rows(dt, n, width, pitch, src, c, s, stream=S)
    refused(-3, rows, dt=3)
    for bad in (dict(n=-1), dict(width=0), dict(pitch=39), dict(width=B.MAX_ROW + 1, pitch=B.MAX_ROW + 1), dict(n=1 << 36), dict(pitch=1 << 41)):
        refused(-2, rows, **bad)
    for missing in ("src", "c", "s"):
        refused(-1, rows, **{missing: None})
        refused(-5, rows, **{missing: Q})
    rows(n=0, src=None)

    def weight(dt=B.DTYPE_BF16, n=2, K=64, N=128, W=P, c=P, s=P):
        B.moe_quant_weight(dt, n, K, N, W, c, s, stream=S)
    refused(-3, weight, dt=3)
    for bad in (dict(n=-1), dict(n=65536), dict(K=0), dict(K=96), dict(N=72), dict(K=1 << 16, N=1 << 15)):
        refused(-2, weight, **bad)
    for missing in ("W", "c", "s"):
        refused(-1, weight, **{missing: None})
        refused(-5, weight, **{missing: Q})
    weight(n=0, W=None)


def test_linear8_refusals():
    ok = dict(T=8, d_in=64, d_out=128, dtype=B.DTYPE_BF16, act=B.ACT_GELU)
    assert B.moe_linear8_workspace_bytes(B.make_linear8(**{**ok, "T": 0})) == 0
    for bad in (dict(T=-1), dict(T=(1 << 24) + 1), dict(d_in=96), dict(d_out=100), dict(d_in=0), dict(d_in=B.MAX_ROW + 64), dict(d_in=1 << 16, d_out=1 << 15)):
        refused(-2, B.moe_linear8_workspace_bytes, B.make_linear8(**{**ok, **bad}))
    for bad in (dict(dtype=3), dict(act=3)):
        refused(-3, B.moe_linear8_workspace_bytes, B.make_linear8(**{**ok, **bad}))

    def fwd(act=B.ACT_GELU, x=P, xs=P, W=P, w=P, Wb=None, wb=None, b=None, bb=None, r=None, y=P, ws=P, n=BIG, **kw):
        B.moe_linear8_fwd(B.make_linear8(**{**ok, "act": act, **kw}), x, xs, W, w, Wb, wb, b, bb, r, y, ws, stream=S, ws_bytes=n)
    for missing in ("x", "xs", "W", "w", "y"):
        refused(-1, fwd, **{missing: None})
    refused(-1, fwd, T=100, ws=None)                 # sums of K parts need room, those of few rows none
    refused(-7, fwd, T=100, n=16)
    for extra in ("Wb", "wb", "bb"):
        refused(-3, fwd, **{extra: P})
    refused(-1, fwd, act=B.ACT_SWIGLU)
    refused(-1, fwd, act=B.ACT_SWIGLU, Wb=P)
    for odd in ("x", "xs", "W", "w", "b", "r", "y", "ws"):
        refused(-5, fwd, **{odd: Q})
    fwd(T=0, x=None)


def test_linear8_workspace_does_for_smaller_calls_too():
    for act in (B.ACT_NONE, B.ACT_SWIGLU):
        for K in (64, 16384, 65536):
            for N in (64, 256, 4096, 16384):
                last = 0
                for T in (0, 1, 15, 32, 33, 64, 65, 513, 5000, 1 << 20):
                    n = B.moe_linear8_workspace_bytes(B.make_linear8(T, K, N, B.DTYPE_BF16, act))
                    assert last <= n <= 512 * 128 * 128 * 4 and (n == 0) == (T <= 32)
                    last = n


def test_expert_ffn8_refusals():
    ok = dict(T=8, d_model=64, d_ff=128, E=4, k=2, dtype=B.DTYPE_BF16, act=B.ACT_SWIGLU)
    n = B.moe_expert_ffn8_workspace_bytes(B.make_cfg(**ok))
    assert n >= 16 * 128 * 3 + 16 * 4
    refused(-3, B.moe_expert_ffn8_workspace_bytes, B.make_cfg(**{**ok, "dtype": B.DTYPE_F32}))
    refused(-2, B.moe_expert_ffn8_workspace_bytes, B.make_cfg(**{**ok, "d_ff": B.MAX_ROW + 64}))
    refused(-2, B.moe_expert_ffn8_workspace_bytes, B.make_cfg(**{**ok, "d_model": 72}))

    def fwd(act=B.ACT_SWIGLU, x=P, xs=P, W1=P, s1=P, W1b=P, s1b=P, W2=P, s2=P, src=P, off=P, kept=P, lo=None, hi=None, y=P, ws=P, m=BIG):
        B.moe_expert_ffn_fwd8(B.make_cfg(**{**ok, "act": act}), x, xs, W1, s1, W1b, s1b, W2, s2, src, off, kept, lo, hi, y, ws, stream=S, ws_bytes=m)
    for missing in ("x", "xs", "W1", "s1", "W1b", "s1b", "W2", "s2", "src", "off", "kept", "y", "ws"):
        refused(-1, fwd, **{missing: None})
        refused(-5, fwd, **{missing: Q})
    refused(-3, fwd, act=B.ACT_GELU)
    refused(-4, fwd, lo=P)
    refused(-7, fwd, m=n - 1)
