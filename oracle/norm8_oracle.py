"""CPU oracle of the norm with its residual, dropout, and products in 8-bit integers (numpy, double precision but where a definition
is one of single precision).  Shares no code with the library."""
from __future__ import annotations

import numpy as np

from oracle.operators_oracle import act as activate

LOW = np.uint64(0xFFFFFFFF)


def philox(c0, c1, c2, c3, k0, k1):
    """Philox 4x32 with ten rounds on arrays of 32-bit words (as uint64)."""
    c = [np.asarray(v, dtype=np.uint64) for v in np.broadcast_arrays(c0, c1, c2, c3)]
    k0, k1 = int(k0), int(k1)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & LOW, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def drop_cut(p):
    return min(65535, int(np.floor(float(np.float32(p)) * 65536 + 0.5)))


def drop_mask(rows, width, p, seed, offset, first_row=0):
    """What every element is multiplied by."""
    cut = drop_cut(p)
    groups = np.arange((width + 7) // 8, dtype=np.uint64)[None, :]
    r = np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None]
    words = philox(groups, r, np.uint64(offset & 0xFFFFFFFF), np.uint64((offset >> 32) & 0xFFFFFFFF), seed & 0xFFFFFFFF, seed >> 32)
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2).reshape(rows, -1)[:, :width]
    return np.where(bits >= cut, 65536.0 / (65536 - cut), 0.0)


def norm_fwd(h, gamma, eps):
    """(y, rstd) of h as it is stored."""
    rstd = 1 / np.sqrt((h * h).mean(axis=1) + eps)
    return h * rstd[:, None] * gamma, rstd


def norm_bwd(dy, h, gamma, eps, dh_add):
    """(dh, dgamma)."""
    rstd = (1 / np.sqrt((h * h).mean(axis=1) + eps))[:, None]
    u, a = h * rstd, gamma * dy
    return rstd * (a - u * (a * u).mean(axis=1, keepdims=True)) + dh_add, (dy * u).sum(axis=0)


def quant_rows(v):
    """(codes int8, scales fp32) of the rows of an fp32 array."""
    v = np.asarray(v, dtype=np.float32)
    top = np.abs(v).max(axis=1)
    bad = ~np.isfinite(top)
    with np.errstate(invalid="ignore", over="ignore"):
        m = np.maximum(np.where(bad, np.float32(1), top), np.float32(2.0 ** -100)).astype(np.float32)
        up = np.float32(127) / m
        codes = np.rint(np.where(bad[:, None], np.float32(0), v) * up[:, None])
    return codes.astype(np.int8), np.where(bad, np.float32(np.nan), m * np.float32(1 / 127)).astype(np.float32)


def lay_weight(codes):
    """The bytes of a matrix [d_in, d_out] in the order in which the products read them, by the formula of the interface."""
    K, N = codes.shape
    r, c = np.meshgrid(np.arange(K), np.arange(N), indexing="ij")
    at = ((c // 16) * (K // 64) + r // 64) * 1024 + (r % 64 // 16) * 256 + (c % 16) * 16 + r % 16
    out = np.empty(K * N, dtype=np.int8)
    out[at.reshape(-1)] = codes.reshape(-1)
    return out


def quant_weight(w):
    """(bytes, scales) of a matrix [d_in, d_out]."""
    codes, scales = quant_rows(np.ascontiguousarray(np.asarray(w, dtype=np.float32).T))
    return lay_weight(codes.T), scales


def linear8(x, xs, w, ws, bias, act, residual):
    """w, ws, bias: lists of one or two.  Sums are whole numbers; also returns the size of what was added up, for tolerances."""
    z, size = [], 1.0
    for W, s, b in zip(w, ws, bias):
        v = (x.astype(np.int64) @ W.astype(np.int64)).astype(np.float64) * np.asarray(xs, np.float64)[:, None] * np.asarray(s, np.float64)[None, :]
        b = np.zeros(W.shape[1]) if b is None else b
        z.append(v + b)
        size = size * (np.abs(v) + np.abs(b))
    y = activate(z, act)
    return y if residual is None else y + residual, size
