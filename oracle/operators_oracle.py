"""CPU oracle (numpy, 64 bits) of the operators beside the expert layer: scored routing, dense products with an epilogue,
activations in 8 bits.  Written from the definitions in include/moe.h; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

try:
    from scipy.special import erfc as _erfc
except ImportError:   # pragma: no cover
    _erfc = np.vectorize(math.erfc)


# ---- scored routing ------------------------------------------------------------------------------------------------

def scores(logits, kind):
    """[T, E] scores; experts that cannot be chosen (-inf, NaN) have none."""
    l = np.asarray(logits, dtype=np.float64).copy()
    shut = ~(l > -np.inf)
    l[np.isposinf(l)] = np.finfo(np.float32).max
    l[shut] = -np.inf
    if kind == "softmax":
        top = l.max(axis=1, keepdims=True)
        with np.errstate(invalid="ignore"):
            ex = np.where(shut, 0.0, np.exp(l - np.where(np.isfinite(top), top, 0.0)))
        z = ex.sum(axis=1, keepdims=True)
        return np.where(z > 0, ex / np.where(z > 0, z, 1.0), 0.0), l
    with np.errstate(over="ignore"):
        return np.where(shut, 0.0, 1.0 / (1.0 + np.exp(-np.where(shut, 0.0, l)))), l


def route(logits, kind, k, balance=None, groups=1, top_groups=1, rank=1, renorm=True, scale=1.0):
    """(idx [T, k], w [T, k]) row by row, from the definition."""
    s, l = scores(logits, kind)
    T, E = s.shape
    idx, w = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    size = E // groups
    for t in range(T):
        # without a bias the scores grow with the logits: the logits order the experts, also where scores round to the same number
        by_logit = balance is None and (groups == 1 or rank == 1)
        key = l[t].copy() if by_logit else s[t] + (0.0 if balance is None else np.minimum(np.asarray(balance, dtype=np.float64), np.finfo(np.float32).max))
        key[~(l[t] > -np.inf)] = -np.inf
        key[np.isnan(key)] = -np.inf
        if groups > 1:
            g = [sum(sorted(key[i * size:(i + 1) * size], reverse=True)[:rank]) for i in range(groups)]
            best = sorted(range(groups), key=lambda i: (-g[i], i))[:top_groups]
            for i in range(groups):
                if i not in best:
                    key[i * size:(i + 1) * size] = -np.inf
        order = [e for e in sorted(range(E), key=lambda e: (-key[e], e)) if key[e] > -np.inf][:k]
        idx[t, :len(order)] = order
        w[t] = weights(l[t], s[t], idx[t], kind, renorm) * scale
    return idx, w


def weights(l, s, idx, kind, renorm):
    """Weights of one token's slots before the scale, from log scores so that ratios of tiny scores survive."""
    p = np.zeros(len(idx))
    live = idx >= 0
    if not live.any():
        return p
    e = idx[live]
    if not renorm:
        p[live] = s[e]
        return p
    log = l[e] if kind == "softmax" else -np.logaddexp(0.0, -l[e])
    q = np.exp(log - log.max())
    p[live] = q / q.sum()
    return p


def route_bwd(logits, kind, idx, dw, renorm=True, scale=1.0):
    s, l = scores(logits, kind)
    out = np.zeros_like(s)
    for t in range(s.shape[0]):
        live = [j for j, e in enumerate(idx[t]) if 0 <= e < s.shape[1] and l[t, e] > -np.inf]
        e = idx[t][live]
        ids = np.full(len(idx[t]), -1)
        ids[live] = e
        p = weights(l[t], s[t], ids, kind, renorm)[live]
        g = np.asarray(dw[t], dtype=np.float64)[live]
        D = (p * g).sum()
        if kind == "softmax" and not renorm:
            out[t] = -scale * s[t] * D
            out[t, e] += scale * p * g
        else:
            out[t, e] = scale * p * (g - D if renorm else g)
            if kind == "sigmoid":
                out[t, e] *= np.exp(-np.logaddexp(0.0, l[t, e]))
    return out


# ---- 8 bits ----------------------------------------------------------------------------------------------------------

E4M3 = sorted({m * 2.0 ** -9 for m in range(8)} | {(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if not (e == 15 and m == 7)})


def _codes(q, fmt):
    """Nearest element of every value, ties to the even code: (bytes, values)."""
    q = np.asarray(q, dtype=np.float64)
    if fmt == "i8":
        c = np.clip(np.rint(q * 64), -127, 127)
        return c.astype(np.int64).astype(np.int8).view(np.uint8), c / 64
    grid = np.array(E4M3)
    a = np.abs(q)
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    lo = hi - 1
    d_lo, d_hi = a - grid[lo], grid[hi] - a
    pick = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    return (pick + np.where(np.signbit(q), 128, 0)).astype(np.uint8), np.where(np.signbit(q), -1.0, 1.0) * grid[pick]


def pack(v, fmt):
    """(codes [rows, blocks * 32], scales [rows, blocks], values [rows, width] before the clamp) of a matrix."""
    v = np.asarray(v, dtype=np.float64)
    rows, width = v.shape
    nb = -(-width // 32)
    u = np.zeros((rows, nb * 32))
    u[:, :width] = v
    u = u.reshape(rows, nb, 32)
    codes, scales, vals = np.zeros((rows, nb, 32), np.uint8), np.zeros((rows, nb), np.uint8), np.zeros((rows, nb, 32))
    largest = 448.0 if fmt == "e4m3" else 127.5 / 64
    for r in range(rows):
        for b in range(nb):
            m = np.abs(u[r, b]).max()
            if not np.isfinite(m):
                scales[r, b], vals[r, b] = 255, np.nan
                continue
            e = -127
            if m > 0:
                e = max(-127, math.frexp(m)[1] - 1 - (8 if fmt == "e4m3" else 0))
                if m > largest * 2.0 ** e or (fmt == "i8" and m == largest * 2.0 ** e):
                    e += 1
                e = min(e, 127)
            codes[r, b], q = _codes(u[r, b] * 2.0 ** -e, fmt)
            scales[r, b], vals[r, b] = e + 127, q * 2.0 ** e
    return codes.reshape(rows, -1), scales, vals.reshape(rows, -1)[:, :width]


# ---- dense products ----------------------------------------------------------------------------------------------------

def act(z, kind):
    if kind == "gelu":
        return 0.5 * z[0] * _erfc(-z[0] / math.sqrt(2))
    if kind == "swiglu":
        return z[0] / (1 + np.exp(-z[0])) * z[1]
    return z[0]


def act_slopes(z, kind):
    """d act / d z of every product."""
    if kind == "gelu":
        return [0.5 * _erfc(-z[0] / math.sqrt(2)) + z[0] * np.exp(-0.5 * z[0] ** 2) / math.sqrt(2 * math.pi)]
    if kind == "swiglu":
        sg = 1 / (1 + np.exp(-z[0]))
        return [z[1] * sg * (1 + z[0] * (1 - sg)), z[0] * sg]
    return [np.ones_like(z[0])]
