"""Cases of the operators around the expert layer: the norm in front of it, dropout on its output, and its products in 8-bit integers.

A case is a dict of plain values with an "op":
  norm     h = residual + dropout(x), y = gamma h / rms(h); `bwd`: then the gradients of h, of x and of gamma.
           T d dtype, stream (type of the residual stream: residual, h and their gradients), p (0: no dropout), residual, bwd
  dropout  y = residual + dropout(x); `bwd`: the gradient of x too, its mask computed anew.  T d dtype p residual bwd
  linear8  y = act(x W + b) + r with W in 8 bits and a scale for each column; x is quantised first, a scale for each token.
           T d n dtype act bias residual
  mlp8     a shared expert as it answers requests: norm of residual + x straight to 8 bits, up-projection, its output to 8 bits,
           down-projection with the residual stream added.  T d n dtype act
  experts8 the routed experts of a layer as they answer requests: tokens to 8 bits, dispatch, both products in 8 bits, combine.
           T E k d f dtype act

Quantising a row (or a column of weights): m = max(largest magnitude, 2^-100), codes round(v * (127 / m)), ties to even, scale m / 127.
Dropout drops an element where 16 bits of a counter generator (Philox 4x32 with ten rounds: key = seed, counter = column / 8, row, offset;
the column's remainder picks half a word) are below round(65536 p), and multiplies the others by 65536 / (65536 - that).

The plain forms below are torch operations in 32 bits.  What an operator stores in between for the next one has the type it is stored in.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def _norm(T, d, dtype="bf16", stream=None, p=0.0, residual=True, bwd=True):
    return dict(op="norm", T=T, d=d, dtype=dtype, stream=stream or dtype, p=p, residual=residual, bwd=bwd)


def _dropout(T, d, dtype="bf16", p=0.1, residual=True, bwd=True):
    return dict(op="dropout", T=T, d=d, dtype=dtype, p=p, residual=residual, bwd=bwd)


def _linear8(T, d, n, dtype="bf16", act="none", bias=False, residual=False):
    return dict(op="linear8", T=T, d=d, n=n, dtype=dtype, act=act, bias=bias, residual=residual)


def _experts8(T, E, k, d, f, dtype="bf16", act="swiglu"):
    return dict(op="experts8", T=T, E=E, k=k, d=d, f=f, dtype=dtype, act=act)


def listed():
    return [
        # generation, a batch of four: only latency counts
        dict(_norm(4, 4096, bwd=False), name="norm_decode"),
        # a large training step: dropout on the branch, the residual stream in full precision
        dict(_norm(16384, 4096, stream="f32", p=0.1), name="norm_step"),
        # ragged: a width no vector divides, an odd number of tokens
        dict(_norm(3001, 1091, dtype="f16"), name="norm_step_ragged"),
        # full precision, a small model
        dict(_norm(300, 516, dtype="f32", p=0.2), name="norm_f32_step"),
        # the end of a block in training, forward and backward
        dict(_dropout(32768, 4096), name="dropout_step"),
        # small, full precision, an odd width, forward alone
        dict(_dropout(300, 517, dtype="f32", p=0.5, residual=False, bwd=False), name="dropout_small"),
        # generation, one token: the up-projection of a shared expert is a read of its weights
        dict(_linear8(1, 4096, 14336, act="swiglu"), name="linear8_decode_up"),
        # a short prompt: ragged token count, widths that are multiples of 64 only, the whole epilogue
        dict(_linear8(3001, 2880, 1088, dtype="f16", act="gelu", bias=True, residual=True), name="linear8_ragged"),
        # the sizes of the framework's benchmark: prompts of a large batch
        dict(_linear8(32768, 4096, 14336, act="swiglu"), name="linear8_large"),
        # generation, a batch of 16: the whole shared expert
        dict(op="mlp8", T=16, d=4096, n=14336, dtype="bf16", act="swiglu", name="mlp8_decode"),
        # generation, a batch of four on a layer of 256 experts: a token or two for each of some thirty of them
        dict(_experts8(4, 256, 8, 2048, 1024), name="experts8_decode"),
        # prompts: 64 experts with uneven loads
        dict(_experts8(16384, 64, 4, 2048, 1024), name="experts8_prompt"),
    ]


def _log_int(rng, lo, hi, mult=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // mult * mult, max(-(-lo // mult) * mult, int(round(v / mult)) * mult))


def draw(rng):
    """One more case of the listed ranges; sizes over their logarithm."""
    while True:
        op = rng.choice(["norm", "norm", "dropout", "linear8", "linear8", "mlp8", "experts8"])
        half = rng.choice(["bf16", "bf16", "f16"])
        dtype = rng.choice([half, half, half, "f32"])
        if op == "norm":
            bwd = rng.random() < 0.7
            c = _norm(_log_int(rng, 64 if bwd else 1, 32768), _log_int(rng, 16, 16384, rng.choice([1, 8, 64])), dtype, rng.choice([dtype, dtype, "f32"]),
                      rng.choice([0.0, 0.1, 0.3]), rng.random() < 0.8, bwd)
        elif op == "dropout":
            c = _dropout(_log_int(rng, 1, 65536), _log_int(rng, 16, 16384, rng.choice([1, 8, 64])), dtype, rng.choice([0.05, 0.1, 0.5]),
                         rng.random() < 0.6, rng.random() < 0.6)
        elif op == "linear8":
            c = _linear8(_log_int(rng, 1, 32768), _log_int(rng, 256, 14336, 64), _log_int(rng, 256, 14336, 64), dtype,
                         rng.choice(["none", "gelu", "swiglu"]), rng.random() < 0.5, rng.random() < 0.5)
        elif op == "mlp8":
            c = dict(op="mlp8", T=_log_int(rng, 1, 16384), d=_log_int(rng, 256, 8192, 64), n=_log_int(rng, 256, 14336, 64), dtype=half,
                     act=rng.choice(["gelu", "swiglu"]))
        else:
            E = _log_int(rng, 4, 256)
            c = _experts8(_log_int(rng, 1, 16384), E, rng.randint(1, min(8, E)), _log_int(rng, 256, 4096, 64), _log_int(rng, 256, 4096, 64), half,
                          rng.choice(["gelu", "swiglu"]))
        w = work(c)
        if w["flops"] <= 7e12 and w["bytes"] <= 1.2e9:
            return c


def work(case):
    """Bytes and operations one pass cannot do without."""
    c = case
    size = lambda name: 4 if name == "f32" else 2  # noqa: E731
    s = size(c["dtype"])
    if c["op"] in ("norm", "dropout"):
        n = c["T"] * c["d"]
        if c["op"] == "dropout":
            return {"bytes": n * s * (2 + c["residual"] + 2 * c["bwd"]), "flops": n * (2 + c["bwd"])}
        t = size(c["stream"])
        keeps = c["residual"] or c["p"] > 0
        fwd = n * (s + t * c["residual"] + t * keeps + s)              # x, residual in, h, y out
        bwd = n * (s + (t if keeps else s) + t + t + s * (c["p"] > 0 or s != t))   # dy, h, dh of the stream in, dh and dx out
        return {"bytes": fwd + (bwd if c["bwd"] else 0), "flops": n * (16 if c["bwd"] else 6)}
    mats = 2 if c["act"] == "swiglu" else 1
    if c["op"] == "linear8":
        T, d, n = c["T"], c["d"], c["n"]
        return {"bytes": T * d * s + mats * d * n + T * n * s * (1 + c["residual"]), "flops": 2 * T * d * n * mats}
    if c["op"] == "mlp8":
        T, d, n = c["T"], c["d"], c["n"]
        return {"bytes": 4 * T * d * s + (mats + 1) * d * n, "flops": 2 * T * d * n * (mats + 1)}
    A, d, f = c["T"] * c["k"], c["d"], c["f"]
    return {"bytes": 2 * c["T"] * d * s + min(A, c["E"]) * (mats + 1) * d * f, "flops": 2 * A * d * f * (mats + 1)}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _normal(gen, shape, std, dtype):
    out = torch.empty(shape, dtype=dtype, device=gen.device)
    flat, step = out.view(-1), 1 << 27
    for i in range(0, flat.numel(), step):
        p = flat[i:i + step]
        p.copy_(torch.randn(p.numel(), generator=gen, device=gen.device).mul_(std))
    return out


def _rows(gen, T, d, dtype):
    """Activations as a residual stream has them: tokens of different sizes, some columns far larger than the others."""
    v = _normal(gen, (T, d), 1.0, torch.float32)
    v *= torch.exp(_normal(gen, (T, 1), 0.5, torch.float32))
    v *= torch.where(torch.rand((1, d), generator=gen, device=v.device) < 0.005, 12.0, 1.0)
    return v.to(dtype)


def _weight8(gen, shape):
    """A matrix (or one for each expert) in 8 bits, with a scale for each column: codes and scales as a quantiser leaves them, and
    the codes in the order in which the matrix cores take them: 16 columns x 64 rows after one another, sixteen rows of a column
    together."""
    d, n = shape[-2:]
    codes = torch.empty(shape, dtype=torch.int8, device=gen.device)
    flat, step = codes.view(-1), 1 << 27
    for i in range(0, flat.numel(), step):
        p = flat[i:i + step]
        p.copy_(torch.randn(p.numel(), generator=gen, device=gen.device).mul_(33.0).round_().clamp_(-127, 127))
    scales = (0.8 + 0.4 * torch.rand((*shape[:-2], n), generator=gen, device=gen.device)) * (d ** -0.5 / 33.0)
    laid = codes.view(-1, d // 64, 4, 16, n // 16, 16).permute(0, 4, 1, 2, 5, 3).contiguous()
    return {"codes": codes, "scales": scales, "laid": laid}


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    td = TYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] in ("norm", "dropout"):
        T, d = c["T"], c["d"]
        ts = TYPES[c.get("stream", c["dtype"])]
        s["x"] = _rows(gen, T, d, td)
        s["residual"] = _rows(gen, T, d, ts) if c["residual"] else None
        s["gamma"] = (1 + 0.2 * _normal(gen, (d,), 1.0, torch.float32)).to(td)
        s["seed"], s["offset"] = (seed * 0x9E3779B97F4A7C15 + 0x1234567) % (1 << 64), (seed * 7919 + (5 << 33)) % (1 << 64)
        if c["bwd"]:
            s["dy"] = _normal(gen, (T, d), 1.0, td)
            s["d_h"] = _normal(gen, (T, d), 1.0, ts)
        return s
    mats = 2 if c["act"] == "swiglu" else 1
    s["x"] = _rows(gen, c["T"], c["d"], td)
    if c["op"] == "linear8":
        s["W"] = [_weight8(gen, (c["d"], c["n"])) for _ in range(mats)]
        s["b"] = [_normal(gen, (c["n"],), 0.1, td) for _ in range(mats)] if c["bias"] else [None] * mats
        s["r"] = _normal(gen, (c["T"], c["n"]), 1.0, td) if c["residual"] else None
    elif c["op"] == "mlp8":
        s["residual"] = _rows(gen, c["T"], c["d"], td)
        s["gamma"] = (1 + 0.2 * _normal(gen, (c["d"],), 1.0, torch.float32)).to(td)
        s["W"] = [_weight8(gen, (c["d"], c["n"])) for _ in range(mats)]
        s["Wd"] = _weight8(gen, (c["n"], c["d"]))
    else:
        T, E, k = c["T"], c["E"], c["k"]
        logits = _normal(gen, (T, E), 1.0, torch.float32) + _normal(gen, (1, E), 0.7, torch.float32)
        top = logits.topk(k, dim=1)
        s["idx"], s["w"] = top.indices.to(torch.int32).contiguous(), torch.softmax(top.values, dim=1).contiguous()
        s["most"] = int(torch.bincount(s["idx"].view(-1).long(), minlength=E).max())   # rows of the busiest expert: the plain form's padding
        s["W"] = [_weight8(gen, (E, c["d"], c["f"])) for _ in range(mats)]
        s["Wd"] = _weight8(gen, (E, c["f"], c["d"]))
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _act(z, act):
    """act of the products z (a list of one, or two for swiglu)."""
    if act == "swiglu":
        return z[0] * torch.sigmoid(z[0]) * z[1]
    return z[0] * 0.5 * torch.erfc(-z[0] * math.sqrt(0.5)) if act == "gelu" else z[0]


def _philox_round(v, k):
    a, b = v[0] * 0xD2511F53, v[2] * 0xCD9E8D57   # 64 bits, signed: the halves below are those of the unsigned products
    low = 0xFFFFFFFF
    return [((b >> 32) & low) ^ v[1] ^ k[0], b & low, ((a >> 32) & low) ^ v[3] ^ k[1], a & low]


def _keep(T, d, p, seed, offset, device):
    """Which elements of a [T, d] matrix dropout keeps, and what it multiplies them by."""
    cut = min(65535, int(math.floor(p * 65536 + 0.5)))
    low = 0xFFFFFFFF
    col = torch.arange((d + 7) // 8, device=device).view(1, -1).expand(T, -1)
    row = torch.arange(T, device=device).view(-1, 1).expand_as(col)
    v = [col, row, torch.full_like(col, offset & low), torch.full_like(col, offset >> 32)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        v = _philox_round(v, k)
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    halves = torch.stack([h for w in v for h in (w & 0xFFFF, w >> 16)], dim=2)
    return halves.view(T, -1)[:, :d] >= cut, 65536 / (65536 - cut)


def _dropped(v, s):
    """dropout(v) in 32 bits."""
    c = s["case"]
    if c["p"] == 0:
        return v.float()
    keep, scale = _keep(c["T"], c["d"], c["p"], s["seed"], s["offset"], v.device)
    return torch.where(keep, v.float() * scale, torch.zeros((), device=v.device))


def _quantise(v):
    """(codes as numbers, scales) of the rows of a matrix in 32 bits."""
    m = v.abs().amax(dim=1, keepdim=True).clamp(min=2.0 ** -100)
    up = torch.full_like(m, 127.0) / m
    return torch.round(v * up), m * (1.0 / 127.0)


def _product8(codes, scales, w):
    return (codes @ w["codes"].float()) * (scales * w["scales"])


def _rms_norm(h, gamma):
    rstd = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
    return h * rstd * gamma.float(), rstd


def _norm_plain(s):
    c, td, ts = s["case"], TYPES[s["case"]["dtype"]], TYPES[s["case"]["stream"]]
    h = _dropped(s["x"], s)
    out = {}
    if s["residual"] is not None or c["p"] > 0:
        h = h if s["residual"] is None else h + s["residual"].float()
        out["h"] = h.to(ts)
        h = out["h"].float()
    y, rstd = _rms_norm(h, s["gamma"])
    out["y"] = y.to(td)
    if c["bwd"]:
        a = s["dy"].float() * s["gamma"].float()
        dh = rstd * (a - h * rstd * rstd * (a * h).mean(dim=1, keepdim=True)) + s["d_h"].float()
        out["dh"] = dh.to(ts)
        if c["p"] > 0 or td != ts:
            out["dx"] = _dropped(dh, s).to(td)
        out["dgamma"] = (s["dy"].float() * h * rstd).sum(dim=0)
    return out


def _dropout_plain(s):
    y = _dropped(s["x"], s)
    out = {"y": (y if s["residual"] is None else y + s["residual"].float()).to(s["x"].dtype)}
    if s["case"]["bwd"]:
        out["dx"] = _dropped(s["dy"], s).to(s["x"].dtype)
    return out


def _linear8_plain(s):
    c = s["case"]
    q, scale = _quantise(s["x"].float())
    z = [_product8(q, scale, w) for w in s["W"]]
    z = [v if b is None else v + b.float() for v, b in zip(z, s["b"])]
    y = _act(z, c["act"])
    return (y if s["r"] is None else y + s["r"].float()).to(s["x"].dtype)


def _mlp8_plain(s):
    td = s["x"].dtype
    h = (s["residual"].float() + s["x"].float()).to(td)
    q, scale = _quantise(_rms_norm(h.float(), s["gamma"])[0])
    hidden = _act([_product8(q, scale, w) for w in s["W"]], s["case"]["act"]).to(td)
    q, scale = _quantise(hidden.float())
    return {"h": h, "out": (_product8(q, scale, s["Wd"]) + h.float()).to(td)}


def _experts8_plain(s):
    c, td = s["case"], s["x"].dtype
    T, E, k, most = c["T"], c["E"], c["k"], s["most"]
    e = s["idx"].view(-1).long()
    order = torch.argsort(e, stable=True)
    es = e[order]
    first = torch.searchsorted(es, torch.arange(E, device=e.device))
    slot = es * most + torch.arange(T * k, device=e.device) - first[es]   # every expert's rows, filled up to those of the busiest
    q, scale = _quantise(s["x"].float())
    rows = torch.zeros((E * most, c["d"]), device=e.device)
    rows[slot] = q[order // k]
    row_scale = torch.zeros((E * most, 1), device=e.device)
    row_scale[slot] = scale[order // k]

    def product(v, v_scale, w):
        return torch.bmm(v.view(E, most, -1), w["codes"].float()) * (v_scale.view(E, most, 1) * w["scales"][:, None, :])

    hidden = _act([product(rows, row_scale, w) for w in s["W"]], c["act"]).to(td)
    q, scale = _quantise(hidden.float().view(E * most, -1))
    y = product(q, scale, s["Wd"]).view(E * most, -1)[slot]
    y = torch.zeros_like(y).index_copy_(0, order, y)
    return (y.view(T, k, -1) * s["w"][:, :, None]).sum(dim=1).to(td)


_RUN_PLAIN = {"norm": _norm_plain, "dropout": _dropout_plain, "linear8": _linear8_plain, "mlp8": _mlp8_plain, "experts8": _experts8_plain}


def run(state):
    return (_RUN_OWN if own else _RUN_PLAIN)[state["case"]["op"]](state)


# ---- the framework's operators -------------------------------------------------------------------------------------

def _buffers(s, make):
    """What a program keeps from call to call: output buffers, the workspace, descriptions of the sizes."""
    if "kept_buffers" not in s:
        s["kept_buffers"] = make()
    return s["kept_buffers"]


def _new(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda:0")


def _space(n):
    return _new(max(256, n), dtype=torch.uint8)


def _types(B):
    return {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16}


def _acts(B):
    return {"none": B.ACT_NONE, "gelu": B.ACT_GELU, "swiglu": B.ACT_SWIGLU}


def _two(ws, key):
    """An argument for each of two matrices, None for the second where there is one."""
    return [w[key] for w in ws] + [None] * (2 - len(ws))


def _own_norm(s):
    from paper_2504_03871_amd import binding as B
    c, td, ts = s["case"], TYPES[s["case"]["dtype"]], TYPES[s["case"]["stream"]]
    T, d, keeps = c["T"], c["d"], s["residual"] is not None or c["p"] > 0

    def make():
        norm = B.make_norm(T, d, _types(B)[c["dtype"]], stream=_types(B)[c["stream"]], eps=EPS)
        b = {"norm": norm, "drop": B.make_drop(c["p"], s["seed"], s["offset"]) if c["p"] > 0 else None, "y": _new(T, d, dtype=td),
             "h": _new(T, d, dtype=ts) if keeps or (c["bwd"] and td != ts) else None, "rstd": _new(T) if c["bwd"] else None}
        if c["bwd"]:
            b.update(dh=_new(T, d, dtype=ts), dx=_new(T, d, dtype=td) if c["p"] > 0 or td != ts else None, dgamma=_new(d),
                     ws=_space(B.moe_norm_bwd_workspace_bytes(norm)))
        return b

    b = _buffers(s, make)
    B.moe_norm_fwd(b["norm"], b["drop"], s["x"], s["residual"], s["gamma"], b["h"], b["rstd"], b["y"], None, None)
    out = {"h": b["h"], "y": b["y"]} if keeps else {"y": b["y"]}
    if c["bwd"]:
        h = s["x"] if b["h"] is None else b["h"]
        B.moe_norm_bwd(b["norm"], b["drop"], s["dy"], h, s["gamma"], b["rstd"], s["d_h"], b["dh"], b["dx"], b["dgamma"], 0, b["ws"])
        out["dh"] = b["dh"]
        if b["dx"] is not None:
            out["dx"] = b["dx"]
        out["dgamma"] = b["dgamma"]
    return out


def _own_dropout(s):
    from paper_2504_03871_amd import binding as B
    c = s["case"]
    dt = _types(B)[c["dtype"]]
    b = _buffers(s, lambda: {"drop": B.make_drop(c["p"], s["seed"], s["offset"]), "y": torch.empty_like(s["x"]),
                             "dx": torch.empty_like(s["x"]) if c["bwd"] else None})
    B.moe_dropout(dt, c["T"], c["d"], b["drop"], s["x"], s["residual"], b["y"])
    if not c["bwd"]:
        return {"y": b["y"]}
    B.moe_dropout(dt, c["T"], c["d"], b["drop"], s["dy"], None, b["dx"])
    return {"y": b["y"], "dx": b["dx"]}


def _own_linear8(s):
    from paper_2504_03871_amd import binding as B
    c, td = s["case"], s["x"].dtype
    T, d, n = c["T"], c["d"], c["n"]

    def make():
        lin = B.make_linear8(T, d, n, _types(B)[c["dtype"]], _acts(B)[c["act"]])
        return {"lin": lin, "ws": _space(B.moe_linear8_workspace_bytes(lin)), "codes": _new(T, d, dtype=torch.int8), "scales": _new(T), "y": _new(T, n, dtype=td)}

    b = _buffers(s, make)
    B.moe_quant_rows(b["lin"].dtype, T, d, d, s["x"], b["codes"], b["scales"])
    W, ws, bias = _two(s["W"], "laid"), _two(s["W"], "scales"), (s["b"] + [None])[:2]
    B.moe_linear8_fwd(b["lin"], b["codes"], b["scales"], W[0], ws[0], W[1], ws[1], bias[0], bias[1], s["r"], b["y"], b["ws"])
    return b["y"]


def _own_mlp8(s):
    from paper_2504_03871_amd import binding as B
    c, td = s["case"], s["x"].dtype
    T, d, n = c["T"], c["d"], c["n"]

    def make():
        dt = _types(B)[c["dtype"]]
        up, down = B.make_linear8(T, d, n, dt, _acts(B)[c["act"]]), B.make_linear8(T, n, d, dt, B.ACT_NONE)
        return {"norm": B.make_norm(T, d, dt, eps=EPS), "up": up, "down": down,
                "ws": _space(max(B.moe_linear8_workspace_bytes(up), B.moe_linear8_workspace_bytes(down))),
                "h": _new(T, d, dtype=td), "codes": _new(T, d, dtype=torch.int8), "scales": _new(T), "hidden": _new(T, n, dtype=td),
                "hidden_codes": _new(T, n, dtype=torch.int8), "hidden_scales": _new(T), "out": _new(T, d, dtype=td)}

    b = _buffers(s, make)
    W, ws = _two(s["W"], "laid"), _two(s["W"], "scales")
    B.moe_norm_fwd(b["norm"], None, s["x"], s["residual"], s["gamma"], b["h"], None, None, b["codes"], b["scales"])
    B.moe_linear8_fwd(b["up"], b["codes"], b["scales"], W[0], ws[0], W[1], ws[1], None, None, None, b["hidden"], b["ws"])
    B.moe_quant_rows(b["up"].dtype, T, n, n, b["hidden"], b["hidden_codes"], b["hidden_scales"])
    B.moe_linear8_fwd(b["down"], b["hidden_codes"], b["hidden_scales"], s["Wd"]["laid"], s["Wd"]["scales"], None, None, None, None, b["h"], b["out"], b["ws"])
    return {"h": b["h"], "out": b["out"]}


def _own_experts8(s):
    from paper_2504_03871_amd import binding as B
    c, td = s["case"], s["x"].dtype
    T, E, k, d, f = c["T"], c["E"], c["k"], c["d"], c["f"]

    def make():
        cfg = B.make_cfg(T, d, f, E, k, _types(B)[c["dtype"]], _acts(B)[c["act"]])
        i32 = lambda n: _new(n, dtype=torch.int32)  # noqa: E731
        return {"cfg": cfg, "ws": _space(max(B.moe_workspace_bytes(cfg), B.moe_expert_ffn8_workspace_bytes(cfg))), "codes": _new(T, d, dtype=torch.int8),
                "scales": _new(T), "counts": i32(E), "kept": i32(E), "offsets": i32(E + 1), "row_of": i32(T * k), "src_of": i32(T * k),
                "y_perm": _new(T * k, d, dtype=td), "out": _new(T, d, dtype=td)}

    b = _buffers(s, make)
    W, ws = _two(s["W"], "laid"), _two(s["W"], "scales")
    B.moe_quant_rows(b["cfg"].dtype, T, d, d, s["x"], b["codes"], b["scales"])
    B.moe_dispatch(b["cfg"], s["x"], s["idx"], None, None, b["counts"], b["kept"], b["offsets"], b["row_of"], b["src_of"], None, b["ws"])
    B.moe_expert_ffn_fwd8(b["cfg"], b["codes"], b["scales"], W[0], ws[0], W[1], ws[1], s["Wd"]["laid"], s["Wd"]["scales"], b["src_of"], b["offsets"],
                          b["kept"], None, None, b["y_perm"], b["ws"])
    B.moe_combine(b["cfg"], b["y_perm"], s["w"], s["idx"], b["row_of"], b["offsets"], b["kept"], None, None, b["out"])
    return b["out"]


_RUN_OWN = {"norm": _own_norm, "dropout": _own_dropout, "linear8": _own_linear8, "mlp8": _own_mlp8, "experts8": _own_experts8}


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------

def _mask64(rows, d, p, seed, offset):
    """What each element is multiplied by: 0, or 65536 / (65536 - cut).  Products of 32-bit numbers from 16-bit halves."""
    def wide(m, x):
        high, low = m * (x >> 16), m * (x & 0xFFFF)
        middle = high + (low >> 16)
        return middle >> 16, ((middle & 0xFFFF) << 16) | (low & 0xFFFF)

    cut = min(65535, round(p * 65536)) if p * 65536 % 1 != 0.5 else int(p * 65536 + 0.5)
    dev = torch.device("cuda:0")
    x0, x1 = torch.meshgrid(torch.arange(rows, device=dev), torch.arange(-(-d // 8), device=dev), indexing="ij")
    x0, x1 = x1.contiguous(), x0.contiguous()
    x2, x3 = torch.full_like(x0, offset % 2 ** 32), torch.full_like(x0, offset // 2 ** 32)
    k0, k1 = seed % 2 ** 32, seed // 2 ** 32
    for i in range(10):
        h0, l0 = wide(0xD2511F53, x0)
        h1, l1 = wide(0xCD9E8D57, x2)
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    out = torch.empty((rows, x0.shape[1], 8), dtype=torch.float64, device=dev)
    for i, w in enumerate((x0, x1, x2, x3)):
        out[:, :, 2 * i] = (w % 65536 >= cut).double()
        out[:, :, 2 * i + 1] = (w // 65536 >= cut).double()
    return out.view(rows, -1)[:, :d] * (65536 / (65536 - cut))


def _codes64(v):
    """Codes of the rows of a matrix, whole numbers in 64 bits, and the scales; the factor 127 / m is a number of 32 bits."""
    m = torch.clamp(torch.linalg.vector_norm(v, ord=float("inf"), dim=1), min=2.0 ** -100)
    up = (127.0 / m).float().double()
    return torch.round((v * up[:, None]).float().double()), m / 127.0


def _gelu64(z):
    return z * torch.special.ndtr(z)


def _silu64(z):
    return z / (1 + torch.exp(-z))


def _act64(z, act):
    return _silu64(z[0]) * z[1] if act == "swiglu" else _gelu64(z[0]) if act == "gelu" else z[0]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    td = TYPES[c["dtype"]]
    x = s["x"].double()
    if c["op"] == "dropout":
        m = _mask64(c["T"], c["d"], c["p"], s["seed"], s["offset"])
        out = {"y": x * m if s["residual"] is None else torch.addcmul(s["residual"].double(), x, m)}
        if c["bwd"]:
            out["dx"] = s["dy"].double() * m
        return out
    if c["op"] == "norm":
        m = _mask64(c["T"], c["d"], c["p"], s["seed"], s["offset"]) if c["p"] > 0 else None
        h = x if m is None else x * m
        out = {}
        if s["residual"] is not None or c["p"] > 0:
            if s["residual"] is not None:
                h = h + s["residual"].double()
            out["h"] = h
            h = h.to(TYPES[c["stream"]]).double()   # the norm is that of h as it is stored
        h = h.detach().requires_grad_(c["bwd"])
        g = s["gamma"].double().requires_grad_(c["bwd"])
        y = g * h / torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / c["d"] + EPS)
        out["y"] = y.detach()
        if c["bwd"]:
            dh, dg = torch.autograd.grad(y, (h, g), s["dy"].double())
            out["dh"] = dh + s["d_h"].double()
            if c["p"] > 0 or TYPES[c["stream"]] != td:
                out["dx"] = out["dh"] if m is None else out["dh"] * m
            out["dgamma"] = dg
        return out
    if c["op"] == "linear8":
        q, scale = _codes64(x)
        z = [torch.mm(q, w["codes"].double()).mul_(scale[:, None]).mul_(w["scales"].double()) for w in s["W"]]
        for v, b in zip(z, s["b"]):
            if b is not None:
                v.add_(b.double())
        y = _act64(z, c["act"])
        return y if s["r"] is None else y + s["r"].double()
    if c["op"] == "mlp8":
        h = s["residual"].double() + x
        v = h.to(td).double()
        q, scale = _codes64(s["gamma"].double() * v / torch.sqrt(v.square().sum(dim=1, keepdim=True) / c["d"] + EPS))
        hidden = _act64([torch.mm(q, w["codes"].double()) * torch.outer(scale, w["scales"].double()) for w in s["W"]], c["act"])
        q, scale = _codes64(hidden.to(td).double())   # as it is stored
        return {"h": h, "out": torch.mm(q, s["Wd"]["codes"].double()) * torch.outer(scale, s["Wd"]["scales"].double()) + v}
    q, scale = _codes64(x)
    out = torch.zeros_like(x)
    for e in range(c["E"]):
        t, j = torch.nonzero(s["idx"] == e, as_tuple=True)
        if t.numel() == 0:
            continue
        hidden = _act64([torch.mm(q[t], w["codes"][e].double()) * torch.outer(scale[t], w["scales"][e].double()) for w in s["W"]], c["act"])
        p, ps = _codes64(hidden.to(td).double())
        y = torch.mm(p, s["Wd"]["codes"][e].double()) * torch.outer(ps, s["Wd"]["scales"][e].double())
        out.index_add_(0, t, y * s["w"][t, j].double()[:, None])
    return out
