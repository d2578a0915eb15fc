"""Cases of the operators beside the expert layer: scored routing, products with an epilogue, activations kept in 8 bits.

A case is a dict of plain values with an "op":
  route   choice of experts from gate logits: scores, balance bias, groups, top-k, weights; `bwd`: the gradient of the logits too.
          T E k, score "softmax" | "sigmoid", groups, top_groups, rank (experts that make a group's score), renorm, scale,
          balance (a selection bias is given), masked (some logits are -inf, some tokens have none left)
  linear  y = act(x W + b) + r, by `what`: "fwd", "step" (forward, then the gradients of x, W and b), "packed" (the gradients from
          pre-activations that were kept in 8 bits).  T d n (x is [T, d], y [T, n]), dtype, act "none" | "gelu" | "swiglu", bias,
          residual, fmt of the packed pre-activations
  pack    a matrix packed to 8 bits and unpacked again.  rows width dtype fmt
  saved   the pre-activations of an expert layer packed after its forward pass, and every plane restored for its backward pass.
          T d f E k dtype act fmt

The plain forms below are torch operations in 32 bits, or in 64 where two values may lie closer together than 32 bits resolve.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 32   # values that share a scale


def _route(T, E, k, score, groups=1, top_groups=1, rank=1, renorm=True, scale=1.0, balance=True, masked=False, bwd=True):
    return dict(op="route", T=T, E=E, k=k, score=score, groups=groups, top_groups=top_groups, rank=rank, renorm=renorm, scale=scale,
                balance=balance, masked=masked, bwd=bwd)


def _linear(what, T, d, n, dtype="bf16", act="none", bias=True, residual=True, fmt="i8"):
    return dict(op="linear", what=what, T=T, d=d, n=n, dtype=dtype, act=act, bias=bias, residual=residual, fmt=fmt)


def listed():
    return [
        # generation: the router of a many-expert layer for a decode batch of four, where only latency counts
        dict(_route(4, 256, 8, "sigmoid", 8, 4, 2, True, 2.5, bwd=False), name="route_decode"),
        # training step of a layer with 64 experts, plain softmax scores, an odd number of tokens of which some are padding
        dict(_route(8191, 64, 6, "softmax", renorm=False, balance=False, masked=True), name="route_softmax_step"),
        # training step of a layer with 256 experts in eight groups, sigmoid scores and a balance bias: a large batch
        dict(_route(32768, 256, 8, "sigmoid", 8, 4, 2, True, 2.5), name="route_groups_step"),
        # generation, one token: the up-projection of a shared expert, which is a read of its weights
        dict(_linear("fwd", 1, 4096, 14336, act="swiglu", bias=False, residual=False), name="linear_decode_up"),
        # generation, a batch of 16: the down-projection, long sums, the routed experts' output added
        dict(_linear("fwd", 16, 14336, 4096, dtype="f16", bias=False), name="linear_decode_down"),
        # full precision, sizes that are multiples of four and nothing more: gradient checks and small models
        dict(_linear("step", 300, 516, 1540, dtype="f32", act="gelu"), name="linear_f32_step"),
        # an ordinary training step of a shared expert's first product
        dict(_linear("step", 8192, 1024, 4096, act="gelu"), name="linear_step"),
        # ragged everything: odd token count, widths that are multiples of 64 only; the second product, with the residual
        dict(_linear("step", 3001, 2880, 1088, dtype="f16"), name="linear_step_ragged"),
        # the sizes of the framework's benchmark, the largest that is run
        dict(_linear("step", 32768, 4096, 14336, act="swiglu", bias=False, residual=False), name="linear_step_large"),
        # the backward of a checkpointed shared expert: its pre-activations lie in 8 bits
        dict(_linear("packed", 4096, 2048, 8192, act="swiglu", residual=False), name="linear_bwd_packed"),
        # a small full-precision activation kept in 8 bits, of a width that no block divides
        dict(op="pack", rows=300, width=516, dtype="f32", fmt="e4m3", name="pack_small"),
        # checkpoints of an expert layer at training size
        dict(op="saved", T=16384, d=2048, f=8192, E=16, k=2, dtype="bf16", act="swiglu", fmt="i8", name="saved_step"),
    ]


def _log_int(rng, lo, hi, mult=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // mult * mult, max(-(-lo // mult) * mult, int(round(v / mult)) * mult))


def draw(rng):
    """One more case of the listed ranges; sizes over their logarithm."""
    while True:
        op = rng.choice(["route", "linear", "linear", "pack", "saved"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op == "route":
            groups = rng.choice([1, 1, 2, 4, 8])
            E = groups * _log_int(rng, max(2, 8 // groups), 256 // groups)
            top = rng.randint(1, groups)
            k = rng.randint(1, min(8, E // groups * top))
            c = _route(_log_int(rng, 1, 32768), E, k, rng.choice(["softmax", "sigmoid"]), groups, top, rng.choice([1, 2]),
                       rng.random() < 0.6, rng.choice([1.0, 2.5]), rng.random() < 0.6, rng.random() < 0.3, rng.random() < 0.7)
        elif op == "linear":
            what = rng.choice(["fwd", "step", "step", "packed"])
            act = rng.choice(["gelu", "swiglu"] if what == "packed" else ["none", "gelu", "swiglu"])
            fmt, bias, residual = rng.choice(["e4m3", "i8"]), rng.random() < 0.5, what != "packed" and rng.random() < 0.5
            lo = 1 if what == "fwd" else 64
            if dtype == "f32":
                c = _linear(what, _log_int(rng, lo, 4096), _log_int(rng, 64, 2048, 4), _log_int(rng, 64, 2048, 4), dtype, act, bias, residual, fmt)
            else:
                c = _linear(what, _log_int(rng, lo, 32768), _log_int(rng, 256, 14336, 64), _log_int(rng, 256, 14336, 64), dtype, act, bias,
                            residual, fmt)
        elif op == "pack":
            c = dict(op="pack", rows=_log_int(rng, 1, 65536), width=_log_int(rng, 4, 14336, 4), dtype=dtype, fmt=rng.choice(["e4m3", "i8"]))
        else:
            E = _log_int(rng, 4, 64)
            c = dict(op="saved", T=_log_int(rng, 16, 16384), d=256, f=_log_int(rng, 256, 8192, 64), E=E, k=rng.randint(1, 4), dtype=dtype,
                     act=rng.choice(["gelu", "swiglu"]), fmt=rng.choice(["e4m3", "i8"]))
        w = work(c)
        if w["flops"] <= 1.2e13 and w["bytes"] <= 4e9:
            return c


def work(case):
    """Bytes and operations one pass cannot do without."""
    c = case
    if c["op"] == "route":
        logits, chosen = c["T"] * c["E"] * 4, c["T"] * c["k"] * 8
        return {"bytes": logits + chosen + (2 * logits + c["T"] * c["k"] * 4 if c["bwd"] else 0), "flops": c["T"] * c["E"] * (20 if c["bwd"] else 10)}
    s = 4 if c["dtype"] == "f32" else 2
    mats = 2 if c.get("act") == "swiglu" else 1
    if c["op"] == "linear":
        T, d, n = c["T"], c["d"], c["n"]
        one, x, w, y = 2 * T * d * n * mats, T * d * s, d * n * s * mats, T * n * s
        fwd = {"bytes": x + w + y + (y if c["residual"] else 0), "flops": one}
        bwd = {"bytes": 2 * x + 2 * w + y, "flops": 2 * one}   # dy, x, W in, dx and dW out
        if c["what"] == "fwd":
            return fwd
        if c["what"] == "packed":
            return {"bytes": bwd["bytes"] + mats * T * n * 33 / 32, "flops": 2 * one}
        keep = 0 if c["act"] == "none" else 2 * mats * y       # the pre-activations, written and read
        return {"bytes": fwd["bytes"] + bwd["bytes"] + keep, "flops": 3 * one}
    if c["op"] == "pack":
        n = c["rows"] * c["width"]
        return {"bytes": 2 * n * (s + 33 / 32), "flops": 4 * n}
    n = c["T"] * c["k"] * c["f"]
    return {"bytes": n * (mats * (s + 33 / 32) + mats * (33 / 32 + s) + s), "flops": 8 * n * mats}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _normal(gen, shape, std, dtype):
    out = torch.empty(shape, dtype=dtype, device=gen.device)
    flat, step = out.view(-1), 1 << 27
    for i in range(0, flat.numel(), step):
        p = flat[i:i + step]
        p.copy_(torch.randn(p.numel(), generator=gen, device=gen.device).mul_(std))
    return out


def prepare(case, seed):
    c, dev = case, torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    s = {"case": c}
    if c["op"] == "route":
        T, E = c["T"], c["E"]
        # gate logits of spread 1.5 around levels that differ from expert to expert; the balance bias in steps of its update
        s["logits"] = _normal(gen, (T, E), 1.5, torch.float32) + _normal(gen, (1, E), 0.5, torch.float32)
        s["balance"] = (_normal(gen, (E,), 30.0, torch.float32).round() * 0.001) if c["balance"] else None
        if c["masked"]:   # experts that are switched off for a token, and padding tokens that have none
            s["logits"].masked_fill_(torch.rand((T, E), generator=gen, device=dev) < 0.05, -math.inf)
            s["logits"].masked_fill_(torch.rand((T, 1), generator=gen, device=dev) < 0.02, -math.inf)
        s["d_w"] = _normal(gen, (T, c["k"]), 1.0, torch.float32) if c["bwd"] else None
        return s
    td = TYPES[c["dtype"]]
    mats = 2 if c.get("act") == "swiglu" else 1
    if c["op"] == "linear":
        T, d, n = c["T"], c["d"], c["n"]
        s["x"] = _normal(gen, (T, d), 1.0, td)
        s["W"] = [_normal(gen, (d, n), d ** -0.5, td) for _ in range(mats)]
        s["b"] = [_normal(gen, (n,), 0.1, td) for _ in range(mats)] if c["bias"] else [None] * mats
        s["r"] = _normal(gen, (T, n), 1.0, td) if c["residual"] else None
        s["dy"] = _normal(gen, (T, n), 1.0, td) if c["what"] != "fwd" else None
        s["packed"] = [_pack(_normal(gen, (T, n), 1.0, td), c["fmt"]) for _ in range(mats)] if c["what"] == "packed" else None
        return s
    if c["op"] == "pack":
        # rows of different sizes, as activations have them, one of zeros
        s["v"] = _normal(gen, (c["rows"], c["width"]), 1.0, td) * torch.exp(_normal(gen, (c["rows"], 1), 1.5, torch.float32)).to(td)
        s["v"][c["rows"] // 2] = 0
        return s
    A = c["T"] * c["k"]
    s["pre"] = _normal(gen, (mats, A, c["f"]), 1.3, td)
    edges = torch.sort(torch.randint(0, A + 1, (c["E"] - 1,), generator=gen, device=dev)).values   # ragged loads, experts without rows too
    s["offsets"] = torch.cat([edges.new_zeros(1), edges, edges.new_full((1,), A)]).to(torch.int32)
    s["kept"] = (s["offsets"][1:] - s["offsets"][:-1]).contiguous()
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _act(z, act):
    """act of the products z (a list of one, or two for swiglu), in the type they have."""
    if act == "swiglu":
        return z[0] * torch.sigmoid(z[0]) * z[1]
    return z[0] * 0.5 * torch.erfc(-z[0] * math.sqrt(0.5)) if act == "gelu" else z[0]


def _act_grad(z, act, dy):
    """The gradients of the products."""
    if act == "swiglu":
        sg = torch.sigmoid(z[0])
        return [dy * z[1] * sg * (1 + z[0] * (1 - sg)), dy * z[0] * sg]
    if act == "gelu":
        return [dy * (0.5 * torch.erfc(-z[0] * math.sqrt(0.5)) + z[0] * torch.exp(-0.5 * z[0] * z[0]) / math.sqrt(2 * math.pi))]
    return [dy]


def _pack(v, fmt):
    """(codes, scale exponents): blocks of 32 along a row with one power of two, the smallest that takes the largest value
    without saturation; codes e4m3, or whole numbers of 64ths.  A block with an infinity or NaN has the exponent 128."""
    rows, width = v.shape
    u = torch.nn.functional.pad(v.float(), (0, -width % BLOCK)).view(rows, -1, BLOCK)
    top = u.abs().amax(dim=2)
    mant, ex = torch.frexp(top)
    e = (ex - 9 + (mant > 0.875).int()) if fmt == "e4m3" else (ex - 1 + (mant >= 127.5 / 128).int())
    e = torch.where(top > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    bad = ~torch.isfinite(top)
    scaled = torch.where(bad[..., None], torch.zeros_like(u), u).double() * torch.exp2(-e.double())[..., None]
    if fmt == "e4m3":
        codes = scaled.float().to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        codes = torch.round(scaled * 64).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return codes.view(rows, -1), torch.where(bad, torch.full_like(e, 128), e).add(127).to(torch.uint8)


def _unpack(packed, width, fmt, dtype):
    """The values in `dtype`, none beyond its largest finite one."""
    codes, e = packed
    value = codes.view(torch.float8_e4m3fn).float().double() if fmt == "e4m3" else codes.view(torch.int8).double() / 64
    e = e.int() - 127
    v = value.view(codes.shape[0], -1, BLOCK) * torch.exp2(e.double())[..., None]
    most = torch.finfo(dtype).max
    v = torch.where((e == 128)[..., None], torch.full_like(v, math.nan), v.clamp(-most, most))
    return v.view(codes.shape[0], -1)[:, :width].to(dtype)


def _route_plain(s):
    c, l = s["case"], s["logits"].double()
    T, E, k = c["T"], c["E"], c["k"]
    open_ = l > -math.inf
    if c["score"] == "sigmoid":
        sc = torch.sigmoid(l)
    else:
        top = l.amax(dim=1, keepdim=True)
        ex = torch.where(open_, torch.exp(l - top), torch.zeros_like(l))
        sc = ex / ex.sum(dim=1, keepdim=True)
    sc = torch.where(open_, sc, torch.zeros_like(sc))
    ch = sc if s["balance"] is None else sc + s["balance"].double()
    ch = torch.where(open_, ch, torch.full_like(ch, -math.inf))
    if c["groups"] > 1:
        gs = ch.view(T, c["groups"], -1).topk(c["rank"], dim=2).values.sum(dim=2)
        best = gs.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        allowed = torch.zeros_like(gs, dtype=torch.bool).scatter_(1, best, True)
        ch = torch.where(allowed.repeat_interleave(E // c["groups"], dim=1), ch, torch.full_like(ch, -math.inf))
    v, idx = ch.sort(dim=1, descending=True, stable=True)
    v, idx = v[:, :k], idx[:, :k]
    live = v > -math.inf
    p = torch.where(live, sc.gather(1, idx), torch.zeros_like(v))
    if c["renorm"]:
        total = p.sum(dim=1, keepdim=True)
        p = torch.where(live, p / total, torch.zeros_like(p))
    out = {"idx": torch.where(live, idx, torch.full_like(idx, -1)).to(torch.int32), "w": (p * c["scale"]).float()}
    if c["bwd"]:
        dw = torch.where(live, s["d_w"].double(), torch.zeros_like(p))
        D = (p * dw).sum(dim=1, keepdim=True)
        if c["renorm"]:
            dl = c["scale"] * p * (dw - D)
            if c["score"] == "sigmoid":
                dl = dl * torch.sigmoid(-l.gather(1, idx))
        elif c["score"] == "sigmoid":
            dl = c["scale"] * p * torch.sigmoid(-l.gather(1, idx)) * dw
        else:
            dl = c["scale"] * p * dw
        dl = torch.where(live, dl, torch.zeros_like(dl))
        dense = torch.zeros_like(l).scatter_(1, idx, dl)
        if c["score"] == "softmax" and not c["renorm"]:
            dense = dense - c["scale"] * sc * D
        out["d_logits"] = dense.float()
    return out


def _linear_plain(s):
    c, td = s["case"], TYPES[s["case"]["dtype"]]
    x, W = s["x"].float(), [w.float() for w in s["W"]]
    out = {}
    if c["what"] == "packed":
        z = [_unpack(p, c["n"], c["fmt"], td).float() for p in s["packed"]]
    else:
        z = [x @ w for w in W]
        z = [v if b is None else v + b.float() for v, b in zip(z, s["b"])]
        y = _act(z, c["act"])
        out["y"] = (y if s["r"] is None else y + s["r"].float()).to(td)
    if c["what"] != "fwd":
        dz = _act_grad(z, c["act"], s["dy"].float())
        dx = dz[0] @ W[0].t()
        out["dx"] = (dx if len(W) == 1 else dx + dz[1] @ W[1].t()).to(td)
        out["dW"] = [(x.t() @ g).to(td) for g in dz]
        out["db"] = [g.sum(dim=0).to(td) for g in dz] if c["bias"] else []
    return out


def run(state):
    s, c = state, state["case"]
    if own:
        return _RUN_OWN[c["op"]](s)
    if c["op"] == "route":
        return _route_plain(s)
    if c["op"] == "linear":
        return _linear_plain(s)
    td = TYPES[c["dtype"]]
    if c["op"] == "pack":
        return _unpack(_pack(s["v"], c["fmt"]), c["width"], c["fmt"], td)
    pre = [_unpack(_pack(p, c["fmt"]), c["f"], c["fmt"], td) for p in s["pre"]]
    return {"pre": pre, "hidden": _act([p.float() for p in pre], c["act"]).to(td)}


# ---- the framework's operators -------------------------------------------------------------------------------------

def _buffers(s, make):
    """What a program keeps from call to call: output buffers, the workspace, descriptions of the sizes."""
    if "kept_buffers" not in s:
        s["kept_buffers"] = make()
    return s["kept_buffers"]


def _own_route(s):
    from paper_2504_03871_amd import binding as B
    c = s["case"]

    def make():
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda:0")  # noqa: E731
        return (B.make_cfg(c["T"], 256, 256, c["E"], c["k"]),
                B.make_score(B.SCORE_SOFTMAX if c["score"] == "softmax" else B.SCORE_SIGMOID, c["groups"], c["top_groups"], c["rank"],
                             c["renorm"], c["scale"]),
                new(c["T"], c["k"], dtype=torch.int32), new(c["T"], c["k"]), new(c["T"], c["E"]) if c["bwd"] else None)

    cfg, score, idx, w, d_logits = _buffers(s, make)
    B.moe_route_scored(cfg, score, None, None, None, s["balance"], s["logits"], None, idx, w)
    if not c["bwd"]:
        return {"idx": idx, "w": w}
    B.moe_route_scored_bwd(cfg, score, None, None, s["logits"], idx, s["d_w"], d_logits, None, None, None)
    return {"idx": idx, "w": w, "d_logits": d_logits}


def _own_linear(s):
    from paper_2504_03871_amd import binding as B
    c, td = s["case"], TYPES[s["case"]["dtype"]]
    mats = len(s["W"])

    def make():
        new = lambda *shape: torch.empty(shape, dtype=td, device="cuda:0")  # noqa: E731
        dt = {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16}[c["dtype"]]
        act = {"none": B.ACT_NONE, "gelu": B.ACT_GELU, "swiglu": B.ACT_SWIGLU}[c["act"]]
        pre = B.PACK_NONE if c["what"] != "packed" else B.PACK_E4M3 if c["fmt"] == "e4m3" else B.PACK_I8
        lin = B.make_linear(c["T"], c["d"], c["n"], dt, act, pre=pre, grad=dt)
        ws = torch.empty(max(256, B.moe_linear_workspace_bytes(lin)), dtype=torch.uint8, device="cuda:0")
        b = {"lin": lin, "ws": ws, "y": new(c["T"], c["n"]) if c["what"] != "packed" else None, "z": [None, None], "zs": [None, None]}
        if c["what"] != "fwd":
            b["dx"] = new(c["T"], c["d"])
            b["dW"] = [new(c["d"], c["n"]) for _ in range(mats)]
            b["db"] = [new(c["n"]) for _ in range(mats)] if c["bias"] else []
            if c["what"] == "packed":
                b["z"], b["zs"] = [p[0] for p in s["packed"]], [p[1] for p in s["packed"]]
            elif c["act"] != "none":
                b["z"] = [new(c["T"], c["n"]) for _ in range(mats)]
        return b

    b = _buffers(s, make)
    two = lambda v: (list(v) + [None, None])[:2]  # noqa: E731
    out = {}
    if c["what"] != "packed":
        B.moe_linear_fwd(b["lin"], s["x"], *two(s["W"]), *two(s["b"]), s["r"], *two(b["z"]), b["y"], b["ws"])
        out["y"] = b["y"]
    if c["what"] != "fwd":
        B.moe_linear_bwd(b["lin"], s["dy"], s["x"], *two(s["W"]), *two(b["z"]), *two(b["zs"]), None, b["dx"], *two(b["dW"]), *two(b["db"]),
                         0, b["ws"])
        out.update(dx=b["dx"], dW=b["dW"], db=b["db"])
    return out


def _own_pack(s):
    from paper_2504_03871_amd import binding as B
    c, v = s["case"], s["v"]
    dt = {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16}[c["dtype"]]
    fmt = B.PACK_E4M3 if c["fmt"] == "e4m3" else B.PACK_I8

    def make():
        codes, scales = B.moe_pack8_bytes(c["rows"], c["width"])
        return [torch.empty(n, dtype=torch.uint8, device="cuda:0") for n in (codes, scales)] + [torch.empty_like(v)]

    codes, scales, back = _buffers(s, make)
    B.moe_pack8(dt, fmt, c["rows"], c["width"], c["width"], v, codes, scales)
    B.moe_unpack8(dt, fmt, c["rows"], c["width"], c["width"], codes, scales, back)
    return back


def _own_saved(s):
    from paper_2504_03871_amd import binding as B
    c, pre = s["case"], s["pre"]
    fmt = B.PACK_E4M3 if c["fmt"] == "e4m3" else B.PACK_I8

    def make():
        dt = {"f32": B.DTYPE_F32, "bf16": B.DTYPE_BF16, "f16": B.DTYPE_F16}[c["dtype"]]
        cfg = B.make_cfg(c["T"], c["d"], c["f"], c["E"], c["k"], dt, B.ACT_SWIGLU if c["act"] == "swiglu" else B.ACT_GELU)
        codes, scales = B.moe_saved_pack8_bytes(cfg)
        return [cfg] + [torch.empty(n, dtype=torch.uint8, device="cuda:0") for n in (codes, scales)] + \
            [torch.empty((pre.shape[0] + 1, *pre.shape[1:]), dtype=pre.dtype, device="cuda:0")]

    cfg, codes, scales, planes = _buffers(s, make)
    B.moe_saved_pack8(cfg, fmt, pre, s["offsets"], s["kept"], None, None, codes, scales)
    B.moe_saved_restore8(cfg, fmt, codes, scales, s["offsets"], s["kept"], None, None, planes)
    return {"pre": [planes[i] for i in range(pre.shape[0])], "hidden": planes[-1]}


_RUN_OWN = {"route": _own_route, "linear": _own_linear, "pack": _own_pack, "saved": _own_saved}


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------

def _nearest8(v, fmt):
    """The value that an element of a [rows, width] matrix in 64 bits stands for after packing: rounded to the nearest multiple
    of its quantum, ties to even."""
    rows, width = v.shape
    u = torch.nn.functional.pad(v, (0, (BLOCK - width % BLOCK) % BLOCK)).reshape(-1, BLOCK)
    largest = u.abs().max(dim=1, keepdim=True).values
    log = torch.floor(torch.log2(largest.clamp(min=1e-300)))
    log = torch.where(torch.exp2(log) > largest, log - 1, log)
    log = torch.where(torch.exp2(log + 1) <= largest, log + 1, log)
    if fmt == "e4m3":
        e = torch.where(largest > 448 * torch.exp2(log - 8), log - 7, log - 8)
    else:
        e = torch.where(largest * 64 >= 127.5 * torch.exp2(log), log + 1, log)
    e = e.clamp(-127, 127)
    q = u / torch.exp2(e)
    if fmt == "e4m3":
        own_log = torch.frexp(q).exponent.double() - 1
        step = torch.exp2(own_log.clamp(min=-6) - 3)
    else:
        step = torch.full_like(q, 1 / 64)
    return (torch.round(q / step) * step * torch.exp2(e)).reshape(rows, -1)[:, :width]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "route":
        lg = s["logits"].double().requires_grad_(True)
        T, E = lg.shape
        shut = torch.isinf(lg.detach())
        if c["score"] == "softmax":
            dead = shut.all(dim=1, keepdim=True)
            prob = torch.softmax(torch.where(dead, torch.zeros_like(lg), lg), dim=1) * (~dead)
        else:
            prob = 1 / (1 + torch.exp(-lg.masked_fill(shut, -700.0)))
        with torch.no_grad():
            key = prob + (0 if s["balance"] is None else s["balance"].double())
            key = key.masked_fill(shut, -math.inf)
            size = E // c["groups"]
            if c["groups"] > 1:
                g = key.view(T, c["groups"], size).sort(dim=2, descending=True).values[:, :, :c["rank"]].sum(dim=2)
                # a group is in where fewer than top_groups are ahead of it
                order = torch.arange(c["groups"], device=g.device)
                ahead = (g[:, None, :] > g[:, :, None]) | ((g[:, None, :] == g[:, :, None]) & (order[None, None, :] < order[None, :, None]))
                key = key.masked_fill((ahead.sum(dim=2) >= c["top_groups"]).repeat_interleave(size, dim=1), -math.inf)
            order = torch.argsort(-key, dim=1, stable=True)[:, :c["k"]]
            live = torch.isfinite(key.gather(1, order))
        w = prob.gather(1, order) * live
        if c["renorm"]:
            w = w / w.sum(dim=1, keepdim=True).clamp(min=1e-300)
        w = w * c["scale"]
        out = {"idx": torch.where(live, order, -1).int(), "w": w.detach()}
        if c["bwd"]:
            grad, = torch.autograd.grad((w * s["d_w"].double()).sum(), lg)
            out["d_logits"] = torch.where(shut, torch.zeros_like(grad), grad)
        return out
    if c["op"] == "linear":
        x, W = s["x"].double(), [w.double() for w in s["W"]]
        td = TYPES[c["dtype"]]
        out = {}
        if c["what"] == "packed":
            value = torch.float8_e4m3fn if c["fmt"] == "e4m3" else torch.int8
            z = [q.view(value).to(torch.float64) * torch.pow(2.0, e.double() - (127 if c["fmt"] == "e4m3" else 133)).repeat_interleave(BLOCK, dim=1)
                 for q, e in s["packed"]]
            z = [v[:, :c["n"]].clamp(-torch.finfo(td).max, torch.finfo(td).max).to(td).double() for v in z]
        else:
            z = [torch.mm(x, w) for w in W]
            z = [v if b is None else v.add_(b.double()) for v, b in zip(z, s["b"])]
        if c["act"] == "gelu":
            phi = torch.special.ndtr(z[0])
            y, slopes = z[0] * phi, [phi + z[0] * torch.exp(-z[0] ** 2 / 2) / math.sqrt(2 * math.pi)]
        elif c["act"] == "swiglu":
            sg = 1 / (1 + torch.exp(-z[0]))
            y, slopes = z[0] * sg * z[1], [z[1] * sg * (1 + z[0] * (1 - sg)), z[0] * sg]
        else:
            y, slopes = z[0], [torch.ones_like(z[0])]
        del z
        if c["what"] != "packed":
            out["y"] = y if s["r"] is None else y + s["r"].double()
        if c["what"] != "fwd":
            g = [s["dy"].double() * sl for sl in slopes]
            del slopes, y
            out["dx"] = sum(torch.mm(a, w.t()) for a, w in zip(g, W))
            out["dW"] = [torch.mm(x.t(), a) for a in g]
            out["db"] = [a.sum(dim=0) for a in g] if c["bias"] else []
        return out
    td = TYPES[c["dtype"]]
    if c["op"] == "pack":
        return _nearest8(s["v"].double(), c["fmt"]).clamp(-torch.finfo(td).max, torch.finfo(td).max).to(td)
    pre = [_nearest8(p.double(), c["fmt"]).clamp(-torch.finfo(td).max, torch.finfo(td).max).to(td) for p in s["pre"]]
    z = [p.double() for p in pre]
    hidden = z[0] * torch.special.ndtr(z[0]) if c["act"] == "gelu" else z[0] / (1 + torch.exp(-z[0])) * z[1]
    return {"pre": pre, "hidden": hidden}
