"""An MoE block with a shared expert: scored routing, routed experts, a dense expert for every token, 8-bit checkpoints.

    h      = silu(x Wg) * (x Wu)                                   the shared expert, moe_linear_fwd
    out    = sum_j w_j expert_{e_j}(x) + h Wd                      routed output as the down-projection's residual
    e, w   = moe_route_scored(x Wr)                                scores, balance bias, groups, renormalised weights

Owns the buffers and issues the library calls in order, as layer.MoELayer does; nothing is computed here but the update of the
balance bias.  With `fmt` (binding.PACK_E4M3 or PACK_I8) the pre-activations of both experts are kept in 8 bits between forward and
backward, and the planes that they are computed in, `moe.saved` and `pre`, are free in between: several blocks that run one after
the other share one set of them, which is what saves memory (a block alone has its codes on top).
"""
from __future__ import annotations

import torch

from . import binding as B
from .layer import MoELayer


class SharedExpertMoE:
    def __init__(self, T, d_model, d_ff, d_shared, E, k, score, dtype=B.DTYPE_BF16, act=B.ACT_SWIGLU, capacity=0, fmt=B.PACK_NONE,
                 saved=None, pre=None, device="cuda:0"):
        """`score`: binding.make_score(...); `d_shared`: hidden width of the shared expert; `saved`, `pre`: another block's
        moe.saved and pre, with `fmt` only."""
        if fmt == B.PACK_NONE and (saved is not None or pre is not None):
            raise ValueError("without a pack format a block's planes hold what its backward reads: they cannot be shared")
        self.score, self.fmt, self.T = score, fmt, T
        m = self.moe = MoELayer(T, d_model, d_ff, E, k, dtype=dtype, act=act, capacity=capacity, device=device, saved=saved)
        td, dev = m.tdtype, m.device
        e = lambda *s, dtype=td: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.balance = torch.zeros(E, dtype=torch.float32, device=dev)
        # parameters (filled by the caller) and their gradients, fp32
        self.Wg, self.Wu, self.Wd = e(d_model, d_shared), e(d_model, d_shared), e(d_shared, d_model)
        self.dWg, self.dWu, self.dWd = (torch.empty(w.shape, dtype=torch.float32, device=dev) for w in (self.Wg, self.Wu, self.Wd))
        self.up = B.make_linear(T, d_model, d_shared, dtype, B.ACT_SWIGLU, pre=fmt)
        self.down = B.make_linear(T, d_shared, d_model, dtype, B.ACT_NONE)
        self.ws = e(max(256, B.moe_linear_workspace_bytes(self.up), B.moe_linear_workspace_bytes(self.down)), dtype=torch.uint8)
        self.h, self.dh = e(T, d_shared), e(T, d_shared)
        if pre is not None:
            good = lambda p: p is not None and p.shape == (T, d_shared) and p.dtype == td and p.device == m.x.device and p.is_contiguous()  # noqa: E731
            if len(pre) != 2 or not all(map(good, pre)) or pre[0].data_ptr() == pre[1].data_ptr():
                raise ValueError(f"pre must be two contiguous planes [{T}, {d_shared}] of {td} on {dev}")
        self.pre, self.scales = [e(T, d_shared), e(T, d_shared)] if pre is None else list(pre), [None, None]
        if fmt != B.PACK_NONE:
            self.dtype = dtype
            n = B.moe_pack8_bytes(T, d_shared)
            self.codes, self.scales = ([e(b, dtype=torch.uint8) for _ in range(2)] for b in n)
            self.moe_codes, self.moe_scales = (e(b, dtype=torch.uint8) for b in B.moe_saved_pack8_bytes(m.cfg))

    def forward(self):
        """out from moe.x; moe.out is the routed part on the way and the block's output at the end."""
        m = self.moe
        B.moe_route_scored(m.cfg, self.score, m.x, m.Wr, m.bias, self.balance, None, m.logits, m.topk_idx, m.topk_w, m.ws)
        m.dispatch()
        m.ffn_fwd()
        m.combine()
        B.moe_linear_fwd(self.up, m.x, self.Wg, self.Wu, None, None, None, *self.pre, self.h, self.ws)
        B.moe_linear_fwd(self.down, self.h, self.Wd, None, None, None, m.out, None, None, m.out, self.ws)
        if self.fmt != B.PACK_NONE:   # from here on `saved` and `pre` are free
            B.moe_saved_pack8(m.cfg, self.fmt, m.saved, m.offsets, m.kept, m.slice_lo, m.slice_hi, self.moe_codes, self.moe_scales)
            for p, c, s in zip(self.pre, self.codes, self.scales):
                B.moe_pack8(self.dtype, self.fmt, self.T, p.shape[1], p.shape[1], p, c, s)

    def backward(self, accumulate=0):
        """moe.dx and every weight gradient from moe.d_out."""
        m = self.moe
        if self.fmt != B.PACK_NONE:
            B.moe_saved_restore8(m.cfg, self.fmt, self.moe_codes, self.moe_scales, m.offsets, m.kept, m.slice_lo, m.slice_hi, m.saved)
        m.combine_bwd()
        m.ffn_bwd(accumulate)
        m.dispatch_bwd()
        B.moe_route_scored_bwd(m.cfg, self.score, m.x, m.Wr, m.logits, m.topk_idx, m.d_topk_w, m.d_logits, m.dWr, m.dx, m.ws, accumulate)
        B.moe_linear_bwd(self.down, m.d_out, self.h, self.Wd, None, None, None, None, None, None, self.dh, self.dWd, None, None, None,
                         accumulate, self.ws)
        pre = self.pre if self.fmt == B.PACK_NONE else self.codes
        B.moe_linear_bwd(self.up, self.dh, m.x, self.Wg, self.Wu, *pre, *self.scales, m.dx, m.dx, self.dWg, self.dWu, None, None, accumulate,
                         self.ws)

    def step(self):
        self.forward()
        self.backward()

    def update_balance(self, rate):
        """Moves the balance bias towards an even load: up for experts below the mean, down for those above."""
        load = self.moe.counts.float()
        self.balance += rate * torch.sign(load.mean() - load)
