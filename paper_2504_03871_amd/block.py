"""MoE blocks with a shared expert, alone and behind their norm, and in 8 bits for inference: scored routing, routed experts, a dense expert for
every token, 8-bit checkpoints.

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


def _torch_type(dtype):
    return {B.DTYPE_BF16: torch.bfloat16, B.DTYPE_F16: torch.float16}.get(dtype, torch.float32)


def _check_rows(name, t, like, rows, d):
    """A caller's tensor, [rows, d] or split further in front of d: kernels take its address alone, and would read past the end of a smaller one."""
    if (not isinstance(t, torch.Tensor) or t.shape[-1:] != (d,) or t.numel() != rows * d or t.dtype != like.dtype or t.device != like.device
            or not t.is_contiguous()):
        raise ValueError(f"{name} must be [{rows}, {d}] of {like.dtype} on {like.device}, contiguous")


class NormedBlock:
    """A SharedExpertMoE with what a network has in front of it, in training: the residual stream takes in the last block's output, with
    dropout, and the block sees its norm.

        h = residual + dropout(branch)      out = block(gamma h / rms(h))      the next block's branch is out, its residual h

    `stream`: type of the residual stream (None: the block's).  Dropout's mask follows from `seed`, `layer` and the number in `step`, a
    64-bit integer on the GPU that the caller advances once per training step, by a kernel, so that captured steps have masks of
    their own."""

    def __init__(self, block, stream=None, p=0.0, seed=0, layer=0, eps=1e-6):
        if not 0 <= p < 1:
            raise ValueError("dropout's probability must be 0 <= p < 1")
        self.block, m = block, block.moe
        T, d, dtype = m.T, m.d, m.cfg.dtype
        self.norm = B.make_norm(T, d, dtype, stream, eps=eps)
        st = _torch_type(self.norm.stream)
        e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device=m.device)  # noqa: E731
        self.step = torch.zeros(1, dtype=torch.int64, device=m.device)
        self.drop = B.make_drop(p, seed, layer << 32, self.step) if p > 0 else None
        self.gamma, self.dgamma = e(d, dtype=m.tdtype), e(d)      # gamma: filled by the caller
        self.h, self.rstd, self.dh = e(T, d, dtype=st), e(T), e(T, d, dtype=st)
        # without dropout and in one type the branch's gradient is the stream's
        self.d_branch = e(T, d, dtype=m.tdtype) if p > 0 or st != m.tdtype else self.dh
        self.ws = e(max(256, B.moe_norm_bwd_workspace_bytes(self.norm)), dtype=torch.uint8)

    def forward(self, branch, residual=None):
        """(out, h).  branch: [T, d] of the block's type, residual: of the stream's."""
        _check_rows("branch", branch, self.block.moe.x, *self.h.shape)
        if residual is not None:
            _check_rows("residual", residual, self.h, *self.h.shape)
        B.moe_norm_fwd(self.norm, self.drop, branch, residual, self.gamma, self.h, self.rstd, self.block.moe.x, None, None)
        self.block.forward()
        return self.block.moe.out, self.h

    def backward(self, d_h=None, accumulate=0):
        """(gradient of branch, gradient of residual) from block.moe.d_out and `d_h`, what reaches h past this block."""
        if d_h is not None:
            _check_rows("d_h", d_h, self.h, *self.h.shape)
        self.block.backward(accumulate)
        B.moe_norm_bwd(self.norm, self.drop, self.block.moe.dx, self.h, self.gamma, self.rstd, d_h, self.dh,
                       None if self.d_branch is self.dh else self.d_branch, self.dgamma, accumulate, self.ws)
        return self.d_branch, self.dh


class ServedBlock:
    """The same block as it answers requests, T tokens at a time: every product with weights and activations in 8 bits, a scale for each
    column and each token.  `source`: a SharedExpertMoE whose weights are quantised here, once; its router is used as it is.  `capacity`: rows
    kept per expert of these T tokens, 0: all of them; the source's counts rows of a training batch, and does not hold here.
    `stream`: type of the residual stream, as in NormedBlock."""

    def __init__(self, source, gamma, T, eps=1e-6, capacity=0, stream=None):
        m, self.T, self.score = source.moe, T, source.score
        dtype, d, f, fs, td = m.cfg.dtype, m.d, m.f, source.Wg.shape[1], m.tdtype
        if dtype == B.DTYPE_F32:
            raise ValueError("8-bit products of experts have results of 16 bits")
        _check_rows("gamma", gamma, m.x, 1, d)
        e = lambda *s, dtype=td: torch.empty(*s, dtype=dtype, device=m.device)  # noqa: E731
        i32 = lambda *s: e(*s, dtype=torch.int32)  # noqa: E731
        f32 = lambda *s: e(*s, dtype=torch.float32)  # noqa: E731
        i8 = lambda *s: e(*s, dtype=torch.int8)  # noqa: E731

        def quantised(W):
            n, (d_in, d_out) = (W.shape[0], W.shape[1:]) if W.dim() == 3 else (1, W.shape)
            codes, scales = i8(n * d_in * d_out), f32(n, d_out)
            B.moe_quant_weight(dtype, n, d_in, d_out, W, codes, scales)
            return codes, scales

        self.W1, self.W1b, self.W2 = quantised(m.W1), (None, None) if m.W1b is None else quantised(m.W1b), quantised(m.W2)
        self.Wg, self.Wu, self.Wd = (quantised(w) for w in (source.Wg, source.Wu, source.Wd))
        self.Wr, self.bias, self.balance, self.gamma = m.Wr, m.bias, source.balance, gamma
        self.cfg = B.make_cfg(T, d, f, m.E, m.k, dtype, m.act, capacity)
        self.norm = B.make_norm(T, d, dtype, stream, eps=eps)
        self.up, self.down = B.make_linear8(T, d, fs, dtype, B.ACT_SWIGLU), B.make_linear8(T, fs, d, dtype)
        A = T * m.k
        self.h, self.y, self.codes, self.scales, self.out = e(T, d, dtype=_torch_type(self.norm.stream)), e(T, d), i8(T, d), f32(T), e(T, d)
        self.logits, self.topk_idx, self.topk_w = f32(T, m.E), i32(T, m.k), f32(T, m.k)
        self.counts, self.kept, self.offsets, self.row_of, self.src_of, self.y_perm = i32(m.E), i32(m.E), i32(m.E + 1), i32(A), i32(A), e(A, d)
        self.hidden, self.hidden_codes, self.hidden_scales = e(T, fs), i8(T, fs), f32(T)
        self.ws = e(max(256, B.moe_workspace_bytes(self.cfg), B.moe_expert_ffn8_workspace_bytes(self.cfg), B.moe_linear8_workspace_bytes(self.up),
                        B.moe_linear8_workspace_bytes(self.down)), dtype=torch.uint8)

    def forward(self, branch, residual=None):
        """(out, h) as NormedBlock's, without dropout."""
        _check_rows("branch", branch, self.y, *self.h.shape)
        if residual is not None:
            _check_rows("residual", residual, self.h, *self.h.shape)
        B.moe_norm_fwd(self.norm, None, branch, residual, self.gamma, self.h, None, self.y, self.codes, self.scales)
        B.moe_route_scored(self.cfg, self.score, self.y, self.Wr, self.bias, self.balance, None, self.logits, self.topk_idx, self.topk_w, self.ws)
        B.moe_dispatch(self.cfg, None, self.topk_idx, None, None, self.counts, self.kept, self.offsets, self.row_of, self.src_of, None, self.ws)
        B.moe_expert_ffn_fwd8(self.cfg, self.codes, self.scales, *self.W1, *self.W1b, *self.W2, self.src_of, self.offsets, self.kept, None, None,
                              self.y_perm, self.ws)
        B.moe_combine(self.cfg, self.y_perm, self.topk_w, self.topk_idx, self.row_of, self.offsets, self.kept, None, None, self.out)
        B.moe_linear8_fwd(self.up, self.codes, self.scales, *self.Wg, *self.Wu, None, None, None, self.hidden, self.ws)
        B.moe_quant_rows(self.up.dtype, self.T, self.hidden.shape[1], self.hidden.shape[1], self.hidden, self.hidden_codes, self.hidden_scales)
        B.moe_linear8_fwd(self.down, self.hidden_codes, self.hidden_scales, *self.Wd, None, None, None, None, self.out, self.out, self.ws)
        return self.out, self.h
