"""A stack of pre-norm MoE blocks with a backward from 8-bit activation checkpoints.

Block i:  h_i = h_{i-1} + m_{i-1},  y = LN_i(h_i),  m_i = MoE_i(y)
Output :  LN_out(h_n + m_n), with h_1 = x + 0.

Every block routes by the gating rule of the stack (``_lib.make_gate_rule``) with a balance bias of
its own in place of an auxiliary loss, and runs its experts through one ``MoELayer`` whose
scratch buffers all blocks share; a pass lends the layer the blocks' weights and tables and takes
them back. What a block keeps for its backward is in 8 bits: its hidden states
h, the experts' [G|U] and their outputs (one byte a value and four per 128 of them), beside the
norm's statistics, the router logits and the picks. The backward makes y and the permuted rows anew
from h, the activations from [G|U], and adds up the gradients in the order of the calls:

  forward : moe_layer_norm_fwd -> moe_route_gate -> moe_dispatch -> moe_expert_ffn_fwd -> moe_ckpt_pack -> moe_combine_fwd
  backward: moe_ckpt_unpack -> moe_layer_norm_fwd -> moe_dispatch -> moe_combine_bwd -> moe_expert_ffn_bwd_ckpt
            -> moe_gate_bwd -> moe_dispatch_bwd -> moe_layer_norm_bwd

It gives gradients and moves the balance biases; the weights' update is the caller's.
"""
from __future__ import annotations

from contextlib import contextmanager

import torch

from . import _lib as L
from .layer import MoELayer


class Checkpoint:
    """8-bit blocks of a [rows, cols] activation."""

    def __init__(self, rows, cols, device):
        self.rows, self.cols = rows, cols
        self.q = torch.empty(rows, cols, dtype=torch.int8, device=device)
        self.scale = torch.empty(rows, L.ckpt_blocks(cols), dtype=torch.float32, device=device)

    def pack(self, dtype, x, stream):
        L.moe_ckpt_pack(self.rows, self.cols, dtype, x, self.q, self.scale, stream=stream)

    def unpack(self, dtype, x, stream):
        L.moe_ckpt_unpack(self.rows, self.cols, dtype, self.q, self.scale, x, stream=stream)

    def nbytes(self):
        return self.q.numel() + 4 * self.scale.numel()


class _Block:
    """Parameters of one block, their gradients, and what it keeps for the backward."""

    def __init__(self, sh, dt, device):
        T, d, E, F, k, P = sh.T, sh.d_model, sh.n_experts, sh.d_ff, sh.top_k, sh.n_parties
        f32 = torch.float32

        def z(*s, dtype=dt):
            return torch.empty(*s, dtype=dtype, device=device)

        self.gamma, self.beta = torch.ones(d, device=device), torch.zeros(d, device=device)
        self.w_router, self.w1, self.w2 = z(P, E, d), z(E, 2 * F, d), z(E, d, F)
        self.balance_bias = torch.zeros(P, E, device=device)
        self.dgamma, self.dbeta = z(d, dtype=f32), z(d, dtype=f32)
        self.dw_router, self.dw1, self.dw2 = torch.empty_like(self.w_router), torch.empty_like(self.w1), torch.empty_like(self.w2)
        self.h = Checkpoint(T, d, device)
        self.gu, self.y_perm = Checkpoint(T * k, 2 * F, device), Checkpoint(T * k, d, device)
        self.mean, self.rstd = z(T, dtype=f32), z(T, dtype=f32)
        self.logits = z(T, E, dtype=f32)
        self.topk_idx, self.topk_w = z(T, k, dtype=torch.int32), z(T, k, dtype=f32)
        self.counts = z(P, E, dtype=torch.int32)

    def params(self):
        return {"gamma": self.gamma, "beta": self.beta, "w_router": self.w_router, "w1": self.w1, "w2": self.w2}

    def grads(self):
        return {"gamma": self.dgamma, "beta": self.dbeta, "w_router": self.dw_router, "w1": self.dw1, "w2": self.dw2}

    def kept_bytes(self):
        small = (self.mean, self.rstd, self.logits, self.topk_idx, self.topk_w, self.counts)
        return sum(c.nbytes() for c in (self.h, self.gu, self.y_perm)) + sum(4 * t.numel() for t in small)


class PreNormMoE:
    def __init__(self, shape, n_blocks: int, rule=None, balance_rate: float = 1e-3, eps: float = 1e-5, device: str = "cuda"):
        """shape: one batch through one block (``MoELayer``'s), no shared experts. rule: default softmax
        over all experts, scale 1. balance_rate: step of the balance bias per backward."""
        if shape.n_shared:
            raise ValueError("the blocks have no shared experts: their activations are not checkpointed")
        if n_blocks < 1:
            raise ValueError("n_blocks must be >= 1")
        self.shape, self.rule = shape, rule if rule is not None else L.make_gate_rule()
        self.eps, self.balance_rate = float(eps), float(balance_rate)
        self.layer = lay = MoELayer(shape, device)
        self.dtype = L.MOE_BF16 if shape.dtype == "bf16" else L.MOE_F32
        T, d = shape.T, shape.d_model
        self.blocks = [_Block(shape, lay.dt, device) for _ in range(n_blocks)]
        self.gamma, self.beta = torch.ones(d, device=device), torch.zeros(d, device=device)
        self.dgamma, self.dbeta = torch.empty(d, device=device), torch.empty(d, device=device)
        self.h_out = Checkpoint(T, d, device)
        self.mean, self.rstd = torch.empty(T, device=device), torch.empty(T, device=device)
        self.out = torch.empty(T, d, dtype=lay.dt, device=device)
        # hidden states in flight, their gradient, dA
        self._h = [torch.empty_like(self.out) for _ in range(2)]
        self._dh = [torch.empty_like(self.out) for _ in range(2)]
        # the normed states and the layer's output: not lay.x and lay.out, in which a caller may hold x
        self._y, self._m = torch.empty_like(lay.x), torch.empty_like(lay.out)
        self._dact = torch.empty_like(lay.act)
        self.ws_bytes = L.moe_layer_norm_workspace_size(T, d)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)

    _LENT = ("x", "out", "w_router", "w1", "w2", "dw1", "dw2", "topk_idx", "topk_w", "counts", "logits")

    @contextmanager
    def _lent(self):
        """The layer for one pass: on the stack's buffers and, block by block (``_use``), their weights and tables; its own
        ones are back afterwards."""
        lay = self.layer
        own = {name: getattr(lay, name) for name in self._LENT}
        lay.x, lay.out = self._y, self._m
        try:
            yield lay
        finally:
            for name, t in own.items():
                setattr(lay, name, t)

    def _use(self, b):
        """The layer runs on block b's weights and tables."""
        lay = self.layer
        lay.w1, lay.w2, lay.dw1, lay.dw2, lay.w_router = b.w1, b.w2, b.dw1, b.dw2, b.w_router
        lay.topk_idx, lay.topk_w, lay.counts, lay.logits = b.topk_idx, b.topk_w, b.counts, b.logits

    def forward(self, x, stream=None):
        """x [T,d] device tensor of the layer's dtype (read only) -> self.out."""
        s = stream if stream is not None else torch.cuda.current_stream()
        with self._lent() as lay:
            return self._forward(x, lay, s)

    def _forward(self, x, lay, s):
        T, d = self.shape.T, self.shape.d_model
        h, m = x, None
        for i, b in enumerate(self.blocks):
            self._use(b)
            into = self._h[i % 2] if m is not None else None
            L.moe_layer_norm_fwd(T, d, self.dtype, h, m, b.gamma, b.beta, self.eps, into, self._y, b.mean, b.rstd, b.h.q,
                                 b.h.scale, stream=s)
            h = into if into is not None else h
            L.moe_route_gate(lay.cfg, self.rule, self._y, b.w_router, None, b.balance_bias, lay._po(), b.logits, lay.probs,
                             b.topk_idx, b.topk_w, b.counts, stream=s)
            lay.dispatch(s)
            lay.ffn_fwd(s)
            b.gu.pack(self.dtype, lay.h_gu, s)
            b.y_perm.pack(self.dtype, lay.y_perm, s)
            lay.combine_fwd(s)
            m = lay.out
        L.moe_layer_norm_fwd(T, d, self.dtype, h, m, self.gamma, self.beta, self.eps, self._h[len(self.blocks) % 2], self.out,
                             self.mean, self.rstd, self.h_out.q, self.h_out.scale, stream=s)
        return self.out

    def backward(self, dout, stream=None):
        """dout [T,d]: the gradient of self.out. Writes every block's gradients and updates its balance
        bias from the batch's counts; returns the gradient of x."""
        s = stream if stream is not None else torch.cuda.current_stream()
        with self._lent() as lay:
            return self._backward(dout, lay, s)

    def _backward(self, dout, lay, s):
        T, d = self.shape.T, self.shape.d_model
        dh = self._dh[0]
        L.moe_layer_norm_bwd(T, d, self.dtype, dout, None, self.h_out.q, self.h_out.scale, self.mean, self.rstd, self.gamma, None,
                             dh, self.dgamma, self.dbeta, self.workspace, self.ws_bytes, stream=s)
        for i in reversed(range(len(self.blocks))):
            b = self.blocks[i]
            self._use(b)
            # y, the permuted rows and the experts' outputs as the checkpoints hold them
            b.h.unpack(self.dtype, self._h[0], s)
            L.moe_layer_norm_fwd(T, d, self.dtype, self._h[0], None, b.gamma, b.beta, self.eps, None, self._y, stream=s)
            lay.dispatch(s)
            b.y_perm.unpack(self.dtype, lay.y_perm, s)
            L.moe_combine_bwd(lay.cfg, dh, lay.y_perm, b.topk_w, lay.slot_of, lay.dy_perm, lay.dtopk_w, stream=s)
            L.moe_expert_ffn_bwd_ckpt(lay.cfg, lay.x_perm, lay.offsets, b.w1, b.w2, b.gu.q, b.gu.scale, lay.dy_perm, self._dact,
                                      lay.act, lay.dh, lay.dx_perm, b.dw1, b.dw2, group_expert=lay.group_expert, stream=s)
            L.moe_gate_bwd(lay.cfg, self.rule, b.logits, b.topk_idx, lay.dtopk_w, None, lay._po(), lay.dlogits, self._y,
                           b.w_router, b.dw_router, None, lay.dx_router, lay.workspace, lay.ws_bytes, stream=s)
            lay.dispatch_bwd(s)
            into = self._dh[1] if dh is self._dh[0] else self._dh[0]
            L.moe_layer_norm_bwd(T, d, self.dtype, lay.dx, None, b.h.q, b.h.scale, b.mean, b.rstd, b.gamma, dh, into, b.dgamma,
                                 b.dbeta, self.workspace, self.ws_bytes, stream=s)
            dh = into
            L.moe_gate_balance(lay.cfg, b.counts, self.balance_rate, b.balance_bias, b.balance_bias, stream=s)
        return dh

    def kept_bytes(self):
        """Device bytes that the blocks keep between their forward and their backward."""
        return sum(b.kept_bytes() for b in self.blocks) + self.h_out.nbytes() + 8 * self.shape.T

    def check_status(self, stream=None):
        self.layer.check_status(stream)
