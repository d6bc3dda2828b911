"""A stack of pre-norm MoE blocks from token ids to the loss of the next ones, and the matrices' orthogonalised update.

``TokenMoE``: h = scale * W[ids] -> ``PreNormMoE`` -> cross entropy of the targets over the vocabulary, W_out the
embedding's own matrix (tied) or another. One pass is

  forward : moe_embed_fwd -> the stack's forward -> moe_vocab_loss (the loss, the gradients of the states and of W_out)
  backward: the stack's backward -> moe_embed_bwd (added to W_out's gradient where the two are tied)

The logits are never in memory. In bf16 a tied matrix's gradient is rounded twice, as the loss's part and again when the embedding's
is added to it (in fp32, to the rounded one). A padding token has id < 0 (its state is zero) and a token whose loss does not count
target < 0.

``Muon``: the update of a set of matrices of one size (the experts' W1 or W2, a router's): momentum, moe_orthogonalise,
moe_sgd_update; ``RoundRobinTrainer(update="muon")`` takes it for the experts.
"""
from __future__ import annotations

import math

import torch

from . import _lib as L
from .block import PreNormMoE


class TokenMoE:
    def __init__(self, shape, vocab: int, n_blocks: int, rule=None, tied: bool = True, scale=None, device: str = "cuda", **stack):
        """shape: one batch through one block (``PreNormMoE``'s). scale: of the embedding, default sqrt(d). stack: further
        arguments of ``PreNormMoE``."""
        if vocab < 1:
            raise ValueError("vocab must be >= 1")
        self.shape, self.vocab, self.tied = shape, int(vocab), bool(tied)
        self.net = PreNormMoE(shape, n_blocks, rule, device=device, **stack)
        self.dtype, dt = self.net.dtype, self.net.out.dtype
        T, d = shape.T, shape.d_model
        self.scale = float(scale) if scale is not None else math.sqrt(d)
        self.w_in = torch.empty(vocab, d, dtype=dt, device=device)
        self.w_out = self.w_in if tied else torch.empty_like(self.w_in)
        self.dw_out = torch.empty_like(self.w_in)
        self.dw_in = self.dw_out if tied else torch.empty_like(self.w_in)
        self.x, self.dh = torch.empty(T, d, dtype=dt, device=device), torch.empty(T, d, dtype=dt, device=device)
        self.loss = torch.empty(1, device=device)
        self.token_loss = torch.empty(T, device=device)
        self.ws_bytes = max(L.moe_embed_workspace_size(T, d, vocab), L.moe_vocab_loss_workspace_size(T, d, vocab, self.dtype, True))
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)

    def params(self):
        return {"w_in": self.w_in} if self.tied else {"w_in": self.w_in, "w_out": self.w_out}

    def grads(self):
        return {"w_in": self.dw_in} if self.tied else {"w_in": self.dw_in, "w_out": self.dw_out}

    def _sizes(self):
        return self.shape.T, self.shape.d_model, self.vocab, self.dtype

    def _states(self, ids, s):
        L.moe_embed_fwd(*self._sizes(), ids, self.w_in, self.scale, self.x, stream=s)
        return self.net.forward(self.x, s)

    def evaluate(self, ids, target, weight=None, stream=None):
        """The loss alone -> self.loss, self.token_loss (ids, target [T] i32, weight [T] f32 or None as in moe_vocab_loss)."""
        s = stream if stream is not None else torch.cuda.current_stream()
        h = self._states(ids, s)
        L.moe_vocab_loss(*self._sizes(), h, self.w_out, target, weight, self.loss, self.token_loss, None, None, self.workspace,
                         self.ws_bytes, stream=s)
        return self.loss

    def step(self, ids, target, weight=None, stream=None):
        """One batch: the loss, and the gradients of W (``grads``) and of every block (``net.blocks[i].grads()``)."""
        s = stream if stream is not None else torch.cuda.current_stream()
        h = self._states(ids, s)
        L.moe_vocab_loss(*self._sizes(), h, self.w_out, target, weight, self.loss, self.token_loss, self.dh, self.dw_out,
                         self.workspace, self.ws_bytes, stream=s)
        dx = self.net.backward(self.dh, s)
        L.moe_embed_bwd(*self._sizes(), ids, dx, self.scale, self.tied, self.dw_in, self.workspace, self.ws_bytes, stream=s)
        return self.loss

    def check_status(self, stream=None):
        self.net.check_status(stream)


class Muon:
    """Orthogonalised updates with momentum of ``groups`` matrices [rows, cols] (``w.shape`` = groups, rows, cols, or rows, cols
    for one): w -= lr * sqrt(max(1, rows / cols)) * out, out of moe_orthogonalise. With counts, groups without tokens keep
    their weights and their momentum."""

    def __init__(self, w, beta: float = 0.95, nesterov: bool = True, steps: int = 5):
        self.groups, (self.rows, self.cols) = (w.shape[0] if w.dim() == 3 else 1), w.shape[-2:]
        self.dtype = L.MOE_BF16 if w.dtype == torch.bfloat16 else L.MOE_F32
        self.beta, self.nesterov, self.steps = float(beta), bool(nesterov), int(steps)
        self.scale = math.sqrt(max(1.0, self.rows / self.cols))
        self.momentum = torch.zeros(w.shape, dtype=torch.float32, device=w.device)
        self.out = torch.empty_like(w)
        self.ws_bytes = L.moe_orthogonalise_workspace_size(self.groups, self.rows, self.cols, self.dtype)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=w.device)

    def update(self, w, dw, lr: float, counts=None, w_master=None, stream=None):
        s = stream if stream is not None else torch.cuda.current_stream()
        L.moe_orthogonalise(self.groups, self.rows, self.cols, self.dtype, dw, self.momentum, self.beta, self.nesterov, counts, self.steps,
                            self.scale, self.momentum, self.out, self.workspace, self.ws_bytes, stream=s)
        L.moe_sgd_update(w, self.out, self.groups, self.rows * self.cols, counts, lr, self.dtype, w_master=w_master, stream=s)
