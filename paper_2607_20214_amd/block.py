"""One attention-block training step around the ELSAA operator.

Alg. 1 and Alg. 6 project the block input with dense matrices before the
operator (Q = X W_Q, K = X W_K, V = X W_V) and project the operator's
output after it (O_head W_O).  This module wires those products
(``elsaa_gemm`` on the matrix cores) to the operator (``elsaa_fwd`` /
``elsaa_bwd``) with every attention tensor in the operator's head-major
[B, H, N, d_h] layout, so no reshape copy runs between them:

    forward   QKV = X W_qkv        -> one [1, 3H, N, d_h] buffer (Q, K, V are
                                      its contiguous head ranges)
              O   = ELSAA(Q, K, V)
              Y   = O W_O
    backward  dO  = dY W_O^T       (head-major)
              dW_O = O^T dY
              dQ, dK, dV = ELSAA backward, written into one [1, 3H, N, d_h]
                                      buffer dQKV
              dX   = dQKV W_qkv^T
              dW_qkv = X^T dQKV

Every buffer is allocated once, in the constructor; ``step()`` only
enqueues library calls on torch's current stream.  Like the rest of the
package it only marshals arguments.

``DecayBlock`` and ``DecayServer`` are a block with linear attention with a
decay for each head in ELSAA's place, for models that answer token by token
(ELSAA sorts whole sequences and keeps no state):

    s   = x + residual,  y = norm(s)     (elsaa_rms_norm_fwd)
    QKV = y W_qkv                        -> one [B, 3H, N, d_h] buffer
    O   = decay attention(Q, K, V)       (elsaa_decay_fwd)
    out = O W_O                          the next block's x; s is its residual

``DecayBlock`` is its training step (bfloat16 products, all gradients),
``DecayServer`` answers with 8-bit weights and activations: a prompt through
the chunked form, which leaves each sequence's state, then single tokens.
"""
from __future__ import annotations

import torch

from . import (Buffers, Config, DecayConfig, bwd, decay_bwd, decay_fwd, decay_step, decay_workspace_bytes, fwd, gemm,
               gemm_i8, gemm_plan, gemm_workspace_bytes, quantize_rows, rms_norm_bwd, rms_norm_fwd, rms_norm_i8,
               rms_norm_workspace_bytes)


class AttentionBlock:
    """Buffers and launch sequence of one block step (B = 1).

    X, dY: [N, d_model] bf16; W_qkv: [d_model, 3 d_model] bf16 (columns
    W_Q | W_K | W_V, head h of each in columns h d_h .. (h+1) d_h - 1);
    W_O: [d_model, d_model] bf16; w_sort, w_race: the operator's hash
    projections (float32, per head).
    """

    def __init__(self, cfg: Config, X, dY, W_qkv, W_O, w_sort, w_race):
        if cfg.B != 1:
            raise ValueError("the block step keeps Q, K, V as heads of one [1, 3H, N, d_h] buffer (B = 1)")
        if cfg.dtype != "bf16":
            raise ValueError("the block step runs with bf16 storage")
        dev = X.device
        H, N, d = cfg.H, cfg.N, cfg.d_h
        dm = H * d
        for name, t, shp in (("X", X, (N, dm)), ("dY", dY, (N, dm)), ("W_qkv", W_qkv, (dm, 3 * dm)),
                             ("W_O", W_O, (dm, dm))):
            if t.shape != torch.Size(shp) or t.dtype != torch.bfloat16 or not t.is_contiguous():
                raise ValueError(f"{name}: expected contiguous bf16 {shp}, got {t.dtype} {tuple(t.shape)}")
        self.cfg = cfg
        self.X, self.dY, self.W_qkv, self.W_O = X, dY, W_qkv, W_O
        self.w_sort, self.w_race = w_sort, w_race
        bf, f32 = torch.bfloat16, torch.float32
        self.qkv = torch.empty(1, 3 * H, N, d, dtype=bf, device=dev)
        self.dqkv = torch.empty_like(self.qkv)
        self.do = torch.empty(1, H, N, d, dtype=bf, device=dev)
        self.q, self.k, self.v = self.qkv[:, :H], self.qkv[:, H:2 * H], self.qkv[:, 2 * H:]
        self.bufs = Buffers(cfg, dev, backward=True)
        self.bufs.dq, self.bufs.dk, self.bufs.dv = self.dqkv[:, :H], self.dqkv[:, H:2 * H], self.dqkv[:, 2 * H:]
        self.Y = torch.empty(N, dm, dtype=f32, device=dev)
        self.dW_O = torch.empty(dm, dm, dtype=f32, device=dev)
        self.dX = torch.empty(N, dm, dtype=f32, device=dev)
        self.dW_qkv = torch.empty(dm, 3 * dm, dtype=f32, device=dev)
        o = self.bufs.o
        plans = [gemm_plan(X, W_qkv, out=self.qkv), gemm_plan(o, W_O, out=self.Y),
                 gemm_plan(dY, W_O, trans_b=True, out=self.do), gemm_plan(o, dY, trans_a=True, out=self.dW_O),
                 gemm_plan(self.dqkv, W_qkv, trans_b=True, out=self.dX),
                 gemm_plan(X, self.dqkv, trans_a=True, out=self.dW_qkv)]
        ws = max(gemm_workspace_bytes(p) for p in plans)
        self.gws = torch.empty(max(ws, 256), dtype=torch.uint8, device=dev)
        self.lse = self.d_lr = self.saved = None

    def project(self):
        """QKV = X W_qkv, written head-major into the operator's input buffer."""
        gemm(self.X, self.W_qkv, out=self.qkv, workspace=self.gws)

    def attend_and_backward(self):
        """Everything of the step after the QKV product: the operator forward,
        Y, dO, dW_O, the operator backward into dQKV, dX and dW_qkv."""
        cfg, b = self.cfg, self.bufs
        o, self.lse, self.d_lr, self.saved = fwd(cfg, self.q, self.k, self.v, self.w_sort, self.w_race, buffers=b)
        gemm(o, self.W_O, out=self.Y, workspace=self.gws)
        gemm(self.dY, self.W_O, trans_b=True, out=self.do, workspace=self.gws)
        gemm(o, self.dY, trans_a=True, out=self.dW_O, workspace=self.gws)
        bwd(cfg, self.q, self.k, self.v, self.w_race, self.do, self.lse, self.d_lr, self.saved, buffers=b)
        gemm(self.dqkv, self.W_qkv, trans_b=True, out=self.dX, workspace=self.gws)
        gemm(self.X, self.dqkv, trans_a=True, out=self.dW_qkv, workspace=self.gws)

    def step(self):
        """One training step of the block (forward and backward)."""
        self.project()
        self.attend_and_backward()


def _check_weights(d_model, **weights):
    for name, (t, shape, dtype) in weights.items():
        if t.shape != torch.Size(shape) or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")


class DecayBlock:
    """Training step of a pre-norm block with decay attention.

    cfg: B sequences of N tokens, H heads of d_h (bfloat16; B * N a multiple of
    8); d_model = H d_h.  norm_w float32 [d_model]; W_qkv [d_model, 3 d_model]
    and W_O [d_model, d_model] bfloat16, columns as in AttentionBlock; log_decay
    float32 [H].  x, residual and their gradients are bfloat16 [B * N, d_model].
    lengths (int32 [B] or None) shortens sequences; rows behind them must be finite
    (the products of the weight gradients read them, with zeros).  Buffers are allocated
    once: what forward() and backward() return is overwritten by the next call.
    """

    def __init__(self, cfg: DecayConfig, norm_w, W_qkv, W_O, log_decay, eps: float = 1e-6, lengths=None):
        B, H, N, d = cfg.B, cfg.H, cfg.N, cfg.d_h
        dm = H * d
        if cfg.dtype != "bf16":
            raise ValueError("the block step runs with bf16 storage")
        bf, f32, dev = torch.bfloat16, torch.float32, W_qkv.device
        _check_weights(dm, norm_w=(norm_w, (dm,), f32), W_qkv=(W_qkv, (dm, 3 * dm), bf), W_O=(W_O, (dm, dm), bf),
                       log_decay=(log_decay, (H,), f32))
        self.cfg, self.eps, self.lengths = cfg, eps, lengths
        self.norm_w, self.W_qkv, self.W_O, self.log_decay = norm_w, W_qkv, W_O, log_decay
        rows = lambda: torch.empty(B * N, dm, dtype=bf, device=dev)          # noqa: E731
        self.s, self.y, self.out, self.dy, self.dx = rows(), rows(), rows(), rows(), rows()
        self.qkv = torch.empty(B, 3 * H, N, d, dtype=bf, device=dev)
        self.dqkv = torch.empty_like(self.qkv)
        self.o, self.do = (torch.empty(B, H, N, d, dtype=bf, device=dev) for _ in range(2))
        self.dW_qkv = torch.empty(dm, 3 * dm, dtype=f32, device=dev)
        self.dW_O = torch.empty(dm, dm, dtype=f32, device=dev)
        self.dnorm_w = torch.empty(dm, dtype=f32, device=dev)
        plans = [gemm_plan(self.y, W_qkv, out=self.qkv), gemm_plan(self.o, W_O, out=self.out),
                 gemm_plan(self.out, W_O, trans_b=True, out=self.do), gemm_plan(self.o, self.out, trans_a=True, out=self.dW_O),
                 gemm_plan(self.dqkv, W_qkv, trans_b=True, out=self.dy),
                 gemm_plan(self.y, self.dqkv, trans_a=True, out=self.dW_qkv)]
        # one workspace for all: the calls of a step follow each other on one stream
        ws = max([gemm_workspace_bytes(p) for p in plans] +
                 [decay_workspace_bytes(cfg, False), decay_workspace_bytes(cfg, True), rms_norm_workspace_bytes(B * N, dm)])
        self.ws = torch.empty(max(ws, 256), dtype=torch.uint8, device=dev)

    def _heads(self, t):
        H = self.cfg.H
        return t[:, :H], t[:, H:2 * H], t[:, 2 * H:]

    def forward(self, x, residual=None):
        """(out, s): the block's output and the residual stream x + residual."""
        _, s = rms_norm_fwd(x, self.norm_w, residual=residual, eps=self.eps, out=self.y, out_sum=self.s)
        gemm(self.y, self.W_qkv, out=self.qkv, workspace=self.ws)
        # (zeros behind a sequence's length keep those rows out of the output and of dW_O)
        decay_fwd(self.cfg, *self._heads(self.qkv), self.log_decay, lengths=self.lengths, out=self.o, want_state=False,
                  workspace=self.ws, zero_tail=True)
        gemm(self.o, self.W_O, out=self.out, workspace=self.ws)
        return self.out, s

    def backward(self, dout, ds=None):
        """Gradients behind the last forward(): dx, the gradient of x and of the
        residual alike, and dW_qkv, dW_O, dnorm_w (float32), as a dict.  ds is the residual stream's
        own gradient."""
        gemm(dout, self.W_O, trans_b=True, out=self.do, workspace=self.ws)
        gemm(self.o, dout, trans_a=True, out=self.dW_O, workspace=self.ws)
        decay_bwd(self.cfg, *self._heads(self.qkv), self.log_decay, self.do, lengths=self.lengths,
                  out=self._heads(self.dqkv), workspace=self.ws)
        gemm(self.dqkv, self.W_qkv, trans_b=True, out=self.dy, workspace=self.ws)
        gemm(self.y, self.dqkv, trans_a=True, out=self.dW_qkv, workspace=self.ws)
        rms_norm_bwd(self.s, self.norm_w, self.dy, dsum=ds, eps=self.eps, out=self.dx, out_dweight=self.dnorm_w,
                     workspace=self.ws)
        return {"dx": self.dx, "dW_qkv": self.dW_qkv, "dW_O": self.dW_O, "dnorm_w": self.dnorm_w}


class DecayServer:
    """The block of DecayBlock answering B sequences with 8-bit projections.

    The weights (as DecayBlock takes them) are quantised once, a scale for each
    output channel; activations are quantised by the norm and behind the attention, a
    scale for each token.  prompt() runs the chunked form over padded prompts and
    leaves every sequence's state, token() moves all states on by one token.
    """

    def __init__(self, B: int, H: int, norm_w, W_qkv, W_O, log_decay, eps: float = 1e-6):
        dm = norm_w.numel()
        if dm % H:
            raise ValueError(f"d_model {dm} does not split into {H} heads")
        bf, f32, dev = torch.bfloat16, torch.float32, W_qkv.device
        _check_weights(dm, norm_w=(norm_w, (dm,), f32), W_qkv=(W_qkv, (dm, 3 * dm), bf), W_O=(W_O, (dm, dm), bf),
                       log_decay=(log_decay, (H,), f32))
        self.B, self.H, self.d_h, self.eps = B, H, dm // H, eps
        self.norm_w, self.log_decay = norm_w, log_decay
        self.w_qkv, self.s_qkv = quantize_rows(W_qkv.t().contiguous())
        self.w_o, self.s_o = quantize_rows(W_O.t().contiguous())
        self.state = torch.zeros(B, H, self.d_h, self.d_h, dtype=f32, device=dev)

    def _attend(self, x, residual, N, attention):
        H, dm = self.H, self.H * self.d_h
        if x.shape != (self.B * N, dm):
            raise ValueError(f"x: expected {(self.B * N, dm)}, got {tuple(x.shape)}")
        q8, sc, s = rms_norm_i8(x, self.norm_w, residual=residual, eps=self.eps)
        qkv = torch.empty(self.B, 3 * H, N, self.d_h, dtype=torch.bfloat16, device=x.device)
        gemm_i8(q8, sc, self.w_qkv, self.s_qkv, out=qkv)
        o8, so = quantize_rows(attention(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:]))
        return gemm_i8(o8, so, self.w_o, self.s_o), x if s is None else s

    def prompt(self, x, residual=None, lengths=None, cont: bool = False):
        """(out, s) of prompts x [B * N, d_model]; the states behind them replace
        those kept (cont: the prompts go on from the states kept).  lengths
        (int32 [B] on the GPU) shortens sequences: rows of out behind them are zero."""
        N = x.shape[0] // self.B
        cfg = DecayConfig(self.B, self.H, N, self.d_h)

        def attention(q, k, v):
            return decay_fwd(cfg, q, k, v, self.log_decay, state=self.state if cont else None, lengths=lengths,
                             out_state=self.state, zero_tail=True)[0]

        return self._attend(x, residual, N, attention)

    def token(self, x, residual=None):
        """(out, s) of one token for each sequence, x [B, d_model]."""
        cfg = DecayConfig(self.B, self.H, 1, self.d_h)
        return self._attend(x, residual, 1, lambda q, k, v: decay_step(cfg, q, k, v, self.log_decay, self.state)[0])
