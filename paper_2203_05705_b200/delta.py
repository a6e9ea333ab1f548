"""Layer of the gated delta rule with its layer norm, driven through the C ABI.

This module only owns buffers and the order of the calls, as `glr.GlrLayer` does for its layer:

  xn = layer norm of x (`ard_layer_norm_fwd`)
  Z = xn W^T + b, one product over all T * B rows (`ard_layer_fwd`): queries | keys | values | forget gates | write gates side by side
  y, the rule along the time axis (`ard_delta_forward`)

and their adjoints in the opposite order (`ard_delta_backward`, `ard_layer_bwd_weight`, `ard_bias_grad`, `ard_layer_bwd_data`, `ard_layer_norm_bwd`).  With
`in_pat`, the row pattern of the layer below, x and its gradient are compact over that layer's kept units, and the product contracts over them only.

The parameters are fp32 with a bf16 copy of the weight for the products; `adamw_rows` hands them to `ard.ard_adamw_step`.
"""
from __future__ import annotations

import torch

from . import ard
from .glr import adamw_entries

BF, F32 = torch.bfloat16, torch.float32


class DeltaLayer:
    def __init__(self, ctx, in_pat, T, B, I, heads, Dk, Dv, W, bias, norm_weight, norm_bias, eps=1e-5, length_eps=1e-6):
        """in_pat: row pattern of the layer below over its I units, or None.  W: [heads * (2 Dk + Dv + 2)][I], rows q | k | v | f | b, each head after head, bias as
        many, norm_weight, norm_bias [I]; all four are copied to fp32 on the GPU."""
        widths = [heads * n for n in (Dk, Dk, Dv, 1, 1)]
        self.N = N = sum(widths)
        for name, v, shape in (("W", W, (N, I)), ("bias", bias, (N,)), ("norm_weight", norm_weight, (I,)), ("norm_bias", norm_bias, (I,))):
            if tuple(v.shape) != shape:
                raise ValueError("%s has shape %s, the layer's is %s" % (name, tuple(v.shape), shape))
        self.ctx, self.in_pat, self.T, self.B, self.I, self.heads, self.Dk, self.Dv = ctx, in_pat, T, B, I, heads, Dk, Dv
        self.eps, self.length_eps, self.scale = eps, length_eps, Dk ** -0.5
        self.H = heads * Dv
        self.pat = ard.ard_pattern_create(ctx, ard.ARD_ROW, I, N, 0)      # stays dense
        self.at = [sum(widths[:k]) for k in range(5)]
        new = lambda *shape, dtype=F32: torch.zeros(shape, dtype=dtype, device="cuda")
        self.p_W, self.p_b, self.p_nw, self.p_nb = (v.to("cuda", F32, copy=True).contiguous() for v in (W, bias, norm_weight, norm_bias))
        self.W = self.p_W.to(BF)
        self.dW, self.db, self.dnw, self.dnb = new(N, I), new(N), new(I), new(I)
        self.Xn, self.dXn, self.dX = (new(T * B, I, dtype=BF) for _ in range(3))
        self.mean, self.rstd = new(T * B), new(T * B)
        self.ld = -(-N // 8) * 8                 # rows on a grid of 16 bytes
        self.Z, self.dZ = new(T * B, self.ld, dtype=BF), new(T * B, self.ld, dtype=BF)
        self.Y = new(T * B, self.H, dtype=BF)
        self.S = new(-(-T // ard.ARD_DELTA_CHUNK), B, heads, Dk, Dv)
        self.hT, self.dh0 = new(B, heads, Dk, Dv), new(B, heads, Dk, Dv)
        self.h = new(B, heads, Dk, Dv)           # the state of step()
        self.work = new(max(1, ard.ard_delta_work_bytes(T, B, heads, Dk, Dv, True)), dtype=torch.uint8)
        self.Wk = new(N, I, dtype=BF) if in_pat is not None else self.W   # packed over the kept inputs
        self.dWk = new(N, I) if in_pat is not None else self.dW
        self.X = None
        self.live = None                         # of padded batches
        self.times = torch.arange(T, device="cuda")[:, None]     # (here: what a capture makes is not there before its replay)
        self.signs = (1 - 2 * (torch.arange(I, device="cuda") % 2)).to(BF)

    def close(self):
        ard.ard_pattern_destroy(self.pat)

    def _blocks(self, t):
        return [t.data_ptr() + 2 * a for a in self.at]

    def pack(self):
        """The weight over the kept inputs, after a new draw or a step of the optimiser.  Nothing to do without in_pat."""
        if self.in_pat is not None:
            ard.ard_compact_weight_cols(self.ctx, self.pat, self.in_pat, ard.ARD_BF16, self.I, self.N, self.W, self.I, self.Wk, self.I)

    def _project(self, X, rows):
        ard.ard_layer_norm_fwd(self.ctx, self.in_pat, ard.ARD_BF16, rows, self.I, self.eps, X, self.I, self.p_nw, self.p_nb, self.Xn, self.I,
                               self.mean, self.rstd)
        ard.ard_layer_fwd(self.ctx, self.pat, self.in_pat, ard.ARD_BF16, rows, self.I, self.N, 1.0, self.Xn, self.I, self.Wk, self.I, self.p_b,
                          self.Z, self.ld, ard.ARD_OUT_COMPACT)

    def _check(self, name, t, shape, dtype):
        if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or t.device != self.Xn.device or not t.is_contiguous()):
            raise ValueError("%s has to be contiguous %s %s on %s, got %s %s on %s"
                             % (name, dtype, shape, self.Xn.device, t.dtype, tuple(t.shape), t.device))

    def _rule(self, T, lens, h0, Y, hT, S):
        z, need = self._blocks(self.Z), ard.ard_delta_work_bytes(T, self.B, self.heads, self.Dk, self.Dv, False)
        ard.ard_delta_forward(self.ctx, ard.ARD_BF16, T, self.B, self.heads, self.Dk, self.Dv, self.scale, self.length_eps, z[0], self.ld, z[1], self.ld,
                              z[2], self.ld, z[3], z[4], self.ld, lens, h0, Y, self.H, hT, S, self.work if need else None, need)

    def forward(self, X, h0=None, lens=None):
        """X: bf16 [T*B][I] (with in_pat compact), kept until backward().  Returns Y [T*B][heads * Dv].  h0: fp32 [B][heads][Dk][Dv] or None; lens: int32
        [B] or None; rows of X and of backward()'s dY behind a sequence's end may hold anything.  The last states are in hT."""
        self._check("X", X, (self.T * self.B, self.I), BF)
        self._check("h0", h0, tuple(self.hT.shape), F32)
        self._check("lens", lens, (self.B,), torch.int32)
        if lens is not None:      # norm and product run over all rows, whose gradients are zero there: they may not be infinite, or all alike
            if self.live is None:
                self.live = torch.empty_like(X)
            torch.where((self.times < lens).view(-1, 1), X, self.signs, out=self.live)
            X = self.live
        self.X, self.lens = X, lens
        self.pack()
        self._project(X, self.T * self.B)
        self._rule(self.T, lens, h0, self.Y, self.hT, self.S)
        return self.Y

    def backward(self, dY, dhT=None):
        """dY: bf16 [T*B][heads * Dv].  Returns dX bf16 [T*B][I] (with in_pat compact); the parameters' gradients are in dW, db, dnw, dnb, that of h0 in
        dh0."""
        ctx, pat, ip, rows, I, N, ld = self.ctx, self.pat, self.in_pat, self.T * self.B, self.I, self.N, self.ld
        if self.X is None:
            raise RuntimeError("backward() before forward()")
        self._check("dY", dY, (rows, self.H), BF)
        self._check("dhT", dhT, tuple(self.hT.shape), F32)
        z, dz = self._blocks(self.Z), self._blocks(self.dZ)
        ard.ard_delta_backward(ctx, ard.ARD_BF16, self.T, self.B, self.heads, self.Dk, self.Dv, self.scale, self.length_eps, z[0], ld, z[1], ld, z[2], ld, z[3],
                               z[4], ld, self.lens, self.S, dY, self.H, dhT, dz[0], ld, dz[1], ld, dz[2], ld, dz[3], dz[4], ld, self.dh0, self.work,
                               self.work.numel())
        ard.ard_layer_bwd_weight(ctx, pat, ip, ard.ARD_BF16, ard.ARD_F32, rows, I, N, 1.0, self.Xn, I, self.dZ, ld, 1, self.dWk, I, 0 if ip is not None else 1)
        if ip is not None:
            ard.ard_expand_weight_grad_cols(ctx, pat, ip, ard.ARD_F32, I, N, self.dWk, I, self.dW, I, 1)
        ard.ard_bias_grad(ctx, pat, ard.ARD_BF16, rows, N, self.dZ, ld, 1, self.db, 1)
        ard.ard_layer_bwd_data(ctx, pat, ip, ard.ARD_BF16, rows, I, N, 1.0, self.dZ, ld, 1, self.Wk, I, None, 0, self.dXn, I)
        ard.ard_layer_norm_bwd(ctx, ip, ard.ARD_BF16, rows, I, self.dXn, I, self.X, I, self.p_nw, self.mean, self.rstd, self.dX, I, self.dnw, self.dnb, 1)
        return self.dX

    def step(self, x):
        """One token of every sequence: x bf16 [B][I]; h is the state before and after.  Returns y [B][heads * Dv].  The weight is the one that pack() or
        forward() packed last.  Uses the buffers of forward(): not between it and its backward()."""
        self._check("x", x, (self.B, self.I), BF)
        self.X = None
        self._project(x, self.B)
        self._rule(1, None, self.h, self.Y, self.h, None)
        return self.Y[:self.B]

    def adamw_rows(self, weight_decay=0.0, state_bits=32):
        """The layer's entries for `ard.adamw_tensors`, with states that begin as zeros; the decay is the weight's alone.  The caller keeps the list."""
        return adamw_entries(((self.p_W, self.dW, self.W, weight_decay), (self.p_b, self.db, None, 0.0), (self.p_nw, self.dnw, None, 0.0),
                              (self.p_nb, self.dnb, None, 0.0)), state_bits)
