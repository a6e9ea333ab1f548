"""Layer of a gated linear recurrence with its layer norm, driven through the C ABI.

This module only owns buffers and the order of the calls, as `lstm.LstmLayer` does for its layer:

  xn = layer norm of x (`ard_layer_norm_fwd`)
  Zf, Zg, Zo = xn Wf^T + bf, ... for the kept units (`ard_layer_fwd`): products over all T * B rows at once
  y = alpha s(Zo) c, c the scan along the time axis (`ard_glr_forward`)

and their adjoints in the opposite order (`ard_glr_backward`, `ard_layer_bwd_weight`, `ard_bias_grad`, `ard_layer_bwd_data`,
`ard_layer_norm_bwd`).  The layer's row pattern is that of its units: dropped ones have no gates, no state and no gradient.  With `in_pat`, the
pattern of the layer below, x and its gradient are compact over that layer's kept units, and so are both sides of the products.

The parameters are fp32 with a bf16 copy of the weight for the products; `adamw_rows` hands them to `ard.ard_adamw_step`.
"""
from __future__ import annotations

import torch

from . import ard

BF, F32 = torch.bfloat16, torch.float32


def adamw_entries(parameters, state_bits):
    """Entries for `ard.adamw_tensors` from (parameter, gradient, bf16 copy or None, decay), with states that begin as zeros."""
    rows = []
    for p, g, w, decay in parameters:
        r, c = p.shape if p.dim() == 2 else (1, p.numel())
        row = dict(rows=r, cols=c, p=p, g=g, w=w, weight_decay=decay)
        if state_bits == 8:
            blocks = -(-r * c // ard.ARD_ADAMW_BLOCK)
            row.update(m=torch.zeros(r * c, dtype=torch.uint8, device="cuda"), v=torch.zeros(r * c, dtype=torch.uint8, device="cuda"),
                       m_scale=torch.zeros(blocks, dtype=F32, device="cuda"), v_scale=torch.zeros(blocks, dtype=F32, device="cuda"))
        else:
            row.update(m=torch.zeros(r * c, dtype=F32, device="cuda"), v=torch.zeros(r * c, dtype=F32, device="cuda"))
        rows.append(row)
    return rows


class GlrLayer:
    def __init__(self, ctx, pat, in_pat, T, B, I, H, W, bias, norm_weight, norm_bias, eps=1e-5):
        """pat: row pattern over the H units (K_dim I); in_pat: that of the layer below over its I units, or None.  W: [3H][I], blocks f | g | o along the
        rows, bias [3H], norm_weight, norm_bias [I]; all four are copied to fp32 on the GPU."""
        if tuple(W.shape) != (3 * H, I):
            raise ValueError("W has shape %s, the layer's is %s" % (tuple(W.shape), (3 * H, I)))
        for name, v, n in (("bias", bias, 3 * H), ("norm_weight", norm_weight, I), ("norm_bias", norm_bias, I)):
            if tuple(v.shape) != (n,):
                raise ValueError("%s has shape %s, the layer's is %s" % (name, tuple(v.shape), (n,)))
        self.ctx, self.pat, self.in_pat, self.T, self.B, self.I, self.H, self.eps = ctx, pat, in_pat, T, B, I, H, eps
        new = lambda *shape, dtype=F32: torch.zeros(shape, dtype=dtype, device="cuda")
        self.p_W, self.p_b, self.p_nw, self.p_nb = (v.to("cuda", F32, copy=True).contiguous() for v in (W, bias, norm_weight, norm_bias))
        self.W = self.p_W.to(BF)
        self.dW, self.db, self.dnw, self.dnb = new(3 * H, I), new(3 * H), new(I), new(I)
        self.Xn, self.dXn, self.dX = (new(T * B, I, dtype=BF) for _ in range(3))
        self.dXs = new(T * B, I)
        self.mean, self.rstd = new(T * B), new(T * B)
        self.Z, self.dZ = new(T * B, 3 * H, dtype=BF), new(T * B, 3 * H, dtype=BF)
        self.Y = new(T * B, H, dtype=BF)
        self.S = new(-(-T // ard.ARD_GLR_CHUNK), B, H)
        self.hT, self.dh0 = new(B, H), new(B, H)
        self.h = new(B, H)       # the state of step()
        self.Wk = new(3 * H, I, dtype=BF) if in_pat is not None else self.W   # packed in both dimensions
        self.dWk = new(3 * H, I) if in_pat is not None else self.dW
        self.X = None
        self.X_live = None       # of padded batches
        self.times = torch.arange(T, device="cuda")[:, None]
        self.signs = (1 - 2 * (torch.arange(I, device="cuda") % 2)).to(BF)

    def _columns(self, t, k):
        return t.data_ptr() + k * self.H * t.element_size()

    def _rows(self, t, k):
        return t.data_ptr() + k * self.H * t.shape[1] * t.element_size()

    def pack(self):
        """The weights over the kept units of both patterns, after a new draw or a step of the optimiser.  Nothing to do without in_pat."""
        if self.in_pat is not None:
            for k in range(3):
                ard.ard_compact_weight_cols(self.ctx, self.pat, self.in_pat, ard.ARD_BF16, self.I, self.H, self._rows(self.W, k), self.I,
                                            self._rows(self.Wk, k), self.I)

    def _gates(self, X, rows):
        I, H = self.I, self.H
        ard.ard_layer_norm_fwd(self.ctx, self.in_pat, ard.ARD_BF16, rows, I, self.eps, X, I, self.p_nw, self.p_nb, self.Xn, I, self.mean,
                               self.rstd)
        for k in range(3):
            ard.ard_layer_fwd(self.ctx, self.pat, self.in_pat, ard.ARD_BF16, rows, I, H, 1.0, self.Xn, I, self._rows(self.Wk, k), I,
                              self._columns(self.p_b, k), self._columns(self.Z, k), 3 * H, ard.ARD_OUT_COMPACT)

    def _check(self, name, t, shape, dtype):
        if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or t.device != self.Xn.device or not t.is_contiguous()):
            raise ValueError("%s has to be contiguous %s %s on %s, got %s %s on %s"
                             % (name, dtype, shape, self.Xn.device, t.dtype, tuple(t.shape), t.device))

    def _live(self, X, lens):
        """X without what a padded batch may hold behind its sequences' ends and the norm cannot carry.  Norm and products run over all rows; the gates'
        gradients are zero there, which a product takes away only if what it is multiplied with is finite.  So there values are held within 2^50 and NaN
        becomes zero; with eps = 0, where a row also has to have a variance, padded rows become +1, -1, +1, ..."""
        T, B, I = self.T, self.B, self.I
        if self.X_live is None:
            self.X_live = torch.empty_like(self.Xn)
        x, out = X.view(T, B, I), self.X_live.view(T, B, I)
        rest = self.signs
        if self.eps > 0:
            rest = torch.clamp(x, -2.0 ** 50, 2.0 ** 50, out=out).nan_to_num_(0.0)
        torch.where((self.times < lens).view(T, B, 1), x, rest, out=out)
        return self.X_live

    def forward(self, X, alpha, h0=None, lens=None):
        """X: bf16 [T*B][I] (with in_pat compact), kept until backward().  Returns Y [T*B][H], compact: the kept units' columns are valid.
        h0: fp32 [B][H] or None; lens: int32 [B] or None, rows of X and of backward()'s dY behind a sequence's end may hold anything; the last
        states are in hT."""
        T, B, H = self.T, self.B, self.H
        self._check("X", X, (T * B, self.I), BF)
        self._check("h0", h0, (B, H), F32)
        self._check("lens", lens, (B,), torch.int32)
        self.X, self.lens = X if lens is None else self._live(X, lens), lens
        self.pack()
        self._gates(self.X, T * B)
        z = [self._columns(self.Z, k) for k in range(3)]
        ard.ard_glr_forward(self.ctx, self.pat, ard.ARD_BF16, T, B, H, alpha, z[0], z[1], z[2], 3 * H, lens, h0, self.Y, H, self.hT, self.S)
        return self.Y

    def backward(self, alpha, dY, dhT=None):
        """dY: bf16 [T*B][H], compact.  Returns dX bf16 [T*B][I] (with in_pat compact); the parameters' gradients (zero at dropped units) are in dW,
        db, dnw, dnb, that of h0 in dh0."""
        ctx, pat, ip, T, B, I, H = self.ctx, self.pat, self.in_pat, self.T, self.B, self.I, self.H
        if self.X is None:
            raise RuntimeError("backward() before forward()")
        self._check("dY", dY, (T * B, H), BF)
        self._check("dhT", dhT, (B, H), F32)
        z, dz = ([self._columns(t, k) for k in range(3)] for t in (self.Z, self.dZ))
        ard.ard_glr_backward(ctx, pat, ard.ARD_BF16, T, B, H, alpha, z[0], z[1], z[2], 3 * H, self.lens, self.S, dY, H, dhT, dz[0], dz[1], dz[2],
                             3 * H, self.dh0)
        for k in range(3):
            ard.ard_layer_bwd_weight(ctx, pat, ip, ard.ARD_BF16, ard.ARD_F32, T * B, I, H, 1.0, self.Xn, I, dz[k], 3 * H, 1,
                                     self._rows(self.dWk, k), I, 0 if ip is not None else 1)
            if ip is not None:
                ard.ard_expand_weight_grad_cols(ctx, pat, ip, ard.ARD_F32, I, H, self._rows(self.dWk, k), I, self._rows(self.dW, k), I, 1)
            ard.ard_bias_grad(ctx, pat, ard.ARD_BF16, T * B, H, dz[k], 3 * H, 1, self._columns(self.db, k), 1)
            # the gates' shares of the input's gradient are added up in fp32 and rounded once: they cancel in part, and the norm's adjoint takes means off
            ard.ard_layer_bwd_data(ctx, pat, ip, ard.ARD_BF16, T * B, I, H, 1.0, dz[k], 3 * H,
                                   1 | ard.ARD_FLAG_OUT_F32 | (ard.ARD_FLAG_ACCUMULATE if k else 0), self._rows(self.Wk, k), I, None, 0, self.dXs, I)
        self.dXn.copy_(self.dXs)
        ard.ard_layer_norm_bwd(ctx, ip, ard.ARD_BF16, T * B, I, self.dXn, I, self.X, I, self.p_nw, self.mean, self.rstd, self.dX, I, self.dnw,
                               self.dnb, 1)
        return self.dX

    def step(self, x, alpha=1.0):
        """One token of every sequence: x bf16 [B][I]; h is the state before and after.  Returns y [B][H], compact.  The weights are those that pack()
        or forward() packed last.  Uses the buffers of forward(): not between it and its backward()."""
        self._check("x", x, (self.B, self.I), BF)
        self.X = None
        self._gates(x, self.B)
        z = [self._columns(self.Z, k) for k in range(3)]
        ard.ard_glr_forward(self.ctx, self.pat, ard.ARD_BF16, 1, self.B, self.H, alpha, z[0], z[1], z[2], 3 * self.H, None, self.h, self.Y,
                            self.H, self.h, None)
        return self.Y[:self.B]

    def adamw_rows(self, weight_decay=0.0, state_bits=32):
        """The layer's entries for `ard.adamw_tensors`, with states that begin as zeros; the decay is the weight's alone.  The caller keeps the list."""
        return adamw_entries(((self.p_W, self.dW, self.W, weight_decay), (self.p_b, self.db, None, 0.0), (self.p_nw, self.dnw, None, 0.0),
                              (self.p_nb, self.dnb, None, 0.0)), state_bits)
