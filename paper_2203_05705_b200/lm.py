"""The two ends of a recurrent language model, driven through the C ABI: tokens to rows below its layers, logits and their loss above them.

Both ends share one table [V][N], as is usual: a token's row goes in, scaled, and the logits are products with all rows.  Buffers and the order of the calls
only:

  x = alpha * table[ids], compact over `in_pat`'s kept units where the input is dropped (`ard_embedding_fwd`)
  ... the layers, any whose last one has N outputs (`glr.GlrLayer`, `delta.DeltaLayer`, `lstm.LstmStack`) ...
  z = y table^T (`ard_layer_fwd`), loss and dz (`ard_distill_loss`)

and backwards dtable = dz^T y (`ard_layer_bwd_weight`), dy (`ard_layer_bwd_data`), and, when the layers have given the gradient of x, its rows added to dtable
(`ard_embedding_bwd`).
"""
from __future__ import annotations

import torch

from . import ard
from .glr import adamw_entries

BF, F32 = torch.bfloat16, torch.float32


class TokenEnds:
    def __init__(self, ctx, in_pat, rows, V, N, table, alpha=1.0):
        """rows: positions of a batch (T * B); table: [V][N], copied to fp32 on the GPU; in_pat: row pattern over the N inputs of the first layer, or None."""
        if tuple(table.shape) != (V, N):
            raise ValueError("table has shape %s, the model's is %s" % (tuple(table.shape), (V, N)))
        self.ctx, self.in_pat, self.rows, self.V, self.N, self.alpha = ctx, in_pat, rows, V, N, float(alpha)
        self.pat = ard.ard_pattern_create(ctx, ard.ARD_ROW, N, V, 0)      # stays dense
        new = lambda *shape, dtype=F32: torch.zeros(shape, dtype=dtype, device="cuda")
        self.p_table = table.to("cuda", F32, copy=True).contiguous()
        self.table, self.dtable = self.p_table.to(BF), new(V, N)
        self.x, self.dy = new(rows, N, dtype=BF), new(rows, N, dtype=BF)
        self.ldz = -(-V // 8) * 8                # rows on a grid of 16 bytes
        self.z = new(rows, self.ldz, dtype=BF)
        self.losses, self.total = new(rows), new(1)
        self.ids = self.y = None
        self.lookups, self.under_loss, self.under_dy = 0, None, None      # which lookup the loss, and then dy, belong to

    def close(self):
        ard.ard_pattern_destroy(self.pat)

    def _check(self, name, t, shape, dtype):
        if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or t.device != self.x.device or not t.is_contiguous()):
            raise ValueError("%s has to be contiguous %s %s on %s, got %s %s on %s"
                             % (name, dtype, shape, self.x.device, t.dtype, tuple(t.shape), t.device))

    def embed(self, ids):
        """ids: int32 [rows], negative: padding.  Returns x bf16 [rows][N] (with in_pat compact).  Fewer rows than the batch's, as decoding has them, are taken too;
        then x has as many.  x is one buffer, which the first layer reads again on its way back: not between a batch's embed() and its embed_backward()."""
        rows = ids.shape[0]
        if rows > self.rows:
            raise ValueError("ids has %d positions, the model %d" % (rows, self.rows))
        self._check("ids", ids, (rows,), torch.int32)
        self.ids, self.lookups = ids, self.lookups + 1
        ard.ard_embedding_fwd(self.ctx, self.in_pat, ard.ARD_BF16, rows, self.V, self.N, self.alpha, ids, self.table, self.N, self.x, self.N)
        return self.x[:rows]

    def logits(self, y):
        """y: bf16 [rows][N], or fewer rows.  Returns z, whose first V columns are the logits.  Not between loss() and its backward()."""
        rows = y.shape[0]
        if rows > self.rows:
            raise ValueError("y has %d rows, the model %d" % (rows, self.rows))
        self._check("y", y, (rows, self.N), BF)
        self.y = None
        ard.ard_layer_fwd(self.ctx, self.pat, None, ard.ARD_BF16, rows, self.N, self.V, 1.0, y, self.N, self.table, self.N, None, self.z, self.ldz,
                          ard.ARD_OUT_COMPACT)
        return self.z[:rows]

    def loss(self, y, labels=None, teacher_ids=None, teacher_logits=None, tau=1.0, hard=1.0, soft=0.0, row_weight=None):
        """The loss of y (kept until backward()) against labels (int32 [rows]) and a teacher's top logits (int32 and fp32 [rows][k]).  Returns total, fp32 [1] on the device; each row's is in
        losses[:rows], and the gradient of the logits takes the logits' place until backward()."""
        rows, k = y.shape[0], 0 if teacher_ids is None else teacher_ids.shape[1]
        self._check("labels", labels, (rows,), torch.int32)
        self._check("teacher_ids", teacher_ids, (rows, k), torch.int32)
        self._check("teacher_logits", teacher_logits, (rows, k), F32)
        self._check("row_weight", row_weight, (rows,), F32)
        if k and teacher_logits is None:
            raise ValueError("teacher_ids without teacher_logits")
        self.logits(y)
        ard.ard_distill_loss(self.ctx, ard.ARD_BF16, rows, self.V, self.z, self.ldz, labels, k, teacher_ids, teacher_logits, k, tau, hard, soft, row_weight,
                             self.losses, self.total, self.z, self.ldz)
        self.y, self.under_loss = y, self.lookups
        return self.total

    def backward(self):
        """Behind loss(): returns dy bf16 [rows][N], what the layers' backward calls start from; the output's share of the table's gradient is in dtable."""
        if self.y is None:
            raise RuntimeError("backward() before loss()")
        rows = self.y.shape[0]
        ard.ard_layer_bwd_weight(self.ctx, self.pat, None, ard.ARD_BF16, ard.ARD_F32, rows, self.N, self.V, 1.0, self.y, self.N, self.z, self.ldz, 1,
                                 self.dtable, self.N, 1)
        ard.ard_layer_bwd_data(self.ctx, self.pat, None, ard.ARD_BF16, rows, self.N, self.V, 1.0, self.z, self.ldz, 1, self.table, self.N, None, 0,
                               self.dy, self.N)
        self.under_dy = self.under_loss
        return self.dy[:rows]

    def embed_backward(self, dx):
        """Behind backward(), once: dx bf16 [rows][N], the gradient of embed()'s x (with in_pat compact), whose share is added to dtable."""
        if self.ids is None:
            raise RuntimeError("embed_backward() before embed()")
        self._check("dx", dx, (self.ids.shape[0], self.N), BF)
        if self.under_dy != self.lookups:
            raise RuntimeError("embed_backward() without a backward() of the last embed()'s loss, or a second time")
        self.under_dy = None
        ard.ard_embedding_bwd(self.ctx, self.in_pat, ard.ARD_BF16, self.ids.shape[0], self.V, self.N, self.alpha, self.ids, dx, self.N, self.dtable, self.N, True)

    def adamw_rows(self, weight_decay=0.0, state_bits=32):
        """The table's entry for `ard.adamw_tensors`."""
        return adamw_entries(((self.p_table, self.dtable, self.table, weight_decay),), state_bits)
