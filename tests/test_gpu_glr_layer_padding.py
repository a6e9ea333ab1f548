"""GlrLayer: what stands in a padded batch behind a sequence's end does not matter."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx
from oracle import pattern as OP
from paper_2203_05705_b200 import ard
from paper_2203_05705_b200.glr import GlrLayer

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _random(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32))


def _layer(ctx, T, B, I, H, drawn, in_drawn, eps):
    pat = ctx.pattern(ard.ARD_ROW, I, H)
    ard.ard_pattern_set(ctx.h, pat, *drawn)
    in_pat = None
    if in_drawn is not None:
        in_pat = ctx.pattern(ard.ARD_ROW, 8, I)
        ard.ard_pattern_set(ctx.h, in_pat, *in_drawn)
    return GlrLayer(ctx.h, pat, in_pat, T, B, I, H, _random(1, 3 * H, I) / I ** 0.5, 0.2 * _random(2, 3 * H), 1 + 0.2 * _random(3, I),
                    0.2 * _random(4, I), eps)


@pytest.mark.parametrize("T,B,I,H,lens,drawn,in_drawn,eps", [
    (35, 4, 64, 128, (35, 1, 0, 20), (1, 1), None, 1e-5), (35, 4, 64, 128, (35, 1, 0, 20), (2, 2), None, 0.0),
    (9, 3, 48, 31, (4, 9, -2), (3, 1), (2, 1), 1e-5), (130, 2, 96, 64, (129, 400), (2, 1), (5, 3), 0.0)])
@pytest.mark.parametrize("rest", [float("nan"), float("inf"), 3e38])
def test_values_behind_a_sequences_end(T, B, I, H, lens, drawn, in_drawn, eps, rest):
    """The same bits whatever the padded rows hold, and a step of the optimiser that is taken."""
    ctx = Ctx(4 * T * B * 4 * max(I, H) + (1 << 20))
    try:
        pad = (np.arange(T)[:, None] >= np.asarray(lens)[None, :]).reshape(-1)
        assert pad.any()
        left = []
        for fill in (None, rest):
            ly = _layer(ctx, T, B, I, H, drawn, in_drawn, eps)
            X, dY = _random(5, T * B, I).to(BF).cuda(), (0.1 * _random(6, T * B, H)).to(BF).cuda()
            if fill is not None:
                X[torch.from_numpy(pad).cuda()] = fill
                dY[torch.from_numpy(pad).cuda()] = fill
            before = X.clone()
            y = ly.forward(X, 2.0, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
            ly.backward(2.0, dY)
            n = len(OP.row_keep(H, *drawn)) if drawn[0] > 1 else H
            ni = I if in_drawn is None else len(OP.row_keep(I, *in_drawn))
            rows = ly.adamw_rows()
            norm = torch.zeros(2, device="cuda")
            table = ard.adamw_tensors(rows)
            ard.ard_grad_norm(ctx.h, table, len(rows), 1.0, norm)
            ard.ard_adamw_step(ctx.h, table, len(rows), 1e-2, 0.9, 0.999, 1e-8, 32, 1, 1, None, None, norm[1:])
            torch.cuda.synchronize()
            assert ard.ard_last_device_status(ctx.h) == 0
            assert torch.equal(before.view(torch.int16), X.view(torch.int16))         # the caller's
            dX = ly.dX[:, :ni]
            assert not bool(dX[torch.from_numpy(pad).cuda()].any())
            left.append([t.clone() for t in (y[:, :n], ly.hT, dX, ly.dW, ly.db, ly.dnw, ly.dnb, ly.dh0, norm, ly.p_W, ly.p_b, ly.p_nw, ly.p_nb)])
            assert all(bool(torch.isfinite(t).all()) for t in left[-1])
        assert all(torch.equal(a, b) for a, b in zip(*left))
    finally:
        ctx.close()
