"""GlrLayer: the gates' shares of the input's gradient are added up in fp32."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host
from oracle import pattern as OP
from paper_2203_05705_b200 import ard
from test_gpu_glr_layer_padding import BF, _layer, _random

pytestmark = pytest.mark.gpu
U, HALF = 2.0 ** -24, 2.0 ** -8


@pytest.mark.parametrize("T,B,I,H,drawn,in_drawn", [
    (35, 8, 64, 128, (1, 1), None), (20, 6, 128, 96, (2, 1), (3, 2)), (7, 3, 37, 50, (2, 2), None), (1, 5, 64, 64, (1, 1), (2, 2))])
def test_the_gates_shares_of_the_inputs_gradient(T, B, I, H, drawn, in_drawn):
    """One rounding to bf16 of a sum in fp32, also where the shares cancel: the weight's blocks differ by little but their signs."""
    ctx = Ctx(4 * T * B * 4 * max(I, H) + (1 << 20))
    try:
        ly = _layer(ctx, T, B, I, H, drawn, in_drawn, 1e-5)
        ly.p_W[H:2 * H] = -ly.p_W[:H] * 1.03
        ly.W.copy_(ly.p_W)
        ly.forward(_random(5, T * B, I).to(BF).cuda(), 1.0)
        ly.backward(1.0, (0.1 * _random(6, T * B, H)).to(BF).cuda())
        torch.cuda.synchronize()
        assert ard.ard_last_device_status(ctx.h) == 0
        keep = np.arange(H) if drawn[0] == 1 else OP.row_keep(H, *drawn)
        keep_in = np.arange(I) if in_drawn is None else OP.row_keep(I, *in_drawn)
        W = host(ly.W).reshape(3, H, I)[:, keep][:, :, keep_in]
        dz = host(ly.dZ).reshape(T * B, 3, H)[..., :len(keep)]
        want = np.einsum("rkn,kni->ri", dz, W)
        # 3 n products and their additions; the tensor cores may cut off where others round
        err = (3 * len(keep) + 4) * 2 * U * np.einsum("rkn,kni->ri", np.abs(dz), np.abs(W))
        off = np.abs(host(ly.dXn)[:, :len(keep_in)] - want)
        assert (off <= HALF * np.abs(want) + (1 + HALF) * err + 1e-37).all(), float((off - HALF * np.abs(want) - err).max())
    finally:
        ctx.close()
