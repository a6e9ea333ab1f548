"""Layer norm over the widest row that an int can count."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
N = 2 ** 31 - 1
U, HALF = 2.0 ** -24, 2.0 ** -8


def test_a_row_of_2_to_the_31_less_one_columns():
    """Values that are zero but at a few places, the last columns among them, so that every sum is exact."""
    ctx = Ctx(0)
    try:
        at = torch.tensor([0, 255, 256, 2 ** 30 + 5, N - 300, N - 256, N - 2, N - 1], device="cuda")
        sign = torch.tensor([1.0, -1, -1, 1, 1, -1, 1, -1], device="cuda")
        x, y = (torch.zeros(N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        x[at] = (8 * sign).to(x.dtype)
        y.fill_(7.0)
        mean, rstd = torch.full((2,), -1.0, device="cuda"), torch.full((2,), -1.0, device="cuda")
        ard.ard_layer_norm_fwd(ctx.h, None, ard.ARD_BF16, 1, N, 0.0, x, N, None, None, y, N, mean, rstd)
        want = np.sqrt(N / (64.0 * len(at)))           # of the mean square 64 * 8 / N
        assert mean.tolist() == [0.0, -1.0]
        assert abs(float(rstd[0]) - want) <= 8 * U * want and float(rstd[1]) == -1.0
        got = y[at].double().cpu().numpy()
        assert (np.abs(got - 8 * want * sign.double().cpu().numpy()) <= (HALF + 16 * U) * 8 * want).all()
        assert int(torch.count_nonzero(y)) == len(at)

        dy, places = torch.zeros_like(x), torch.tensor([1, N - 1], device="cuda")
        dy[places] = torch.tensor([1.0, -1.0], device="cuda").to(x.dtype)
        y.fill_(7.0)
        ard.ard_layer_norm_bwd(ctx.h, None, ard.ARD_BF16, 1, N, dy, N, x, N, None, mean, rstd, y, N, None, None, 0)
        torch.cuda.synchronize()
        assert ard.ard_last_device_status(ctx.h) == 0
        xh = torch.zeros(2, dtype=torch.float64)
        xh[1] = -8 * want                              # of the last column, and none of column 1
        s2 = float(-xh[1]) / N                         # the mean of e * xh; that of e is zero
        dx = lambda e, h: want * (e - h * s2)  # noqa: E731
        for place, e, h in ((1, 1.0, 0.0), (N - 1, -1.0, -8 * want), (0, 0.0, 8 * want), (N - 256, 0.0, -8 * want)):
            assert abs(float(y[place].double()) - dx(e, h)) <= (HALF + 32 * U) * abs(dx(e, h)) + 32 * U * want * abs(h * s2), place
        assert int(torch.count_nonzero(y)) == len(at) + 1
        with pytest.raises(ard.ArdError) as e:
            ard.ard_layer_norm_bwd(ctx.h, None, ard.ARD_BF16, 1, N, dy, N, x, N, None, mean, rstd, y, N, mean, None, 0)
        assert e.value.status == ard.ARD_ERR_UNSUPPORTED
    finally:
        ctx.close()
