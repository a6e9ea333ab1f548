"""The gated delta rule's write gates near 1: their gradients keep their digits."""
import numpy as np
import pytest

from gpu_helpers import Ctx, host
from oracle import delta as OD
from test_gpu_delta import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [6, 100])
@pytest.mark.parametrize("zb", [(-4.0, 4.0), (8.0, 18.0), (18.0, 60.0)])
def test_gradients_of_write_gates_near_one(T, zb):
    """dZb = (1 - b) du.u, entry by entry.  du.u is allowed what the other tests allow the gates' gradients, 4 * 2^-12 of its root mean square; 1 - b, which is
    exp(-z) b, a relative error of 2^-16 (the product z log2(e) is rounded: |z| 2^-24 of the exponential, and some units); the output's rounding 2^-8."""
    ctx = Ctx()
    case = Case(T, 2, 2, 32, 40)
    case.fill(case.zb, case.h, case.rng.uniform(*zb, size=(T, 2, 2)))
    case.forward(ctx)
    case.backward(ctx)
    x, dy = case.inputs()
    _, S, u = OD.fwd(*x, np.float32(case.scale), np.float32(case.eps), None, host(case.h0))
    want = OD.bwd(*x, np.float32(case.scale), np.float32(case.eps), S, u, dy, None, host(case.dhT))[4]
    left = OD.logistic(x[4])[1]
    along = want / left
    bound = (2.0 ** -8 + 2.0 ** -16) * np.abs(want) + left * 4 * 2.0 ** -12 * np.sqrt((along ** 2).mean())
    off = np.abs(host(case.dzb).reshape(want.shape) - want)
    assert (off <= bound).all(), float((off / bound).max())
    ctx.close()
