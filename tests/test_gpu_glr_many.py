"""The gated linear recurrence over more sequences, and over more units, than an int counts with a block's added."""
import pytest
import torch

from gpu_helpers import Ctx
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = Ctx(0)
    yield c
    c.close()


@pytest.mark.parametrize("B", [2 ** 30 + 10])
def test_more_than_2_to_the_30_sequences(ctx, B):
    """Of one unit and one step: f = 1/2."""
    g = torch.Generator(device="cuda").manual_seed(1)
    zf, zg = torch.zeros(B, dtype=BF, device="cuda"), torch.randn(B, generator=g, device="cuda", dtype=BF)
    y, hT = torch.full((B + 8,), 7.0, dtype=BF, device="cuda"), torch.full((B + 8,), 7.0, device="cuda")
    ard.ard_glr_forward(ctx.h, None, ard.ARD_BF16, 1, B, 1, 1.0, zf, zg, None, 1, None, None, y, 1, hT, None)
    torch.cuda.synchronize()
    assert ard.ard_last_device_status(ctx.h) == 0
    assert torch.equal(y[:B], zg * 0.5) and bool((y[B:] == 7).all()) and bool((hT[B:] == 7).all())
    assert torch.equal(hT[:B], hT[:B].to(BF).float()) and torch.equal(hT[:B].to(BF), y[:B])


# in pairs of columns, and one by one
@pytest.mark.parametrize("H", [2 ** 31 - 2, 2 ** 31 - 1])
@pytest.mark.parametrize("T", [1, 2])
def test_units_up_to_2_to_the_31(ctx, T, H):
    """Candidates and gradients that are zero but at a few units, the last ones among them."""
    at = torch.tensor([0, 127, 128, 2 ** 30 - 1, H - 300, H - 129, H - 2, H - 1], device="cuda")
    new = lambda: torch.zeros((T, H), dtype=BF, device="cuda")  # noqa: E731
    zf, zg, dy = new(), new(), new()
    zg[0, at] = torch.arange(1.0, 9.0, device="cuda").to(BF)
    dy[0, at[1:]] = 2.0
    y, S = new().fill_(7.0), torch.full((1, H), 7.0, device="cuda")
    ard.ard_glr_forward(ctx.h, None, ard.ARD_BF16, T, 1, H, 1.0, zf, zg, None, H, None, None, y, H, None, S)
    c = torch.arange(1.0, 9.0, device="cuda") / 2
    assert torch.equal(y[0, at].float(), c) and int(torch.count_nonzero(y[0])) == len(at) and int(torch.count_nonzero(S)) == 0
    if T == 2:
        assert torch.equal(y[1, at].float(), c / 2) and int(torch.count_nonzero(y[1])) == len(at)
    dzf, dzg = y.fill_(7.0), new().fill_(7.0)
    ard.ard_glr_backward(ctx.h, None, ard.ARD_BF16, T, 1, H, 1.0, zf, zg, None, H, None, S, dy, H, None, dzf, dzg, None, H, None)
    torch.cuda.synchronize()
    assert ard.ard_last_device_status(ctx.h) == 0
    # dzg = d / 2, dzf = d (0 - zg) / 4
    assert torch.equal(dzg[0, at[1:]].float(), torch.ones(7, device="cuda")) and int(torch.count_nonzero(dzg)) == 7
    assert torch.equal(dzf[0, at[1:]].float(), -c[1:]) and int(torch.count_nonzero(dzf)) == 7
