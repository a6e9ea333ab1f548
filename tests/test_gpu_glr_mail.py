"""The recurrence in clusters of CTAs: maps that arrive from other CTAs, over many rounds and many repeats, beside other work on the device."""
import pytest
import torch

from paper_2203_05705_b200 import ard
from test_gpu_glr import BF16, F32, Case, _both, _ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,T,B,H,lens", [
    (BF16, 8192, 1, 64, None), (BF16, 4100, 1, 256, None), (F32, 3000, 2, 70, [3000, 1111]), (BF16, 2500, 3, 640, [2500, 64, 1300]), (F32, 1500, 9, 256, None)])
def test_many_rounds_many_times(dtype, T, B, H, lens):
    c = Case(dtype, T, B, H, True, lens=lens, seed=T)
    _both(c)
    first = [t.clone() for t in c.outputs()]
    other, busy = torch.cuda.Stream(), torch.randn(2048, 2048, device="cuda")
    same = lambda a, b: torch.equal(torch.nan_to_num(a, 3.0), torch.nan_to_num(b, 3.0))  # noqa: E731
    for k in range(60):
        for t in c.outputs():
            t.fill_(float("nan"))
        other.wait_stream(torch.cuda.current_stream())
        if k % 2:
            with torch.cuda.stream(other):
                busy @ busy
        c.forward(_ctx().h)
        c.backward(_ctx().h)
        assert all(same(a, b) for a, b in zip(first, c.outputs())), k
    assert ard.ard_last_device_status(_ctx().h) == 0
