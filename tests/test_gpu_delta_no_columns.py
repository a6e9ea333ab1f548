"""The gated delta rule over heads without keys' or without values' columns."""
import pytest
import torch

from gpu_helpers import Ctx
from paper_2203_05705_b200 import ard
from test_gpu_delta import BF, BF16, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 16, 70])
@pytest.mark.parametrize("Dk,Dv", [(0, 24), (16, 0), (0, 0)])
def test_heads_without_columns(T, Dk, Dv):
    """Sums over no keys, or for no values, are zero: all that has columns is written, and nothing beside it."""
    ctx = Ctx()
    case = Case(T, 3, 2, max(Dk, 1), max(Dv, 1), lens=[T, 0, T // 2], pad=3, off=1)
    case.Dk, case.Dv = Dk, Dv
    case.forward(ctx)
    case.backward(ctx)
    for t, n in ((case.y, Dv), (case.dq, Dk), (case.dk, Dk), (case.dv, Dv), (case.dzf, 1), (case.dzb, 1)):
        assert bool((t[:, :2 * n] == 0).all()) and bool(torch.isnan(t[:, 2 * n:]).all())
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_OK
    ctx.close()


def test_heads_without_columns_from_a_graph():
    ctx = Ctx()
    T, B, h, Dv, ld = 40, 2, 3, 8, 32
    e = torch.randn((T * B, ld), device="cuda").to(BF)
    y = torch.empty((T * B, ld), dtype=BF, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ard.ard_delta_forward(ctx.h, BF16, T, B, h, 0, Dv, 1.0, 0.0, e, ld, e, ld, e, ld, e, e, ld, None, None, y, ld, None, None, None, 0, stream=side.cuda_stream)
    y.fill_(float("nan"))
    graph.replay()
    assert bool((y[:, :h * Dv] == 0).all()) and bool(torch.isnan(y[:, h * Dv:]).all())
    ctx.close()
