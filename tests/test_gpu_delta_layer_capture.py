"""DeltaLayer over a padded batch whose first call is captured, then called eagerly before any replay."""
import pytest
import torch

from gpu_helpers import Ctx
from test_gpu_delta_layer import BF, make

pytestmark = pytest.mark.gpu


def test_first_call_in_a_capture():
    ctx = Ctx(1 << 24)
    T, B, I, heads, Dk, Dv = 20, 3, 64, 2, 16, 32
    seen = []
    for captured in (False, True):
        layer, _ = make(ctx, None, T, B, I, heads, Dk, Dv)
        g = torch.Generator(device="cuda").manual_seed(0)
        X, dY = torch.randn((T * B, I), generator=g, device="cuda").to(BF), torch.randn((T * B, heads * Dv), generator=g, device="cuda").to(BF)
        lens = torch.tensor([20, 0, 7], dtype=torch.int32, device="cuda")
        behind = (torch.arange(T, device="cuda")[:, None] >= lens).view(-1)
        X[behind] = float("nan")
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                layer.forward(X, lens=lens)
                layer.backward(dY)
        y = layer.forward(X, lens=lens).clone()
        seen.append((y, layer.backward(dY).clone(), layer.dW.clone()))
        if captured:
            graph.replay()
            seen.append((layer.Y.clone(), layer.dX.clone(), layer.dW.clone()))
        torch.cuda.synchronize()
        layer.close()
    for other in seen[1:]:
        for a, b in zip(seen[0], other):
            assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
    ctx.close()
