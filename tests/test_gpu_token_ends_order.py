"""TokenEnds: the lookup whose gradient is asked for is the one that the loss stands above."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx
from paper_2203_05705_b200 import ard
from paper_2203_05705_b200.lm import TokenEnds

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def make():
    ctx = Ctx(1 << 24)
    g = torch.Generator(device="cuda").manual_seed(0)
    ends = TokenEnds(ctx.h, None, 16, 40, 32, torch.randn((40, 32), generator=g, device="cuda"))
    ids, other, labels = (torch.randint(0, 40, (16,), generator=g, device="cuda", dtype=torch.int32) for _ in range(3))
    y, dx = (torch.randn((16, 32), generator=g, device="cuda").to(BF) for _ in range(2))
    return ctx, ends, ids, other, labels, y, dx


@pytest.mark.parametrize("rows", [16, 4])
@pytest.mark.parametrize("behind", ["loss", "backward"])
def test_a_lookup_between_the_loss_and_the_gradient(rows, behind):
    """The other lookup's rows took the place of what the gradient is of: refused, and the table's gradient is left alone."""
    ctx, ends, ids, other, labels, y, dx = make()
    ends.embed(ids)
    ends.loss(y, labels)
    if behind == "loss":
        ends.embed(other[:rows])
    ends.backward()
    if behind == "backward":
        ends.embed(other[:rows])
    before = ends.dtable.clone()
    with pytest.raises(RuntimeError):
        ends.embed_backward(dx[:rows])
    assert torch.equal(ends.dtable, before)
    ends.close()
    ctx.close()


def test_a_share_is_added_once():
    ctx, ends, ids, other, labels, y, dx = make()
    ends.embed(other)            # lookups without a gradient, as in decoding
    ends.embed(ids)
    with pytest.raises(RuntimeError):
        ends.embed_backward(dx)  # before any backward()
    ends.loss(y, labels)
    ends.backward()
    out = ends.dtable.clone()
    ends.embed_backward(dx)
    once = ends.dtable.clone()
    with pytest.raises(RuntimeError):
        ends.embed_backward(dx)
    assert torch.equal(ends.dtable, once)
    share = torch.zeros_like(out)
    ard.ard_embedding_bwd(ctx.h, None, ard.ARD_BF16, 16, 40, 32, 1.0, ids, dx, 32, share, 32, True)
    # a sum of at most 16 rows and what stood there, 17 additions here and 17 there
    assert bool(((once - out - share).abs() <= 34 * 2.0 ** -24 * (out.abs() + 16 * dx.abs().max())).all())
    # and another step goes on as the first did
    ends.embed(ids)
    ends.loss(y, labels)
    ends.backward()
    ends.embed_backward(dx)
    assert torch.equal(ends.dtable, once)
    ends.close()
    ctx.close()
