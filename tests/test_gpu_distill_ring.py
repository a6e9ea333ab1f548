"""The loss over rows that come through the ring: rows that are skipped beside rows whose copy takes its time, rows so long that the ring holds two or one of them,
and the longest."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host
from paper_2203_05705_b200 import ard
from test_gpu_distill import BF16, F32, Case

pytestmark = pytest.mark.gpu


def both(case, V):
    """Twice the same bits, near the definition."""
    ctx = Ctx()
    z = host(case.z)[:, :V]
    case.call(ctx)
    case.check(z)
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_OK
    first = [case.loss.clone(), case.total.clone(), case.dz.clone()]
    if case.dz is not case.z:
        case.call(ctx)
        for a, b in zip(first, (case.loss, case.total, case.dz)):
            assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
    ctx.close()


@pytest.mark.parametrize("V", [9000, 14000, 20000, 33000, 100003])
@pytest.mark.parametrize("k", [0, 20])
@pytest.mark.parametrize("skipped", [lambda r: r % 2 == 0, lambda r: r % 2 == 1, lambda r: r % 4 != 1, lambda r: r % 3 != 0], ids=["even", "odd", "three_of_4", "two_of_3"])
def test_rows_that_are_skipped(V, k, skipped):
    """A CTA's rows come to its teams in turn; a row without weight is there at once, a copy later than that of a row asked for behind it."""
    case = Case(BF16, 148 * 5, V, k, hard=1.0 if k == 0 else 0.5, soft=0.0 if k == 0 else 0.5, weights=False)
    case.labels[:] = np.abs(case.labels)
    n = np.arange(case.rows) // 148          # which of its CTA's rows (without clusters)
    case.w = np.where(skipped(n), 0, 1).astype(np.float32)
    both(case, V)


@pytest.mark.parametrize("dtype,V,rows", [(BF16, 151936, 100), (F32, 120001, 70), (F32, 200000, 70), (F32, 300000, 70), (BF16, 590001, 70)])
@pytest.mark.parametrize("k,how", [(0, dict(hard=1.0)), (1024, dict(hard=0.4, soft=0.6, tau=2.0))], ids=["labels", "both"])
@pytest.mark.parametrize("place", [dict(), dict(off=3, pad=1, off_out=5), dict(in_place=True, off=1)], ids=["apart", "unaligned", "in_place"])
def test_long_rows(dtype, V, rows, k, how, place):
    """Clusters of four and eight, with three slots, two or one; more rows than clusters have teams, so that slots and mail are used again."""
    both(Case(dtype, rows, V, k, **how, **place), V)


@pytest.mark.parametrize("dtype,k,most", [(BF16, 0, 913415), (F32, 0, 456707), (BF16, 1024, 651271), (F32, 1024, 325635)])
def test_the_longest_rows(dtype, k, most):
    """A CTA's part of a row, 1784 * 128 bytes or, beside the entries of two teams, 1272 * 128; eight parts."""
    how = dict(hard=0.5, soft=0.5, tau=1.5) if k else dict()
    both(Case(dtype, 3, most, k, **how), most)
    ctx = Ctx()
    case = Case(dtype, 1, most + 1, k, **how)
    with pytest.raises(ard.ArdError) as e:
        case.call(ctx)
    assert e.value.status == ard.ARD_ERR_UNSUPPORTED
    ctx.close()
