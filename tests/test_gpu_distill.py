"""ard_distill_loss against the definition in fp64, with the errors that fp32 may make."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host, tdtype
from oracle import distill as OD
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
F32, BF16 = ard.ARD_F32, ard.ARD_BF16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
UNIT = 2.0 ** -24


class Case:
    def __init__(self, dtype, rows, V, k, tau=1.0, hard=1.0, soft=0.0, pad=0, off=0, off_out=None, weights=True, seed=0, scale=2.0, in_place=False):
        self.dtype, self.rows, self.V, self.k, self.tau, self.hard, self.soft = dtype, rows, V, k, tau, hard, soft
        rng = np.random.default_rng(seed + V)
        self.ld = V + pad
        self.z = self.buf(off)
        self.z[:, :V] = torch.from_numpy(rng.normal(size=(rows, V)).astype(np.float32) * scale).to(tdtype(dtype))
        self.labels = rng.integers(0, V, rows).astype(np.int32)
        self.labels[rng.random(rows) < 0.2] = -1
        self.ids = rng.integers(0, V, (rows, k)).astype(np.int32)        # tokens may come up twice
        self.t = (rng.normal(size=(rows, k)) * 2).astype(np.float32)
        self.w = rng.random(rows).astype(np.float32) if weights else None
        if weights:
            self.w[rng.random(rows) < 0.1] = 0
        self.dz = self.z if in_place else self.buf(off if off_out is None else off_out)
        self.loss, self.total = torch.full((rows,), float("nan"), device="cuda"), torch.full((1,), float("nan"), device="cuda")

    def buf(self, off):
        n = self.rows * self.ld
        return torch.full((n + off + 64,), float("nan"), dtype=tdtype(self.dtype), device="cuda")[off:off + n].view(self.rows, self.ld)

    def call(self, ctx, gradient=True):
        put = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
        self.keep = [put(x) for x in (self.labels, self.ids, self.t, self.w)]
        labels, ids, t, w = self.keep
        ard.ard_distill_loss(ctx.h, self.dtype, self.rows, self.V, self.z, self.ld, labels, self.k, ids if self.k else None, t if self.k else None,
                             self.k, self.tau, self.hard, self.soft, w, self.loss, self.total, self.dz if gradient else None, self.ld)

    def check(self, z, gradient=True):
        V, tau = self.V, self.tau
        loss, dz = host(self.loss), host(self.dz)
        half = HALF_STEP[self.dtype]
        total, total_err = 0.0, 0.0
        for r in range(self.rows):
            w = 1.0 if self.w is None else float(self.w[r])
            got = None if w == 0 else OD.row(z[r], int(self.labels[r]), self.ids[r], self.t[r], tau, self.hard, self.soft)
            if got is None:
                assert loss[r] == 0 and (not gradient or (dz[r, :V] == 0).all())
                continue
            L, g, q1, qt, less = got
            # Of an exponential: two units, and its argument's: the difference from the maximum (one), its product with a constant that is rounded itself
            # (two), |argument| times each.  Of a sum: one an addition, of those that one thread makes and of the tree's.
            with np.errstate(invalid="ignore"):
                far1, fart = np.abs(z[r] - z[r].max()), np.abs(z[r] - z[r].max()) / tau
            far1, fart = np.minimum(far1, 1000.0), np.minimum(fart, 1000.0)    # exp(-1000) is zero
            some = 96 + V / 128
            e1, et = (some + 4 * far1) * np.exp(q1) * abs(self.hard), (some + 4 * fart) * np.exp(qt) * abs(self.soft) * tau
            bound = half * np.abs(w * g) + (1 + half) * UNIT * w * (e1 + et + 40 * np.abs(less)) + 1e-37
            if gradient:
                assert (np.abs(dz[r, :V] - w * g) <= bound).all(), (r, float(np.abs(dz[r, :V] - w * g).max()))
            span = float(np.max(np.abs(q1[q1 > -1e30])))
            err = UNIT * (abs(self.hard) + abs(self.soft) * tau * tau) * (some + 16 + 16 * span + (8 * np.abs(self.t[r][np.isfinite(self.t[r])]).max() / tau if self.k else 0))
            assert abs(loss[r] - L) <= err or loss[r] == L, (r, loss[r], L, err)
            total += w * L
            total_err += w * err + abs(w * L) * 2 * UNIT
        assert abs(float(self.total) - total) <= total_err + abs(total) * UNIT + 1e-37 or float(self.total) == total
        if gradient:
            assert bool(torch.isnan(self.dz[:, V:]).all())


SIZES = [(BF16, 3, 1), (F32, 64, 10), (BF16, 33, 32), (BF16, 40, 33), (F32, 9, 127), (BF16, 5, 128), (BF16, 37, 129), (F32, 20, 1000), (BF16, 5, 4096),
         (F32, 6, 4100), (BF16, 7, 8800), (BF16, 5, 16390), (F32, 4, 16500), (BF16, 3, 32768), (BF16, 3, 33001), (F32, 2, 70001), (BF16, 2, 100003)]


@pytest.mark.parametrize("dtype,rows,V", SIZES)
@pytest.mark.parametrize("kind", ["labels", "teacher", "both", "both_tau", "both_2", "both_4"])
def test_sizes(dtype, rows, V, kind):
    ctx = Ctx()
    how = {"labels": dict(k=0), "teacher": dict(k=min(5, 2 * V), tau=3.0, hard=0.0, soft=1.0), "both": dict(k=16, tau=1.0, hard=0.5, soft=0.25),
           "both_tau": dict(k=70, tau=0.7, hard=0.3, soft=0.6), "both_2": dict(k=3, tau=2.0, hard=0.4, soft=0.6),
           "both_4": dict(k=130, tau=4.0, hard=0.4, soft=0.6)}[kind]
    case = Case(dtype, rows, V, pad=V % 3, off=V % 5, **how)
    z = host(case.z)[:, :V]
    case.call(ctx)
    case.check(z)
    first = case.dz.clone()
    case.call(ctx)
    assert torch.equal(first[:, :V], case.dz[:, :V])
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_OK
    ctx.close()


@pytest.mark.parametrize("dtype,rows,V,k", [(BF16, 9000, 12, 3), (F32, 5000, 100, 0), (BF16, 3000, 520, 8), (BF16, 1500, 4500, 4)])
def test_more_rows_than_a_grid(dtype, rows, V, k):
    ctx = Ctx()
    case = Case(dtype, rows, V, k=k, tau=2.0, hard=0.5, soft=0.5 if k else 0.0)
    z = host(case.z)
    case.call(ctx)
    case.check(z)
    ctx.close()


@pytest.mark.parametrize("V", [20, 300, 9000, 40000])
@pytest.mark.parametrize("off_out,pad", [(0, 0), (1, 1), (3, 0)])
def test_gradient_in_place_or_elsewhere_or_not_at_all(V, off_out, pad):
    ctx = Ctx()
    how = dict(k=9, tau=1.5, hard=0.5, soft=0.5, pad=pad)
    case = Case(BF16, 12, V, off_out=off_out, **how)
    z = host(case.z)[:, :V]
    case.call(ctx)
    case.check(z)
    inside = Case(BF16, 12, V, off=off_out, in_place=True, **how)
    inside.call(ctx)
    inside.check(z)
    if off_out == 0:    # (a row's sums are cut by where it begins)
        assert torch.equal(inside.dz[:, :V], case.dz[:, :V])
    without = Case(BF16, 12, V, **how)
    without.call(ctx, gradient=False)
    without.check(z, gradient=False)
    assert torch.equal(without.loss, case.loss) and bool(torch.isnan(without.dz).all())
    ctx.close()


@pytest.mark.parametrize("dtype,V", [(F32, 24), (BF16, 90), (BF16, 1000), (F32, 9000), (BF16, 50000)])
def test_masked_classes(dtype, V):
    """Logits of -infinity and of the type's lowest value; rows of nothing else."""
    ctx = Ctx()
    lowest = torch.finfo(tdtype(dtype)).min
    case = Case(dtype, 6, V, k=6, tau=2.0, hard=0.5, soft=0.5, weights=False)
    case.labels[:] = np.arange(6)
    case.ids[:] = np.arange(6)
    case.z[0, V // 2:V] = float("-inf")
    case.z[1, V // 2:V] = lowest
    case.z[2, 10:V] = float("-inf")
    case.z[3, :V] = lowest              # every class as likely as any other
    case.t[4, 2:] = float("-inf")
    case.ids[5, :] = -1
    z = host(case.z)[:, :V]
    case.call(ctx)
    case.check(z)
    # a label without probability, and rows that say nothing
    case.z[0, 0] = float("-inf")
    case.z[1, :V] = float("-inf")
    case.z[2, 3] = float("nan")
    case.labels[3], case.ids[3] = -1, -5
    case.labels[4], case.t[4] = -1, float("-inf")
    case.z[3, 5] = case.z[4, 5] = float("nan")    # not read
    case.call(ctx)
    loss, dz = host(case.loss), host(case.dz)[:, :V]
    assert loss[0] == np.inf and np.isfinite(dz[0]).all()
    assert np.isnan(loss[1]) and np.isnan(loss[2]) and np.isnan(dz[2]).all()
    assert (loss[3:5] == 0).all() and (dz[3:5] == 0).all()
    ctx.close()


def test_large_logits_keep_their_differences():
    ctx = Ctx()
    case = Case(F32, 8, 2000, k=4, tau=1.0, hard=1.0, soft=1.0, weights=False)
    case.z += 8192.0
    z = host(case.z)
    case.call(ctx)
    case.check(z)
    ctx.close()


def test_weight_zero_is_not_read():
    ctx = Ctx()
    case = Case(BF16, 5, 700, k=3, tau=1.0, hard=1.0, soft=1.0)
    case.w[:] = [0, 1, 0, 2, 0]
    case.z[[0, 2, 4]] = float("nan")
    z = host(case.z)
    case.call(ctx)
    case.check(z)
    ctx.close()


@pytest.mark.parametrize("V", [50, 600])
def test_tokens_out_of_range_are_reported_and_count_as_absent(V):
    for what in ("labels", "ids"):
        ctx = Ctx()
        case = Case(BF16, 7, V, k=3, tau=2.0, hard=1.0, soft=1.0)
        case.w[:] = 1
        getattr(case, what).flat[4] = V if what == "labels" else 2 ** 31 - 1
        z = host(case.z)
        case.call(ctx)
        case.check(z)
        assert ard.ard_last_device_status(ctx.h) == ard.ARD_ERR_INVALID_ARG
        ctx.close()


@pytest.mark.parametrize("V", [12, 777])
def test_gradient_against_differences(V):
    ctx = Ctx()
    case = Case(F32, 4, V, k=5, tau=2.0, hard=0.7, soft=0.4, weights=False)
    case.call(ctx)
    z, g = host(case.z), host(case.dz)
    rng = np.random.default_rng(5)
    d = rng.normal(size=z.shape)
    h = 1e-4
    total = lambda x: sum(0.0 if got is None else got[0] for got in (OD.row(x[r], int(case.labels[r]), case.ids[r], case.t[r], 2.0, 0.7, 0.4) for r in range(4)))  # noqa: E731
    slope = (total(z + h * d) - total(z - h * d)) / (2 * h)
    # the difference quotient's own error is h^2 / 6 times a third derivative, at most the logits' spread cubed
    assert abs(slope - (g * d).sum()) <= 1e-6 * (1 + np.abs(d).max() ** 3)
    ctx.close()


def test_more_than_2_to_the_32_elements():
    V, rows = 70000, 62000
    ctx = Ctx()
    z = torch.zeros((rows, V), dtype=torch.bfloat16, device="cuda")
    labels = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    labels[0], labels[-1] = 1, V - 1
    loss, total = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
    ard.ard_distill_loss(ctx.h, BF16, rows, V, z, V, labels, 0, None, None, 0, 1.0, 1.0, 0.0, None, loss, total, z, V)
    assert abs(float(loss[-1]) - np.log(V)) <= 1e-5 and abs(float(total) - 2 * np.log(V)) <= 2e-5
    assert float(z[-1, V - 1]) == -1.0 and abs(float(z[-1, 0]) * V - 1) <= 2.0 ** -8
    assert int(torch.count_nonzero(z[1:-1])) == 0
    ctx.close()


def test_no_rows():
    ctx = Ctx()
    total = torch.full((1,), 7.0, device="cuda")
    e = torch.empty(1, device="cuda")
    ard.ard_distill_loss(ctx.h, F32, 0, 10, e, 10, None, 0, None, None, 0, 1.0, 1.0, 0.0, None, e, total, None, 0)
    assert float(total) == 0.0
    ctx.close()


@pytest.mark.parametrize("V", [40, 9000, 60000])
def test_on_a_stream_and_from_a_graph(V):
    """Captured on another stream than the current one and replayed on other logits: scratch and counters are as the call before left them."""
    ctx = Ctx()
    case = Case(BF16, 300, V, 5, tau=2.0, hard=0.6, soft=0.4, weights=False)
    case.call(ctx)
    labels, ids, t, w = case.keep
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        for _ in range(2):           # the second one begins where the first one ended
            ard.ard_distill_loss(ctx.h, BF16, case.rows, V, case.z, V, labels, 5, ids, t, 5, 2.0, 0.6, 0.4, w, case.loss, case.total, case.dz, V,
                                 stream=side.cuda_stream)
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        case.z.copy_(torch.randn(case.z.shape, generator=g, device="cuda") * 2)
        case.total.fill_(float("nan"))
        graph.replay()
        case.check(host(case.z))
    ctx.close()


@pytest.mark.parametrize("dtype,rows,V,k", [(BF16, 40, 80, 80), (F32, 9, 100, 128), (BF16, 20, 700, 65), (F32, 7, 900, 128), (BF16, 6, 2000, 100), (BF16, 5, 4096, 128),
                                            (F32, 3, 2040, 90), (BF16, 5, 300, 129)])
@pytest.mark.parametrize("tau", [1.0, 2.7])
def test_many_entries_over_short_rows(dtype, rows, V, k, tau):
    ctx = Ctx()
    case = Case(dtype, rows, V, k, tau=tau, hard=0.4, soft=0.6, pad=1, off=1)
    case.call(ctx)
    case.check(host(case.z[:, :V]))
    ctx.close()
