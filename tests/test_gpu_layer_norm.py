"""ard_layer_norm_fwd / ard_layer_norm_bwd against the fp64 statement: types, odd sizes, leading dimensions and alignments, kept columns."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host, tdtype
from oracle import layer_norm as ON
from oracle import pattern as OP
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
F32, BF16 = ard.ARD_F32, ard.ARD_BF16
U = 2.0 ** -24
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}      # of the type of an output, relative


def _buffer(rows, n, ld, dtype, off, values=None):
    """[rows][ld] that starts `off` elements into its memory, NaN outside the values."""
    t = torch.full((rows * ld + off + 64,), float("nan"), dtype=tdtype(dtype), device="cuda")[off:off + rows * ld].view(rows, ld)
    if values is not None:
        t[:, :n] = torch.from_numpy(values).to(tdtype(dtype))
    return t


def _run(ctx, pat, dtype, rows, N, dp=1, b=1, ld=(0, 0, 0, 0), off=0, affine=True, eps=1e-5, shift=0.3, zero_fill=1, seed=0):
    keep = np.arange(N) if dp == 1 else OP.row_keep(N, dp, b)
    n = len(keep)
    rng = np.random.default_rng(seed)
    X = _buffer(rows, n, N + ld[0], dtype, off, (rng.normal(size=(rows, n)) * 1.5 + shift).astype(np.float32))
    dY = _buffer(rows, n, N + ld[1], dtype, off, (rng.normal(size=(rows, n)) * 0.3).astype(np.float32))
    Y, dX = _buffer(rows, n, N + ld[2], dtype, off), _buffer(rows, n, N + ld[3], dtype, off)
    weight = torch.from_numpy((rng.normal(size=N) * 0.2 + 1).astype(np.float32)).cuda() if affine else None
    bias = torch.from_numpy((rng.normal(size=N) * 0.2).astype(np.float32)).cuda() if affine else None
    mean, rstd, dw, db = (torch.full((k,), float("nan"), device="cuda") for k in (rows, rows, N, N))
    ard.ard_layer_norm_fwd(ctx, pat, dtype, rows, N, eps, X, N + ld[0], weight, bias, Y, N + ld[2], mean, rstd)
    ard.ard_layer_norm_bwd(ctx, pat, dtype, rows, N, dY, N + ld[1], X, N + ld[0], weight, mean, rstd, dX, N + ld[3], dw, db, zero_fill)
    x, dy = host(X)[:, :n], host(dY)[:, :n]
    w, bb = (host(weight)[keep], host(bias)[keep]) if affine else (np.ones(n), np.zeros(n))
    y0, mean0, rstd0 = ON.fwd(x, w, bb, eps)
    dx0, dw0, db0 = ON.bwd(dy, x, w, mean0, rstd0)
    # fp32 sums: at most n / 32 additions in a lane and a tree of ten behind them; K covers that and the handful of operations around
    K = 24 + n / 32
    size = np.abs(x).max(axis=1)
    e_mean = K * U * size
    assert (np.abs(host(mean) - mean0) <= e_mean).all()
    # d = x - mean is off by e_mean and a unit of x; the variance doubles that relative to the deviation
    e_rstd = rstd0 * (K * U + 2 * rstd0 * (e_mean + U * size))
    assert (np.abs(host(rstd) - rstd0) <= e_rstd).all()
    xh = (x - mean0[:, None]) * rstd0[:, None]
    e_xh = np.abs(xh) * (e_rstd / rstd0 + 4 * U)[:, None] + (rstd0 * (e_mean + U * size))[:, None]
    tol = HALF_STEP[dtype] * np.abs(y0) + 1.01 * (e_xh * np.abs(w) + 4 * U * (np.abs(xh * w) + np.abs(bb)))
    assert (np.abs(host(Y)[:, :n] - y0) <= tol).all()
    e = np.abs(dy * w)
    m1, m2 = e.mean(axis=1, keepdims=True), (e * np.abs(xh)).mean(axis=1, keepdims=True)
    e_m2 = K * U * m2 + (e * e_xh).mean(axis=1, keepdims=True)
    inner = e + m1 + np.abs(xh) * m2
    tol = rstd0[:, None] * ((K * U) * (e + m1) + e_xh * m2 + np.abs(xh) * e_m2 + 6 * U * inner) + np.abs(dx0) * (e_rstd / rstd0)[:, None]
    tol = HALF_STEP[dtype] * np.abs(dx0) + 1.01 * tol
    assert (np.abs(host(dX)[:, :n] - dx0) <= tol).all()
    Kr = 24 + rows / 4              # rows: at most a quarter of them one after the other
    dws, dbs = host(dw), host(db)
    assert (np.abs(dws[keep] - dw0) <= Kr * U * (np.abs(dy) * np.abs(xh)).sum(axis=0) + (np.abs(dy) * e_xh).sum(axis=0)).all()
    assert (np.abs(dbs[keep] - db0) <= Kr * U * np.abs(dy).sum(axis=0)).all()
    for t, ldt in ((Y, N + ld[2]), (dX, N + ld[3])):        # nothing behind the columns
        assert bool(torch.isnan(t[:, n:]).all())
    dropped = np.setdiff1d(np.arange(N), keep)
    for g in (dws, dbs):
        assert (g[dropped] == 0).all() if zero_fill else np.isnan(g[dropped]).all()
    return Y, dX, dw, db


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 31), (64, 256), (129, 255), (33, 1000), (7, 1024), (300, 1025), (64, 2048), (20, 4100), (9, 8192), (5, 8200),
          (3, 16384), (2, 16400), (2, 40000), (2000, 64), (4097, 24), (700, 1500)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,N", SHAPES)
def test_shapes(dtype, rows, N):
    ctx = Ctx(0)
    try:
        _run(ctx.h, None, dtype, rows, N, seed=rows + N)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,N,ld,off", [(40, 64, (8, 16, 24, 32), 0), (40, 65, (7, 0, 1, 2), 0), (40, 64, (0, 0, 0, 0), 1), (13, 520, (0, 8, 0, 8), 8),
                                           (13, 2046, (2, 2, 2, 2), 0), (50, 1500, (4, 4, 4, 4), 0), (30, 96, (1, 0, 0, 0), 0),
                                           (30, 96, (0, 0, 0, 3), 0), (11, 8192, (0, 8, 0, 0), 0)])
def test_strides_and_alignment(dtype, rows, N, ld, off):
    ctx = Ctx(0)
    try:
        _run(ctx.h, None, dtype, rows, N, ld=ld, off=off, seed=N)
        _run(ctx.h, None, dtype, rows, N, ld=ld, off=off, seed=N, affine=False, eps=0.5)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,N,dp,b,ld", [(700, 1500, 2, 2, 4), (64, 2048, 3, 1, 0), (17, 100, 7, 5, 0), (9, 40, 40, 40, 0), (33, 8192, 2, 1, 0),
                                            (33, 4096, 16, 16, 8), (128, 256, 1, 1, 0), (5, 16384, 5, 3, 0), (12, 33, 32, 2, 7)])
def test_kept_columns(dtype, rows, N, dp, b, ld):
    ctx = Ctx(0)
    try:
        pat = ctx.pattern(ard.ARD_ROW, 16, N)
        ard.ard_pattern_set(ctx.h, pat, dp, b)
        _run(ctx.h, pat, dtype, rows, N, dp, b, ld=(ld,) * 4, seed=N + dp)
        _run(ctx.h, pat, dtype, rows, N, dp, b, ld=(ld,) * 4, zero_fill=0, seed=N + dp + 1)
    finally:
        ctx.close()


def test_a_large_mean_does_not_spoil_the_variance():
    ctx = Ctx(0)
    try:
        _run(ctx.h, None, F32, 50, 768, shift=1000.0, seed=1)
        _run(ctx.h, None, F32, 50, 1001, shift=-4000.0, seed=2)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_row_that_is_not_finite_spoils_itself_alone(dtype):
    ctx = Ctx(0)
    try:
        rows, N = 70, 512
        X, dY = torch.randn(rows, N, device="cuda").to(tdtype(dtype)), torch.randn(rows, N, device="cuda").to(tdtype(dtype))
        out = []
        for bad in (False, True):
            if bad:
                X[13, 5], X[40, 500] = float("nan"), float("inf")
            Y, dX = torch.empty_like(X), torch.empty_like(X)
            mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            ard.ard_layer_norm_fwd(ctx.h, None, dtype, rows, N, 1e-5, X, N, None, None, Y, N, mean, rstd)
            ard.ard_layer_norm_bwd(ctx.h, None, dtype, rows, N, dY, N, X, N, None, mean, rstd, dX, N, None, None, 0)
            out.append((Y, dX))
        fine = [r for r in range(rows) if r not in (13, 40)]
        for a, b in zip(*out):
            assert torch.equal(a[fine], b[fine]) and bool(torch.isnan(b[[13, 40]]).all())
    finally:
        ctx.close()


@pytest.mark.parametrize("rows,N", [(0, 16), (5, 0), (0, 0)])
def test_nothing_to_do(rows, N):
    ctx = Ctx(0)
    try:
        x, y = torch.ones(64, device="cuda"), torch.full((64,), 7.0, device="cuda")
        dw, db = torch.full((16,), 7.0, device="cuda"), torch.full((16,), 7.0, device="cuda")
        ard.ard_layer_norm_fwd(ctx.h, None, F32, rows, N, 1e-5, x, 16, None, None, y, 16, None, None)
        ard.ard_layer_norm_bwd(ctx.h, None, F32, rows, N, x, 16, x[32:], 16, None, x, x, y, 16, dw, db, 1)
        assert bool((y == 7).all())
        for g in (dw, db):                   # a sum over no rows is zero
            assert bool((g[:N] == 0).all()) and bool((g[N:] == 7).all())
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype,rows,N", [(F32, 200, 384), (BF16, 333, 1024), (BF16, 50, 1501)])
def test_outputs_that_are_not_wanted(dtype, rows, N):
    ctx = Ctx(0)
    try:
        X, dY = torch.randn(rows, N, device="cuda").to(tdtype(dtype)), torch.randn(rows, N, device="cuda").to(tdtype(dtype))
        w = torch.randn(N, device="cuda")
        Y, mean, rstd = torch.empty_like(X), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        ard.ard_layer_norm_fwd(ctx.h, None, dtype, rows, N, 1e-5, X, N, w, None, Y, N, mean, rstd)
        Y2 = torch.empty_like(X)
        ard.ard_layer_norm_fwd(ctx.h, None, dtype, rows, N, 1e-5, X, N, w, None, Y2, N, None, None)
        assert torch.equal(Y, Y2)
        full = [torch.empty_like(X), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")]
        ard.ard_layer_norm_bwd(ctx.h, None, dtype, rows, N, dY, N, X, N, w, mean, rstd, full[0], N, full[1], full[2], 0)
        for want in ([1, 0, 0], [0, 1, 0], [0, 0, 1], [0, 1, 1], [1, 1, 0], [0, 0, 0]):
            got = [torch.full_like(t, 7.0) for t in full]
            a = [t if k else None for t, k in zip(got, want)]
            ard.ard_layer_norm_bwd(ctx.h, None, dtype, rows, N, dY, N, X, N, w, mean, rstd, a[0], N, a[1], a[2], 0)
            for t, f, k in zip(got, full, want):
                assert torch.equal(t, f) if k else bool((t == 7).all())
    finally:
        ctx.close()


def test_patterns_of_other_kinds_are_refused():
    ctx, other = Ctx(0), Ctx(0)
    try:
        x = torch.zeros(64 * 64, device="cuda")
        y = torch.zeros(64 * 64, device="cuda")
        pats = ((ctx.pattern(ard.ARD_TILE, 64, 64, 32), ard.ARD_ERR_INVALID_ARG), (other.pattern(ard.ARD_ROW, 64, 64), ard.ARD_ERR_INVALID_ARG),
                (ctx.pattern(ard.ARD_ROW, 64, 63), ard.ARD_ERR_SHAPE))
        n0 = ard.ard_launch_count(ctx.h)          # (making a pattern launches its dense draw)
        for pat, status in pats:
            for call in (lambda: ard.ard_layer_norm_fwd(ctx.h, pat, F32, 4, 64, 1e-5, x, 64, None, None, y, 64, None, None),
                         lambda: ard.ard_glr_forward(ctx.h, pat, F32, 2, 2, 64, 1.0, x, x, None, 64, None, None, y, 64, None, None)):
                with pytest.raises(ard.ArdError) as e:
                    call()
                assert e.value.status == status
        assert ard.ard_launch_count(ctx.h) == n0
    finally:
        ctx.close()
        other.close()


@pytest.mark.parametrize("dtype,rows,N", [(BF16, 3000, 512), (F32, 700, 1500), (BF16, 130, 8192), (BF16, 700, 1501), (BF16, 64, 256)])
def test_graph_replays_and_repeats_give_the_same_bits(dtype, rows, N):
    ctx = Ctx(0)
    try:
        td = tdtype(dtype)
        X, dY, w = torch.randn(rows, N, device="cuda").to(td), torch.randn(rows, N, device="cuda").to(td), torch.randn(N, device="cuda")
        outs = [torch.empty_like(X), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(X),
                torch.empty(N, device="cuda"), torch.empty(N, device="cuda")]

        def call():
            ard.ard_layer_norm_fwd(ctx.h, None, dtype, rows, N, 1e-5, X, N, w, w, outs[0], N, outs[1], outs[2])
            ard.ard_layer_norm_bwd(ctx.h, None, dtype, rows, N, dY, N, X, N, w, outs[1], outs[2], outs[3], N, outs[4], outs[5], 0)
        call()
        first = [t.clone() for t in outs]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for k in range(3):
            for t in outs:
                t.fill_(float("nan"))
            graph.replay() if k else call()
            assert all(torch.equal(a, b) for a, b in zip(first, outs))
        X.mul_(2.0)                     # other inputs in the same memory
        dY.neg_()
        call()
        second = [t.clone() for t in outs]
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(second, outs)) and not torch.equal(first[3], second[3])
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,N,ld,off", [(1300, 255, (0, 0, 0, 0), 0), (1300, 64, (1, 2, 3, 5), 1), (1250, 1, (0, 1, 2, 3), 3), (1400, 31, (4, 2, 1, 0), 2),
                                           (1300, 1000, (0, 0, 0, 0), 4), (1200, 8, (0, 0, 0, 0), 5), (200, 2999, (2, 0, 4, 6), 3), (40, 8191, (0, 0, 0, 0), 0),
                                           (1190, 520, (8, 8, 4, 8), 0), (1300, 2048, (2, 2, 2, 2), 6), (3, 2056, (1, 3, 5, 7), 7), (5000, 130, (0, 0, 0, 0), 0),
                                           (37, 4096, (4, 4, 4, 4), 0)])
def test_rows_that_begin_anywhere(dtype, rows, N, ld, off):
    """More or longer rows than a CTA each is made for, off the 16-byte grid: their copies start ahead of them and end behind them, in NaN."""
    ctx = Ctx(0)
    try:
        _run(ctx.h, None, dtype, rows, N, ld=ld, off=off, seed=N + off)
        _run(ctx.h, None, dtype, rows, N, ld=ld, off=off, seed=N, affine=False)
        if N >= 16:
            pat = ctx.pattern(ard.ARD_ROW, 16, N)
            ard.ard_pattern_set(ctx.h, pat, 3, 2)
            _run(ctx.h, pat, dtype, rows, N, 3, 2, ld=ld, off=off, seed=N + 1)
        assert ard.ard_last_device_status(ctx.h) == 0
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [147, 148, 149, 1183, 1184, 1185])
@pytest.mark.parametrize("N", [2048, 2047, 2056])
def test_where_the_kernels_change(dtype, rows, N):
    ctx = Ctx(0)
    try:
        _run(ctx.h, None, dtype, rows, N, seed=rows)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,N,ld,off", [(1185, 64, (0, 0, 0, 0), 0), (20000, 33, (0, 1, 2, 3), 1), (5000, 128, (8, 0, 8, 16), 0), (3000, 129, (0, 0, 0, 0), 0),
                                           (9000, 256, (0, 8, 0, 8), 0), (2500, 250, (6, 6, 6, 6), 0), (40000, 8, (0, 0, 0, 0), 0), (30000, 3, (0, 0, 0, 0), 0),
                                           (1200, 100, (4, 4, 4, 4), 0), (4000, 257, (0, 0, 0, 0), 3), (19000, 256, (1, 1, 1, 1), 0)])
def test_many_short_rows(dtype, rows, N, ld, off):
    ctx = Ctx(0)
    try:
        _run(ctx.h, None, dtype, rows, N, ld=ld, off=off, seed=N + off)
        if N >= 16:
            pat = ctx.pattern(ard.ARD_ROW, 16, N)
            ard.ard_pattern_set(ctx.h, pat, 2, 2)
            _run(ctx.h, pat, dtype, rows, N, 2, 2, ld=ld, off=off, zero_fill=0, seed=N + 1)
    finally:
        ctx.close()
