"""ard_embedding_fwd / ard_embedding_bwd against the definition in fp64."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host, tdtype
from oracle import embedding as OE
from oracle import pattern as OP
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
F32, BF16 = ard.ARD_F32, ard.ARD_BF16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def tokens(rng, rows, V, kind):
    if kind == "one":
        return np.full(rows, V // 2, np.int32)
    if kind == "zipf":
        return np.minimum(((V + 1.0) ** rng.random(rows) - 1).astype(np.int32), V - 1)
    ids = rng.integers(0, V, rows).astype(np.int32)
    if kind == "padded":
        ids[rng.random(rows) < 0.3] = -1
        ids[: rows // 10] = -(2 ** 31)
    return ids


def matrix(rng, rows, cols, ld, off, dtype, full=None):
    """[rows][ld] beginning `off` elements behind an aligned address, NaN outside the first `cols` columns."""
    t = torch.full((rows * ld + off + 64,), float("nan"), dtype=tdtype(dtype), device="cuda")[off:off + rows * ld].view(rows, ld)
    if rng is not None:
        t[:, :cols] = torch.from_numpy(rng.normal(size=(rows, cols)).astype(np.float32)).to(tdtype(dtype))
    return t


CASES = [
    # dtype, rows, V, N, (dp, b), ld beyond N, offset in elements, tokens, accumulate
    (BF16, 1, 1, 1, (1, 1), 0, 0, "any", False),
    (BF16, 5, 7, 3, (1, 1), 2, 1, "any", False),
    (F32, 64, 10, 128, (1, 1), 0, 0, "any", False),
    (F32, 33, 50, 129, (1, 1), 4, 3, "padded", True),
    (BF16, 700, 880, 1500, (2, 2), 0, 0, "zipf", False),
    (BF16, 700, 880, 1500, (2, 1), 0, 0, "zipf", True),
    (BF16, 257, 400, 1000, (3, 2), 8, 8, "padded", False),
    (BF16, 100, 30, 131, (7, 7), 0, 0, "any", False),
    (BF16, 3000, 11, 512, (1, 1), 0, 0, "any", False),
    (F32, 2000, 5000, 260, (1, 1), 0, 2, "zipf", False),
    (BF16, 20000, 300, 136, (1, 1), 0, 0, "one", False),
    (BF16, 40000, 3000, 72, (1, 1), 0, 0, "zipf", False),
    (BF16, 40000, 3000, 70, (1, 1), 1, 0, "padded", True),
    (F32, 17000, 2, 8, (1, 1), 0, 0, "any", False),
    (BF16, 16385, 1, 64, (1, 1), 0, 0, "any", True),
    (BF16, 200, 300000, 16, (1, 1), 0, 0, "any", False),
    (BF16, 0, 40, 24, (1, 1), 0, 0, "any", False),
    # few tokens: some clusters of CTAs, one token each
    (BF16, 50000, 3, 24, (1, 1), 0, 0, "padded", False),
    (F32, 5000, 2, 300, (1, 1), 1, 1, "any", True),
    (BF16, 9000, 5, 1000, (3, 2), 8, 0, "zipf", False),
    (F32, 3000, 7, 4, (1, 1), 0, 0, "any", False),
    (BF16, 3, 2, 8, (1, 1), 0, 0, "any", False),
    (BF16, 0, 2, 130, (2, 1), 0, 0, "any", False),
    # tokens of more than one digit of the sort, lists that fill up several times
    (BF16, 30000, 9000, 1500, (1, 1), 0, 0, "any", False),
    (F32, 30000, 200000, 136, (1, 1), 0, 0, "zipf", True),
]


def test_on_a_stream_and_from_a_graph():
    """On another stream than the current one, captured, and replayed on other tokens and gradients."""
    ctx = Ctx()
    rows, V, N = 3000, 500, 260
    rng = np.random.default_rng(4)
    ids = torch.from_numpy(tokens(rng, rows, V, "zipf")).cuda()
    table, y, dy, dtable = matrix(rng, V, N, N, 0, BF16), matrix(None, rows, N, N, 0, BF16), matrix(rng, rows, N, N, 0, BF16), matrix(None, V, N, N, 0, F32)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def both():
        s = torch.cuda.current_stream().cuda_stream
        ard.ard_embedding_fwd(ctx.h, None, BF16, rows, V, N, 1.0, ids, table, N, y, N, stream=s)
        ard.ard_embedding_bwd(ctx.h, None, BF16, rows, V, N, 1.0, ids, dy, N, dtable, N, 0, stream=s)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        both()
    for seed in (5, 6):
        rng = np.random.default_rng(seed)
        ids.copy_(torch.from_numpy(tokens(rng, rows, V, "padded")))
        dy.copy_(matrix(rng, rows, N, N, 0, BF16))
        graph.replay()
        got = y.clone(), dtable.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            both()
        side.synchronize()
        assert torch.equal(got[0], y) and torch.equal(got[1], dtable)
        want, size, count = OE.bwd(ids.cpu().numpy(), host(dy), V, N, 1.0, np.arange(N))
        assert (np.abs(host(dtable) - want) <= (count[:, None] + 3) * 2.0 ** -24 * size).all()
    ctx.close()


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_%dx%dx%d_dp%d_%s%s" % ("f32" if c[0] == F32 else "bf16", c[1], c[2], c[3], c[4][0], c[7],
                                                                               "_add" if c[8] else ""))
def test_both_ways(case):
    dtype, rows, V, N, (dp, b), pad, off, kind, accumulate = case
    rng = np.random.default_rng(rows + V)
    ctx = Ctx()
    pat = None if dp == 1 else ctx.pattern(ard.ARD_ROW, N, N)
    if pat is not None:
        ard.ard_pattern_set(ctx.h, pat, dp, b)
    keep = np.arange(N) if dp == 1 else OP.row_keep(N, dp, b)
    n, ld, alpha = len(keep), N + pad, 1.7
    ids = tokens(rng, rows, V, kind)
    d_ids = torch.from_numpy(ids).cuda()
    table = matrix(rng, V, N, ld, off, dtype)
    y = matrix(None, rows, n, ld, off, dtype)
    ard.ard_embedding_fwd(ctx.h, pat, dtype, rows, V, N, alpha, d_ids, table, ld, y, ld)
    want = OE.fwd(ids, host(table[:, :N]), np.float32(alpha), keep)
    half = HALF_STEP[dtype]
    assert (np.abs(host(y)[:, :n] - want) <= (half + 2.0 ** -24) * np.abs(want)).all()
    assert bool(torch.isnan(y[:, n:]).all())
    dy = matrix(rng, rows, n, ld, off, dtype)
    dtable = matrix(rng if accumulate else None, V, N, ld, off, F32)
    before = host(dtable)[:, :N]
    ard.ard_embedding_bwd(ctx.h, pat, dtype, rows, V, N, alpha, d_ids, dy, ld, dtable, ld, accumulate)
    first = dtable.clone()
    want, size, count = OE.bwd(ids, host(dy)[:, :n], V, N, np.float32(alpha), keep)
    if accumulate:
        want, size = want + before, size + np.abs(before)
    # one rounding an addition (of a sum no larger than the terms' sizes), one for the factor, one for what stood there
    bound = (count[:, None] + 3) * 2.0 ** -24 * size
    assert (np.abs(host(dtable)[:, :N] - want) <= bound).all()
    dropped = np.setdiff1d(np.arange(N), keep)
    if not accumulate:
        assert (host(dtable)[:, :N][:, dropped] == 0).all() and (host(dtable)[:, :N][count == 0] == 0).all()
    else:
        assert (host(dtable)[:, :N][:, dropped] == before[:, dropped]).all()
    assert bool(torch.isnan(dtable[:, N:]).all())
    # the same bits again
    if accumulate:
        dtable[:, :N] = torch.from_numpy(before).float().cuda()
    else:
        dtable.fill_(3.0)
    ard.ard_embedding_bwd(ctx.h, pat, dtype, rows, V, N, alpha, d_ids, dy, ld, dtable, ld, accumulate)
    assert torch.equal(dtable[:, :N], first[:, :N])
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_OK
    ctx.close()


def test_tokens_out_of_range_are_reported_and_count_as_padding():
    ctx = Ctx()
    V, N, rows = 9, 40, 50
    rng = np.random.default_rng(1)
    ids = rng.integers(0, V, rows).astype(np.int32)
    ids[[3, 17]] = V, 2 ** 31 - 1
    d_ids = torch.from_numpy(ids).cuda()
    table, y = matrix(rng, V, N, N, 0, F32), matrix(None, rows, N, N, 0, F32)
    ard.ard_embedding_fwd(ctx.h, None, F32, rows, V, N, 1.0, d_ids, table, N, y, N)
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_ERR_INVALID_ARG
    assert np.array_equal(host(y), OE.fwd(ids, host(table), 1.0, np.arange(N)))
    dy, dtable = matrix(rng, rows, N, N, 0, F32), matrix(None, V, N, N, 0, F32)
    ard.ard_embedding_bwd(ctx.h, None, F32, rows, V, N, 1.0, d_ids, dy, N, dtable, N, 0)
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_ERR_INVALID_ARG
    want, size, count = OE.bwd(ids, host(dy), V, N, 1.0, np.arange(N))
    assert (np.abs(host(dtable) - want) <= (count[:, None] + 2) * 2.0 ** -24 * size).all()
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_OK
    ctx.close()


def test_gradient_against_differences():
    """The lookup is linear in the table: <dY, lookup(table + d) - lookup(table)> is <dtable, d>."""
    ctx = Ctx()
    rng = np.random.default_rng(2)
    rows, V, N = 300, 40, 96
    ids = torch.from_numpy(tokens(rng, rows, V, "padded")).cuda()
    dy = matrix(rng, rows, N, N, 0, F32)
    dtable, y0, y1 = matrix(None, V, N, N, 0, F32), matrix(None, rows, N, N, 0, F32), matrix(None, rows, N, N, 0, F32)
    ard.ard_embedding_bwd(ctx.h, None, F32, rows, V, N, 0.5, ids, dy, N, dtable, N, 0)
    a, d = matrix(rng, V, N, N, 0, F32), matrix(rng, V, N, N, 0, F32)
    b = a + d
    ard.ard_embedding_fwd(ctx.h, None, F32, rows, V, N, 0.5, ids, a, N, y0, N)
    ard.ard_embedding_fwd(ctx.h, None, F32, rows, V, N, 0.5, ids, b, N, y1, N)
    terms = host(dy) * (host(y1) - host(y0))
    assert abs(terms.sum() - (host(dtable) * (host(b) - host(a))).sum()) <= 400 * 2.0 ** -24 * np.abs(terms).sum()
    ctx.close()


def test_more_than_2_to_the_32_elements():
    """A table past every 32-bit offset, with more tokens than a CTA can count where its columns fill the device."""
    V, N, rows = 270000, 16384, 400
    ctx = Ctx()
    ids = torch.randint(V - 300, V, (rows,), dtype=torch.int32, device="cuda")
    ids[:3] = torch.tensor([0, V - 1, V // 2], dtype=torch.int32)
    dy = torch.randn((rows, N), device="cuda").to(torch.bfloat16)
    dtable = torch.full((V, N), float("nan"), device="cuda")
    ard.ard_embedding_bwd(ctx.h, None, BF16, rows, V, N, 2.0, ids, dy, N, dtable, N, 0)
    want = torch.zeros((V - (V - 300), N), dtype=torch.float64, device="cuda")
    live = ids >= V - 300
    want.index_add_(0, (ids[live] - (V - 300)).long(), 2.0 * dy[live].double())
    assert float((dtable[V - 300:].double() - want).abs().max()) <= 400 * 2.0 ** -24 * 2 * float(want.abs().max())
    assert torch.equal(dtable[0], 2.0 * dy[0].float()) and torch.equal(dtable[V // 2], 2.0 * dy[2].float())
    dtable[0] = dtable[V // 2] = 0
    assert int(torch.count_nonzero(dtable[:V - 300])) == 0
    table = dtable.view(torch.bfloat16).view(V, 2 * N)     # any bits do: what is looked up comes back as it is
    table[ids.long()] = torch.randn((rows, 2 * N), device="cuda").to(torch.bfloat16)
    y = torch.empty((rows, 2 * N), dtype=torch.bfloat16, device="cuda")
    ard.ard_embedding_fwd(ctx.h, None, BF16, rows, V, 2 * N, 1.0, ids, table, 2 * N, y, 2 * N)
    assert torch.equal(y, table[ids.long()])
    ctx.close()
