"""Layer norm and the optimiser where elements lie more than 2^32 apart, and layer norm of long rows over kept units."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx
from paper_2203_05705_b200 import ard
from test_gpu_layer_norm import _run

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = Ctx(0)
    yield c
    c.close()


# a CTA a row; rings on the 16-byte grid and off it; rows by lanes; rows too long for rings
@pytest.mark.parametrize("rows,N,ld", [(70, 512, 1 << 26), (1500, 320, 3 << 20), (1500, 320, (3 << 20) + 1), (1500, 64, 3 << 20), (1500, 65, (3 << 20) + 3), (70, 20000, 1 << 26)])
def test_layer_norm(ctx, rows, N, ld):
    """The same bits as from rows that lie together, on the same grid."""
    assert rows * ld > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(rows + N)
    x, dy = (torch.randn((rows, N), generator=g, device="cuda").to(BF) for _ in range(2))
    w, b = (torch.randn(N, generator=g, device="cuda") for _ in range(2))
    left = []
    for p in (N + (ld - N) % 8, ld):
        X, dY, out = (torch.empty(rows * p, dtype=BF, device="cuda").view(rows, p) for _ in range(3))
        X[:, :N], dY[:, :N] = x, dy
        mean, rstd, dw, db = (torch.empty(k, device="cuda") for k in (rows, rows, N, N))
        ard.ard_layer_norm_fwd(ctx.h, None, ard.ARD_BF16, rows, N, 1e-5, X, p, w, b, out, p, mean, rstd)
        y = out[:, :N].clone()
        ard.ard_layer_norm_bwd(ctx.h, None, ard.ARD_BF16, rows, N, dY, p, X, p, w, mean, rstd, out, p, dw, db, 1)
        torch.cuda.synchronize()
        left.append((y, out[:, :N].clone(), mean, rstd, dw, db))
    assert ard.ard_last_device_status(ctx.h) == 0
    assert all(torch.equal(a, b) for a, b in zip(*left)) and bool(torch.isfinite(left[0][1]).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_optimiser_rows_far_apart(ctx, bits):
    """The same bits as of rows that lie together."""
    rows, cols, ld = 70, 1001, 1 << 26
    g = torch.Generator(device="cuda").manual_seed(5)
    p, gr = torch.randn((rows, cols), generator=g, device="cuda"), torch.randn((rows, cols), generator=g, device="cuda").to(BF)
    n = rows * cols
    left = []
    for apart in (False, True):
        if apart:
            P, G, W = (torch.empty(rows * ld, dtype=t, device="cuda").view(rows, ld) for t in (F32, BF, BF))
            P[:, :cols], G[:, :cols] = p, gr
        else:
            P, G, W = p.clone(), gr.clone(), torch.empty_like(gr)
        state = F32 if bits == 32 else torch.uint8
        m, v = torch.zeros(n, dtype=state, device="cuda"), torch.zeros(n, dtype=state, device="cuda")
        ms, vs = torch.zeros(-(-n // 128), device="cuda"), torch.zeros(-(-n // 128), device="cuda")
        at = ld if apart else cols
        table = ard.adamw_tensors([dict(rows=rows, cols=cols, p=P, ldp=at, g=G, ldg=at, w=W, ldw=at, m=m, v=v, m_scale=ms, v_scale=vs, weight_decay=0.1)])
        out = torch.zeros(2, device="cuda")
        for t in (1, 2):
            ard.ard_grad_norm(ctx.h, table, 1, 1.0, out)
            ard.ard_adamw_step(ctx.h, table, 1, 1e-2, 0.9, 0.999, 1e-8, bits, 3, t, None, None, out[1:])
        torch.cuda.synchronize()
        left.append([P[:, :cols].clone(), W[:, :cols].clone(), m, v, ms, vs, out])
    assert all(torch.equal(a, b) for a, b in zip(*left))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_parameter_of_more_than_2_to_the_32_elements(ctx, bits):
    n = 2 ** 32 + 128 * 33 + 5
    at = torch.tensor([0, 127, 2 ** 31 + 3, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 128 * 20, n - 6, n - 1], device="cuda")    # one a block, or two of equal size
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=BF, device="cuda")
    g[at] = torch.tensor([1.0, -1, 2, -2, 4, -4, 8, -8], device="cuda").to(BF)
    state = F32 if bits == 32 else torch.uint8
    m, v = torch.zeros(n, dtype=state, device="cuda"), torch.zeros(n, dtype=state, device="cuda")
    ms, vs = torch.zeros(-(-n // 128), device="cuda"), torch.zeros(-(-n // 128), device="cuda")
    table = ard.adamw_tensors([dict(rows=1, cols=n, p=p, g=g, m=m, v=v, m_scale=ms, v_scale=vs)])
    out = torch.zeros(2, device="cuda")
    ard.ard_grad_norm(ctx.h, table, 1, 0.0, out)
    ard.ard_adamw_step(ctx.h, table, 1, 1e-2, 0.9, 0.999, 1e-12, bits, 3, 1)
    torch.cuda.synchronize()
    assert ard.ard_last_device_status(ctx.h) == 0
    want = np.sqrt(2 * (1 + 4 + 16 + 64))
    assert abs(float(out[0]) - want) <= 2 * U * want
    # a first step's length is the rate's, by the gradient's sign
    assert bool(((p[at].double() + 1e-2 * torch.sign(g[at].double())).abs() <= 40 * U * 1e-2).all())
    count = lambda t: sum(int(torch.count_nonzero(part)) for part in t.split(2 ** 30))  # noqa: E731  (a count is taken in 32 bits)
    assert count(m) == len(at) and count(v) == len(at) and count(p) == len(at)
    if bits == 8:
        # a block's largest value is 448 times its scale; the last two share a block
        assert bool((m[at].view(torch.float8_e4m3fn).float().abs() == 448).all()) and bool((v[at].view(torch.float8_e4m3fn).float() == 448).all())
        scale = 0.1 * g[at].double().abs() / 448
        assert bool(((ms[at // 128].double() - scale).abs() <= 4 * U * scale).all())


@pytest.mark.parametrize("dtype", [ard.ARD_F32, ard.ARD_BF16])
@pytest.mark.parametrize("rows,N,dp,b", [(37, 16384, 2, 1), (300, 8200, 1, 1), (1300, 9000, 2, 2), (1300, 16381, 5, 3), (40, 20000, 3, 1)])
def test_long_rows_over_kept_units(ctx, dtype, rows, N, dp, b):
    pat = ctx.pattern(ard.ARD_ROW, 16, N)
    ard.ard_pattern_set(ctx.h, pat, dp, b)
    _run(ctx.h, pat, dtype, rows, N, dp=dp, b=b, seed=N + rows)
