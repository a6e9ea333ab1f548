"""ard_adamw_step with states in 8 bits where second moments leave fp32's normal range, ard_grad_norm with the smallest bounds."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx
from oracle import adamw as OA
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
U, F = 2.0 ** -24, np.float32
LR, B1, B2 = 1e-2, 0.9, 0.999
INVERSE = F(1) / F(OA.LARGEST)      # a block's largest value times this is its scale
_held = []


def _h():
    if not _held:
        _held.append(Ctx(0))
    return _held[0].h


def _tensor(g, decay=0.0, p=0.0):
    n = g.numel()
    new = lambda k, dt=torch.float32: torch.zeros(k, dtype=dt, device="cuda")  # noqa: E731
    return dict(rows=1, cols=n, p=new(n) + p, g=g.cuda(), m=new(n, torch.uint8), v=new(n, torch.uint8), m_scale=new(-(-n // 128)),
                v_scale=new(-(-n // 128)), weight_decay=decay)


def _step(t, number, lr=LR, b1=B1, eps=1e-8):
    ard.ard_adamw_step(_h(), ard.adamw_tensors([t]), 1, lr, b1, B2, eps, 8, 3, number)
    torch.cuda.synchronize()
    assert ard.ard_last_device_status(_h()) == 0


def _root(t):
    return t["v"].view(torch.float8_e4m3fn).float().cpu().numpy() * np.repeat(t["v_scale"].cpu().numpy(), 128)[:t["cols"]]


# whole tiles, and a block that ends the tensor inside a tile
@pytest.mark.parametrize("n,at", [(4096, 700), (1300, 1290)])
@pytest.mark.parametrize("huge", [1e21, -3e30])
def test_a_second_moment_beyond_fp32_leaves_its_parameter_to_decay(n, at, huge):
    """v = infinity: m / (sqrt(v) + eps) = 0, as with states in 32 bits; in this step and in later ones, and no other block notices."""
    g = torch.from_numpy(np.random.default_rng(n).normal(size=n).astype(F))
    calm, t = _tensor(g, 0.1, 0.5), _tensor(g, 0.1, 0.5)
    t["g"][at] = huge
    block = slice(at // 128 * 128, min(n, at // 128 * 128 + 128))
    want = 0.5
    for k in range(1, 5):
        _step(calm, k)
        _step(t, k)
        want *= 1 - LR * 0.1
        # a product and a difference a step, of numbers about a half
        assert abs(float(t["p"][at]) - want) <= 2 * k * U
        assert bool(torch.isfinite(t["p"]).all()) and bool(torch.isfinite(t["v_scale"]).all()) and bool(torch.isfinite(t["m_scale"]).all())
        # the square of what is held is beyond fp32 still
        assert float(_root(t)[at]) >= 2.0 ** 64
        for key in ("p", "m", "v"):
            a, b = calm[key].clone(), t[key].clone()
            a[block] = b[block] = 0
            assert torch.equal(a, b), key
        t["g"][at] = 1.0       # what comes afterwards does not bring it back, as it does not in 32 bits


def test_a_second_moment_beyond_fp32_beside_roots_that_are_zero():
    g = torch.zeros(256)
    g[3] = 1e22
    t = _tensor(g, 0.0, 1.0)
    for k in range(1, 4):
        _step(t, k)
        assert bool((t["p"] == 1).all())
    t["g"][7] = 1.0            # a root that was zero begins: its first step is of the formula's length
    _step(t, 4)
    m, v = 1 - B1, 1 - B2
    want = 1 - LR * (m / (1 - B1 ** 4)) / (np.sqrt(v / (1 - B2 ** 4)) + 1e-8)
    assert abs(float(t["p"][7]) - want) <= 2 * U + 40 * U * abs(1 - want)


@pytest.mark.parametrize("eps", [0.0, 1e-30])
def test_second_moments_below_the_normal_range(eps):
    """Gradients of 1e-21 to 1e-17: v is subnormal in fp32, its root is not."""
    blocks = 4000
    rng = np.random.default_rng(2)
    values = (np.exp(rng.uniform(np.log(2e-21), np.log(1e-17), size=blocks)) * rng.choice([-1, 1], size=blocks)).astype(F)
    g = np.zeros((blocks, 128), F)
    g[:, 9] = values
    t = _tensor(torch.from_numpy(g.reshape(-1)))
    _step(t, 1, eps=eps)
    v = (F(1.0 - B2) * values).astype(F) * values
    assert (v > 0).all() and (v < 2.0 ** -126).mean() > 0.5
    want = np.sqrt(v.astype(np.float64))
    got = t["v_scale"].cpu().numpy().astype(np.float64) / float(INVERSE)
    assert (np.abs(got - want) <= 4 * U * want).all()
    m, lift1, lift2 = (1 - B1) * values.astype(np.float64), 1 / (1 - B1), 1 / (1 - B2)
    p = -LR * m * lift1 / (want * np.sqrt(lift2) + eps)
    assert (np.abs(t["p"].cpu().numpy().reshape(-1, 128)[:, 9] - p) <= 40 * U * np.abs(p)).all()


@pytest.mark.parametrize("big", [8.4e37, 8.6e37, 3.3e38])
def test_first_moments_up_to_fp32s_end(big):
    """m = g; without a rate the parameters stay."""
    g = torch.zeros(1024)
    g[::128] = torch.tensor([1, -1, 1, -1, 1, -1, 1, -1.0]) * big
    g[1::128] = big / 7
    t = _tensor(g, 0.0, 1.0)
    _step(t, 1, lr=0.0, b1=0.0)
    codes = t["m"].view(torch.float8_e4m3fn).float()
    assert bool((codes[::128].abs() == 448).all()) and bool((codes[::128].sign() == t["g"][::128].sign()).all())
    assert bool((codes[1::128] == 64).all())      # 448 / 7: on the grid, and the division by 7 is off by less than a random word's half step
    want = np.full(8, F(big)) * INVERSE
    assert (np.abs(t["m_scale"].cpu().numpy() - want) <= np.spacing(want)).all()
    assert bool((t["p"] == 1).all())


@pytest.mark.parametrize("most", [1e-45, 7e-46, 1e-60, 5e-324])
def test_bounds_that_fp32_does_not_hold(most):
    g = torch.full((1000,), 1e-3, device="cuda")
    out = torch.zeros(2, device="cuda")
    ard.ard_grad_norm(_h(), ard.adamw_tensors([{"rows": 1, "cols": 1000, "p": None, "g": g, "m": None, "v": None}]), 1, most, out)
    norm, factor = OA.norm([g.double().cpu().numpy()], most)
    assert abs(float(out[0]) - norm) <= 2 * U * norm and abs(float(out[1]) - factor) <= 2.0 ** -149
