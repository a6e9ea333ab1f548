"""ard_adamw_step and ard_grad_norm against the fp64 statement (oracle/adamw.py): states in 32 and 8 bits, many tensors, strides, ragged ends,
factors on the device, graphs."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host
from oracle import adamw as OA
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LR, B1, B2, EPS = 2e-3, 0.9, 0.999, 1e-8
BF = torch.bfloat16
_held = []


def _h():
    if not _held:
        _held.append(Ctx(0))
    return _held[0].h


def _place(rows, cols, ld, off, dtype, values):
    """[rows][ld] NaN outside `values` [rows][cols], from element `off` of its memory."""
    t = torch.full((rows * ld + off + 64,), float("nan"), dtype=dtype, device="cuda")[off:off + rows * ld].view(rows, ld)
    if values is not None:
        t[:, :cols] = torch.from_numpy(np.asarray(values, np.float32)).to(dtype)
    return t


class Param:
    def __init__(self, rows, cols, bits=32, gd=torch.float32, ld=(0, 0, 0), off=0, decay=0.1, copy=True, seed=0, first=False, gscale=1e-2):
        rng = np.random.default_rng(seed)
        self.rows, self.cols, self.n, self.bits, self.decay, self.ld, self.off = rows, cols, rows * cols, bits, decay, ld, off
        n = self.n
        self.p = _place(rows, cols, cols + ld[0], off, torch.float32, rng.normal(size=(rows, cols)) * 0.1)
        g = rng.normal(size=(rows, cols)) * gscale * np.exp(rng.normal(size=(rows, 1)))
        g[:, ::7] = 0.0
        self.g = _place(rows, cols, cols + ld[1], off, gd, g)
        self.w = _place(rows, cols, cols + ld[2], off, BF, None) if copy else None
        m, v = rng.normal(size=n) * 3e-3, rng.normal(size=n) ** 2 * 1e-4
        if first:
            m[:], v[:] = 0, 0
        if bits == 32:
            self.m, self.v = _place(1, n, n, off, torch.float32, m[None]), _place(1, n, n, off, torch.float32, v[None])
            self.ms = self.vs = None
        else:
            blocks = -(-n // 128)
            for x, code, scale in ((m, "m", "ms"), (np.sqrt(v), "v", "vs")):
                s = OA.scales(x).astype(np.float32)
                q = np.zeros(n)
                live = np.repeat(s, 128)[:n] > 0
                q[live] = (x / np.maximum(np.repeat(s, 128)[:n], 1e-38))[live]
                t = torch.zeros(n + off + 64, dtype=torch.uint8, device="cuda")
                t[off + n:] = 0x5A
                t[off:off + n] = torch.from_numpy(q).float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cuda()
                setattr(self, code, t)
                sc = torch.full((blocks + 3,), -5.0, device="cuda")
                sc[:blocks] = torch.from_numpy(s)
                setattr(self, scale, sc)
        self.before = self.state()

    def state(self):
        """p, m, v as fp64 vectors."""
        p = host(self.p)[:, :self.cols].reshape(-1)
        if self.bits == 32:
            return p, host(self.m).reshape(-1)[:self.n], host(self.v).reshape(-1)[:self.n]
        m, r = self.codes()
        return p, m * self.wide(self.ms), (r * self.wide(self.vs)) ** 2

    def codes(self):
        return tuple(t[self.off:self.off + self.n].view(torch.float8_e4m3fn).double().cpu().numpy() for t in (self.m, self.v))

    def wide(self, scale):
        return np.repeat(host(scale)[:-(-self.n // 128)], 128)[:self.n]

    def entry(self):
        part = lambda t: t if self.bits == 32 else t[self.off:]  # noqa: E731
        return {"rows": self.rows, "cols": self.cols, "p": self.p, "ldp": self.cols + self.ld[0], "g": self.g, "ldg": self.cols + self.ld[1],
                "w": self.w, "ldw": self.cols + self.ld[2], "m": part(self.m), "v": part(self.v), "m_scale": self.ms, "v_scale": self.vs,
                "weight_decay": self.decay}

    def check(self, t, number, seed=0, gf=1.0, lr=LR):
        n = self.n
        g = host(self.g)[:, :self.cols].reshape(-1) * gf
        p0, m0, v0 = self.before
        m, v = OA.moments(m0, v0, g, B1, B2)
        p = OA.step(p0, m, v, lr, B1, B2, EPS, self.decay, t)
        # eight bits: the value of a state is a product of two fp32 numbers (and v its square); constants in fp32 are off by half a unit
        em = 8 * U * (np.abs(B1 * m0) + np.abs((1 - B1) * g))
        ev = 12 * U * v
        got = host(self.p)[:, :self.cols].reshape(-1)
        lift1, lift2 = 1 / (1 - B1 ** t), 1 / (1 - B2 ** t)
        den = np.sqrt(v * lift2) + EPS
        tol = 1.5 * U * np.abs(p) + lr * (8 * U * self.decay * np.abs(p0) + (em + 24 * U * np.abs(m)) * lift1 / den)
        assert (np.abs(got - p) <= tol + 1e-44).all()
        if self.w is not None:
            assert torch.equal(self.w[:, :self.cols], self.p[:, :self.cols].to(BF))
            assert bool(torch.isnan(self.w[:, self.cols:]).all())
        assert bool(torch.isnan(self.p[:, self.cols:]).all())
        if self.bits == 32:
            gm, gv = host(self.m).reshape(-1)[:n], host(self.v).reshape(-1)[:n]
            assert (np.abs(gm - m) <= em + 1e-44).all() and (np.abs(gv - v) <= ev + 1e-44).all()
            return
        words = OA.words(n, seed, t, number)
        for x, err, q, scale, r, root in ((m, em, self.codes()[0], self.ms, words & np.uint64(0xFFFF), False),
                                          (np.sqrt(v), 12 * U * np.sqrt(v), self.codes()[1], self.vs, words >> np.uint64(16), True)):
            want = OA.scales(x)
            s = host(scale)[:len(want)]
            blocks = lambda a: np.concatenate([a, np.zeros(-n % 128)]).reshape(-1, 128).max(axis=1)  # noqa: E731
            assert (np.abs(s - want) <= 4 * U * want + blocks(err) / OA.LARGEST).all()
            # the 8-bit value is the rounding of a number no further from the true one than err, times a scale as it came out
            off = err + 8 * U * np.abs(x)
            lo = OA.rounded(np.sign(x) * np.maximum(np.abs(x) - off, 0), s, r, root)
            hi = OA.rounded(np.sign(x) * (np.abs(x) + off), s, r, root)
            assert ((np.minimum(lo, hi) <= q) & (q <= np.maximum(lo, hi))).all()
            assert (q == OA.rounded(x, s, r, root)).mean() > 0.999 or n < 2000
        for x in (self.m, self.v):
            assert bool((x[self.off + n:] == 0x5A).all())
        assert bool((self.ms[-(-n // 128):] == -5).all()) and bool((self.vs[-(-n // 128):] == -5).all())


SIZES = [(1, 1), (1, 3), (1, 4), (1, 127), (1, 128), (1, 129), (1, 2048), (1, 2049), (3, 5), (10, 2048), (64, 33), (257, 129), (100, 1000), (1, 300001), (128, 4096)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gd", [torch.float32, BF])
def test_sizes(bits, gd):
    """Each alone, then all of them in one call; a step from zero states among them."""
    for k, (r, c) in enumerate(SIZES):
        q = Param(r, c, bits, gd, seed=k, first=k % 3 == 0, copy=k % 2 == 0)
        ard.ard_adamw_step(_h(), ard.adamw_tensors([q.entry()]), 1, LR, B1, B2, EPS, bits, 5 + k, 1 + k)
        q.check(1 + k, 0, 5 + k)
    qs = [Param(r, c, bits, gd, seed=40 + k, decay=0.01 * k, copy=k % 2 == 1) for k, (r, c) in enumerate(SIZES)]
    ard.ard_adamw_step(_h(), ard.adamw_tensors([q.entry() for q in qs]), len(qs), LR, B1, B2, EPS, bits, (7 << 33) + 1, 3)
    for k, q in enumerate(qs):
        q.check(3, k, (7 << 33) + 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ld,off", [((0, 0, 0), 1), ((0, 0, 0), 4), ((3, 0, 0), 0), ((0, 5, 0), 0), ((0, 0, 1), 0), ((4, 8, 16), 0), ((1, 2, 3), 3)])
def test_strides_and_alignment(bits, ld, off):
    qs = [Param(r, c, bits, gd, ld=ld, off=off, seed=r + c) for r, c in ((5, 64), (33, 100), (1, 77), (2, 2050)) for gd in (torch.float32, BF)]
    ard.ard_adamw_step(_h(), ard.adamw_tensors([q.entry() for q in qs]), len(qs), LR, B1, B2, EPS, bits, 9, 4)
    for k, q in enumerate(qs):
        q.check(4, k, 9)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [16, 17, 216, 217, 500])
def test_many_tensors(bits, count):
    """More than one table of the launch; empty tensors among them."""
    qs = [None if k % 11 == 5 else Param(1 + k % 3, 1 + (k * 37) % 300, bits, seed=k) for k in range(count)]
    empty = {"rows": 0, "cols": 4, "p": None, "g": None, "g_dtype": 0, "m": None, "v": None}
    n0 = ard.ard_launch_count(_h())
    table = ard.adamw_tensors([empty if q is None else q.entry() for q in qs])
    ard.ard_adamw_step(_h(), table, count, LR, B1, B2, EPS, bits, 21, 2)
    assert ard.ard_launch_count(_h()) - n0 == (1 if count <= 217 else 3)
    for k, q in enumerate(qs):
        if q is not None:
            q.check(2, k, 21)
    out = torch.zeros(2, device="cuda")
    ard.ard_grad_norm(_h(), table, count, 0.5, out)
    want, factor = OA.norm([host(q.g)[:, :q.cols] for q in qs if q is not None], 0.5)
    assert abs(float(out[0]) - want) <= 2 * U * want and abs(float(out[1]) - factor) <= 4 * U * factor


def test_several_steps_against_the_librarys():
    """Fifteen steps of torch.optim.AdamW in fp64 from zero states: the step's number, its corrections, states carried on."""
    rng = np.random.default_rng(3)
    p0 = rng.normal(size=(40, 50)).astype(np.float32)
    tp = torch.tensor(p0, dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([tp], lr=LR, betas=(B1, B2), eps=EPS, weight_decay=0.1)
    p, g = torch.from_numpy(p0).cuda(), torch.empty(40, 50, device="cuda")
    m, v = torch.zeros(2000, device="cuda"), torch.zeros(2000, device="cuda")
    table = ard.adamw_tensors([{"rows": 40, "cols": 50, "p": p, "g": g, "m": m, "v": v, "weight_decay": 0.1}])
    for t in range(1, 16):
        gr = rng.normal(size=(40, 50)).astype(np.float32)
        tp.grad = torch.tensor(gr, dtype=torch.float64)
        opt.step()
        g.copy_(torch.from_numpy(gr))
        ard.ard_adamw_step(_h(), table, 1, LR, B1, B2, EPS, 32, 0, t)
    # a step moves by about LR; each is off by some 30 units of that and rounds p once
    assert np.abs(host(p) - tp.detach().numpy()).max() <= 15 * (40 * U * 4 * LR + 2 * U * np.abs(p0).max())


@pytest.mark.parametrize("bits", [32, 8])
def test_counter_and_factors_on_the_device(bits):
    counter = torch.tensor([4], dtype=torch.int64, device="cuda")
    lrf, gf = torch.tensor([0.25], device="cuda"), torch.tensor([0.125], device="cuda")
    q = Param(30, 70, bits, seed=1)
    ard.ard_adamw_step(_h(), ard.adamw_tensors([q.entry()]), 1, LR, B1, B2, EPS, bits, 3, 2, counter, lrf, gf)
    q.check(6, 0, 3, gf=0.125, lr=0.25 * LR)
    # a factor that is not finite, or a step of number zero: nothing moves
    for bad, step in ((float("nan"), 2), (float("inf"), 2), (0.5, 0)):
        q = Param(30, 70, bits, seed=2)
        old = [t.clone() for t in (q.p, q.m, q.v)]
        ard.ard_adamw_step(_h(), ard.adamw_tensors([q.entry()]), 1, LR, B1, B2, EPS, bits, 3, step, None, None,
                           torch.tensor([bad], device="cuda"))
        same = lambda a, b: torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))  # noqa: E731
        assert all(same(a, b) for a, b in zip(old, (q.p, q.m, q.v))) and bool(torch.isnan(q.w).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_constants_at_their_ends(bits):
    """No first moment, no second moment, no rate."""
    for b1, b2, lr in ((0.0, 0.999, LR), (0.9, 0.0, LR), (0.0, 0.0, LR), (0.9, 0.999, 0.0)):
        q = Param(1, 600, bits, seed=7)
        g = host(q.g).reshape(-1)
        p0, m0, v0 = q.before
        ard.ard_adamw_step(_h(), ard.adamw_tensors([q.entry()]), 1, lr, b1, b2, 1e-6, bits, 3, 5)
        m, v = OA.moments(m0, v0, g, b1, b2)
        p = OA.step(p0, m, v, lr, b1, b2, 1e-6, q.decay, 5)
        assert np.abs(host(q.p).reshape(-1) - p).max() <= 2 * U * np.abs(p).max() + 64 * U * lr * max(1.0, np.abs((p - p0)).max() / max(lr, 1e-30))


def test_blocks_of_zeros_and_of_tiny_values():
    n = 1024
    g = torch.zeros(n, device="cuda")
    g[256:384] = 1e-38
    g[384:512] = 1e-30
    g[512] = 3e4
    g[513:640] = 1e-8
    p, m, v = torch.ones(n, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    table = ard.adamw_tensors([{"rows": 1, "cols": n, "p": p, "g": g, "m": m, "v": v, "m_scale": ms, "v_scale": vs}])
    for t in range(1, 40):
        ard.ard_adamw_step(_h(), table, 1, 1e-2, B1, B2, EPS, 8, 3, t)
    assert bool(torch.isfinite(p).all())
    assert bool((p[:256] == 1).all()) and not bool(m[:384].any()) and not bool(v[:256].any())
    # beside a gradient 3e12 times as large a small one's root is held as the smallest value, so its steps are short, not wild
    assert bool((v[513:640].view(torch.float8_e4m3fn).float() >= 2.0 ** -9).all())
    assert float((p[513:640] - 1).abs().max()) <= 40 * 1e-2 * 1.01


def test_a_value_that_is_not_a_number_spoils_its_block_alone():
    q = Param(1, 1024, 8, seed=5)
    q.g[0, 300] = float("nan")
    ard.ard_adamw_step(_h(), ard.adamw_tensors([q.entry()]), 1, LR, B1, B2, EPS, 8, 3, 5)
    bad = torch.isnan(q.p[0]).nonzero().reshape(-1).tolist()
    assert bad == [300]
    assert torch.isnan(q.ms[:8]).nonzero().reshape(-1).tolist() == [2] == torch.isnan(q.vs[:8]).nonzero().reshape(-1).tolist()


@pytest.mark.parametrize("gd", [torch.float32, BF])
def test_norm(gd):
    for shapes, scale in (([(1, 1)], 1.0), ([(1, 5), (300, 1000), (7, 33)], 1e-3), ([(1, 4096)] * 5, 1e15), ([(33, 65)], 1e-25)):
        qs = [Param(r, c, 32, gd, seed=k, gscale=scale, ld=(0, 3 * (k % 2), 0)) for k, (r, c) in enumerate(shapes)]
        qs[0].g[0, 0] = scale
        table = ard.adamw_tensors([q.entry() for q in qs])
        for most in (1.0, 1e-4, 0.0, -1.0, 1e30):
            out = torch.full((3,), 7.0, device="cuda")
            ard.ard_grad_norm(_h(), table, len(qs), most, out)
            want, factor = OA.norm([host(q.g)[:, :q.cols] for q in qs], most)
            assert abs(float(out[0]) - want) <= 2 * U * want
            assert abs(float(out[1]) - factor) <= 4 * U * factor and float(out[2]) == 7
    for bad in (float("nan"), float("inf"), -float("inf")):
        qs[0].g[1, 2] = bad
        ard.ard_grad_norm(_h(), table, len(qs), 1.0, out)
        assert not np.isfinite(float(out[0])) and np.isnan(float(out[1]))
    ard.ard_grad_norm(_h(), table, 0, 1.0, out)            # no gradients
    assert out.tolist() == [0.0, 1.0, 7.0]


@pytest.mark.parametrize("gd", [torch.float32, BF])
@pytest.mark.parametrize("n", [8191, 8192, 8193, 16384, 100000, 2 ** 20 + 8])
def test_norm_of_whole_and_ragged_tiles(n, gd):
    """Every element counts once: gradients of which one alone is not zero, at the tiles' borders, and all of them."""
    g = torch.zeros(n, device="cuda", dtype=gd)
    out = torch.zeros(2, device="cuda")
    table = ard.adamw_tensors([{"rows": 1, "cols": n, "p": None, "g": g, "m": None, "v": None}])
    for at in {0, 1, 3, 4, 7, 8, 1023, 1024, 2047, 2048, 4095, 4096, 8190, n // 2, n - 9, n - 2, n - 1} | set(range(8176, min(n, 8208))):
        for value in (3.0, 2e-30):
            g[at] = value
            ard.ard_grad_norm(_h(), table, 1, 1.0, out)
            g[at] = 0.0
            want = float(torch.tensor(value).to(gd))
            assert abs(float(out[0]) - want) <= 2 * U * want, at
    g.copy_(torch.randn(n, device="cuda"))
    ard.ard_grad_norm(_h(), table, 1, 1.0, out)
    want, factor = OA.norm([host(g)], 1.0)
    # sums of eight squares are off by at most eight units each, those over all of them by far less
    assert abs(float(out[0]) - want) <= 2 * U * want and abs(float(out[1]) - factor) <= 4 * U * factor


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_follows_counter_and_gradients(bits):
    """Norm, clip and step in one graph, the counter advanced between replays, against the same calls made eagerly: the same bits."""
    made = []
    for graphed in (False, True):
        q = [Param(64, 65, bits, seed=1, first=True), Param(1, 65, bits, BF, seed=2, first=True, decay=0.0)]
        counter, out = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")
        table = ard.adamw_tensors([x.entry() for x in q])

        def call():
            ard.ard_grad_norm(_h(), table, 2, 0.1, out)
            ard.ard_adamw_step(_h(), table, 2, LR, B1, B2, EPS, bits, 4, 1, counter, None, out[1:])
        if graphed:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                call()
        for t in range(5):
            graph.replay() if graphed else call()
            counter += 1
            q[0].g.neg_()
        made.append([x for r in q for x in (r.p, r.m, r.v, r.w)] + [out])
    for a, b in zip(*made):
        assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))


def _eight(n, off, seed, g):
    """Tensors for one step with states in 8 bits from zeros, the scales `off` floats into their memory."""
    blocks = -(-n // 128)
    new = lambda k, dt=torch.float32: torch.zeros(k, dtype=dt, device="cuda")  # noqa: E731
    return dict(rows=1, cols=n, p=new(n), g=g, w=None, m=new(n, torch.uint8), v=new(n, torch.uint8), m_scale=new(blocks + off)[off:],
                v_scale=new(blocks + off)[off:], weight_decay=0.0)


def _steps(t, k=2):
    table = ard.adamw_tensors([t])
    for step in range(1, k + 1):
        ard.ard_adamw_step(_h(), table, 1, LR, B1, B2, EPS, 8, 9, step)
    torch.cuda.synchronize()


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("n", [512 * 40, 512 * 7 + 130, 128 * 3, 77])
def test_scales_on_any_four_bytes(n, off):
    """A tensor's scales among others' in one buffer: the same bits as on a 16-byte grid."""
    g = torch.from_numpy(np.random.default_rng(n).normal(size=n).astype(np.float32)).cuda()
    a, b = _eight(n, 0, 1, g), _eight(n, off, 1, g)
    _steps(a)
    _steps(b)
    for k in ("p", "m", "v", "m_scale", "v_scale"):
        assert torch.equal(a[k], b[k]), k


def test_states_in_eight_bits_are_rounded_from_what_the_formulas_give_in_fp32():
    """The scale of a block with one value is that value times 1 / 448.  m: every operation rounded, bit for bit.  The root: to the last bit but for values
    within 2^-46 of the middle between two numbers, of which there is one in millions."""
    n, f = 128 * 20000, np.float32
    rng = np.random.default_rng(4)
    values = (np.exp(rng.uniform(-25, 10, size=20000)) * rng.choice([-1, 1], size=20000)).astype(f)
    g = np.zeros((20000, 128), f)
    g[:, 5] = values
    t = _eight(n, 0, 1, torch.from_numpy(g.reshape(-1)).cuda())
    _steps(t, 1)
    inverse = f(1) / f(448)
    m = (f(1.0 - B1) * values).astype(f)
    assert np.array_equal(t["m_scale"].cpu().numpy(), (np.abs(m) * inverse).astype(f))
    v = ((f(1.0 - B2) * values).astype(f) * values).astype(f)
    want, got = (np.sqrt(v) * inverse).astype(f), t["v_scale"].cpu().numpy()
    same = got == want
    assert same.mean() > 0.999 and (np.abs(got - want) <= np.spacing(want)).all()
    # a second step: beta1 m + (1 - beta1) g of three roundings, m being its code times its scale
    code = t["m"].view(torch.float8_e4m3fn).float().cpu().numpy().reshape(-1, 128)[:, 5]
    before = (code * t["m_scale"].cpu().numpy()).astype(f)
    ard.ard_adamw_step(_h(), ard.adamw_tensors([t]), 1, LR, B1, B2, EPS, 8, 9, 2)
    torch.cuda.synchronize()
    m = ((f(B1) * before).astype(f) + (f(1.0 - B1) * values).astype(f)).astype(f)
    assert np.array_equal(t["m_scale"].cpu().numpy(), (np.abs(m) * inverse).astype(f))
