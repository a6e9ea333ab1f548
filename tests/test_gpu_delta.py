"""ard_delta_forward / ard_delta_backward against the recurrence in fp64 (oracle/delta.py).

Errors allowed.  States are fp32 throughout: a step adds to a state what rounds by some units of 2^-24 of its size, at random, and nothing
enlarges what is there (|I - b k k^T| <= 1, f <= 1), so after T steps 64 + 16 sqrt(T) units of the state's 2-norm.  Outputs in bf16: half a step of the
value, and what products of two bf16 parts leave out: 2^-18 an operand and term, against the output's root mean square 2^-12 with the sums' own
roundings and some ten products one behind the other.  The gates' gradients are differences of sums over a chunk: four times that.
"""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host
from oracle import delta as OD
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
BF16, BF, F32 = ard.ARD_BF16, torch.bfloat16, torch.float32


class Case:
    def __init__(self, T, B, h, Dk, Dv, lens=None, eps=1e-6, pad=0, off=0, first=True, last=True, seed=0, shift=3.0, packed=False):
        self.T, self.B, self.h, self.Dk, self.Dv, self.eps = T, B, h, Dk, Dv, eps
        self.scale = Dk ** -0.5
        self.rng = rng = np.random.default_rng(seed + T + 7 * Dk + Dv)
        self.lens = None if lens is None else np.asarray(lens, np.int32)
        self.d_lens = None if lens is None else torch.from_numpy(self.lens).cuda()
        self.live = OD._inside(T, B, self.lens)
        self.pad, self.off = pad, off
        self.base = None
        if packed:
            self.base = self.buf(h * (2 * Dk + Dv))
            self.ld = (self.base.shape[1],) * 3
            self.q, self.k, self.v = (self.base[:, a:b] for a, b in ((0, h * Dk), (h * Dk, 2 * h * Dk), (2 * h * Dk, h * (2 * Dk + Dv))))
        else:
            self.q, self.k, self.v = self.buf(h * Dk), self.buf(h * Dk), self.buf(h * Dv)
            self.ld = tuple(x.shape[1] for x in (self.q, self.k, self.v))
        self.zf, self.zb, self.dy = self.buf(h), self.buf(h), self.buf(h * Dv)
        size = Dk ** -0.5 if eps < 0 else 1.0     # as they are: of length one or so, and never above where it matters
        for x, n, s, m in ((self.q, h * Dk, 1.0, 0.0), (self.k, h * Dk, size * 0.7, 0.0), (self.v, h * Dv, 1.0, 0.0), (self.zf, h, 1.5, shift), (self.zb, h, 1.0, 0.0),
                           (self.dy, h * Dv, 1.0, 0.0)):
            self.fill(x, n, rng.normal(size=(T, B, n)) * s + m)
        state = lambda: torch.from_numpy(rng.normal(size=(B, h, Dk, Dv)).astype(np.float32)).cuda()  # noqa: E731
        self.h0, self.dhT = (state() if first else None), (state() if last else None)
        self.y = self.buf(h * Dv)
        self.S = torch.full((-(-T // ard.ARD_DELTA_CHUNK), B, h, Dk, Dv), float("nan"), device="cuda")
        self.hT, self.dh0 = (torch.full((B, h, Dk, Dv), float("nan"), device="cuda") for _ in range(2))
        self.dq, self.dk, self.dv, self.dzf, self.dzb = (self.buf(n) for n in (h * Dk, h * Dk, h * Dv, h, h))

    def buf(self, n):
        ld, rows = n + self.pad, self.T * self.B
        return torch.full((rows * ld + self.off + 64,), float("nan"), dtype=BF, device="cuda")[self.off:self.off + rows * ld].view(rows, ld)

    def fill(self, t, n, x):
        x = np.where(self.live[..., None], x, np.nan).astype(np.float32)      # rows behind the end: not to be read
        t[:, :n] = torch.from_numpy(x.reshape(self.T * self.B, n)).to(BF)

    def work(self, backward):
        n = ard.ard_delta_work_bytes(self.T, self.B, self.h, self.Dk, self.Dv, backward)
        w = torch.full((n + 16,), 0xFF, dtype=torch.uint8, device="cuda")
        return w[5:5 + n], n

    def forward(self, ctx, save=True, hT=True, **more):
        w, n = self.work(False)
        out = self.hT if hT is True else hT
        ard.ard_delta_forward(ctx.h, BF16, self.T, self.B, self.h, self.Dk, self.Dv, self.scale, self.eps, self.q, self.ld[0], self.k, self.ld[1], self.v,
                              self.ld[2], self.zf, self.zb, self.zf.shape[1], self.d_lens, self.h0, self.y, self.y.shape[1], out,
                              self.S if save else None, w if n else None, n, **more)

    def backward(self, ctx, dh0=True, **more):
        w, n = self.work(True)
        out = self.dh0 if dh0 is True else dh0
        ard.ard_delta_backward(ctx.h, BF16, self.T, self.B, self.h, self.Dk, self.Dv, self.scale, self.eps, self.q, self.ld[0], self.k, self.ld[1], self.v,
                               self.ld[2], self.zf, self.zb, self.zf.shape[1], self.d_lens, self.S, self.dy, self.dy.shape[1], self.dhT, self.dq,
                               self.dq.shape[1], self.dk, self.dk.shape[1], self.dv, self.dv.shape[1], self.dzf, self.dzb, self.dzf.shape[1], out, w, n, **more)

    def outputs(self):
        return [self.y, self.hT, self.dq, self.dk, self.dv, self.dzf, self.dzb, self.dh0]

    def inputs(self):
        T, B, h, Dk, Dv = self.T, self.B, self.h, self.Dk, self.Dv
        on = self.live[..., None]
        of = lambda t, n: np.where(on, host(t)[:, :n].reshape(T, B, n), 0.0)  # noqa: E731
        return (of(self.q, h * Dk).reshape(T, B, h, Dk), of(self.k, h * Dk).reshape(T, B, h, Dk), of(self.v, h * Dv).reshape(T, B, h, Dv), of(self.zf, h),
                of(self.zb, h)), of(self.dy, h * Dv).reshape(T, B, h, Dv)

    def near(self, name, got, want, tol=2.0 ** -12, whole=None):
        """whole: what the output is a difference of, where it may be much smaller than that (one key of one element has no gradient at all)."""
        n = want.reshape(self.T, self.B, -1).shape[-1]
        got, want = host(got), want.reshape(self.T * self.B, n)
        rms = np.sqrt(((want if whole is None else whole) ** 2).mean()) if want.size else 0.0
        off = np.abs(got[:, :n] - want)
        assert (off <= 2.0 ** -8 * np.abs(want) + tol * rms + 1e-37).all(), (name, float((off - 2.0 ** -8 * np.abs(want)).max() / max(rms, 1e-300)), rms)
        assert np.isnan(got[:, n:]).all(), name
        assert (got[:, :n].reshape(self.T, self.B, n)[~self.live] == 0).all(), name

    def near_state(self, name, got, want):
        units = 64 + 16 * np.sqrt(max(self.T, 1))
        norm, off = np.sqrt((want ** 2).sum()), np.sqrt(((host(got) - want) ** 2).sum())
        assert off <= units * 2.0 ** -24 * norm + 1e-37, (name, off / norm * 2 ** 24, units)

    def check(self, gradient=True):
        x, dy = self.inputs()
        h0, dhT = (None if t is None else host(t) for t in (self.h0, self.dhT))
        y, S, u = OD.fwd(*x, np.float32(self.scale), np.float32(self.eps), self.lens, h0)
        self.near("y", self.y, y)
        self.near_state("hT", self.hT, S[-1])
        if gradient:
            dq, dk, dv, dzf, dzb, dh0, whole_q, whole_k = OD.bwd(*x, np.float32(self.scale), np.float32(self.eps), S, u, dy, self.lens, dhT)
            for name, got, want, tol, whole in (("dv", self.dv, dv, 1, None), ("dq", self.dq, dq, 1, whole_q), ("dk", self.dk, dk, 1, whole_k),
                                                ("dzb", self.dzb, dzb, 4, None), ("dzf", self.dzf, dzf, 4, None)):
                self.near(name, got, want, tol * 2.0 ** -12, whole)
            self.near_state("dh0", self.dh0, dh0)


SHAPES = [(1, 3, 2, 128, 128), (1, 1, 1, 1, 1), (2, 2, 3, 5, 7), (16, 2, 2, 128, 128), (17, 2, 2, 128, 128), (33, 3, 2, 64, 64), (64, 2, 2, 64, 128), (65, 2, 2, 128, 64),
          (130, 2, 1, 40, 99), (100, 1, 3, 8, 16), (200, 2, 2, 128, 128), (300, 1, 2, 33, 31), (70, 2, 2, 65, 66), (19, 40, 8, 16, 8), (129, 1, 1, 127, 1), (90, 2, 1, 1, 128)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("how", [dict(), dict(pad=3, off=1), dict(packed=True, pad=8, off=8)], ids=["plain", "unaligned", "packed"])
def test_both_ways(shape, how):
    ctx = Ctx()
    case = Case(*shape, **how)
    case.forward(ctx)
    case.backward(ctx)
    case.check()
    first = [t.clone() for t in case.outputs()]
    case.forward(ctx)
    case.backward(ctx)
    for a, b in zip(first, case.outputs()):
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
    ctx.close()


@pytest.mark.parametrize("T,lens", [(5, [0, 5, 3, -2]), (16, [16, 1, 99, 0]), (64, [64, 63, 0, 1]), (150, [150, 64, 65, 128]), (150, [0, 0, 0, 0]), (200, [2 ** 31 - 1, -(2 ** 31), 130, 7])])
def test_lengths(T, lens):
    ctx = Ctx()
    case = Case(T, 4, 2, 48, 40, lens=lens, pad=2)
    case.forward(ctx)
    case.backward(ctx)
    case.check()
    ctx.close()


@pytest.mark.parametrize("T", [4, 140])
def test_states_that_are_absent_or_in_place(T):
    ctx = Ctx()
    case = Case(T, 2, 2, 32, 24, first=False, last=False)
    case.forward(ctx)
    case.backward(ctx)
    case.check()
    case = Case(T, 2, 2, 32, 24)
    h0, dhT = case.h0.clone(), case.dhT.clone()
    case.forward(ctx, hT=case.h0)
    case.backward(ctx, dh0=case.dhT)
    case.hT, case.h0, case.dh0, case.dhT = case.h0, h0, case.dhT, dhT
    case.check()
    y = case.y.clone()
    case.forward(ctx, save=False, hT=None)
    assert torch.equal(y, case.y)
    case.backward(ctx, dh0=None)
    case.check()
    ctx.close()


@pytest.mark.parametrize("T", [6, 100, 200])
@pytest.mark.parametrize("eps", [1e-6, 0.0, -1.0])
def test_gates_at_their_ends(T, eps):
    """Gates of exactly 0 and 1, rows of zeros."""
    ctx = Ctx()
    case = Case(T, 2, 2, 32, 40, eps=eps)
    inf = float("inf")
    zf, zb = case.zf.view(T, 2, -1), case.zb.view(T, 2, -1)
    zf[::5, 0] = -inf
    zf[1::3, 1, 0] = inf
    zb[::4, 0] = -inf
    zb[2::7, 1] = inf
    zf[3, 0], zb[3, 1] = -200.0, -200.0
    case.k.view(T, 2, -1)[2::9, 0] = 0
    case.q.view(T, 2, -1)[4::9, 1] = 0
    case.forward(ctx)
    case.backward(ctx)
    case.check()
    ctx.close()


def test_the_past_ends_at_a_gate_of_zero():
    """What comes before a gate of -infinity changes nothing behind it, however large."""
    ctx = Ctx()
    T, cut = 150, 77
    a = Case(T, 1, 2, 64, 64)
    a.zf[cut] = float("-inf")
    a.forward(ctx)
    a.backward(ctx)
    b = Case(T, 1, 2, 64, 64)
    b.zf[cut] = float("-inf")
    b.v[:cut] *= 1e4
    b.h0 *= 1e6
    b.forward(ctx)
    b.backward(ctx)
    assert torch.equal(a.hT, b.hT) and torch.equal(a.y[cut:], b.y[cut:])
    assert bool((a.dh0 == b.dh0).all()) and bool((a.dzf[cut] == 0).all())
    a.check()
    ctx.close()


@pytest.mark.parametrize("scale_v", [2.0 ** -100, 2.0 ** 60])
def test_values_of_any_size(scale_v):
    """The rule is linear in v and the state."""
    ctx = Ctx()
    case = Case(100, 1, 2, 64, 48)
    case.v *= scale_v
    case.h0 *= scale_v
    case.forward(ctx)
    case.check(gradient=False)
    ctx.close()


def test_keys_that_repeat():
    """Steps that all write to the same place: the triangular system at its fullest."""
    ctx = Ctx()
    case = Case(128, 2, 1, 64, 64, shift=6.0)
    case.k.view(128, 2, -1)[:] = case.k.view(128, 2, -1)[0]
    case.zb[:] = 4.0
    case.forward(ctx)
    case.backward(ctx)
    case.check()
    ctx.close()


def test_token_by_token_is_the_whole_sequence():
    ctx = Ctx()
    T, B, h, Dk, Dv = 40, 3, 2, 128, 96
    case = Case(T, B, h, Dk, Dv)
    case.forward(ctx)
    state, y = case.h0.clone(), torch.empty_like(case.y)
    for t in range(T):
        r = slice(t * B, (t + 1) * B)
        ard.ard_delta_forward(ctx.h, BF16, 1, B, h, Dk, Dv, case.scale, case.eps, case.q[r], h * Dk, case.k[r], h * Dk, case.v[r], h * Dv, case.zf[r], case.zb[r], h,
                              None, state, y[r], h * Dv, state, None, None, 0)
    x, _ = case.inputs()
    want = OD.fwd(*x, np.float32(case.scale), np.float32(case.eps), None, host(case.h0))
    case.near("y", y, want[0])
    case.near_state("state", state, want[1][-1])
    case.check(gradient=False)
    ctx.close()


def test_gradient_against_differences():
    """Directions in v, the first state and (by what the gates are) their pre-activations, by differences of the formulas in fp64."""
    ctx = Ctx()
    case = Case(90, 1, 2, 24, 20)
    case.forward(ctx)
    case.backward(ctx)
    x, dy = case.inputs()
    h0, dhT = host(case.h0), host(case.dhT)
    got = [host(t).reshape(s.shape) for t, s in zip((case.dq, case.dk, case.dv, case.dzf, case.dzb), x)] + [host(case.dh0)]

    def loss(x, h0):
        y, S, _ = OD.fwd(*x, np.float32(case.scale), np.float32(case.eps), None, h0)
        return (y * dy).sum() + (S[-1] * dhT).sum()
    rng = np.random.default_rng(3)
    for i in range(6):
        d = rng.normal(size=got[i].shape)
        move = lambda e: loss([a + (e * d if j == i else 0) for j, a in enumerate(x)], h0 + (e * d if i == 5 else 0))  # noqa: E731
        slope = (move(1e-5) - move(-1e-5)) / 2e-5
        want = (got[i] * d).sum()
        # roundings of the gradient's entries, half a step each at random signs, five times their standard deviation; and the quotient's own error
        assert abs(slope - want) <= 5 * 2.0 ** -8 * np.sqrt(((got[i] * d) ** 2).sum()) + 1e-6 * np.abs(got[i] * d).sum(), i
    ctx.close()


def test_no_steps():
    ctx = Ctx()
    h = torch.randn((2, 3, 16, 8), device="cuda")
    out, e = torch.empty_like(h), torch.empty(8, dtype=BF, device="cuda")
    ard.ard_delta_forward(ctx.h, BF16, 0, 2, 3, 16, 8, 1.0, 0.0, e, 48, e, 48, e, 24, e, e, 3, None, h, e, 24, out, None, None, 0)
    assert torch.equal(out, h)
    out.fill_(7)
    ard.ard_delta_backward(ctx.h, BF16, 0, 2, 3, 16, 8, 1.0, 0.0, e, 48, e, 48, e, 24, e, e, 3, None, None, e, 24, None, e, 48, e, 48, e, 24, e, e, 3, out, None, 0)
    assert bool((out == 0).all())
    ctx.close()


@pytest.mark.parametrize("T", [9, 100])
def test_two_graphs_over_one_workspace(T):
    """Two captured forward and backward passes of different sizes that share their work, replayed in turn on other inputs, on a stream of their own."""
    ctx = Ctx()
    cases = [Case(T, 3, 2, 64, 72, lens=[T, T // 2, 0]), Case(2 * T, 1, 5, 128, 128, seed=1)]
    need = max(ard.ard_delta_work_bytes(c.T, c.B, c.h, c.Dk, c.Dv, True) for c in cases)
    shared = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    side, graphs = torch.cuda.Stream(), []
    for c in cases:
        c.work = lambda backward, c=c: (shared, ard.ard_delta_work_bytes(c.T, c.B, c.h, c.Dk, c.Dv, backward))
        side.wait_stream(torch.cuda.current_stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            c.forward(ctx, stream=side.cuda_stream)
            c.backward(ctx, stream=side.cuda_stream)
    for seed in (8, 9):
        rng = np.random.default_rng(seed)
        for c in cases:
            c.fill(c.v, c.h * c.Dv, rng.normal(size=(c.T, c.B, c.h * c.Dv)))
            c.fill(c.zf, c.h, rng.normal(size=(c.T, c.B, c.h)) * 1.5 + 3)
            c.fill(c.dy, c.h * c.Dv, rng.normal(size=(c.T, c.B, c.h * c.Dv)))
        for g in graphs:
            g.replay()
        for c in cases:
            c.check()
    ctx.close()


def test_rows_that_lie_2_to_the_32_elements_apart():
    """Column blocks of one matrix whose offsets pass 32 bits, in elements."""
    T, B, h, Dk, Dv = 70, 1, 2, 16, 24
    ld = 1 << 26
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("two matrices of 9.4 GB")
    ctx = Ctx()
    case = Case(T, B, h, Dk, Dv)
    n = h * Dk
    big, grad = (torch.empty((T, ld), dtype=BF, device="cuda") for _ in range(2))
    at = (0, n, 2 * n, ld - 2 * h, ld - h)
    widths = (n, n, h * Dv, h, h)
    parts = [big[:, a:a + w] for a, w in zip(at, widths)]
    for part, x in zip(parts, (case.q, case.k, case.v, case.zf, case.zb)):
        part.copy_(x)
    q, k, v, zf, zb = parts
    outs = [grad[:, a:a + w] for a, w in zip(at, widths)]
    w, size = case.work(True)
    args = (ctx.h, BF16, T, B, h, Dk, Dv, case.scale, case.eps, q, ld, k, ld, v, ld, zf, zb, ld, None)
    ard.ard_delta_forward(*args, case.h0, case.y, h * Dv, case.hT, case.S, w, size)
    ard.ard_delta_backward(*args, case.S, case.dy, h * Dv, case.dhT, outs[0], ld, outs[1], ld, outs[2], ld, outs[3], outs[4], ld, case.dh0, w, size)
    for mine, there in zip((case.dq, case.dk, case.dv, case.dzf, case.dzb), outs):
        mine.copy_(there)
    case.check()
    ctx.close()
