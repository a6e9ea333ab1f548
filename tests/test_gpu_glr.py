"""ard_glr_forward / ard_glr_backward against the recurrence in fp64, with bounds carried through it (oracle/glr.py)."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host, tdtype
from oracle import glr as OR
from oracle import pattern as OP
from paper_2203_05705_b200 import ard

pytestmark = pytest.mark.gpu
F32, BF16 = ard.ARD_F32, ard.ARD_BF16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


class Case:
    def __init__(self, dtype, T, B, H, gate, lens=None, dp=1, b=1, ldz=0, ldy=0, lddz=0, off=0, alpha=1.5, seed=0, shift=1.0):
        self.dtype, self.T, self.B, self.H, self.gate, self.alpha = dtype, T, B, H, gate, alpha
        self.keep = np.arange(H) if dp == 1 else OP.row_keep(H, dp, b)
        self.n = n = len(self.keep)
        self.ldz, self.ldy, self.lddz, self.off = H + ldz, H + ldy, H + lddz, off
        self.lens = None if lens is None else np.asarray(lens, np.int32)
        rng = np.random.default_rng(seed)
        live = np.ones((T, B), bool) if lens is None else np.arange(T)[:, None] < np.clip(self.lens, 0, T)[None, :]
        fill = lambda x: np.where(live[..., None], x, np.nan).astype(np.float32)  # noqa: E731  (rows behind the end: not to be read)
        self.zf = self.buf(self.ldz, fill(rng.normal(size=(T, B, n)) * 2 + shift))
        self.zg = self.buf(self.ldz, fill(rng.normal(size=(T, B, n))))
        self.zo = self.buf(self.ldz, fill(rng.normal(size=(T, B, n)))) if gate else None
        self.dy = self.buf(self.ldy, fill(rng.normal(size=(T, B, n))))
        self.h0, self.dhT = (torch.from_numpy(rng.normal(size=(B, H)).astype(np.float32)).cuda() for _ in range(2))
        self.y = self.buf(self.ldy)
        self.dz = [self.buf(self.lddz) for _ in range(3 if gate else 2)] + ([] if gate else [None])
        self.S = torch.full((-(-T // ard.ARD_GLR_CHUNK), B, H), float("nan"), device="cuda")
        self.hT, self.dh0 = (torch.full((B, H), float("nan"), device="cuda") for _ in range(2))
        self.dlens = None if lens is None else torch.from_numpy(self.lens).cuda()

    def buf(self, ld, values=None):
        T, B = self.T, self.B
        t = torch.full((T * B * ld + self.off + 64,), float("nan"), dtype=tdtype(self.dtype), device="cuda")
        t = t[self.off:self.off + T * B * ld].view(T, B, ld)
        if values is not None:
            t[..., :self.n] = torch.from_numpy(values).to(tdtype(self.dtype))
        return t

    def forward(self, ctx, pat=None):
        ard.ard_glr_forward(ctx, pat, self.dtype, self.T, self.B, self.H, self.alpha, self.zf, self.zg, self.zo, self.ldz, self.dlens, self.h0,
                            self.y, self.ldy, self.hT, self.S)

    def backward(self, ctx, pat=None):
        ard.ard_glr_backward(ctx, pat, self.dtype, self.T, self.B, self.H, self.alpha, self.zf, self.zg, self.zo, self.ldz, self.dlens, self.S,
                             self.dy, self.ldy, self.dhT, *self.dz, self.lddz, self.dh0)

    def outputs(self):
        return [t for t in [self.y, self.hT, self.S, self.dh0] + self.dz if t is not None]

    def check(self):
        n, T = self.n, self.T
        z = [np.nan_to_num(host(t)[..., :n], posinf=np.inf, neginf=-np.inf) if t is not None else None for t in (self.zf, self.zg, self.zo)]
        dy = np.nan_to_num(host(self.dy)[..., :n])
        h0, dhT = host(self.h0)[:, self.keep], host(self.dhT)[:, self.keep]
        y, c, ey, ec = OR.fwd(*z, self.alpha, self.lens, h0)
        grads, errs = OR.bwd(*z, self.alpha, c, ec, dy, self.lens, dhT)
        half = HALF_STEP[self.dtype]

        def near(got, want, err, half):
            off = np.abs(got - want)
            assert (off <= half * np.abs(want) + (1 + half) * err + 1e-37).all(), float(np.nanmax(off))
        near(host(self.y)[..., :n], y, ey, half)
        near(host(self.hT)[:, self.keep], c[-1], ec[-1], 0.0)
        for g, want, err in zip(self.dz, grads[:3], errs[:3]):
            if g is not None:
                near(host(g)[..., :n], want, err, half)
        near(host(self.dh0)[:, self.keep], grads[3], errs[3], 0.0)
        for t in [self.y] + self.dz:
            if t is not None:
                assert bool(torch.isnan(t[..., n:]).all())            # nothing behind the columns
                if self.lens is not None and T:
                    for b, L in enumerate(np.clip(self.lens, 0, T)):
                        assert bool((t[L:, b, :n] == 0).all())
        dropped = np.setdiff1d(np.arange(self.H), self.keep)
        for t in (self.hT, self.dh0):
            assert bool(torch.isnan(t[:, dropped]).all())
        assert ard.ard_last_device_status(_ctx().h) == 0


_held = []


def _ctx():
    if not _held:
        _held.append(Ctx(0))
    return _held[0]


def _both(case, pat=None):
    case.forward(_ctx().h, pat)
    case.backward(_ctx().h, pat)
    case.check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("T,B,H", [(1, 1, 1), (1, 3, 65), (2, 2, 64), (3, 1, 7), (7, 4, 33), (8, 2, 128), (17, 3, 130), (63, 2, 96), (64, 1, 64),
                                   (65, 2, 64), (128, 2, 32), (129, 1, 31), (200, 5, 100), (511, 1, 62), (1025, 2, 40), (4096, 1, 18), (35, 64, 256)])
def test_shapes(dtype, gate, T, B, H):
    _both(Case(dtype, T, B, H, gate, seed=T + B + H))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,lens", [(1, [0, 1, 5]), (5, [5, 0, 2, -3, 9]), (64, [64, 63, 1, 0]), (130, [130, 65, 64, 0, 129]), (700, [0, 700, 333, 64]),
                                    (300, [0, 0, 0])])
@pytest.mark.parametrize("H,gate", [(48, True), (33, False)])
def test_padded_batches(dtype, T, lens, H, gate):
    _both(Case(dtype, T, len(lens), H, gate, lens=lens, seed=T))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,B,H,dp,b,lens,ld", [(35, 16, 1024, 2, 1, None, 0), (70, 3, 100, 3, 3, [70, 0, 41], 0), (9, 2, 64, 64, 50, None, 8),
                                                (300, 1, 257, 5, 2, [299], 1), (1, 8, 96, 4, 4, None, 0), (130, 2, 200, 1, 1, None, 0)])
def test_kept_units(dtype, T, B, H, dp, b, lens, ld):
    pat = _ctx().pattern(ard.ARD_ROW, 16, H)
    ard.ard_pattern_set(_ctx().h, pat, dp, b)
    _both(Case(dtype, T, B, H, True, lens=lens, dp=dp, b=b, ldz=ld, ldy=ld, lddz=ld, alpha=float(dp), seed=H), pat)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ldz,ldy,lddz,off", [(6, 10, 2, 0), (1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (0, 0, 0, 2), (8, 8, 8, 8)])
def test_strides_and_alignment(dtype, ldz, ldy, lddz, off):
    _both(Case(dtype, 77, 3, 50, True, ldz=ldz, ldy=ldy, lddz=lddz, off=off, seed=ldz + off))


def test_gate_blocks_of_one_matrix():
    T, B, H = 90, 2, 64
    c = Case(BF16, T, B, H, True, seed=4)
    Z = torch.stack([c.zf, c.zg, c.zo], dim=2).contiguous()              # [T][B][3][H]
    dZ = torch.empty_like(Z)
    c.zf, c.zg, c.zo = (Z[:, :, k] for k in range(3))
    c.dz = [dZ[:, :, k] for k in range(3)]
    c.ldz = c.lddz = 3 * H
    _both(c)


@pytest.mark.parametrize("T", [1, 5, 64, 200])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gates_at_their_ends(T, dtype):
    """Gates shut and open to the last bit: -infinity starts anew, +infinity holds, 100 is as good as either."""
    c = Case(dtype, T, 2, 40, True, seed=T)
    for k, v in enumerate((-np.inf, np.inf, 100.0, -100.0)):
        c.zf[k % T::4, :, k::5] = v
        c.zo[(k + 1) % T::4, :, k::5] = v
    _both(c)


def test_a_closed_gate_hides_what_came_before():
    T = 150
    outs = []
    for first in (1.0, 1e30):
        c = Case(F32, T, 1, 64, False, seed=1)
        c.h0.fill_(first)
        c.zg[:70].mul_(first)
        c.zf[70] = -np.inf
        c.forward(_ctx().h)
        c.backward(_ctx().h)
        outs.append([t.clone() for t in (c.y[70:], c.dz[0][71:], c.dz[1][70:])])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("dtype,T", [(F32, 300), (BF16, 65), (BF16, 2)])
def test_a_sequence_in_pieces(dtype, T):
    """The state handed from call to call, in place, and tokens one by one, against the whole sequence."""
    B, H = 3, 48
    whole = Case(dtype, T, B, H, True, seed=9)
    _both(whole)
    for cuts in ([T // 2], list(range(1, T)) if T <= 65 else [1, 2, 3, 67, 200]):
        state, y = whole.h0.clone(), torch.full_like(whole.y, float("nan"))
        ends = [0] + cuts + [T]
        for t0, t1 in zip(ends, ends[1:]):
            ard.ard_glr_forward(_ctx().h, None, dtype, t1 - t0, B, H, whole.alpha, whole.zf[t0:], whole.zg[t0:], whole.zo[t0:], H, None, state,
                                y[t0:], H, state, None)
        z = [host(t) for t in (whole.zf, whole.zg, whole.zo)]
        yo, c, ey, ec = OR.fwd(*z, whole.alpha, None, host(whole.h0))
        assert (np.abs(host(state) - c[-1]) <= ec[-1]).all()
        assert (np.abs(host(y) - yo) <= HALF_STEP[dtype] * np.abs(yo) + 1.01 * ey).all()


def test_states_and_gradients_that_are_left_out():
    T, B, H = 100, 2, 32
    c = Case(F32, T, B, H, False, seed=3)
    c.h0.zero_()
    c.dhT.zero_()
    _both(c)
    y, dz, dh0 = c.y.clone(), [t.clone() for t in c.dz if t is not None], c.dh0.clone()
    c.y.fill_(7.0)
    h = _ctx().h
    ard.ard_glr_forward(h, None, F32, T, B, H, c.alpha, c.zf, c.zg, None, H, None, None, c.y, H, None, None)
    assert torch.equal(y, c.y)
    ard.ard_glr_backward(h, None, F32, T, B, H, c.alpha, c.zf, c.zg, None, H, None, c.S, c.dy, H, None, c.dz[0], c.dz[1], None, H, None)
    assert all(torch.equal(a, b) for a, b in zip(dz, c.dz))
    q = c.dhT.clone()                                      # in place
    ard.ard_glr_backward(h, None, F32, T, B, H, c.alpha, c.zf, c.zg, None, H, None, c.S, c.dy, H, q, c.dz[0], c.dz[1], None, H, q)
    assert torch.equal(q, dh0)


def test_no_steps_no_sequences():
    h = _ctx().h
    z = torch.zeros(64, device="cuda")
    h0 = torch.randn(2, 16, device="cuda")
    y, hT, dh0 = (torch.full((2, 16), 7.0, device="cuda") for _ in range(3))
    ard.ard_glr_forward(h, None, F32, 0, 2, 16, 1.0, z, z[16:], None, 16, None, h0, y, 16, hT, None)
    ard.ard_glr_backward(h, None, F32, 0, 2, 16, 1.0, z, z[16:], None, 16, None, z, z, 16, h0, y, hT.new_zeros(32), None, 16, dh0)
    assert torch.equal(hT, h0) and torch.equal(dh0, h0) and bool((y == 7).all())
    for B, H in ((0, 16), (2, 0)):
        ard.ard_glr_forward(h, None, F32, 3, B, H, 1.0, z, z[16:], None, 16, None, h0, y, 16, hT, None)
    assert torch.equal(hT, h0) and bool((y == 7).all())


@pytest.mark.parametrize("dtype,T,B,H,lens", [(BF16, 2000, 1, 64, None), (F32, 130, 3, 70, [130, 7, 99]), (BF16, 35, 64, 1024, None)])
def test_graph_replays_and_repeats_give_the_same_bits(dtype, T, B, H, lens):
    c = Case(dtype, T, B, H, True, lens=lens, seed=5)
    h = _ctx().h
    c.forward(h)
    c.backward(h)
    first = [t.clone() for t in c.outputs()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.forward(h)
        c.backward(h)
    same = lambda a, b: torch.equal(torch.nan_to_num(a, 3.0), torch.nan_to_num(b, 3.0))  # noqa: E731
    for _ in range(2):
        for t in c.outputs():
            t.fill_(float("nan"))
        graph.replay()
        assert all(same(a, b) for a, b in zip(first, c.outputs()))
    c.h0.add_(1.0)                                         # other inputs in the same memory
    graph.replay()
    assert not same(first[0], c.y)
    c.check()


def test_a_captured_draw_is_followed():
    """A pattern drawn inside the graph: every replay runs over the units that it drew."""
    T, B, H = 20, 4, 96
    h = _ctx().h
    pat = _ctx().pattern(ard.ARD_ROW, 16, H)
    K = np.zeros(4)
    K[[0, 1, 3]] = 1 / 3
    ard.ard_set_distribution(h, 3, K)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    c = Case(F32, T, B, H, True, seed=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ard.ard_sample_pattern_counter(h, pat, 3, 11, 0, counter, 1, 0)
        c.forward(h, pat)
        c.backward(h, pat)
    seen = set()
    for _ in range(8):
        for t in c.outputs():
            t.fill_(float("nan"))
        graph.replay()
        dp, b, nk, idx = ard.ard_pattern_to_host(pat, H)
        c.keep, c.n = idx, nk
        c.check()
        seen.add(dp)
    assert len(seen) > 1


def test_offsets_beyond_32_bits():
    """2^31 elements lie between the first and the last step: 33 steps of one row each in a matrix with a pitch of 2^26."""
    T, H, ld = 33, 64, 1 << 26
    h = _ctx().h
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn((T, 1, 2 * H), generator=g, device="cuda").to(torch.bfloat16)
    big = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, 1, ld)
    big[..., :2 * H] = z
    y = torch.empty((T, 1, H), dtype=torch.bfloat16, device="cuda")
    want = torch.empty_like(y)
    ard.ard_glr_forward(h, None, BF16, T, 1, H, 1.0, big, big[..., H:], None, ld, None, None, y, H, None, None)
    ard.ard_glr_forward(h, None, BF16, T, 1, H, 1.0, z, z[..., H:], None, 2 * H, None, None, want, H, None, None)
    assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("T,B,H,lens,ld,off", [(300, 6, 320, None, 0, 0), (700, 6, 320, [700, 0, 64, 65, 321, 1], 0, 0), (129, 3, 450, [129, 128, 127], 6, 0),
                                               (200, 6, 321, None, 0, 1), (65, 20, 64, None, 0, 0), (1100, 2, 640, None, 0, 0)])
def test_clusters_of_whole_warps(dtype, gate, T, B, H, lens, ld, off):
    """Between 19 and 74 units of a warp's channels: clusters share the sequences, and would fill the device without half warps."""
    _both(Case(dtype, T, B, H, gate, lens=lens, ldz=ld, ldy=ld, lddz=ld, off=off, seed=T + H))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,B,H,dp,b,lens", [(300, 6, 640, 2, 2, None), (400, 2, 200, 3, 1, [400, 333]), (1000, 1, 64, 16, 5, None), (257, 3, 33, 33, 33, [0, 257, 129])])
def test_clusters_over_kept_units(dtype, T, B, H, dp, b, lens):
    pat = _ctx().pattern(ard.ARD_ROW, 16, H)
    ard.ard_pattern_set(_ctx().h, pat, dp, b)
    _both(Case(dtype, T, B, H, True, lens=lens, dp=dp, b=b, seed=T + dp), pat)


@pytest.mark.parametrize("dtype,T,B,H,lens", [(BF16, 500, 1, 256, None), (F32, 300, 2, 64, [300, 40]), (BF16, 300, 6, 320, None),
                                              (BF16, 30, 3, 64, [30, 0, 7]), (F32, 1, 3, 64, None)])
def test_states_in_place(dtype, T, B, H, lens):
    """hT may be h0, dh0 may be dhT: the same bits as in places of their own."""
    c = Case(dtype, T, B, H, True, lens=lens, seed=T)
    _both(c)
    want, grad, y = c.hT.clone(), c.dh0.clone(), c.y.clone()
    c.hT, c.dh0 = c.h0, c.dhT
    c.forward(_ctx().h)
    c.backward(_ctx().h)
    assert torch.equal(c.hT, want) and torch.equal(c.dh0, grad) and torch.equal(c.y, y)


@pytest.mark.parametrize("T,B,H", [(300, 1, 128), (300, 6, 320), (20, 2, 64)])
def test_the_first_call_of_a_context_may_be_captured(T, B, H):
    c, fresh = Case(BF16, T, B, H, True, seed=1), Ctx(0)
    try:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.forward(fresh.h)
            c.backward(fresh.h)
        graph.replay()
        torch.cuda.synchronize()
        c.check()
        del graph
    finally:
        fresh.close()


def test_two_streams_at_once():
    """Calls on two streams share nothing but the inputs."""
    cases = [Case(BF16, 900, 1, 256, True, seed=k) for k in range(2)] + [Case(BF16, 40, 30, 256, True, seed=k) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.forward(_ctx().h)
                c.backward(_ctx().h)
    torch.cuda.synchronize()
    for c in cases:
        c.check()
