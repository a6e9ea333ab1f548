"""Pins for oracle/layer_norm.py, oracle/glr.py and oracle/adamw.py."""
import numpy as np
import pytest
import torch

from oracle import adamw as OA
from oracle import glr as OR
from oracle import layer_norm as ON
from oracle import pattern as OP


def _t(x, grad=False):
    return torch.tensor(np.asarray(x), dtype=torch.float64, requires_grad=grad)


def test_layer_norm_is_the_librarys():
    rng = np.random.default_rng(1)
    X, w, b, dY = rng.normal(0.4, 2, (7, 33)), rng.normal(1, 0.2, 33), rng.normal(0, 1, 33), rng.normal(size=(7, 33))
    x, tw, tb = _t(X, True), _t(w, True), _t(b, True)
    y = torch.nn.functional.layer_norm(x, (33,), tw, tb, 1e-5)
    y.backward(_t(dY))
    Y, mean, rstd = ON.fwd(X, w, b, 1e-5)
    got = (Y,) + ON.bwd(dY, X, w, mean, rstd)
    for a, r in zip(got, (y.detach(), x.grad, tw.grad, tb.grad)):
        assert np.abs(a - r.numpy()).max() <= 1e-12
    h = 1e-6                      # a difference quotient of <dY, Y> along one direction of each input
    for k, at in enumerate((X, w, b)):
        D = rng.normal(size=at.shape)
        args = [X, w, b]
        f = lambda s: (dY * ON.fwd(*[a + s * h * D if q == k else a for q, a in enumerate(args)], 1e-5)[0]).sum()  # noqa: E731
        assert abs((f(1) - f(-1)) / (2 * h) - (got[1 + k] * D).sum()) <= 1e-5


def _torch_glr(zf, zg, zo, alpha, lens, h0):
    c, ys = h0, []
    for t in range(zf.shape[0]):
        f = torch.sigmoid(zf[t])
        live = torch.tensor(t < np.asarray(lens))[:, None]
        c = torch.where(live, f * c + (1 - f) * zg[t], c)
        ys.append(torch.where(live, alpha * c * (1 if zo is None else torch.sigmoid(zo[t])), torch.zeros_like(c)))
    return torch.stack(ys), c


@pytest.mark.parametrize("gate", [True, False])
def test_recurrence_is_what_autograd_makes_of_it(gate):
    rng = np.random.default_rng(2)
    T, B, n, alpha, lens = 9, 4, 5, 1.7, [9, 0, 3, 12]
    z = [rng.normal(size=(T, B, n)) * 2 for _ in range(3)]
    if not gate:
        z[2] = None
    h0, dy, dhT = rng.normal(size=(B, n)), rng.normal(size=(T, B, n)), rng.normal(size=(B, n))
    tz, th = [None if a is None else _t(a, True) for a in z], _t(h0, True)
    y, hT = _torch_glr(*tz, alpha, lens, th)
    ((y * _t(dy)).sum() + (hT * _t(dhT)).sum()).backward()
    Y, c, _, ec = OR.fwd(*z, alpha, lens, h0)
    grads, _ = OR.bwd(*z, alpha, c, ec, dy, lens, dhT)
    assert np.abs(Y - y.detach().numpy()).max() <= 1e-12 and np.abs(c[-1] - hT.detach().numpy()).max() <= 1e-12
    for a, r in zip(grads, tz + [th]):
        assert (a is None) == (r is None)
        if a is not None:
            assert np.abs(a - r.grad.numpy()).max() <= 1e-12
    h = 1e-6
    args = z[:2] + ([z[2]] if gate else [])
    for k in range(len(args) + 1):
        D = rng.normal(size=h0.shape if k == len(args) else args[k].shape)

        def f(s):
            a = [x + s * h * D if q == k else x for q, x in enumerate(args)] + ([] if gate else [None])
            Yk, ck, _, _ = OR.fwd(*a, alpha, lens, h0 + s * h * D if k == len(args) else h0)
            return (Yk * dy).sum() + (ck[-1] * dhT).sum()
        want = grads[3] if k == len(args) else grads[k]
        assert abs((f(1) - f(-1)) / (2 * h) - (want * D).sum()) <= 1e-5


def test_recurrence_padded_and_cut():
    rng = np.random.default_rng(3)
    T, B, n = 11, 2, 3
    z = [rng.normal(size=(T, B, n)) for _ in range(3)]
    h0 = rng.normal(size=(B, n))
    y, c, _, _ = OR.fwd(*z, 1.0, None, h0)
    y1, c1, _, _ = OR.fwd(*[a[:4] for a in z], 1.0, None, h0)
    y2, c2, _, _ = OR.fwd(*[a[4:] for a in z], 1.0, None, c1[-1])
    assert np.array_equal(np.concatenate([y1, y2]), y) and np.array_equal(c2[-1], c[-1])
    yp, cp, _, _ = OR.fwd(*z, 1.0, [4, 11], h0)
    assert np.array_equal(yp[:4, 0], y1[:, 0]) and not yp[4:, 0].any() and np.array_equal(cp[-1, 0], c1[-1, 0])
    z[0][5] = -np.inf                                    # the past does not enter
    ya, _, _, _ = OR.fwd(*z, 1.0, None, h0)
    yb, _, _, _ = OR.fwd(*z, 1.0, None, h0 + 7.0)
    assert np.array_equal(ya[5:], yb[5:]) and np.array_equal(ya[5], (1 / (1 + np.exp(-z[2][5]))) * z[1][5])


def test_optimiser_is_the_librarys():
    rng = np.random.default_rng(4)
    p0 = rng.normal(size=50)
    tp = _t(p0, True)
    opt = torch.optim.AdamW([tp], lr=0.01, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    p, m, v = p0, np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.normal(size=50)
        tp.grad = _t(g)
        opt.step()
        m, v = OA.moments(m, v, g, 0.9, 0.99)
        p = OA.step(p, m, v, 0.01, 0.9, 0.99, 1e-8, 0.1, t)
        assert np.abs(p - tp.detach().numpy()).max() <= 1e-12


def test_random_words_are_the_generators():
    w = OA.words(10, (5 << 32) + 9, (3 << 32) + 2, 6)
    for e in range(10):
        assert int(w[e]) == OP.philox4x32_10((2, 3, e // 4, 7), (9, 5))[e % 4]


def test_eight_bit_floats():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()   # 0 .. 448
    assert codes[-1] == OA.LARGEST and (np.diff(codes) > 0).all()
    one = np.array([1.0])
    for r in (0, 1, 65535):                                # a value on the grid stays
        pad = np.concatenate([codes, [0.0]])
        assert np.array_equal(OA.rounded(pad, one, np.full(128, r)), pad)
    rng = np.random.default_rng(5)
    x = np.exp(rng.uniform(np.log(1e-4), np.log(440), 128))
    below = codes[np.searchsorted(codes, x, side="right") - 1]
    above = codes[np.searchsorted(codes, x, side="right")]
    r = rng.integers(0, 65536, (4096, 128))
    got = np.stack([OA.rounded(x, one, w) for w in r])
    assert ((got == below) | (got == above)).all()
    # the mean of 4096 draws: six standard errors of a value that is one of two, half a step of the 16 bits
    spread = 6 * (above - below) / 2 / 64 + (above - below) / 65536
    assert (np.abs(got.mean(axis=0) - x) <= spread).all()
    assert OA.rounded(np.full(128, 1e-9), one, np.zeros(128), root=True).min() == 2.0 ** -9
    assert not OA.rounded(np.full(128, 1e-9), one, np.zeros(128)).any()
    assert OA.scales(np.array([0.0, -896.0] + [1.0] * 127)).tolist() == [2.0, 1 / 448]
    assert OA.scales(np.full(3, 2.0 ** -111)).tolist() == [0.0]


def test_a_second_moment_held_in_eight_bits_decays():
    """448 gradients of one size, then none for 600 steps except in the block's first element: the mean of the squares follows
    0.999^600 = 0.549 (rounding to nearest would leave every root where it was)."""
    n, t = 1024, 0
    r, s = np.zeros(n), np.zeros(n // 128)
    keep = np.arange(n) % 128 == 0
    start = None
    for t in range(1, 1049):
        g = np.where(keep | (t <= 448), 1.0, 0.0)
        _, v = OA.moments(0.0, (r * np.repeat(s, 128)) ** 2, g, 0.9, 0.999)
        root = np.sqrt(v)
        s = OA.scales(root)
        r = OA.rounded(root, s, OA.words(n, 77, t, 0) >> np.uint64(16), root=True)
        if t == 448:
            start = (r * np.repeat(s, 128)) ** 2
    end = (r * np.repeat(s, 128)) ** 2
    # a move of the root by a step of at most an eighth of it, with chance 0.0005 * 8, adds 6e-5 of the square to its mean in a step: 4 % in
    # 600 steps; the mean of 1016 squares that scatter by less than their size adds 10 %
    ratio = end[~keep].mean() / start[~keep].mean()
    assert 0.45 < ratio < 0.70, ratio
