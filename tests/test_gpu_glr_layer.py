"""The operators of a recurrent layer run together (paper_2203_05705_b200/glr.py): norm, gate products, recurrence, their gradients, the norm of all
gradients and the optimiser's step; two layers, the upper one over the kept units of the lower.  Every stage is held against its statement in fp64 on
what the stage before it left on the device, within that stage's own roundings."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host
from oracle import adamw as OA
from oracle import glr as OR
from oracle import layer_norm as ON
from oracle import pattern as OP
from paper_2203_05705_b200 import ard
from paper_2203_05705_b200.glr import GlrLayer

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
U, HALF = 2.0 ** -24, 2.0 ** -8
SUM = 2 * U            # of a term, per addition: the tensor cores may cut off where others round


def _close(got, want, err, half=HALF):
    off = np.abs(got - want)
    assert (off <= half * np.abs(want) + (1 + half) * err + 1e-37).all(), float(np.nanmax(off - half * np.abs(want) - err))


def _layer(ctx, pat, in_pat, T, B, I, H, seed):
    rng = np.random.default_rng(seed)
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))  # noqa: E731
    return GlrLayer(ctx, pat, in_pat, T, B, I, H, f(3 * H, I) / np.sqrt(I), f(3 * H) * 0.2, 1 + 0.2 * f(I), 0.2 * f(I))


class Stack:
    """Two layers under patterns that the test sets or draws."""

    def __init__(self, T, B, dims, seed=0, lens=None, full=True):
        self.ctx = Ctx(4 * T * B * 4 * max(dims) + (1 << 20))
        self.T, self.B, self.dims = T, B, dims
        I, H1, H2 = dims
        self.pats = [self.ctx.pattern(ard.ARD_ROW, I, H1), self.ctx.pattern(ard.ARD_ROW, H1, H2)]
        h = self.ctx.h
        self.layers = [_layer(h, self.pats[0], None, T, B, I, H1, seed), _layer(h, self.pats[1], self.pats[0], T, B, H1, H2, seed + 1)]
        rng = np.random.default_rng(seed + 2)
        new = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
        self.X, self.dY = new(T * B, I).to(BF), (new(T * B, H2) * 0.1).to(BF)
        self.h0, self.dhT = new(B, H2), new(B, H2)
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.alpha = (1.5, 2.0)

    def run(self):
        a, b = self.layers
        a.forward(self.X, self.alpha[0], lens=self.lens)
        b.forward(a.Y, self.alpha[1], h0=self.h0, lens=self.lens)
        b.backward(self.alpha[1], self.dY, self.dhT)
        a.backward(self.alpha[0], b.dX)

    def keeps(self, drawn):
        return [np.arange(n) if dp == 1 else OP.row_keep(n, dp, b) for n, (dp, b) in zip(self.dims[1:], drawn)]

    def check(self, drawn):
        torch.cuda.synchronize()
        assert ard.ard_last_device_status(self.ctx.h) == 0
        k1, k2 = self.keeps(drawn)
        lens = None if self.lens is None else self.lens.cpu().numpy()
        a, b = self.layers
        zero = np.zeros((self.B, len(k1)))
        check_forward(a, self.X, self.T, np.arange(self.dims[0]), k1, self.alpha[0], zero, lens)
        check_forward(b, a.Y, self.T, k1, k2, self.alpha[1], host(self.h0)[:, k2], lens)
        check_backward(b, a.Y, k1, k2, self.alpha[1], host(self.h0)[:, k2], lens, self.dY, host(self.dhT)[:, k2])
        check_backward(a, self.X, np.arange(self.dims[0]), k1, self.alpha[0], zero, lens, b.dX, zero)


def _gates_of(ly, T, n):
    z = host(ly.Z)[:T * ly.B].reshape(T, ly.B, 3, ly.H)[..., :n]
    return [z[:, :, k] for k in range(3)]


def check_forward(ly, X, T, keep_in, keep, alpha, h0, lens, hT=None):
    rows, ni, n = T * ly.B, len(keep_in), len(keep)
    x, w, b = host(X)[:rows, :ni], host(ly.p_nw)[keep_in], host(ly.p_nb)[keep_in]
    xn0, mean, rstd = ON.fwd(x, w, b, ly.eps)
    # as the norm's own tests: K units for fp32 sums and the operations around them
    K, size = 24 + ni / 32, np.abs(x).max(axis=1)
    e_rstd = K * U + 2 * rstd * (K + 1) * U * size                     # relative
    xh = (x - mean[:, None]) * rstd[:, None]
    e_xh = np.abs(xh) * (e_rstd + 4 * U)[:, None] + (rstd * (K + 1) * U * size)[:, None]
    xn = host(ly.Xn)[:rows, :ni]
    _close(xn, xn0, e_xh * np.abs(w) + 4 * U * (np.abs(xh * w) + np.abs(b)))
    W = host(ly.W).reshape(3, ly.H, ly.I)[:, keep][:, :, keep_in]
    bias = host(ly.p_b).reshape(3, ly.H)[:, keep]
    z = _gates_of(ly, T, n)
    for k in range(3):
        _close(z[k].reshape(rows, n), xn @ W[k].T + bias[k], (ni + 2) * SUM * (np.abs(xn) @ np.abs(W[k]).T + np.abs(bias[k])))
    y, c, ey, ec = OR.fwd(*z, alpha, lens, h0)
    _close(host(ly.Y)[:rows, :n].reshape(T, ly.B, n), y, ey)
    _close(host(ly.hT if hT is None else hT)[:, keep], c[-1], ec[-1], 0.0)
    return c, ec


def check_backward(ly, X, keep_in, keep, alpha, h0, lens, dY, dhT):
    T, B, I, H = ly.T, ly.B, ly.I, ly.H
    rows, ni, n = T * B, len(keep_in), len(keep)
    z = _gates_of(ly, T, n)
    _, c, _, ec = OR.fwd(*z, alpha, lens, h0)
    grads, errs = OR.bwd(*z, alpha, c, ec, host(dY)[:, :n].reshape(T, B, n), lens, dhT)
    dz = host(ly.dZ).reshape(T, B, 3, H)[..., :n]
    for k in range(3):
        _close(dz[:, :, k], grads[k], errs[k])
    _close(host(ly.dh0)[:, keep], grads[3], errs[3], 0.0)
    dz = [dz[:, :, k].reshape(rows, n) for k in range(3)]
    xn = host(ly.Xn)[:, :ni]
    W = host(ly.W).reshape(3, H, I)[:, keep][:, :, keep_in]
    dW, db = host(ly.dW).reshape(3, H, I), host(ly.db).reshape(3, H)
    dxn, rounded, err = 0.0, 0.0, 0.0
    for k in range(3):
        _close(dW[k][np.ix_(keep, keep_in)], dz[k].T @ xn, (rows + 2) * SUM * (np.abs(dz[k]).T @ np.abs(xn)), 0.0)
        _close(db[k][keep], dz[k].sum(axis=0), (rows + 2) * SUM * np.abs(dz[k]).sum(axis=0), 0.0)
        dxn = dxn + dz[k] @ W[k]
        rounded = rounded + np.abs(dxn)                               # every partial sum is rounded to bf16
        err = err + (n + 2) * SUM * (np.abs(dz[k]) @ np.abs(W[k]))
    got = host(ly.dXn)[:, :ni]
    assert (np.abs(got - dxn) <= 1.02 * (HALF * rounded + err) + 1e-37).all()
    gone = np.ones((H, I), bool)
    gone[np.ix_(keep, keep_in)] = False
    assert not dW[:, gone].any() and not np.delete(db, keep, axis=1).any()
    x, w = host(X)[:, :ni], host(ly.p_nw)[keep_in]
    mean, rstd = host(ly.mean), host(ly.rstd)
    dx0, dw0, db0 = ON.bwd(got, x, w, mean, rstd)
    xh = (x - mean[:, None]) * rstd[:, None]
    e_xh = 4 * U * (np.abs(xh) + (rstd * np.abs(x).max(axis=1))[:, None])
    e, K = np.abs(got * w), 24 + ni / 32
    m1, m2 = e.mean(axis=1, keepdims=True), (e * np.abs(xh)).mean(axis=1, keepdims=True)
    tol = K * U * (e + m1) + e_xh * m2 + np.abs(xh) * (K * U * m2 + (e * e_xh).mean(axis=1, keepdims=True)) + 6 * U * (e + m1 + np.abs(xh) * m2)
    _close(host(ly.dX)[:, :ni], dx0, rstd[:, None] * tol)
    Kr = 24 + rows / 4
    dw, db = host(ly.dnw), host(ly.dnb)
    _close(dw[keep_in], dw0, Kr * U * (np.abs(got) * np.abs(xh)).sum(axis=0) + (np.abs(got) * e_xh).sum(axis=0), 0.0)
    _close(db[keep_in], db0, Kr * U * np.abs(got).sum(axis=0), 0.0)
    assert not np.delete(dw, keep_in).any() and not np.delete(db, keep_in).any()


@pytest.mark.parametrize("T,B,dims,drawn,lens", [
    (35, 8, (64, 128, 192), ((2, 1), (3, 2)), None), (35, 8, (64, 128, 192), ((1, 1), (1, 1)), None),
    (70, 3, (40, 96, 64), ((5, 5), (2, 2)), (70, 0, 33)), (1, 5, (64, 64, 64), ((2, 2), (4, 1)), None),
    (9, 4, (37, 50, 31), ((2, 1), (3, 3)), (9, 1, 4, 20)), (130, 2, (256, 520, 136), ((16, 7), (1, 1)), None)])
def test_two_layers(T, B, dims, drawn, lens):
    s = Stack(T, B, dims, lens=lens)
    try:
        for pat, d in zip(s.pats, drawn):
            ard.ard_pattern_set(s.ctx.h, pat, *d)
        s.run()
        s.check(drawn)
    finally:
        s.ctx.close()


def test_two_layers_of_1024_units_over_35_steps():
    s = Stack(35, 64, (1024, 1024, 1024))
    try:
        for pat, d in zip(s.pats, ((2, 2), (3, 1))):
            ard.ard_pattern_set(s.ctx.h, pat, *d)
        s.run()
        s.check(((2, 2), (3, 1)))
    finally:
        s.ctx.close()


def test_tokens_one_by_one():
    """step() over the tokens of sequences: every one against its statement, the state handed on in place."""
    T, B, dims = 6, 4, (64, 128, 192)
    s = Stack(T, B, dims, seed=7)
    try:
        X = s.X.view(T, B, -1)
        for ly in s.layers:
            ly.pack()
        a, b = s.layers
        for t in range(T):
            before = [host(ly.h) for ly in s.layers]
            x = X[t].contiguous()
            y = a.step(x).contiguous()
            out = b.step(y)
            torch.cuda.synchronize()
            check_forward(a, x, 1, np.arange(dims[0]), np.arange(dims[1]), 1.0, before[0], None, hT=a.h)
            check_forward(b, y, 1, np.arange(dims[1]), np.arange(dims[2]), 1.0, before[1], None, hT=b.h)
            assert out.shape == (B, dims[2])
    finally:
        s.ctx.close()


K_DRAW = (0.3, 0.4, 0.3)


def _training(graphed, bits, steps=4):
    """Draw, forward, backward, gradient norm, step; everything that it leaves, and the patterns drawn."""
    s = Stack(20, 6, (64, 96, 128), seed=3, lens=(20, 3, 0, 20, 11, 19))
    try:
        h = s.ctx.h
        ard.ard_set_distribution(h, 1, np.array(K_DRAW))
        rows = s.layers[0].adamw_rows(0.1, bits) + s.layers[1].adamw_rows(0.1, bits)
        table, counter, norm = ard.adamw_tensors(rows), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")

        def call():
            ard.ard_sample_pattern_counter(h, s.pats[0], 1, 5, 0, counter, 0, 1)
            ard.ard_sample_pattern_counter(h, s.pats[1], 1, 5, 0, counter, 1, 2)
            s.run()
            ard.ard_grad_norm(h, table, len(rows), 0.5, norm)
            ard.ard_adamw_step(h, table, len(rows), 1e-2, 0.9, 0.999, 1e-8, bits, 17, 0, counter, None, norm[1:])
        if graphed:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                call()
        seen, out = [], []
        for t in range(steps):
            before = [host(r["p"]) for r in rows]
            moments = [(host(r["m"]), host(r["v"])) for r in rows] if bits == 32 else None
            weights = [ly.W.clone() for ly in s.layers]
            graph.replay() if graphed else call()
            torch.cuda.synchronize()
            seen.append(tuple(tuple(ard.ard_pattern_to_host(p, n)[:2]) for p, n in zip(s.pats, s.dims[1:])))
            out += [r["p"].clone() for r in rows] + [norm.clone(), s.layers[0].dX.clone()] + [ly.W.clone() for ly in s.layers]
            if bits == 32:
                for r, p0, (m0, v0) in zip(rows, before, moments):
                    check_step(r, p0.reshape(-1), m0, v0, t + 1, float(norm[1].double()))
                total = OA.norm([host(r["g"]) for r in rows], 0.5)
                got = host(norm)
                assert abs(got[0] - total[0]) <= 2 * U * total[0] * 8 and abs(got[1] - total[1]) <= 16 * U * total[1]
            now = [ly.W.clone() for ly in s.layers]
            for ly, w in zip(s.layers, weights):       # the stages were computed with the weights before the step
                ly.W.copy_(w)
            p_now = [r["p"].clone() for r in rows]
            for r, p0 in zip(rows, before):
                r["p"].copy_(torch.from_numpy(p0).reshape(r["p"].shape))
            s.check(seen[-1])
            for r, p in zip(rows, p_now):
                r["p"].copy_(p)
            for ly, w in zip(s.layers, now):
                ly.W.copy_(w)
                assert torch.equal(ly.W, ly.p_W.to(BF))
        return out, seen
    finally:
        s.ctx.close()


def check_step(r, p0, m0, v0, t, gf):
    lr, b1, b2, eps, decay = 1e-2, 0.9, 0.999, 1e-8, r["weight_decay"]
    g = host(r["g"]).reshape(-1) * gf
    m, v = OA.moments(m0, v0, g, b1, b2)
    want = OA.step(p0, m, v, lr, b1, b2, eps, decay, t)
    em = 8 * U * (np.abs(b1 * m0) + np.abs((1 - b1) * g))
    lift1, den = 1 / (1 - b1 ** t), np.sqrt(v / (1 - b2 ** t)) + eps
    _close(host(r["p"]).reshape(-1), want, 1.5 * U * np.abs(want) + lr * (8 * U * decay * np.abs(p0) + (em + 24 * U * np.abs(m)) * lift1 / den), 0.0)
    _close(host(r["m"]), m, em, 0.0)
    _close(host(r["v"]), v, 12 * U * v, 0.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_training_steps_eager_and_replayed(bits):
    """Four steps with patterns drawn on the device; the captured step, replayed, leaves the same bits as the calls made one by one."""
    eager, drawn = _training(False, bits)
    replayed, again = _training(True, bits)
    assert drawn == again and len(set(drawn)) > 1
    assert all(torch.equal(a, b) for a, b in zip(eager, replayed))


def test_refusals():
    ctx = Ctx(1 << 20)
    try:
        pat = ctx.pattern(ard.ARD_ROW, 16, 24)
        z = torch.zeros
        with pytest.raises(ValueError):
            GlrLayer(ctx.h, pat, None, 2, 2, 16, 24, z(24, 16), z(72), z(16), z(16))
        with pytest.raises(ValueError):
            GlrLayer(ctx.h, pat, None, 2, 2, 16, 24, z(72, 16), z(72), z(24), z(16))
        ly = GlrLayer(ctx.h, pat, None, 2, 2, 16, 24, z(72, 16), z(72), z(16), z(16))
        x = z(4, 16, dtype=BF, device="cuda")
        with pytest.raises(RuntimeError):
            ly.backward(1.0, z(4, 24, dtype=BF, device="cuda"))
        for bad in (x[:3], x.float(), x.cpu(), z(16, 4, dtype=BF, device="cuda").t()):
            with pytest.raises(ValueError):
                ly.forward(bad, 1.0)
        for bad in (dict(h0=z(2, 24, dtype=BF, device="cuda")), dict(h0=z(2, 16, device="cuda")), dict(lens=z(2, dtype=torch.int64, device="cuda")),
                    dict(lens=z(3, dtype=torch.int32, device="cuda")), dict(lens=z(2, dtype=torch.int32))):
            with pytest.raises(ValueError):
                ly.forward(x, 1.0, **bad)
        ly.forward(x, 1.0)
        with pytest.raises(ValueError):
            ly.backward(1.0, z(4, 24, device="cuda"))
        with pytest.raises(ValueError):
            ly.backward(1.0, z(4, 24, dtype=BF, device="cuda"), z(2, 24, dtype=BF, device="cuda"))
        ly.step(x[:2])
        with pytest.raises(RuntimeError):
            ly.backward(1.0, z(4, 24, dtype=BF, device="cuda"))
    finally:
        ctx.close()
