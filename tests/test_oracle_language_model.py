"""Pins for oracle/embedding.py, oracle/distill.py and oracle/delta.py: autograd in fp64, and definitions written another way."""
import numpy as np
import torch

from oracle import delta as OD
from oracle import distill as OL
from oracle import embedding as OE


def _t(x, grad=True):
    return torch.tensor(np.asarray(x), dtype=torch.float64, requires_grad=grad)


def test_embedding():
    rng = np.random.default_rng(0)
    ids = np.array([3, 0, 3, -1, 5, 3, 6, 0], np.int32)
    table, dy, keep = rng.normal(size=(6, 7)), rng.normal(size=(8, 3)), np.array([1, 4, 5])
    w = _t(table)
    live = [i for i, v in enumerate(ids) if 0 <= v < 6]
    y = 1.5 * torch.nn.functional.embedding(torch.tensor(ids[live]).long(), w)[:, keep]
    want = np.zeros((8, 3))
    want[live] = y.detach().numpy()
    assert np.abs(OE.fwd(ids, table, 1.5, keep) - want).max() <= 1e-12
    y.backward(_t(dy[live], False))
    g, size, count = OE.bwd(ids, dy, 6, 7, 1.5, keep)
    assert np.abs(g - w.grad.numpy()).max() <= 1e-12
    assert count.tolist() == [2, 0, 0, 3, 0, 1] and (size >= np.abs(g) - 1e-12).all()


def test_loss():
    rng = np.random.default_rng(1)
    for tau in (1.0, 0.7, 3.0):
        z, t = rng.normal(size=11) * 2, rng.normal(size=4)
        ids = np.array([2, 9, 2, 5])                   # one token twice
        x = _t(z)
        ce = torch.nn.functional.cross_entropy(x[None], torch.tensor([5]))
        p = torch.softmax(_t(t, False) / tau, 0)
        lq = torch.log_softmax(x / tau, 0)[torch.tensor(ids)]
        L = 0.4 * ce + 0.6 * tau ** 2 * (p * (p.log() - lq)).sum()
        L.backward()
        got, g, _, _, less = OL.row(z, 5, ids, t, tau, 0.4, 0.6)
        assert abs(got - L.item()) <= 1e-12 and np.abs(g - x.grad.numpy()).max() <= 1e-12
        assert np.count_nonzero(less) == 3
    assert OL.row(z, -1, ids, t, 1.0, 1.0, 0.0) is None and OL.row(z, 11, [], [], 1.0, 1.0, 1.0) is None
    assert OL.row(z, -1, [-1, 20], [0.0, 0.0], 1.0, 1.0, 1.0) is None and OL.row(z, -1, [3], [-np.inf], 1.0, 1.0, 1.0) is None


def _torch_delta(q, k, v, zf, zb, scale, eps, lens, S):
    if eps >= 0:
        q, k = (x / torch.sqrt((x * x).sum(-1, keepdim=True) + eps) for x in (q, k))
    ys = []
    for t in range(q.shape[0]):
        f, b = torch.sigmoid(zf[t])[..., None, None], torch.sigmoid(zb[t])[..., None, None]
        kk, vv = k[t][..., :, None], v[t][..., None, :]
        new = f * (S - b * kk @ (kk.transpose(-1, -2) @ S)) + b * kk @ vv          # the rule as a product with I - b k k^T
        live = torch.tensor(t < np.asarray(lens))[:, None, None, None]
        S = torch.where(live, new, S)
        ys.append(torch.where(live[..., 0], scale * (q[t][..., None, :] @ S)[..., 0, :], torch.zeros_like(v[t])))
    return torch.stack(ys), S


def test_delta_rule():
    rng = np.random.default_rng(2)
    T, B, h, Dk, Dv = 9, 3, 2, 5, 4
    lens = [9, 4, 0]
    for eps in (1e-3, -1.0):
        x = [rng.normal(size=s) * (0.5 if eps < 0 else 1.0) for s in ((T, B, h, Dk), (T, B, h, Dk), (T, B, h, Dv), (T, B, h), (T, B, h), (B, h, Dk, Dv))]
        dy, dhT = rng.normal(size=(T, B, h, Dv)), rng.normal(size=(B, h, Dk, Dv))
        xs = [_t(a) for a in x]
        y, S = _torch_delta(*xs[:5], 0.3, eps, lens, xs[5])
        (y * _t(dy, False)).sum().add((S * _t(dhT, False)).sum()).backward()
        got_y, states, u = OD.fwd(*x[:5], 0.3, eps, lens, x[5])
        assert np.abs(got_y - y.detach().numpy()).max() <= 1e-12 and np.abs(states[-1] - S.detach().numpy()).max() <= 1e-12
        grads = OD.bwd(*x[:5], 0.3, eps, states, u, dy, lens, dhT)
        for a, b in zip(grads, xs):
            assert np.abs(a - b.grad.numpy()).max() <= 1e-11


def test_delta_rule_of_zero_lengths():
    x, r = OD.unit(np.zeros((2, 3)), 0.0)
    assert (x == 0).all() and (r == 0).all()
