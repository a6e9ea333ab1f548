"""The operators of a language model run together: tokens, lookup over kept inputs, a gated linear recurrence, a layer of the delta rule, logits, loss against labels
and a teacher, all gradients into one table, and the optimiser's step."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host
from oracle import distill as OL
from oracle import embedding as OE
from oracle import pattern as OP
from paper_2203_05705_b200 import ard
from paper_2203_05705_b200.delta import DeltaLayer
from paper_2203_05705_b200.glr import GlrLayer
from paper_2203_05705_b200.lm import TokenEnds
from paper_2203_05705_b200.lstm import LstmStack
from test_oracle_language_model import _torch_delta

pytestmark = pytest.mark.gpu
BF, D, HALF = torch.bfloat16, torch.float64, 2.0 ** -8


class Model:
    def __init__(self, T=24, B=4, V=203, N=96, heads=2, seed=0):
        self.ctx = ctx = Ctx(1 << 25)
        self.T, self.B, self.V, self.N = T, B, V, N
        rng = np.random.default_rng(seed)
        f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))  # noqa: E731
        self.in_pat, self.glr_pat = ctx.pattern(ard.ARD_ROW, N, N), ctx.pattern(ard.ARD_ROW, N, N)
        ard.ard_pattern_set(ctx.h, self.in_pat, 2, 2)
        ard.ard_pattern_set(ctx.h, self.glr_pat, 3, 1)
        self.keep = OP.row_keep(N, 2, 2)
        self.ends = TokenEnds(ctx.h, self.in_pat, T * B, V, N, f(V, N) / N ** 0.5, alpha=2.0 * N ** 0.5)
        self.glr = GlrLayer(ctx.h, self.glr_pat, self.in_pat, T, B, N, N, f(3 * N, N) / N ** 0.5, f(3 * N) * 0.2, 1 + 0.2 * f(N), 0.2 * f(N))
        Dk, Dv = 16, N // heads
        n = heads * (2 * Dk + Dv + 2)
        self.delta = DeltaLayer(ctx.h, self.glr_pat, T, B, N, heads, Dk, Dv, f(n, N) / N ** 0.5, f(n) * 0.2, 1 + 0.2 * f(N), 0.2 * f(N))
        put = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        self.h_ids = np.minimum(((V + 1.0) ** rng.random(T * B) - 1).astype(np.int32), V - 1)
        self.h_ids[5::11] = -1
        self.ids = put(self.h_ids)
        self.h_labels = rng.integers(0, V, T * B).astype(np.int32)
        self.h_labels[::7] = -1
        self.labels = put(self.h_labels)
        self.h_tid, self.h_t = rng.integers(0, V, (T * B, 6)).astype(np.int32), (rng.standard_normal((T * B, 6)) * 2).astype(np.float32)
        self.tid, self.t = put(self.h_tid), put(self.h_t)
        self.weight = torch.full((T * B,), 1.0 / (T * B), device="cuda")
        rows = sum((m.adamw_rows(weight_decay=0.1, state_bits=8) for m in (self.ends, self.glr, self.delta)), [])
        self.rows, self.table = rows, ard.adamw_tensors(rows)
        self.norm = torch.zeros(2, device="cuda")

    def gradients(self):
        e = self.ends
        y = self.delta.forward(self.glr.forward(e.embed(self.ids), 3.0))
        e.loss(y, self.labels, self.tid, self.t, tau=2.0, hard=0.5, soft=0.5, row_weight=self.weight)
        e.embed_backward(self.glr.backward(3.0, self.delta.backward(e.backward())))

    def step(self):
        self.gradients()
        ard.ard_grad_norm(self.ctx.h, self.table, len(self.rows), 1.0, self.norm)
        ard.ard_adamw_step(self.ctx.h, self.table, len(self.rows), 1e-3, 0.9, 0.999, 1e-8, 8, 1, 1, None, None, self.norm[1:])

    def close(self):
        self.ends.close()
        self.delta.close()
        self.ctx.close()


def test_each_end_on_what_the_layers_hand_it():
    m = Model()
    m.gradients()
    e, V, N = m.ends, m.V, m.N
    n = len(m.keep)
    alpha = np.float32(e.alpha)
    want = OE.fwd(m.h_ids, host(e.table), alpha, m.keep)
    assert (np.abs(host(e.x)[:, :n] - want) <= (HALF + 2.0 ** -24) * np.abs(want)).all()
    # the logits again, since the gradient took their place
    y = m.delta.Y
    z = host(e.logits(y))[:, :V]
    exact = host(y) @ host(e.table).T
    assert (np.abs(z - exact) <= HALF * np.abs(exact) + N * 2.0 ** -23 * (np.abs(host(y)) @ np.abs(host(e.table)).T)).all()
    e.loss(y, m.labels, m.tid, m.t, tau=2.0, hard=0.5, soft=0.5, row_weight=m.weight)
    dz = host(e.z)[:, :V]
    total, w = 0.0, float(m.weight[0])
    for r in range(len(z)):
        L, g, q1, qt, less = OL.row(z[r], int(m.h_labels[r]), m.h_tid[r], m.h_t[r], 2.0, 0.5, 0.5)
        total += w * L
        size = w * (np.exp(q1) + np.exp(qt) + less)
        assert (np.abs(dz[r] - w * g) <= HALF * np.abs(w * g) + 2.0 ** -16 * size + 1e-37).all()
    assert abs(float(e.total) - total) <= 1e-5 * abs(total)
    dy = host(e.backward())
    exact = dz @ host(e.table)
    assert (np.abs(dy - exact) <= HALF * np.abs(exact) + V * 2.0 ** -23 * (np.abs(dz) @ np.abs(host(e.table)))).all()
    out = dz.T @ host(y)
    size = np.abs(dz).T @ np.abs(host(y))
    assert (np.abs(host(e.dtable) - out) <= 200 * 2.0 ** -23 * size + 1e-37).all()
    before = host(e.dtable)
    e.embed_backward(m.glr.dX)
    g, size, count = OE.bwd(m.h_ids, host(m.glr.dX)[:, :n], V, N, alpha, m.keep)
    assert (np.abs(host(e.dtable) - (before + g)) <= (count[:, None] + 3) * 2.0 ** -24 * (size + np.abs(before))).all()
    assert ard.ard_last_device_status(m.ctx.h) == ard.ARD_OK
    m.close()


def exact_loss(m, table):
    """The model in fp64 from the parameters as the products see them, and a table [V][N] that may ask for its gradient."""
    T, B, N, V = m.T, m.B, m.N, m.V
    wide = lambda t: t.detach().cpu().to(D)  # noqa: E731
    keep, kept = torch.from_numpy(m.keep), torch.from_numpy(OP.row_keep(N, 3, 1))
    ids = torch.from_numpy(m.h_ids).long()
    x = float(np.float32(m.ends.alpha)) * table[ids.clamp_min(0)][:, keep] * (ids >= 0)[:, None]
    ln = lambda x, layer, on: torch.nn.functional.layer_norm(x, (len(on),), wide(layer.p_nw)[on], wide(layer.p_nb)[on], layer.eps)  # noqa: E731
    g = m.glr
    z = [ln(x, g, keep) @ wide(g.W)[k * N:(k + 1) * N][kept][:, keep].T + wide(g.p_b)[k * N:(k + 1) * N][kept] for k in range(3)]
    f, v, o = (a.view(T, B, -1) for a in z)
    c, out = torch.zeros(B, len(kept), dtype=D), []
    for t in range(T):
        s = torch.sigmoid(f[t])
        c = s * c + (1 - s) * v[t]
        out.append(3.0 * torch.sigmoid(o[t]) * c)
    d = m.delta
    z = ln(torch.stack(out).view(T * B, -1), d, kept) @ wide(d.W)[:, kept].T + wide(d.p_b)
    cut = [d.at[k] for k in range(5)] + [d.N]
    q, k, v, zf, zb = (z[:, cut[i]:cut[i + 1]].reshape(T, B, d.heads, -1) for i in range(5))
    y, _ = _torch_delta(q, k, v, zf[..., 0], zb[..., 0], d.scale, d.length_eps, [T] * B, torch.zeros(B, d.heads, d.Dk, d.Dv, dtype=D))
    z = y.reshape(T * B, N) @ table.T
    labels, tid = torch.from_numpy(m.h_labels).long(), torch.from_numpy(m.h_tid).long()
    ce = torch.nn.functional.cross_entropy(z, labels, ignore_index=-1, reduction="sum")
    p = torch.softmax(torch.from_numpy(m.h_t).to(D) / 2.0, 1)
    kl = (p * (p.log() - torch.log_softmax(z / 2.0, 1).gather(1, tid))).sum()
    return (0.5 * ce + 0.5 * 4.0 * kl) / (T * B)


def test_the_tables_gradient_and_the_loss_along_it():
    """Against the whole model in fp64: its gradient, within what some 24 roundings to bf16 one behind the other may make of it, 24 half-steps in the 2-norm; and how the loss moves along that
    gradient, there and here, within a tenth."""
    m = Model()
    m.gradients()
    e = m.ends
    g, base = e.dtable.clone(), float(e.total)
    w = e.table.detach().cpu().to(D).requires_grad_()
    loss = exact_loss(m, w)
    loss.backward()
    assert abs(base - loss.item()) <= 24 * HALF
    want = w.grad.numpy()
    assert np.linalg.norm(host(g) - want) <= 24 * HALF * np.linalg.norm(want)
    h = 0.04 / float((g * g).sum())
    losses, exact = [], []
    for sign in (1, -1):
        e.table.copy_((e.p_table + sign * h * g).to(BF))
        y = m.delta.forward(m.glr.forward(e.embed(m.ids), 3.0))
        losses.append(float(e.loss(y, m.labels, m.tid, m.t, tau=2.0, hard=0.5, soft=0.5, row_weight=m.weight)))
        exact.append(float(exact_loss(m, e.table.detach().cpu().to(D))))
    assert losses[0] > base > losses[1]
    assert abs((losses[0] - losses[1]) / (exact[0] - exact[1]) - 1) <= 0.1, (losses, exact)
    m.close()


def test_steps_eager_and_from_a_graph():
    a, b = Model(), Model()
    a.step()
    a.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.step()
        graph.replay()
        graph.replay()
    side.synchronize()
    torch.cuda.synchronize()
    for x, y in ((a.ends.p_table, b.ends.p_table), (a.glr.p_W, b.glr.p_W), (a.delta.p_W, b.delta.p_W), (a.ends.total, b.ends.total), (a.norm, b.norm)):
        assert torch.equal(x, y)
    assert bool(torch.isfinite(a.ends.p_table).all())
    a.close()
    b.close()


def test_decoding():
    m = Model()
    e = m.ends
    m.glr.pack(), m.delta.pack()
    for t in range(5):
        ids = m.ids[t * m.B:(t + 1) * m.B].contiguous()
        y = m.delta.step(m.glr.step(e.embed(ids), 3.0))
        last = host(e.logits(y))[:, :m.V]
    whole = m.delta.forward(m.glr.forward(e.embed(m.ids), 3.0))
    want = host(e.logits(whole))[4 * m.B:5 * m.B, :m.V]
    # both round the same values to bf16, summed up in other orders: a few half-steps along some six roundings
    assert np.linalg.norm(last - want) <= 8 * HALF * np.linalg.norm(want)
    m.close()


def test_refusals():
    m = Model()
    e = m.ends
    for bad in (m.ids.long(), m.ids.cpu(), torch.zeros(m.T * m.B + 1, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            e.embed(bad)
    y = torch.zeros((m.T * m.B, m.N), dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        e.logits(y.float())
    with pytest.raises(ValueError):
        e.loss(y, m.labels[:-1])
    with pytest.raises(ValueError):
        e.loss(y, m.labels, teacher_ids=m.tid)
    with pytest.raises(ValueError):
        e.loss(y, m.labels, teacher_ids=m.tid, teacher_logits=m.t[:, :5])
    e.embed(m.ids)
    with pytest.raises(ValueError):
        e.embed_backward(y[:, :-1])
    with pytest.raises(ValueError):
        TokenEnds(m.ctx.h, None, 4, 10, 8, torch.zeros(10, 9))
    e.loss(y, m.labels)
    e.logits(y)                      # takes the place of the gradient
    with pytest.raises(RuntimeError):
        e.backward()
    fresh = TokenEnds(m.ctx.h, None, 4, 10, 8, torch.zeros(10, 8))
    with pytest.raises(RuntimeError):
        fresh.backward()
    with pytest.raises(RuntimeError):
        fresh.embed_backward(fresh.x)
    fresh.close()
    m.close()


def test_an_lstm_stack_fed_with_tokens():
    """load_tokens puts the same values where forward(X) puts them."""
    T, B, V, dims = 6, 8, 50, [32, 64, 64]
    ctx = Ctx(1 << 24)
    g = torch.Generator(device="cuda").manual_seed(0)
    weights = [(torch.randn((4 * dims[l + 1], dims[l] + dims[l + 1]), generator=g, device="cuda") * 0.1).to(BF) for l in range(2)]
    stack = LstmStack(ctx.h, T, B, dims, weights)
    table = torch.randn((V, dims[0]), generator=g, device="cuda").to(BF)
    ids = torch.randint(0, V, (T, B), generator=g, device="cuda", dtype=torch.int32)
    ids[2, 3] = -1
    X = (table[ids.clamp_min(0).long()].float() * 0.5).to(BF) * (ids >= 0)[..., None]
    want = stack.forward(X, [1.0, 1.0]).clone()
    stack.layers[0].XH[:, :, :dims[0]] = float("nan")
    stack.layers[0].load_tokens(ids, table, 0.5)
    assert torch.equal(stack.layers[0].XH[:T, :, :dims[0]], X)
    assert torch.equal(stack.forward(None, [1.0, 1.0]), want)
    for bad in (ids.long(), ids[:-1], ids.t()):
        with pytest.raises(ValueError):
            stack.layers[0].load_tokens(bad, table)
    with pytest.raises(ValueError):
        stack.layers[0].load_tokens(ids, table.float())
    torch.cuda.synchronize()
    stack.close()
    ctx.close()
