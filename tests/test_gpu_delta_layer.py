"""DeltaLayer (paper_2203_05705_b200/delta.py) against its formulas under autograd in fp64.

Tolerance: forward a value passes five roundings to bf16 (norm, weight, product, rule, and what the rule does with rounded gates), backward as many again, each half a
step, 2^-8 of its size at most, and what is rounded is handed on without growing much; together, in the 2-norm, 16 * 2^-8."""
import numpy as np
import pytest
import torch

from gpu_helpers import Ctx, host
from oracle import pattern as OP
from paper_2203_05705_b200 import ard
from paper_2203_05705_b200.delta import DeltaLayer
from test_oracle_language_model import _torch_delta

pytestmark = pytest.mark.gpu
BF, D = torch.bfloat16, torch.float64
TOL = 16 * 2.0 ** -8


def rel(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def make(ctx, in_pat, T, B, I, heads, Dk, Dv, seed=0):
    rng = np.random.default_rng(seed)
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))  # noqa: E731
    N = heads * (2 * Dk + Dv + 2)
    bias = f(N) * 0.2
    bias[heads * (2 * Dk + Dv):heads * (2 * Dk + Dv + 1)] += 2.0         # gates that remember
    return DeltaLayer(ctx.h, in_pat, T, B, I, heads, Dk, Dv, f(N, I) / I ** 0.5, bias, 1 + 0.2 * f(I), 0.2 * f(I)), rng


def reference(layer, X, keep, lens, h0, dY, dhT):
    """Everything in fp64 on the CPU from the parameters as the products see them."""
    T, B, h, Dk, Dv, I = layer.T, layer.B, layer.heads, layer.Dk, layer.Dv, layer.I
    W, b, nw, nb = (t.detach().cpu().to(D).requires_grad_() for t in (layer.W.float(), layer.p_b, layer.p_nw, layer.p_nb))
    x = X[:, :len(keep)].detach().cpu().to(D).requires_grad_()
    s0 = h0.cpu().to(D).requires_grad_()
    xn = torch.nn.functional.layer_norm(x, (len(keep),), nw[keep], nb[keep], layer.eps)
    z = xn @ W[:, keep].T + b
    cut = [layer.at[k] for k in range(5)] + [layer.N]
    q, k, v, zf, zb = (z[:, cut[i]:cut[i + 1]].reshape(T, B, h, -1) for i in range(5))
    y, S = _torch_delta(q, k, v, zf[..., 0], zb[..., 0], layer.scale, layer.length_eps, lens, s0)
    loss = (y.reshape(T * B, -1) * dY.cpu().to(D)).sum() + (S * dhT.cpu().to(D)).sum()
    loss.backward()
    return y.detach().reshape(T * B, -1).numpy(), S.detach().numpy(), [t.grad.numpy() for t in (x, W, b, nw, nb, s0)]


@pytest.mark.parametrize("shape,dp,ragged", [((70, 3, 64, 2, 32, 40), 1, False), ((40, 2, 96, 3, 24, 16), 2, False), ((12, 4, 64, 2, 16, 32), 1, True),
                                             ((100, 2, 80, 1, 128, 64), 3, True)])
def test_forward_and_gradients(shape, dp, ragged):
    T, B, I, heads, Dk, Dv = shape
    ctx = Ctx(1 << 24)
    in_pat, keep = None, np.arange(I)
    if dp > 1:
        in_pat = ctx.pattern(ard.ARD_ROW, I, I)
        ard.ard_pattern_set(ctx.h, in_pat, dp, 1)
        keep = OP.row_keep(I, dp, 1)
    layer, rng = make(ctx, in_pat, T, B, I, heads, Dk, Dv)
    put = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    X, dY, h0, dhT = put(T * B, I).to(BF), put(T * B, heads * Dv).to(BF), put(B, heads, Dk, Dv), put(B, heads, Dk, Dv) * 0.1
    lens = [T] * B
    d_lens = None
    clean_x, clean_dy = X.clone(), dY.clone()
    if ragged:
        lens = [max(0, T - 3 * b) if b else T for b in range(B)]
        lens[-1] = 0
        d_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        behind = (torch.arange(T, device="cuda")[:, None] >= d_lens).view(-1)
        clean_dy[behind] = 0
        X[behind], dY[behind] = float("nan"), float("inf")
    y = layer.forward(X, h0=h0, lens=d_lens)
    dx = layer.backward(dY, dhT)
    want_y, want_S, want = reference(layer, clean_x, keep, lens, h0, clean_dy, dhT)
    assert rel(host(y), want_y) <= TOL and rel(host(layer.hT), want_S) <= TOL
    got = [dx[:, :len(keep)], layer.dW, layer.db, layer.dnw, layer.dnb, layer.dh0]
    for name, a, b in zip(("dx", "dW", "db", "dnw", "dnb", "dh0"), got, want):
        assert rel(host(a), b) <= TOL, (name, rel(host(a), b))
    dropped = np.setdiff1d(np.arange(I), keep)
    assert (host(layer.dW)[:, dropped] == 0).all() and (host(layer.dnw)[dropped] == 0).all()
    assert ard.ard_last_device_status(ctx.h) == ard.ARD_OK
    layer.close()
    ctx.close()


def test_token_by_token():
    """Steps from the layer's own state are the whole sequence, up to what the product's tiles do with 2 rows in place of 60."""
    ctx = Ctx(1 << 24)
    T, B, I, heads, Dk, Dv = 30, 2, 64, 2, 32, 48
    layer, rng = make(ctx, None, T, B, I, heads, Dk, Dv)
    X = torch.from_numpy(rng.standard_normal((T * B, I)).astype(np.float32)).cuda().to(BF)
    whole = host(layer.forward(X))
    state = host(layer.hT)
    parts = np.concatenate([host(layer.step(X[t * B:(t + 1) * B])) for t in range(T)])
    assert rel(parts, whole) <= 2.0 ** -7 and rel(host(layer.h), state) <= 2.0 ** -7
    layer.close()
    ctx.close()


def test_what_the_layer_refuses():
    ctx = Ctx(1 << 24)
    layer, _ = make(ctx, None, 4, 2, 32, 1, 8, 8)
    x = torch.zeros((8, 32), dtype=BF, device="cuda")
    with pytest.raises(RuntimeError):
        layer.backward(torch.zeros((8, 8), dtype=BF, device="cuda"))
    for bad in (x.float(), x[:7], x.t().contiguous().t(), x.cpu()):
        with pytest.raises(ValueError):
            layer.forward(bad)
    with pytest.raises(ValueError):
        layer.forward(x, lens=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        layer.forward(x, h0=torch.zeros((2, 1, 8, 9), device="cuda"))
    with pytest.raises(ValueError):
        DeltaLayer(ctx.h, None, 4, 2, 32, 1, 8, 8, torch.zeros(25, 32), torch.zeros(26), torch.ones(32), torch.zeros(32))
    layer.close()
    ctx.close()
