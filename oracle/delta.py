"""The gated delta rule and its adjoint, step by step.  TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  fp64.

  S_t = f S_{t-1} + k u^T,  u = b (v - f S_{t-1}^T k),  y = scale S_t^T q;  f = s(zf), b = s(zb), q and k divided by sqrt(sum of squares + eps)
  (eps < 0: as they are); rows behind a sequence's end: y = 0, S stays.

q, k [T][B][h][Dk], v [T][B][h][Dv], zf, zb [T][B][h], states [B][h][Dk][Dv].
"""
from __future__ import annotations

import numpy as np


def logistic(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))


def unit(x, eps):
    """x divided by its length, and one over that."""
    if eps < 0:
        return x, np.ones(x.shape[:-1] + (1,))
    s = (x * x).sum(-1, keepdims=True) + eps
    r = np.where(s > 0, 1.0 / np.sqrt(np.where(s > 0, s, 1.0)), 0.0)
    return x * r, r


def _inside(T, B, lens):
    return np.arange(T)[:, None] < (np.full(B, T) if lens is None else np.clip(lens, 0, T))[None, :]


def fwd(q, k, v, zf, zb, scale, eps, lens=None, h0=None):
    """y [T][B][h][Dv], the states [T+1] and the updates u [T]."""
    T, B, h, Dk = q.shape
    Dv = v.shape[-1]
    inside = _inside(T, B, lens)
    q, k = unit(q, eps)[0], unit(k, eps)[0]
    f, b = logistic(zf)[0], logistic(zb)[0]
    S = np.zeros((T + 1, B, h, Dk, Dv))
    S[0] = 0.0 if h0 is None else h0
    u, y = np.zeros((T, B, h, Dv)), np.zeros((T, B, h, Dv))
    for t in range(T):
        on = inside[t][:, None, None]
        u[t] = np.where(on, b[t][..., None] * (v[t] - f[t][..., None] * np.einsum("bhkv,bhk->bhv", S[t], k[t])), 0.0)
        new = f[t][..., None, None] * S[t] + k[t][..., :, None] * u[t][..., None, :]
        S[t + 1] = np.where(on[..., None], new, S[t])
        y[t] = np.where(on, scale * np.einsum("bhkv,bhk->bhv", S[t + 1], q[t]), 0.0)
    return y, S, u


def bwd(q, k, v, zf, zb, scale, eps, S, u, dy, lens=None, dhT=None):
    """dq, dk, dv, dzf, dzb, dh0, and what dq and dk are before their parts along q and k are taken off."""
    T, B, h, Dk = q.shape
    inside = _inside(T, B, lens)
    (qn, rq), (kn, rk) = unit(q, eps), unit(k, eps)
    (f, nf), (b, nb) = logistic(zf), logistic(zb)
    D = np.zeros(S.shape[1:]) if dhT is None else np.array(dhT, np.float64)
    dq, dk, dv, dzf, dzb = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros_like(zf), np.zeros_like(zb)
    for t in reversed(range(T)):
        on = inside[t][:, None, None]
        g = np.where(on, scale * dy[t], 0.0)
        E = D + qn[t][..., :, None] * g[..., None, :]
        du = np.einsum("bhkv,bhk->bhv", E, kn[t])
        dq[t] = np.where(on, np.einsum("bhkv,bhv->bhk", S[t + 1], g), 0.0)
        db = b[t][..., None] * du
        dk[t] = np.where(on, np.einsum("bhkv,bhv->bhk", E, u[t]) - f[t][..., None] * np.einsum("bhkv,bhv->bhk", S[t], db), 0.0)
        dv[t] = np.where(on, db, 0.0)
        dzb[t] = np.where(on[..., 0], (du * u[t]).sum(-1) * nb[t], 0.0)
        E = E - kn[t][..., :, None] * db[..., None, :]
        dzf[t] = np.where(on[..., 0], f[t] * nf[t] * (E * S[t]).sum((-1, -2)), 0.0)
        D = np.where(on[..., None], f[t][..., None, None] * E, D)
    whole_q, whole_k = rq * dq, rk * dk
    if eps >= 0:
        dq, dk = rq * (dq - qn * (qn * dq).sum(-1, keepdims=True)), rk * (dk - kn * (kn * dk).sum(-1, keepdims=True))
    return dq, dk, dv, dzf, dzb, D, whole_q, whole_k
