"""The gated linear recurrence and its adjoint, step by step.  TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  fp64.

  f = s(zf), c_t = f c_{t-1} + (1 - f) zg, y = alpha s(zo) c_t; rows behind a sequence's end: y = 0, c stays.

Beside each value stands how far a computation in fp32 may be from it, carried through the recurrences: `unit` per operation
(2^-24), gates within (16 + 2 |z|) units of their own size (the exponential's argument is off by |z| units, the
exponential, sum and reciprocal by 2 to 4 each).
"""
from __future__ import annotations

import numpy as np

UNIT = 2.0 ** -24


def gates(z):
    """s(z), 1 - s(z), and the relative error that fp32 may make in either."""
    z = np.asarray(z, np.float64)
    with np.errstate(over="ignore"):
        f, i = 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))
    return f, i, (16 + 2 * np.minimum(np.abs(z), 200.0)) * UNIT


def _inside(T, B, lens):
    lens = np.full(B, T) if lens is None else np.clip(lens, 0, T)
    return (np.arange(T)[:, None] < lens[None, :])[..., None]


def fwd(zf, zg, zo, alpha, lens=None, h0=None):
    """y [T][B][n], the states c [T+1][B][n] (c[0] = h0), and the errors allowed of both."""
    T, B, n = zf.shape
    inside = _inside(T, B, lens)
    f, i, ef = gates(zf)
    c = np.zeros((T + 1, B, n))
    ec = np.zeros((T + 1, B, n))
    c[0] = 0.0 if h0 is None else h0
    for t in range(T):
        now = f[t] * c[t] + i[t] * zg[t]
        err = f[t] * ec[t] + (2 * ef[t] + 4 * UNIT) * (f[t] * np.abs(c[t]) + i[t] * np.abs(zg[t]))
        c[t + 1] = np.where(inside[t], now, c[t])
        ec[t + 1] = np.where(inside[t], err, ec[t])
    o, _, eo = (np.float64(1.0), 0.0, 0.0) if zo is None else gates(zo)
    y = np.where(inside, alpha * o * c[1:], 0.0)
    ey = np.where(inside, abs(alpha) * o * (ec[1:] + (eo + 4 * UNIT) * np.abs(c[1:])), 0.0)
    return y, c, ey, ec


def bwd(zf, zg, zo, alpha, c, ec, dy, lens=None, dhT=None):
    """dzf, dzg, dzo (None without zo), dh0 and the errors allowed of each."""
    T, B, n = zf.shape
    inside = _inside(T, B, lens)
    f, i, ef = gates(zf)
    o, no, eo = (np.ones_like(f), None, 0.0) if zo is None else gates(zo)
    a = np.where(inside, alpha * o * np.where(inside, dy, 0.0), 0.0)   # arrives at c_t from y_t
    q = np.zeros((B, n)) if dhT is None else np.array(dhT, np.float64)
    eq = np.zeros((B, n))
    d, ed = np.zeros_like(f), np.zeros_like(f)
    for t in reversed(range(T)):
        ins = inside[t]
        d[t] = a[t] + q
        ed[t] = (eo[t] if zo is not None else 0.0) * np.abs(a[t]) + 4 * UNIT * (np.abs(a[t]) + np.abs(q)) + eq
        eq = np.where(ins, f[t] * (ed[t] + (2 * ef[t] + 4 * UNIT) * np.abs(d[t])), eq)
        q = np.where(ins, f[t] * d[t], q)
    gap = c[:-1] - zg
    dzf, dzg = np.where(inside, d * gap * f * i, 0.0), np.where(inside, d * i, 0.0)
    ezg = np.where(inside, i * (ed + (ef + 4 * UNIT) * np.abs(d)), 0.0)
    ezf = np.where(inside, f * i * (ed * np.abs(gap) + np.abs(d) * (ec[:-1] + 2 * UNIT * (np.abs(c[:-1]) + np.abs(zg))
                                                                   + (2 * ef + 8 * UNIT) * np.abs(gap))), 0.0)
    if zo is None:
        return (dzf, dzg, None, q), (ezf, ezg, None, eq)
    dzo = np.where(inside, a * c[1:] * no, 0.0)
    ezo = np.where(inside, np.abs(a) * no * (ec[1:] + (2 * eo + 8 * UNIT) * np.abs(c[1:])), 0.0)
    return (dzf, dzg, dzo, q), (ezf, ezg, ezo, eq)
