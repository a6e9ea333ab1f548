"""The optimiser's step, with states in 32 bits or as 8-bit floats.  TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  fp64.

8-bit floats ("e4m3"): 0, and 1.mmm x 2^e from 2^-6 to 448, below that steps of 2^-9.  A block of 128 elements shares a scale, its largest value
/ 448.  A value between two neighbours goes up with the probability of its place between them: floor(x / step + r), r = (word + 1/2) / 2^16.
"""
from __future__ import annotations

import numpy as np

BLOCK, LARGEST, TINY = 128, 448.0, 2.0 ** -110


def moments(m, v, g, beta1, beta2):
    return beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g


def step(p, m, v, lr, beta1, beta2, eps, decay, t):
    """The parameter after the step; m, v as moments() gives them."""
    return p - lr * (decay * p + m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps))


def philox(counter, key):
    """Philox4x32-10 (Salmon et al., SC'11) of arrays of counters [n][4], one key."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    c = [np.array(counter[:, k], u) for k in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        a, b = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        c = [(b >> u(32)) ^ c[1] ^ u(k0), b & low, (a >> u(32)) ^ c[3] ^ u(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, axis=1)


def words(n, seed, t, number):
    """One word per element of a tensor of n elements, the `number`-th (from 0) of the call."""
    quads = (n + 3) // 4
    ctr = np.zeros((quads, 4), np.uint64)
    ctr[:, 0], ctr[:, 1], ctr[:, 2], ctr[:, 3] = t & 0xFFFFFFFF, t >> 32, np.arange(quads), 1 + number
    return philox(ctr, (seed & 0xFFFFFFFF, seed >> 32)).reshape(-1)[:n]


def scales(x):
    """Of the blocks of x [n]."""
    pad = np.concatenate([np.abs(x), np.zeros(-len(x) % BLOCK)]).reshape(-1, BLOCK)
    big = pad.max(axis=1)
    return np.where(big >= TINY, big / LARGEST, 0.0)


def rounded(x, scale, random16, root=False):
    """The 8-bit floats (their values, without the scale) of x [n] with the blocks' scales."""
    s = np.repeat(scale, BLOCK)[:len(x)]
    a = np.where(s > 0, np.abs(x) / np.where(s > 0, s, 1.0), 0.0)
    quantum = np.exp2(np.maximum(np.floor(np.log2(np.maximum(a, 1e-300))), -6.0) - 3)
    q = np.floor(a / quantum + (np.asarray(random16, np.float64) + 0.5) / 65536) * quantum
    if root:
        q = np.where((a > 0) & (q == 0), 2.0 ** -9, q)
    return np.minimum(q, LARGEST) * np.sign(x)


def norm(gradients, max_norm):
    n = np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in gradients))
    return n, (min(1.0, max_norm / (n + 1e-6)) if max_norm > 0 else 1.0)
