"""Loss of rows of logits against labels and a teacher's top logits, with its gradient.  TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  fp64.

  L = hard (lse(z) - z[label]) + soft tau^2 sum_i p_i (log p_i - log softmax(z / tau)[id_i]),  p = softmax(t / tau)

Labels, and teacher's entries, outside 0 .. V-1 are absent, entries whose logit is -infinity too.
"""
from __future__ import annotations

import numpy as np


def log_softmax(x):
    x = x - x.max()
    return x - np.log(np.exp(x).sum())


def row(z, label, ids, t, tau, hard, soft):
    """(L, dL/dz, softmax(z), softmax(z / tau), what falls on the label and the teacher's tokens).  None for a row with neither."""
    z = np.asarray(z, np.float64)
    V = len(z)
    if hard == 0 or not 0 <= label < V:
        label = -1
    live = [i for i in range(len(ids)) if 0 <= ids[i] < V and t[i] != -np.inf] if soft != 0 else []
    if label < 0 and not live:
        return None
    with np.errstate(invalid="ignore", divide="ignore"):
        q1, qt = log_softmax(z), log_softmax(z / tau)
        L, g, less = 0.0, np.zeros(V), np.zeros(V)
        if label >= 0:
            L -= hard * q1[label]
            g += hard * np.exp(q1)
            less[label] += hard
        if live:
            lp = log_softmax(np.asarray(t, np.float64)[live] / tau)
            for i, l in zip(live, lp):
                if np.exp(l) > 0:
                    L += soft * tau * tau * np.exp(l) * (l - qt[ids[i]])
                less[ids[i]] += soft * tau * np.exp(l)
            g += soft * tau * np.exp(qt)
    return L, g - less, q1, qt, less
