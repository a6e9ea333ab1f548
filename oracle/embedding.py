"""Rows of a table by token and the table's gradient.  TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  fp64.

A token outside 0 .. V-1 is padding: its row is zero and adds nothing.  keep: the kept columns, ascending.
"""
from __future__ import annotations

import numpy as np


def fwd(ids, table, alpha, keep):
    table = np.asarray(table, np.float64)[:, keep]
    y = np.zeros((len(ids), len(keep)))
    live = (ids >= 0) & (ids < len(table))
    y[live] = alpha * table[ids[live]]
    return y


def bwd(ids, dy, V, N, alpha, keep):
    """The gradient [V][N], the sum of its terms' sizes, and how many there are for each token."""
    g, size = np.zeros((V, N)), np.zeros((V, N))
    live = np.flatnonzero((ids >= 0) & (ids < V))
    part, parts = np.zeros((V, len(keep))), np.zeros((V, len(keep)))
    np.add.at(part, ids[live], np.asarray(dy, np.float64)[live])
    np.add.at(parts, ids[live], np.abs(np.asarray(dy, np.float64)[live]))
    g[:, keep], size[:, keep] = alpha * part, abs(alpha) * parts
    return g, size, np.bincount(ids[live], minlength=V)
