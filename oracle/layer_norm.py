"""Layer norm over the rows of a matrix and its adjoint.  TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).  fp64."""
from __future__ import annotations

import numpy as np


def fwd(X, weight, bias, eps):
    """(Y, mean, rstd) of X [rows][n]; weight, bias [n]."""
    X = np.asarray(X, np.float64)
    mean = X.mean(axis=1)
    rstd = 1.0 / np.sqrt(((X - mean[:, None]) ** 2).mean(axis=1) + eps)
    return (X - mean[:, None]) * rstd[:, None] * weight + bias, mean, rstd


def bwd(dY, X, weight, mean, rstd):
    """(dX, dweight, dbias)."""
    dY = np.asarray(dY, np.float64)
    xh = (np.asarray(X, np.float64) - mean[:, None]) * rstd[:, None]
    e = dY * weight
    n = X.shape[1]
    dX = rstd[:, None] * (e - e.sum(axis=1, keepdims=True) / n - xh * (e * xh).sum(axis=1, keepdims=True) / n)
    return dX, (dY * xh).sum(axis=0), dY.sum(axis=0)
