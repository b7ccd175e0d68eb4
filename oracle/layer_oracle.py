"""Plain fp64 oracle of what surrounds a layer's router and experts (test infrastructure only): the layer norm and its
gradients. Functions take and return numpy arrays (float64)."""
from __future__ import annotations

import numpy as np


def norm(S, w, b, eps):
    """(Y, mean, rstd) of rows S [T, d]."""
    mean = S.mean(1)
    rstd = 1.0 / np.sqrt(((S - mean[:, None]) ** 2).mean(1) + eps)
    Y = (S - mean[:, None]) * rstd[:, None] * w
    return (Y if b is None else Y + b), mean, rstd


def norm_bwd(dY, S, mean, rstd, w, residual=None):
    """(dX, dw, db) with the statistics given."""
    h = (S - mean[:, None]) * rstd[:, None]
    a = dY * w
    dX = rstd[:, None] * (a - a.mean(1)[:, None] - h * (a * h).mean(1)[:, None])
    return (dX if residual is None else dX + residual), (dY * h).sum(0), dY.sum(0)
