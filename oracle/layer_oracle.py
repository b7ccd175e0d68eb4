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


def expert_balance(g, topk_idx, sample_offsets, scale=1.0):
    """Expert-level load-balance loss of gate values g [T, E] per sample: (loss, counts [B, E], d_gate [B, E], the gradient
    of scale * loss at every g [T, E]). Selections outside [0, E) are not counted; tokens without any take no part."""
    T, E = g.shape
    B = len(sample_offsets) - 1
    counts, d_gate, grad, loss = np.zeros((B, E), dtype=np.int64), np.zeros((B, E)), np.zeros((T, E)), 0.0
    for s in range(B):
        a, b = sample_offsets[s], sample_offsets[s + 1]
        idx = topk_idx[a:b]
        good = (idx >= 0) & (idx < E)
        on = good.any(1)
        counts[s] = np.bincount(idx[good], minlength=E)
        if not on.any():
            continue
        f, n = E * counts[s] / counts[s].sum(), on.sum()
        loss += (f * g[a:b][on].sum(0) / n).sum() / B
        d_gate[s] = scale * f / (B * n)
        grad[a:b][on] = d_gate[s]
    return loss, counts, d_gate, grad


def gate_grad_logits(g, t, slope):
    """Gradient at the logits of <t, g>: slope = 1 (softmax gate) or 1 - s (g = s / sum s, s = sigmoid(z))."""
    return slope * g * (t - (g * t).sum(1, keepdims=True))
