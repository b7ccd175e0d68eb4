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


MX_SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_quantise(x):
    """(codes [..., n / 2], scales [..., n / 32]) of finite x [..., n], and the byte 255 where a block is not finite: every
    value to the nearest of the sizes, a tie to the even code."""
    b = x.reshape(-1, 32)
    good = np.isfinite(b).all(1)
    b = np.where(good[:, None], b, 0.0)
    top = np.abs(b).max(1)
    e = np.where(top > 0, np.floor(np.log2(np.where(top > 0, top, 1.0))), -1000.0)
    e = np.where(top < 2.0 ** e, e - 1, np.where(top >= 2.0 ** (e + 1), e + 1, e))      # log2 rounds near powers of two
    e = np.maximum(e - 2, -127)
    v = np.abs(b) * 2.0 ** -e[:, None]
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])          # the first of equal distances: an even code
    codes = order[np.argmin(np.abs(v[..., None] - MX_SIZES[order]), -1)] + 8 * np.signbit(b)
    codes[~good] = 0
    pairs = codes.reshape(-1, 16, 2)
    q = (pairs[..., 0] + 16 * pairs[..., 1]).astype(np.uint8).reshape(x.shape[:-1] + (-1,))
    return q, np.where(good, e + 127, 255).astype(np.uint8).reshape(x.shape[:-1] + (-1,))


def mx_values(codes, scales):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(-1, 32)
    s = scales.reshape(-1, 1).astype(np.float64)
    v = np.where(c >= 8, -1.0, 1.0) * MX_SIZES[c & 7] * np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return v.reshape(codes.shape[:-1] + (-1,))
