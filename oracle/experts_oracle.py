"""Plain fp64 oracle of the expert layer (test infrastructure only): the selections in expert order, the
rows' movement with weights, the experts' products and the gradients, token by token and expert by expert.

Functions take numpy arrays (float64, integer maps) and return numpy arrays. Rows that belong to no
expert are zero in every result."""
from __future__ import annotations

import numpy as np
from scipy.special import erf

NONE, SILU, GELU = 0, 1, 2


def sort(topk_idx, E):
    """(expert_offsets [E+1], row_slot [R], slot_row [T, k]); selections outside [0, E) take no part."""
    T, k = topk_idx.shape
    row_slot = np.full(T * k, -1, dtype=np.int32)
    slot_row = np.full(T * k, -1, dtype=np.int32)
    offsets = np.zeros(E + 1, dtype=np.int32)
    flat = topk_idx.reshape(-1)
    at = 0
    for e in range(E):
        mine = np.nonzero(flat == e)[0]
        row_slot[at:at + len(mine)] = mine
        slot_row[mine] = np.arange(at, at + len(mine))
        at += len(mine)
        offsets[e + 1] = at
    return offsets, row_slot, slot_row.reshape(T, k)


def dispatch(X, row_slot, k):
    Xs = np.zeros((len(row_slot), X.shape[1]))
    there = row_slot >= 0
    Xs[there] = X[row_slot[there] // k]
    return Xs


def back(rows, slot_row, w=None, residual=None):
    """residual + sum over the slots of w * row (w = 1 without weights)."""
    T, k = slot_row.shape
    out = np.zeros((T, rows.shape[1])) if residual is None else residual.copy()
    for s in range(k):
        t = np.nonzero(slot_row[:, s] >= 0)[0]
        out[t] += (1.0 if w is None else w[t, s][:, None]) * rows[slot_row[t, s]]
    return out


def combine_bwd(dY, Ys, w, slot_row):
    dYs, dw = np.zeros_like(Ys), np.zeros(slot_row.shape)
    for s in range(slot_row.shape[1]):
        t = np.nonzero(slot_row[:, s] >= 0)[0]
        r = slot_row[t, s]
        dYs[r] = w[t, s][:, None] * dY[t]
        dw[t, s] = (dY[t] * Ys[r]).sum(1)
    return dYs, dw


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


def act(kind, z):
    if kind == SILU:
        return z * _sigmoid(z)
    if kind == GELU:
        return 0.5 * z * (1.0 + erf(z / np.sqrt(2.0)))
    return z.copy()


def act_slope(kind, z):
    if kind == SILU:
        s = _sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    if kind == GELU:
        return 0.5 * (1.0 + erf(z / np.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    return np.ones_like(z)


def linear(X, W, offsets, bias=None, kind=NONE, gated=False, residual=None):
    """(out, z) of the rows in expert order."""
    E, n_z, _ = W.shape
    n_out = n_z // 2 if gated else n_z
    z, out = np.zeros((len(X), n_z)), np.zeros((len(X), n_out))
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        z[a:b] = X[a:b] @ W[e].T + (0.0 if bias is None else bias[e])
        y = act(kind, z[a:b, :n_out]) * (z[a:b, n_out:] if gated else 1.0)
        out[a:b] = y + (0.0 if residual is None else residual[a:b])
    return out, z


def act_bwd(dOut, z, offsets, kind, gated):
    """(dZ, db)."""
    n_out = dOut.shape[1]
    n = offsets[-1]
    dZ = np.zeros((len(dOut), 2 * n_out if gated else n_out))
    g, d = z[:n, :n_out], dOut[:n]
    dZ[:n, :n_out] = d * act_slope(kind, g) * (z[:n, n_out:] if gated else 1.0)
    if gated:
        dZ[:n, n_out:] = d * act(kind, g)
    return dZ, np.stack([dZ[offsets[e]:offsets[e + 1]].sum(0) for e in range(len(offsets) - 1)])


def linear_bwd(dZ, X, W, offsets):
    """(dX, dW)."""
    dX, dW = np.zeros((len(dZ), W.shape[2])), np.zeros(W.shape)
    for e in range(len(W)):
        a, b = offsets[e], offsets[e + 1]
        dX[a:b] = dZ[a:b] @ W[e]
        dW[e] = dZ[a:b].T @ X[a:b]
    return dX, dW
