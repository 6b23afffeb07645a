"""Float64 CPU oracle for layers of experts and for clipped gradients.  TEST INFRASTRUCTURE ONLY (see kfac_oracle.py).

Plain numpy, assignment by assignment, from the definitions:

  * sort: assignment i = t K + k goes to row place[i], expert e's rows are offsets[e] .. offsets[e + 1] - 1 with its assignments
    ascending, order[row] = i (-1 behind the last row); an expert outside 0 .. E - 1 is no assignment (place -1);
  * dispatch: xs[place[i]] = x[t];  combine: y[t] = sum_k w[t, k] ys[place[t, k]];  their gradients;
  * the experts' Kronecker factors: F_e = scale * sum over expert e's rows of abar abar^T, abar the row with a trailing 1 if it
    has a bias, scale 1 / (its rows) unless given, 0 without rows; S_e <- decay S_e + (1 - decay) F_e, S_e as it was without rows;
  * norm = sqrt(sum g^2) over all tensors, infinite if it rounds beyond the largest float; out = g min(1, max_norm / norm), g itself if
    the norm is not finite.
"""
from __future__ import annotations

import numpy as np


def expert_sort(expert, experts: int):
    """(offsets, order, place) of a (T, K) array of experts."""
    flat = np.asarray(expert).reshape(-1)
    lists = [[] for _ in range(experts)]
    for i, e in enumerate(flat.tolist()):
        if 0 <= e < experts:
            lists[e].append(i)
    offsets = np.zeros(experts + 1, np.int64)
    order, place = np.full(flat.size, -1, np.int64), np.full(flat.size, -1, np.int64)
    row = 0
    for e, mine in enumerate(lists):
        for i in mine:
            order[row], place[i] = i, row
            row += 1
        offsets[e + 1] = row
    return offsets, order, place.reshape(np.asarray(expert).shape)


def _routed(place):
    T, K = place.shape
    return [(t, k, int(place[t, k])) for t in range(T) for k in range(K) if 0 <= place[t, k] < T * K]


def expert_dispatch(x, place, xs) -> np.ndarray:
    """`xs` with the tokens' rows in it."""
    xs = np.array(xs, dtype=np.float64)
    for t, _, row in _routed(place):
        xs[row] = x[t]
    return xs


def expert_combine(ys, weights, place, dim: int) -> np.ndarray:
    y = np.zeros((place.shape[0], dim))
    for t, k, row in _routed(place):
        y[t] += (1.0 if weights is None else float(weights[t, k])) * np.asarray(ys[row], dtype=np.float64)
    return y


def expert_combine_backward(dy, ys, weights, place, dys):
    """(dys with the gradients in it, dweights)."""
    dys, dweights = np.array(dys, dtype=np.float64), np.zeros(place.shape)
    for t, k, row in _routed(place):
        dys[row] = (1.0 if weights is None else float(weights[t, k])) * np.asarray(dy[t], dtype=np.float64)
        if ys is not None:
            dweights[t, k] = np.dot(np.asarray(dy[t], dtype=np.float64), np.asarray(ys[row], dtype=np.float64))
    return dys, dweights


def expert_factor(x, offsets, has_bias=False, scale: float = 0.0, running=None, decay: float = 0.0) -> np.ndarray:
    x = np.asarray(x, dtype=np.float64)
    E, d = len(offsets) - 1, x.shape[1] + int(has_bias)
    out = np.zeros((E, d, d))
    for e in range(E):
        rows = x[int(offsets[e]):int(offsets[e + 1])]
        if has_bias:
            rows = np.concatenate([rows, np.ones((rows.shape[0], 1))], axis=1)
        n = rows.shape[0]
        if n:
            out[e] = (scale if scale else 1.0 / n) * (rows.T @ rows)
        if running is not None:
            old = np.asarray(running[e], dtype=np.float64)
            out[e] = float(decay) * old + (1.0 - float(decay)) * out[e] if n else old
    return out


def grad_norm(grads) -> float:
    norm = float(np.sqrt(sum(float(np.sum(np.asarray(g, dtype=np.float64) ** 2)) for g in grads)))
    return np.inf if norm >= 2.0 ** 128 - 2.0 ** 103 else norm               # (half a step beyond the largest float)


def grad_clip(grads, max_norm: float, norm=None):
    """(clipped gradients, norm); norm: None, or the one to clip by."""
    norm = grad_norm(grads) if norm is None else float(norm)
    scale = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return [np.asarray(g, dtype=np.float64) * scale for g in grads], norm
