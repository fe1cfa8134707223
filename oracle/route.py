"""The router in 64 bits, token by token: SoftMax, choice, gates, counts, balance loss and the logits' gradient.  Written from
the formulas; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np


def takes_part(z, mask_value) -> bool:
    return bool(mask_value) and not all(v == -math.inf for v in z)


def softmax(z) -> np.ndarray:
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or (z == math.inf).any():
        return np.full(z.shape, math.nan)
    e = np.exp(z - z.max())
    return e / e.sum()


def choose(z, k: int) -> list[int]:
    """Largest first, ties to the lower id, NaN behind everything."""
    return sorted(range(len(z)), key=lambda e: (math.isnan(z[e]), -z[e] if not math.isnan(z[e]) else 0.0, e))[:k]


def forward(logits: np.ndarray, k: int, mask=None, normalize=False):
    """ids [T, k], gates [T, k], counts [E], loss."""
    T, E = logits.shape
    ids, gates = np.zeros((T, k), np.int64), np.zeros((T, k))
    counts, p_sum, n = np.zeros(E, np.int64), np.zeros(E), 0
    for t in range(T):
        ids[t] = choose(logits[t], k)
        if not takes_part(logits[t], True if mask is None else mask[t]):
            continue
        p = softmax(logits[t])
        g = p[ids[t]]
        gates[t] = g / g.sum() if normalize else g
        for e in ids[t]:
            counts[e] += 1
        p_sum += p
        n += 1
    loss = E * sum(counts[e] / (n * k) * (p_sum[e] / n) for e in range(E)) if n else 0.0
    return ids, gates, counts, loss


def backward(logits: np.ndarray, ids: np.ndarray, counts: np.ndarray, d_gates=None, d_loss=0.0, mask=None, normalize=False):
    T, E = logits.shape
    k = ids.shape[1]
    n = counts.sum() / k
    out = np.zeros((T, E))
    for t in range(T):
        if not takes_part(logits[t], True if mask is None else mask[t]):
            continue
        p = softmax(logits[t])
        dp = np.array([d_loss * E / n * counts[e] / (n * k) if n else 0.0 for e in range(E)])
        if d_gates is not None:
            q = p[ids[t]]
            for j in range(k):
                d = d_gates[t, j]
                if normalize:
                    d = (d - (d_gates[t] * q).sum() / q.sum()) / q.sum()
                dp[ids[t, j]] += d
        out[t] = p * (dp - (p * dp).sum())
    return out
