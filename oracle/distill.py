"""The distillation loss and its gradient in fp64, a column at a time: logits z[V], teacher entries (class, logit)."""

import math

import numpy as np


def _softmax(x):
    m = np.max(x)
    if m == -np.inf:
        return np.zeros_like(x)
    e = np.exp(x - m)
    return e / e.sum()


def column(z, idx, t, label, temperature, weight):
    """(loss, dloss/dz, the sum of the absolute values of the loss's terms)."""
    V, T = len(z), temperature
    loss, size, dz = 0.0, 0.0, np.zeros(V)
    if np.max(z) == -np.inf:
        return loss, dz, size
    ok = [j for j, v in enumerate(idx) if 0 <= v < V]
    if weight > 0 and ok and max(t[j] for j in ok) > -np.inf:
        p, q = _softmax(np.array([t[j] for j in ok]) / T), _softmax(z / T)
        zT = (z - np.max(z)) / T
        lse = math.log(np.exp(zT).sum())
        dz += weight * T * q
        for pj, j in zip(p, ok):
            if pj > 0:
                logq = zT[idx[j]] - lse
                loss += weight * T * T * pj * (math.log(pj) - logq)
                size += weight * T * T * pj * (abs(math.log(pj)) + abs(logq))
                dz[idx[j]] -= weight * T * pj
    if weight < 1 and 0 <= label < V:
        logq = z[label] - np.max(z) - math.log(np.exp(z - np.max(z)).sum())
        loss -= (1 - weight) * logq
        size += (1 - weight) * abs(logq)
        dz += (1 - weight) * _softmax(z)
        dz[label] -= 1 - weight
    return loss, dz, size


def batch(Z, idx, t, labels, temperature, weight):
    """Z[V][B], idx and t [top][B], labels[B] -> loss[B], dZ[V][B] (of the sum), size[B]."""
    B = Z.shape[1]
    cols = [column(Z[:, b], idx[:, b], t[:, b], -1 if labels is None else labels[b], temperature, weight)
            for b in range(B)]
    return np.array([c[0] for c in cols]), np.stack([c[1] for c in cols], 1), np.array([c[2] for c in cols])
