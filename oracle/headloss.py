"""Softmax cross entropy of a head layer, in fp64. Tokens are rows here: X[B][K], W[V][K]; a label outside 0 .. V - 1 is
none. keep[K] of 0 / 1."""

import numpy as np


def forward(X, W, bias, labels, keep):
    """loss[B] and the probabilities q[B][V]."""
    z = (X * keep) @ (W * keep).T + (0.0 if bias is None else bias)
    top = z.max(1, keepdims=True)
    none = top[:, 0] == -np.inf
    e = np.exp(z - np.where(none[:, None], 0.0, top))
    total = e.sum(1, keepdims=True)
    on = (labels >= 0) & (labels < W.shape[0]) & ~none
    loss = np.zeros(len(X))
    rows = np.flatnonzero(on)
    loss[rows] = np.log(total[rows, 0]) + top[rows, 0] - z[rows, labels[rows]]
    return loss, np.divide(e, total, out=np.zeros_like(e), where=total > 0), on


def backward(X, W, bias, labels, keep, dloss):
    """dX, dW, dbias."""
    _, q, on = forward(X, W, bias, labels, keep)
    dz = q.copy()
    rows = np.flatnonzero(on)
    dz[rows, labels[rows]] -= 1.0
    dz = dz * (dloss * on)[:, None]
    return dz @ (W * keep) * keep, dz.T @ (X * on[:, None] * keep), dz.sum(0)
