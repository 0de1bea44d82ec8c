"""Root-mean-square norm of a sum, in fp64. Tokens are rows here: x[B][K], gain[K]."""

import numpy as np


def forward(x, r, gain, eps):
    """s, y and the reciprocal root of each row."""
    s = x if r is None else x + r
    inv = 1.0 / np.sqrt((s * s).mean(1) + eps)
    return s, s * inv[:, None] * gain, inv


def backward(s, gain, eps, dY, dS=None):
    """dX and dgain of y(s), dS added to the former: the derivative of s / sqrt(mean s^2 + eps) written out."""
    root = np.sqrt((s * s).mean(1) + eps)[:, None]
    u = dY * gain
    dX = u / root - s * (u * s).mean(1)[:, None] / root ** 3
    return dX if dS is None else dX + dS, (dY * s / root).sum(0)
