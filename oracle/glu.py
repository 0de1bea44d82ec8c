"""Gated feed-forward layer under a row pattern, in fp64: h = scale act(W0 x + b0) (W1 x + b1) on kept units, 0 on
dropped ones. Samples are rows here: X[B][K], W[2][N][K], keep[N] of 0 / 1."""

import numpy as np
from scipy.special import erf

SQRT2PI = np.sqrt(2.0 * np.pi)


def act(name, g):
    """The activation, its derivative, and the sum of the absolute values of the derivative's terms."""
    if name == "relu":
        d = (g > 0).astype(np.float64)
        return np.maximum(g, 0.0), d, d
    if name == "gelu":
        cdf, pdf = 0.5 * (1.0 + erf(g / np.sqrt(2.0))), np.exp(-0.5 * g * g) / SQRT2PI
        return g * cdf, cdf + g * pdf, cdf + np.abs(g) * pdf
    s = np.where(g >= 0, 1.0 / (1.0 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1.0 + np.exp(-np.abs(g))))
    if name == "sigmoid":
        return s, s * (1.0 - s), s * (1.0 - s)
    return g * s, s * (1.0 + g * (1.0 - s)), s * (1.0 + np.abs(g) * (1.0 - s))


def forward(X, W, bias, keep, scale, name):
    """H[B][N] and Z[2][B][N] (before dropping)."""
    b = np.zeros((2, W.shape[1])) if bias is None else bias
    Z = np.stack([X @ W[i].T + b[i] for i in (0, 1)])
    return scale * act(name, Z[0])[0] * Z[1] * keep, Z


def derivatives(Z, dH, keep, scale, name):
    """dG, dU [B][N] from the given pre-activations."""
    a, d, _ = act(name, Z[0])
    m = scale * dH * keep
    return m * Z[1] * d, m * a


def backward(X, W, Z, dH, keep, scale, name):
    dG, dU = derivatives(Z, dH, keep, scale, name)
    return dG @ W[0] + dU @ W[1], np.stack([dG.T @ X, dU.T @ X]), np.stack([dG.sum(0), dU.sum(0)])
