"""Linear attention with a decay for each head, token after token in fp64. One sequence and one head at a time:
q, k [T][Dk], v [T][Dv], S [Dk][Dv], a the decay itself (not its logarithm)."""

import numpy as np


def forward(q, k, v, a, S, scale):
    S = S.copy()
    o = np.zeros((q.shape[0], v.shape[1]))
    for t in range(q.shape[0]):
        S = a * S + np.outer(k[t], v[t])
        o[t] = scale * (q[t] @ S)
    return o, S


def backward(q, k, v, a, S, scale, do, dS):
    """dq, dk, dv and the derivative of the first state."""
    T = q.shape[0]
    dq, dk, dv, G = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), dS.copy()
    S = S.copy()
    for t in range(T):
        S = a * S + np.outer(k[t], v[t])
        dq[t] = scale * (S @ do[t])
    for t in reversed(range(T)):
        G = G + scale * np.outer(q[t], do[t])
        dk[t], dv[t] = G @ v[t], k[t] @ G
        G = a * G
    return dq, dk, dv, G
