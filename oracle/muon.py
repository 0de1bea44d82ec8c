"""The orthogonalised momentum update of a dense block, in fp64. Rows are outputs, columns inputs."""

import numpy as np

COEFFS = (3.4445, -4.7750, 2.0315)


def polynomial(U, eps, iterations, coeffs=COEFFS):
    """U / (|U| + eps), and each iterate after it."""
    a, b, c = coeffs
    xs = [U / (np.sqrt((U * U).sum()) + eps)]
    for _ in range(iterations):
        X = xs[-1]
        A = X @ X.T
        xs.append(a * X + b * (A @ X) + c * (A @ (A @ X)))
    return xs


def update(W, V, G, lr, momentum, decay, nesterov, eps, iterations, coeffs=COEFFS):
    """New W and V."""
    V = momentum * V + G
    X = polynomial(G + momentum * V if nesterov else V, eps, iterations, coeffs)[-1]
    return (1.0 - lr * decay) * W - lr * np.sqrt(max(1.0, W.shape[0] / W.shape[1])) * X, V
