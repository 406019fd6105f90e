"""Oracle of the orthogonalised update: momentum, Frobenius normalisation and the quintic Newton-Schulz iteration of one
matrix, plain numpy in 64 bits, step by step as defined."""
import numpy as np

A, B, C = 3.4445, -4.7750, 2.0315


def iterate(u, steps, eps=1e-7):
    u = np.asarray(u, np.float64)
    tall = u.shape[0] > u.shape[1]
    x = u.T if tall else u
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        g = x @ x.T
        x = A * x + (B * g + C * (g @ g)) @ x
    return x.T if tall else x


def orthogonalize(grad, momentum, mu, nesterov, steps, eps=1e-7):
    """(update, new momentum) of one matrix; momentum None: the gradient itself is orthogonalised."""
    g = np.asarray(grad, np.float64)
    if momentum is None:
        return iterate(g, steps, eps), None
    m = mu * np.asarray(momentum, np.float64) + g
    return iterate(g + mu * m if nesterov else m, steps, eps), m
