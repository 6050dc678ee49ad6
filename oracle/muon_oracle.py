"""Orthogonal updates from their definition, in fp64 numpy.  Test infrastructure only."""
import math

import numpy as np

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonalise(g, steps, eps):
    g = np.asarray(g, np.float64)
    x = g / (np.sqrt((g * g).sum()) + eps)
    a, b, c = COEFFICIENTS
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            s = x @ x.T
            x = a * x + (b * s + c * (s @ s)) @ x
        else:
            s = x.T @ x
            x = a * x + x @ (b * s + c * (s @ s))
    return x


def orthogonalise_by_svd(g, steps, eps):
    """The same through the singular values alone, which the steps act on one by one."""
    u, s, v = np.linalg.svd(np.asarray(g, np.float64), full_matrices=False)
    s = s / (np.sqrt((s * s).sum()) + eps)
    a, b, c = COEFFICIENTS
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return (u * s) @ v


def muon_step(grad, momentum, master, lr, mu, weight_decay, eps, nesterov, steps):
    """grad [rows][cols] -> new momentum, new master"""
    grad, momentum, master = (np.asarray(t, np.float64) for t in (grad, momentum, master))
    momentum = mu * momentum + grad
    x = orthogonalise(grad + mu * momentum if nesterov else momentum, steps, eps)
    rows, cols = x.shape
    return momentum, (1.0 - lr * weight_decay) * master - lr * math.sqrt(max(1.0, rows / cols)) * x
