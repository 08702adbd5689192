"""One update with orthogonalised momentum in 64 bits, written as the formulas stand."""
import math

import numpy as np

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonalise(u, eps=1e-7):
    a, b, c = COEFFICIENTS
    x = u / (np.linalg.norm(u) + eps)
    tall = u.shape[0] > u.shape[1]
    x = x.T if tall else x
    for _ in range(5):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.T if tall else x


def step(p, m, g, lr, beta=0.95, decay=0.01, eps=1e-7, nesterov=True, scale=1.0):
    """(p, m, X) after a step."""
    g = g * scale
    m = beta * m + (1 - beta) * g
    u = (1 - beta) * g + beta * m if nesterov else m
    x = orthogonalise(u, eps)
    return p * (1 - lr * decay) - lr * 0.2 * math.sqrt(max(p.shape)) * x, m, x
