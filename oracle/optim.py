"""The global gradient norm, clipping and AdamW over many tensors in 64 bits."""
from __future__ import annotations

import math

import numpy as np


def grad_norm(grads, inf=False):
    if inf:
        return max((float(np.abs(g).max()) for g in grads if g.size), default=0.0)
    return math.sqrt(math.fsum(float((g.astype(np.float64) ** 2).sum()) for g in grads))


def clip_factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6))


def adamw(theta, g, m, v, step, lr, beta1, beta2, eps, weight_decay):
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    update = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return theta - lr * (update + weight_decay * theta), m, v
