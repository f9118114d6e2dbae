"""Global gradient norm, clipping and the AdamW step in fp64.  Test infrastructure.

    norm = sqrt(sum over all tensors of g^2),  s = min(1, max_norm / (norm + 1e-6))
    m' = b1 m + (1 - b1) s g,  v' = b2 v + (1 - b2) (s g)^2
    p' = p (1 - lr decay) - lr (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps)
"""
import math

import numpy as np


def grad_norm(grads):
    return math.sqrt(math.fsum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))


def clip_factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6)) if max_norm > 0 else 1.0


def adamw(p, m, v, g, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, factor=1.0):
    """One step of one tensor -> (p', m', v')."""
    p, m, v, g = (np.asarray(a, dtype=np.float64) for a in (p, m, v, g))
    x = factor * g
    m = beta1 * m + (1.0 - beta1) * x
    v = beta2 * v + (1.0 - beta2) * x * x
    step_m, step_v = m / (1.0 - beta1 ** step), v / (1.0 - beta2 ** step)
    return p * (1.0 - lr * decay) - lr * step_m / (np.sqrt(step_v) + eps), m, v
