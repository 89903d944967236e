"""Root-mean-square norm and its gradients in float64 (test infrastructure only)."""
import numpy as np


def rmsnorm(x, res, w, eps):
    """x [R, d], res [R, d] or None, w [d], all float64 -> (s, rstd [R], y)."""
    s = x if res is None else x + res
    rstd = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
    return s, rstd, s * rstd[:, None] * w


def rmsnorm_backward(dy, s, w, rstd, dres=None):
    """dL/ds (with the skip path's gradient dres added) and dL/dw of y = s * rstd * w, rstd a function of s."""
    g = dy * w
    proj = (g * s).mean(axis=1) * rstd ** 3
    dx = g * rstd[:, None] - s * proj[:, None]
    return (dx if dres is None else dx + dres), (dy * s * rstd[:, None]).sum(axis=0)
