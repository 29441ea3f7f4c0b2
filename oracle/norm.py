"""fp64 numpy definitions of group normalisation with an activation, and of the
norm of many gradients and clipping by it.

Written from the formulas: statistics over the explicit group axis, the
activation's derivative in closed form, the input gradient by the chain rule
through mean and variance term by term.
"""

import numpy as np
from scipy.special import erf


def _act(name, z):
    if name == "none":
        return z, np.ones_like(z)
    if name == "relu":
        return np.where(z > 0, z, 0.0), (z > 0).astype(np.float64)
    if name == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * z))
        return z * s, s + z * s * (1.0 - s)
    if name == "gelu":
        cdf = 0.5 * (1.0 + erf(z / np.sqrt(2.0)))
        return z * cdf, cdf + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    raise ValueError(name)


def _normalised(x, G, weight, bias, eps):
    B, C = x.shape[:2]
    v = x.astype(np.float64).reshape(B, G, -1)
    mean = v.mean(axis=2)
    centred = v - mean[:, :, None]
    rstd = 1.0 / np.sqrt((centred ** 2).mean(axis=2) + eps)
    xh = (centred * rstd[:, :, None]).reshape(x.shape)
    side = (1, C) + (1,) * (x.ndim - 2)
    w = np.ones(C) if weight is None else weight.astype(np.float64)
    b = np.zeros(C) if bias is None else bias.astype(np.float64)
    return mean, rstd, xh, w.reshape(side), b.reshape(side)


def group_norm_forward(x, G, weight=None, bias=None, eps=1e-5, activation="none"):
    """(y, mean, rstd) of x[B, C, ...]."""
    mean, rstd, xh, w, b = _normalised(x, G, weight, bias, eps)
    return _act(activation, xh * w + b)[0], mean, rstd


def group_norm_preactivation(x, G, weight=None, bias=None, eps=1e-5):
    _, _, xh, w, b = _normalised(x, G, weight, bias, eps)
    return xh * w + b


def group_norm_backward(dy, x, G, weight=None, bias=None, eps=1e-5, activation="none"):
    """(dx, dweight, dbias)."""
    B = x.shape[0]
    mean, rstd, xh, w, b = _normalised(x, G, weight, bias, eps)
    dz = dy.astype(np.float64) * _act(activation, xh * w + b)[1]
    axes = (0,) + tuple(range(2, x.ndim))
    dxh = (dz * w).reshape(B, G, -1)
    n = dxh.shape[2]
    centred = x.astype(np.float64).reshape(B, G, -1) - mean[:, :, None]
    r = rstd[:, :, None]
    # d/dvar of (x - mean) (var + eps)^(-1/2), then d/dmean (the variance's own
    # dependence on the mean sums to zero)
    dvar = -0.5 * (dxh * centred).sum(axis=2, keepdims=True) * r ** 3
    dmean = -(dxh * r).sum(axis=2, keepdims=True)
    dx = dxh * r + dvar * 2.0 * centred / n + dmean / n
    return dx.reshape(x.shape), (dz * xh).sum(axis=axes), dz.sum(axis=axes)


def grad_norm(grads, p=2.0):
    with np.errstate(over="ignore"):
        flat = [np.abs(np.asarray(g, dtype=np.float64)).ravel() for g in grads]
    flat = np.concatenate(flat) if flat else np.zeros(0)
    if not flat.size:
        return 0.0
    if p == float("inf"):
        return float(np.max(flat))
    return float(np.sum(flat ** p) ** (1.0 / p))


def grad_clip(grads, max_norm, p=2.0):
    """(norm, clipped gradients)."""
    norm = grad_norm(grads, p)
    k = max_norm / (norm + 1e-6)
    k = 1.0 if k > 1.0 else k
    return norm, [np.asarray(g, dtype=np.float64) * k for g in grads]
