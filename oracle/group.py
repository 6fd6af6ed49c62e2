"""fp64 statement of the group norm with an activation (channels last) and of clipping by the global norm.

Group norm: over the v voxels and the c / groups channels of a group of a sample, biased variance; then
t = (x - mean) rstd w + b and z = act(t).  Arrays x, z, dz [n, v, c]; w, b [c]."""
import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(t, name, slope=0.0):
    """(act(t), its derivative); the derivative of the leaky ReLU at 0 is `slope`."""
    t = np.asarray(t, dtype=np.float64)
    if name == "none":
        return t, np.ones_like(t)
    if name == "leaky_relu":
        return np.where(t > 0, t, slope * t), np.where(t > 0, 1.0, slope)
    if name == "silu":
        s = 0.5 * (1.0 + np.tanh(0.5 * t))
        return t * s, s + t * s * 0.5 * (1.0 - np.tanh(0.5 * t))
    if name == "gelu":
        below = 0.5 * _erfc(-t / math.sqrt(2.0))
        return t * below, below + t * np.exp(-0.5 * t * t) / math.sqrt(2.0 * math.pi)
    raise ValueError(name)


def _split(x, groups):
    n, v, c = x.shape
    return x.reshape(n, v, groups, c // groups)


def statistics(x, groups, eps):
    """mean, rstd [n, groups]"""
    g = _split(np.asarray(x, dtype=np.float64), groups)
    mean = g.mean(axis=(1, 3))
    var = ((g - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def normalise(x, mean, rstd):
    """xhat [n, v, c] with given statistics [n, groups]"""
    x = np.asarray(x, dtype=np.float64)
    g = _split(x, mean.shape[1])
    return ((g - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)


def group_norm_act_fwd(x, groups, w, b, name, slope=0.0, eps=1e-5):
    mean, rstd = statistics(x, groups, eps)
    return act(normalise(x, mean, rstd) * w + b, name, slope)[0], mean, rstd


def group_norm_act_bwd(dz, x, mean, rstd, w, b, name, slope=0.0):
    """dx, dw, db; mean and rstd are functions of x (their gradient is part of dx)."""
    groups = mean.shape[1]
    xhat = normalise(x, mean, rstd)
    dt = np.asarray(dz, dtype=np.float64) * act(xhat * w + b, name, slope)[1]
    wd, xg = _split(dt * w, groups), _split(xhat, groups)
    level, along = wd.mean(axis=(1, 3), keepdims=True), (wd * xg).mean(axis=(1, 3), keepdims=True)
    dx = (wd - level - xg * along) * rstd[:, None, :, None]
    return dx.reshape(x.shape), (dt * xhat).sum(axis=(0, 1)), dt.sum(axis=(0, 1))


def clip(grads, max_norm):
    """(norm, factor, clipped gradients)"""
    norm = math.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))
    factor = 1.0 if norm <= max_norm else max_norm / norm
    return norm, factor, [np.asarray(g, dtype=np.float64) * factor for g in grads]
