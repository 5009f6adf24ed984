"""Operators of a residual block of dense layers in float64: layer norm, dropout from splitmix64 by position, dense layers with
bias, activation, dropout and residual, and all their gradients.  Matrices are [rows, N]."""
import numpy as np
from scipy.special import expit, ndtr

_STEP = 0x9E3779B97F4A7C15
_M64 = (1 << 64) - 1


def splitmix64(seed, n, first=0):
    """Outputs first .. first+n-1 of the sequence started from `seed` (uint64 array)."""
    state = (np.arange(n, dtype=np.uint64) + np.uint64((first + 1) & _M64)) * np.uint64(_STEP) + np.uint64(seed & _M64)
    z = (state ^ (state >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def kept(rng, m, n, p):
    """Mask [m, n] of the elements dropout keeps; rng = (seed, offset)."""
    if p == 0:
        return np.ones((m, n), bool)
    half = (n + 1) // 2
    words = splitmix64(int(splitmix64(int(rng[0]), 1)[0]), m * half, int(rng[1])).reshape(m, half)
    bits = np.stack((words & np.uint64(0xFFFFFFFF), words >> np.uint64(32)), 2).reshape(m, 2 * half)[:, :n]
    return bits >= np.uint64(round(p * 2.0 ** 32))


def dropout(x, p, rng):
    return np.where(kept(rng, *x.shape, p), x / (1 - p), 0.0)


def act(z, name):
    if name == "relu":
        return np.where(z > 0, z, 0.0)
    if name == "gelu":
        return z * ndtr(z)
    if name == "gelu_tanh":
        return z * expit(2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3))
    if name == "silu":
        return z * expit(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return ndtr(z) + z * np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    if name == "gelu_tanh":
        s = expit(2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3))
        return s + z * s * (1 - s) * 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = expit(z)
        return s + z * s * (1 - s)
    return np.ones_like(z)


def layernorm(x, gamma=None, beta=None, eps=1e-5):
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / np.sqrt((d * d).mean(1) + eps)
    y = d * rstd[:, None]
    y = y if gamma is None else y * gamma
    return (y if beta is None else y + beta), mean, rstd


def layernorm_backward(dy, x, gamma, mean, rstd, addend=None):
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    return dx if addend is None else dx + addend, (dy * xhat).sum(0), dy.sum(0)


def linear(x, w, bias=None, name="none", p=0.0, rng=None, residual=None):
    z = x @ w.T
    z = z if bias is None else z + bias
    y = dropout(act(z, name), p, rng)
    return (y if residual is None else y + residual), z


def linear_dgrad(dz, w, name="none", z=None, p=0.0, rng=None):
    dx = dropout(dz @ w, p, rng)
    return dx if name == "none" else dx * slope(z, name)


def linear_wgrad(dz, x):
    return dz.T @ x, dz.sum(0)


def mlp_block(x, params, name, p, rngs, eps=1e-5):
    """x + drop(drop(act(LN(x) w1' + b1)) w2' + b2); params = gamma, beta, w1, b1, w2, b2 -> y and what the backward pass needs."""
    gamma, beta, w1, b1, w2, b2 = params
    n, mean, rstd = layernorm(x, gamma, beta, eps)
    h, z1 = linear(n, w1, b1, name, p, rngs[0])
    y, _ = linear(h, w2, b2, "none", p, rngs[1], x)
    return y, (n, mean, rstd, h, z1)


def mlp_block_backward(dy, x, params, saved, name, p, rngs):
    """-> dx and the gradients of params."""
    gamma, _, w1, _, w2, _ = params
    n, mean, rstd, h, z1 = saved
    dz2 = dropout(dy, p, rngs[1])
    dw2, db2 = linear_wgrad(dz2, h)
    dz1 = linear_dgrad(dz2, w2, name, z1, p, rngs[0])
    dw1, db1 = linear_wgrad(dz1, n)
    dx, dgamma, dbeta = layernorm_backward(linear_dgrad(dz1, w1), x, gamma, mean, rstd, dy)
    return dx, (dgamma, dbeta, dw1, db1, dw2, db2)
