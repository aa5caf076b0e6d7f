"""Group norm with an activation in 64 bits, and its gradients, written from the definition."""

from __future__ import annotations

import numpy as np


def _rows(p, n, s):
    """[sets][channels] as [samples][1][channels]"""
    return np.repeat(p, n // len(p), axis=0)[:, None, :]


def _groups(v, g):
    n, s, c = v.shape
    return v.reshape(n, s, g, c // g)


def activation(u, act):
    with np.errstate(over="ignore"):
        return u if act == "none" else np.where(u > 0, u, 0.0) if act == "relu" else u / (1 + np.exp(-u))


def slope(u, act):
    if act == "none":
        return np.ones_like(u)
    if act == "relu":
        return (u > 0).astype(np.float64)
    with np.errstate(over="ignore"):
        q = 1 / (1 + np.exp(-u))
    return q * (1 + u * (1 - q))


def forward(x, gamma, beta, g, eps, act):
    """y, mean [n][g], rstd [n][g] and the value before the activation."""
    n, s, c = x.shape
    q = _groups(np.asarray(x, np.float64), g)
    mean = q.mean((1, 3))
    rstd = 1 / np.sqrt(((q - mean[:, None, :, None]) ** 2).mean((1, 3)) + eps)
    h = ((q - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(n, s, c)
    u = h * _rows(gamma, n, s) + _rows(beta, n, s)
    return activation(u, act), mean, rstd, u


def backward(dy, x, gamma, beta, mean, rstd, g, act):
    """dx, dgamma, dbeta for given mean and rstd; then h, u and du, for error bounds."""
    n, s, c = x.shape
    m, r = mean[:, None, :, None], rstd[:, None, :, None]
    h = ((_groups(np.asarray(x, np.float64), g) - m) * r).reshape(n, s, c)
    u = h * _rows(gamma, n, s) + _rows(beta, n, s)
    du = dy * slope(u, act)
    sets = len(gamma)
    per = lambda v: v.reshape(sets, n // sets * s, c).sum(1)  # noqa: E731
    dh = _groups(du * _rows(gamma, n, s), g)
    one, two = dh.mean((1, 3), keepdims=True), (dh * _groups(h, g)).mean((1, 3), keepdims=True)
    dx = (r * (dh - one - _groups(h, g) * two)).reshape(n, s, c)
    return dx, per(du * h), per(du), h, u, du
