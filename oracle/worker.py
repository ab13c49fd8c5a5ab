"""Plain definitions, in 64 bits, of what a worker computes before it has a gradient: layer norm, linear layer, distillation
loss, each with its gradient.  Test infrastructure only; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np


def layer_norm(x, weight, bias, eps):
    """y, mean, 1 / sqrt(variance + eps) of every row."""
    mean = x.mean(axis=1)
    var = ((x - mean[:, None]) ** 2).mean(axis=1)
    with np.errstate(divide="ignore", invalid="ignore"):
        rstd = 1.0 / np.sqrt(var + eps)
        y = (x - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd):
    """dx, dweight, dbias."""
    h = (x - mean[:, None]) * rstd[:, None]
    c = dy if weight is None else dy * weight
    dx = rstd[:, None] * (c - c.mean(axis=1, keepdims=True) - h * (c * h).mean(axis=1, keepdims=True))
    return dx, (dy * h).sum(axis=0), dy.sum(axis=0)


_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, kind):
    if kind == "relu":
        return np.where(z > 0, z, 0.0)
    if kind == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    return z


def act_slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return np.ones_like(z)


def linear(x, weight, bias=None, kind="none", residual=None):
    """y and what the activation is applied to."""
    z = x @ weight.T
    if bias is not None:
        z = z + bias
    y = act(z, kind)
    return (y if residual is None else y + residual), z


def linear_dgrad(dy, weight, kind="none", z=None, residual=None):
    dx = dy @ weight
    if kind != "none":
        dx = dx * act_slope(z, kind)
    return dx if residual is None else dx + residual


def linear_wgrad(dy, x):
    return dy.T @ x, dy.sum(axis=0)


def distill(logits, t_idx, t_val, temperature, dloss=None, scale=1.0):
    """Loss of every row and its gradient, row by row and entry by entry as the header defines them."""
    n, v = logits.shape
    loss = np.zeros(n)
    grad = np.zeros((n, v))
    for i in range(n):
        entries = [(int(j), float(t)) for j, t in zip(t_idx[i], t_val[i]) if j >= 0]
        if any(j >= v for j, _ in entries):
            loss[i] = math.nan
            continue
        if all(t == -math.inf for _, t in entries):
            continue
        t = np.array([t for _, t in entries])
        with np.errstate(invalid="ignore", divide="ignore"):       # a NaN or +Inf among them: every q is NaN
            q = np.exp((t - t.max()) / temperature)
            log_q = (t - t.max()) / temperature - np.log(q.sum())
            q = q / q.sum()
        with np.errstate(invalid="ignore", divide="ignore"):
            u = (logits[i] - logits[i].max()) / temperature
            log_p = u - np.log(np.exp(u).sum())
        for k, (j, _) in enumerate(entries):
            if q[k] != 0:
                loss[i] += temperature * temperature * q[k] * (log_q[k] - log_p[j])
        w = scale * (1.0 if dloss is None else float(dloss[i]))
        if w != 0.0:
            g = np.exp(log_p)
            for k, (j, _) in enumerate(entries):
                g[j] -= q[k]
            grad[i] = w * temperature * g
    return loss, grad
