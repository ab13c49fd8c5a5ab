"""Plain definitions, in 64 bits, of what a worker computes before it has a gradient: layer norm, linear layer, distillation
loss, root-mean-square norm, dropout, log probabilities of tokens, each with its gradient, and of matrices in 8 bits.  Test infrastructure only; shares no code with the library."""
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


def rms_norm(s, weight, eps):
    """y and 1 / sqrt(mean square + eps) of every row of s, the sum of input and residual."""
    with np.errstate(divide="ignore", invalid="ignore"):
        rstd = 1.0 / np.sqrt((s * s).mean(axis=1) + eps)
        y = s * rstd[:, None]
    return (y if weight is None else y * weight), rstd


def rms_norm_backward(dy, s, weight, rstd, residual=None):
    """The gradient of s, and dweight."""
    h = s * rstd[:, None]
    c = dy if weight is None else dy * weight
    ds = rstd[:, None] * (c - h * (c * h).mean(axis=1, keepdims=True))
    return (ds if residual is None else ds + residual), (dy * h).sum(axis=0)


E4M3 = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])   # codes 0 to 126; 127 is the NaN


def e4m3(v):
    """The nearest e4m3 value of magnitudes up to 448, ties to the even code."""
    a = np.abs(v)
    hi = np.minimum(np.searchsorted(E4M3, a), len(E4M3) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isnan(v), np.nan, np.copysign(E4M3[code], v))


def quantize(x):
    """e4m3 entries and the scale of every row; rows with a NaN or an infinity are NaN."""
    most = np.abs(x).max(axis=1)
    scale = np.where(np.isfinite(x).all(axis=1), np.maximum(most / 448.0, 2.0 ** -100), np.nan)
    with np.errstate(invalid="ignore", divide="ignore"):      # not over the scale, whose rounding would move what lies half way between two values
        v = np.where(scale[:, None] > 2.0 ** -100, x * 448.0 / most[:, None], x * 2.0 ** 100)
    return e4m3(np.where(np.isnan(scale[:, None]), np.nan, v)), scale


def dropout_keep(n, d, least, seed, step, stream, row0=0):
    """Which entries of n rows and d columns are kept: half j % 8 of the Philox block of the row and j / 8 is at least `least`."""
    from oracle.philox import philox4x32_10
    keep = np.zeros((n, d), dtype=bool)
    for i in range(n):
        for b in range(-(-d // 8)):
            words = philox4x32_10((step, stream, row0 + i, 1 + b), (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
            for k in range(min(8, d - 8 * b)):
                keep[i, 8 * b + k] = (words[k // 2] >> (16 * (k % 2)) & 0xFFFF) >= least
    return keep


def dropout(x, p, seed, step, stream=0, row0=0, residual=None):
    least = int(np.floor(p * 65536 + 0.5))
    y = np.where(dropout_keep(*x.shape, least, seed, step, stream, row0), x / (1.0 - least / 65536.0), 0.0)
    return y if residual is None else y + residual


def token_logprobs(logits, tokens, top, temperature):
    """logprob, entropy, top_idx, top_logprob, (greatest, log of the sum, entropy), row by row."""
    n, v = logits.shape
    logprob, h = np.zeros(tokens.shape), np.full(n, math.nan)
    top_idx, top_logprob, stats = np.full((n, top), -1), np.full((n, top), math.nan), np.full((n, 3), math.nan)
    for i in range(n):
        s = logits[i]
        good = not np.isnan(s).any() and s.max() != math.inf and s.max() != -math.inf
        log_p = np.full(v, math.nan)
        if good:
            u = (s - s.max()) / temperature
            log_s = math.log(np.exp(u).sum())
            log_p = u - log_s
            p = np.exp(log_p)
            h[i] = -(p[p > 0] * log_p[p > 0]).sum()
            stats[i] = s.max(), log_s, h[i]
            order = np.argsort(-s, kind="stable")[:top]
            order = order[s[order] > -math.inf]
            top_logprob[i] = -math.inf
            top_idx[i, :len(order)] = order
            top_logprob[i, :len(order)] = log_p[order]
        for k, t in enumerate(tokens[i]):
            logprob[i, k] = 0.0 if t < 0 else math.nan if t >= v else log_p[t]
    return logprob, h, top_idx, top_logprob, stats


def token_logprobs_backward(logits, tokens, dlogprob, top_idx, dtop, dentropy, temperature):
    """The gradient in the logits, row by row and token by token."""
    n, v = logits.shape
    grad = np.zeros((n, v))
    for i in range(n):
        g = [(t, w) for ts, ws in ((tokens, dlogprob), (top_idx, dtop)) if ts is not None for t, w in zip(ts[i], ws[i]) if 0 <= t < v]
        h = 0.0 if dentropy is None else float(dentropy[i])
        if h == 0.0 and all(w == 0 for _, w in g):
            continue
        s = logits[i]
        if np.isnan(s).any() or abs(s.max()) == math.inf:
            grad[i] = math.nan
            continue
        u = (s - s.max()) / temperature
        log_p = u - math.log(np.exp(u).sum())
        p = np.exp(log_p)
        live = p > 0
        d = -p * sum(w for _, w in g)
        d[live] -= h * p[live] * (log_p[live] - (p[live] * log_p[live]).sum())
        for t, w in g:
            d[t] += w
        grad[i] = d / temperature
    return grad
