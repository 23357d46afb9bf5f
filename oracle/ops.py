"""Top logits, the distillation loss and group normalisation, in float64.

Top logits of a row z at temperature T: the K largest values in descending
order with their classes (equal values: the lower class first; -inf is never
listed; slots left over hold -inf and -1), and the log-sum of e^{z_c / T} over
the classes not listed.

Distillation loss of a row against a teacher's list (y_k, t_k) and the log-sum
b of its other logits, slot by slot as written in ``distill_row``:

    w_k = e^{t_k / T},  p_k = w_k / (sum w + e^b),  rho = e^b / (sum w + e^b)
    q = softmax(z / T),  s = sum of q over the unlisted classes
    loss = sum_k p_k log(p_k / q_{y_k}) + rho log(rho / s),  0 log 0 = 0

Group normalisation over the rows of a sample and the channels of a group,
with an activation; its gradients are the chain rule of that definition.

Pinned by: torch autograd of the same loss written as a dense KL divergence,
torch's group_norm and its autograd, central differences (tests).
"""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


# ------------------------------------------------------------- top logits ----

def top_logits(Z: np.ndarray, top: int, temperature: float):
    """(values [n, top], ids [n, top], tail_lse [n]) of the rows of Z."""
    n, C = Z.shape
    values, ids = np.full((n, top), -np.inf), np.full((n, top), -1, np.int64)
    tail = np.full(n, -np.inf)
    for r in range(n):
        z = np.asarray(Z[r], np.float64)
        able = [c for c in range(C) if z[c] > -np.inf]                 # NaN is not
        able.sort(key=lambda c: (-z[c], c))
        chosen = able[:top]
        values[r, :len(chosen)], ids[r, :len(chosen)] = z[chosen], chosen
        rest = np.delete(z, chosen) / temperature
        if np.isnan(rest).any():
            tail[r] = np.nan
        elif len(rest) and rest.max() == np.inf:
            tail[r] = np.inf
        elif len(rest) and rest.max() > -np.inf:
            tail[r] = rest.max() + np.log(np.exp(rest - rest.max()).sum())
    return values, ids, tail


# ---------------------------------------------------------- distillation -----

def _lse(x):
    x = np.asarray(x, np.float64)
    m = x.max() if x.size else -np.inf
    return m if m == -np.inf else m + np.log(np.exp(x - m).sum())


def distill_row(z, values, ids, tail, label, temperature, soft_scale, hard_scale):
    """(loss, gradient) of one row; ``tail`` None: none is given; ``label`` < 0: none.

    The logits of z may be -inf (masked classes)."""
    z = np.asarray(z, np.float64)
    C, T = len(z), float(temperature)
    loss, g = 0.0, np.zeros(C)
    first = {}
    for y, t in zip(ids, values):
        if y >= 0 and y not in first:                                  # the lowest slot of a class counts
            first[int(y)] = float(t)
    listed = np.zeros(C, bool)
    listed[list(first)] = True
    if any(t > -np.inf for t in first.values()):
        t = np.array(list(first.values())) / T
        total = _lse(t) if tail is None else _lse(np.append(t, tail))
        log_p = {y: v / T - total for y, v in first.items()}
        log_rho = -np.inf if tail is None else float(tail) - total
        lse = _lse(z / T)
        log_q = z / T - lse
        log_s = _lse(z[~listed] / T) - lse
        p = np.zeros(C)
        for y, lp in log_p.items():
            p[y] = np.exp(lp)
            if p[y] > 0:
                loss += soft_scale * p[y] * (lp - log_q[y])
        rho = np.exp(log_rho)
        if rho > 0:
            loss += soft_scale * rho * (log_rho - log_s)
        q = np.exp(log_q)
        within = np.where(z > -np.inf, np.exp(z / T - _lse(z[~listed] / T)), 0.0) if log_s > -np.inf else np.zeros(C)
        g += soft_scale / T * np.where(listed, q - p, q - rho * within)
    if label >= 0:
        lse1 = _lse(z)
        loss += hard_scale * (lse1 - z[label])
        h = np.exp(z - lse1)
        h[label] -= 1.0
        g += hard_scale * h
    return loss, g


def distill(Z, values, ids, tail, labels, temperature, soft_scale, hard_scale):
    """(loss summed over the rows, J) of ``distill_row``."""
    J, loss = np.zeros(Z.shape), 0.0
    for r in range(len(Z)):
        l, J[r] = distill_row(Z[r], values[r], ids[r], None if tail is None else tail[r],
                              -1 if labels is None else int(labels[r]), temperature, soft_scale, hard_scale)
        loss += l
    return loss, J


# ------------------------------------------------------------- group norm ----

def act(u: np.ndarray, kind: str) -> np.ndarray:
    if kind == "relu":
        return np.maximum(u, 0.0)
    if kind == "silu":
        return u / (1.0 + np.exp(-u))
    if kind == "gelu":
        return 0.5 * u * (1.0 + _erf(u / math.sqrt(2.0)))
    assert kind == "none"
    return u


def act_slope(u: np.ndarray, kind: str) -> np.ndarray:
    if kind == "relu":
        return (u > 0.0).astype(np.float64)
    if kind == "silu":
        g = 1.0 / (1.0 + np.exp(-u))
        return g * (1.0 + u * (1.0 - g))
    if kind == "gelu":
        return 0.5 * (1.0 + _erf(u / math.sqrt(2.0))) + u * np.exp(-0.5 * u * u) / math.sqrt(2.0 * math.pi)
    assert kind == "none"
    return np.ones_like(u)


def _split(x, samples, groups):
    rows, f = x.shape
    return x.reshape(samples, rows // samples, groups, f // groups)


def group_norm_forward(X, gamma, beta, samples: int, groups: int, eps: float, kind: str):
    """(Y, mean, rstd); X is [rows, channels], mean and rstd are [samples, groups]."""
    x = _split(np.asarray(X, np.float64), samples, groups)
    mean = x.mean(axis=(1, 3))
    d = x - mean[:, None, :, None]
    rstd = 1.0 / np.sqrt((d * d).mean(axis=(1, 3)) + eps)
    u = (d * rstd[:, None, :, None]).reshape(X.shape) * gamma + beta
    return act(u, kind), mean, rstd


def group_norm_backward(X, J, gamma, beta, mean, rstd, samples: int, groups: int, kind: str, slope=None):
    """(dX, dgamma, dbeta).  ``slope`` replaces act'(u) where given (a decided ReLU mask)."""
    r = rstd[:, None, :, None]
    xhat = (_split(np.asarray(X, np.float64), samples, groups) - mean[:, None, :, None]) * r
    u = xhat.reshape(X.shape) * gamma + beta
    du = J * (act_slope(u, kind) if slope is None else slope)
    dbeta, dgamma = du.sum(axis=0), (du * xhat.reshape(X.shape)).sum(axis=0)
    dx = _split(du * gamma, samples, groups)
    c1 = dx.mean(axis=(1, 3), keepdims=True)
    c2 = (dx * xhat).mean(axis=(1, 3), keepdims=True)
    return (r * (dx - c1 - xhat * c2)).reshape(X.shape), dgamma, dbeta
