"""The operators of include/pconv_dense.h written out in float64 numpy, from their formulas (test infrastructure only)."""
from __future__ import annotations

import math

import numpy as np

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, name):
    z = np.asarray(z, np.float64)
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "gelu":
        return z * 0.5 * (1 + _erf(z / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + np.exp(-z))
    return z


def act_slope(z, name):
    z = np.asarray(z, np.float64)
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def linear(x, w, bias=None, residual=None, name="none", first=False):
    """(y, z)"""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    if residual is not None and first:
        z = z + np.asarray(residual, np.float64)
    y = act(z, name)
    if residual is not None and not first:
        y = y + np.asarray(residual, np.float64)
    return y, z


def linear_grad_input(dz, w, z=None, name="none", add=None):
    dx = np.asarray(dz, np.float64) @ np.asarray(w, np.float64)
    if name != "none":
        dx = dx * act_slope(z, name)
    return dx if add is None else dx + np.asarray(add, np.float64)


def linear_grad_weight(dz, x):
    """(dw, db)"""
    dz = np.asarray(dz, np.float64)
    return dz.T @ np.asarray(x, np.float64), dz.sum(0)


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd)"""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    return (y if beta is None else y + np.asarray(beta, np.float64)), mean, rstd


def layer_norm_grad(dy, x, gamma=None, eps=1e-5):
    """(dx, dgamma, dbeta)"""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    _, mean, rstd = layer_norm(x, eps=eps)
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def distill(logits, indices, values, T, weight=None):
    """(loss, grad) row by row, as the header states them."""
    s = np.asarray(logits, np.float64)
    R, V = s.shape
    loss, grad = np.zeros(R), np.zeros((R, V))
    for r in range(R):
        w = 1.0 if weight is None else float(weight[r])
        there = (indices[r] >= 0) & (indices[r] < V)
        i, t = np.asarray(indices[r])[there].astype(np.int64), np.asarray(values[r], np.float64)[there] / T
        if w == 0 or not np.any(~(t == -np.inf)):
            continue
        with np.errstate(invalid="ignore", divide="ignore"):
            log_p = t - np.nanmax(t)
            log_p = log_p - np.log(np.exp(log_p).sum())
            z = s[r] / T
            log_q = z - z.max()
            log_q = log_q - np.log(np.exp(log_q).sum())
            p = np.exp(log_p)
            terms = np.where(p == 0, 0.0, p * (log_p - log_q[i]))
            loss[r] = w * T * T * terms.sum()
            g = np.exp(log_q) * (p.sum() / p.sum())
            np.subtract.at(g, i, p)
            grad[r] = w * T * g
    return loss, grad
