"""CPU oracle of the dense operators -- TEST INFRASTRUCTURE ONLY.

The linear layer with bias, activation and residual, the cross entropy of a
linear layer's logits and the clipping of gradients, each with its gradient, in
fp64 numpy from the definitions.  Shares no code with the HIP kernels.
"""
from __future__ import annotations

import math

import numpy as np

NONE, RELU, GELU, SILU = 0, 1, 2, 3
_erf = np.vectorize(math.erf, otypes=[np.float64])
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(code, z):
    z = np.asarray(z, np.float64)
    if code == RELU:
        return np.where(z > 0, z, 0.0)
    if code == GELU:
        return 0.5 * z * _erfc(-z / math.sqrt(2.0))
    if code == SILU:
        with np.errstate(over="ignore"):
            return z / (1.0 + np.exp(-z))
    return z


def slope(code, z):
    z = np.asarray(z, np.float64)
    if code == RELU:
        return (z > 0).astype(np.float64)
    if code == GELU:
        return 0.5 * _erfc(-z / math.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if code == SILU:
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def linear(x, W, bias=None, code=NONE, residual=None):
    """(out, z)"""
    z = np.asarray(x, np.float64) @ np.asarray(W, np.float64)
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    out = act(code, z)
    return (out if residual is None else out + np.asarray(residual, np.float64)), z


def linear_backward(dout, x, W, pre=None, code=NONE):
    """(dx, dW, db, dz)"""
    dz = np.asarray(dout, np.float64)
    if code != NONE:
        dz = dz * slope(code, pre)
    return dz @ np.asarray(W, np.float64).T, np.asarray(x, np.float64).T @ dz, dz.sum(0), dz


def cross_entropy(x, W, labels, bias=None, weight=None):
    """dict of loss, lse, dx, dW, db and, for the live rows, the list of rows, z, q and dz.
    A row whose label is outside of [0, V) is left out of everything."""
    x, W = np.asarray(x, np.float64), np.asarray(W, np.float64)
    labels = np.asarray(labels, np.int64)
    n, V = x.shape[0], W.shape[0]
    live = np.flatnonzero((labels >= 0) & (labels < V))
    z = x[live] @ W.T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        m = z.max(1, initial=-np.inf)
        m0 = np.where(np.isfinite(m), m, 0.0)
        e = np.exp(z - m0[:, None])
        lse_l = m0 + np.log(e.sum(1))
        lse_l = np.where(np.isposinf(m), np.nan, lse_l)
        q = np.where(np.isneginf(lse_l)[:, None], 0.0, np.exp(z - lse_l[:, None]))
        at = np.take_along_axis(z, labels[live][:, None], 1)[:, 0]
        loss_l = np.where(np.isneginf(at) & ~np.isnan(lse_l), np.inf, lse_l - at)
    w = np.ones(n) if weight is None else np.asarray(weight, np.float64)
    dz = q.copy()
    dz[np.arange(len(live)), labels[live]] -= 1.0
    dz *= w[live][:, None]
    loss, lse, dx = np.zeros(n), np.zeros(n), np.zeros_like(x)
    loss[live], lse[live], dx[live] = loss_l, lse_l, dz @ W
    return dict(loss=loss, lse=lse, dx=dx, dW=dz.T @ x[live], db=dz.sum(0), live=live, z=z, q=q,
                dz=dz)


def clip(grads, max_norm):
    """(norm, clipped gradients)"""
    grads = [np.asarray(g, np.float64) for g in grads]
    norm = math.sqrt(sum(float((g * g).sum()) for g in grads))
    factor = 1.0 if norm <= max_norm else max_norm / norm
    return norm, [g * factor for g in grads]
