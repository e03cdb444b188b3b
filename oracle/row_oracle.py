"""CPU oracle of the row operators -- TEST INFRASTRUCTURE ONLY.

Embedding rows, layer norm and distillation from a teacher's top logits, each
with its gradient, in fp64 numpy from the definitions.  Shares no code with the
HIP kernels.
"""
from __future__ import annotations

import numpy as np


def embed(E, ids, scale=1.0, add=None):
    """scale * E[id] (+ add); an id outside [0, len(E)) has no row."""
    E = np.asarray(E, np.float64)
    ids = np.asarray(ids, np.int64)
    there = (ids >= 0) & (ids < len(E))
    out = np.where(there[:, None], E[np.where(there, ids, 0)] * scale, 0.0)
    return out if add is None else out + np.asarray(add, np.float64)


def embed_backward(dY, ids, R, scale=1.0, pad_id=-1):
    """dE [R][C]: scale times the sum of the rows of every id but pad_id."""
    dY = np.asarray(dY, np.float64)
    ids = np.asarray(ids, np.int64)
    keep = (ids >= 0) & (ids < R) & (ids != pad_id)
    dE = np.zeros((R, dY.shape[1]))
    np.add.at(dE, ids[keep], dY[keep])
    return dE * scale


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd) per row."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(1) + eps)
    y = d * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) for the given mean and rstd."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    rstd = np.asarray(rstd, np.float64)[:, None]
    h = (x - np.asarray(mean, np.float64)[:, None]) * rstd
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    if x.shape[0]:
        dx = rstd * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    else:
        dx = np.zeros_like(x)
    return dx, (dy * h).sum(0), dy.sum(0)


def teacher(ids, top, V, T):
    """(p, log p, present, live): the teacher's distribution over its entries."""
    ids, top = np.asarray(ids, np.int64), np.asarray(top, np.float64)
    with np.errstate(invalid="ignore"):
        there = (ids >= 0) & (ids < V) & ~(top == -np.inf)
        t = np.where(there, top, -np.inf)
        live = there.any(1)
        m = np.where(live, t.max(1), 0.0)[:, None]
        e = np.where(there, np.exp((t - m) / T), 0.0)
        s = np.where(live, e.sum(1), 1.0)[:, None]
        return e / s, (t - m) / T - np.log(s), there, live


def student(z, T):
    """(q, log q, lse) of the logits; a logit of -inf has q = 0."""
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        m = z.max(1)
        m = np.where(m == -np.inf, 0.0, m)[:, None]
        e = np.where(z == -np.inf, 0.0, np.exp((z - m) / T))
        s = e.sum(1, keepdims=True)
        q = np.where(s == 0.0, 0.0, e / np.where(s == 0.0, 1.0, s))
        lq = np.where(z == -np.inf, -np.inf, (z - m) / T - np.log(s))
        return q, lq, (m / T + np.log(s))[:, 0]


def distill(z, ids, top, T, w=None):
    """(loss, lse, dz): rows without entries have loss 0, lse 0 and gradient 0."""
    n, V = np.asarray(z).shape
    p, lp, there, live = teacher(ids, top, V, T)
    q, lq, lse = student(z, T)
    at = np.where(there, ids, 0).astype(np.int64)
    with np.errstate(invalid="ignore"):
        terms = np.where(there & ~(p == 0.0), p * (lp - np.take_along_axis(lq, at, 1)), 0.0)
    loss = np.where(live, T * T * terms.sum(1), 0.0)
    d = q.copy()
    np.subtract.at(d, (np.repeat(np.arange(n), ids.shape[1]), at.reshape(-1)), p.reshape(-1))
    w = np.ones(n) if w is None else np.asarray(w, np.float64)
    dz = np.where(live[:, None], d * (T * w)[:, None], 0.0)
    return loss, np.where(live, lse, 0.0), dz
