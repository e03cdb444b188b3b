"""Error bounds of the dense operators' GPU tests, derived from the kernels'
arithmetic.  u = 2^-24 is the rounding unit of fp32.

A sum of K exact products in fp32, in any order, is off by at most K u times the
sum of their magnitudes.  Split fp32 products leave out at most 2^-22 of a product
(2^-23 and the terms' own rounding), the five small ones of the six are at most
2^-7 of it each and are summed first: 1.1 K roundings cover them.  The bounds are
first-order; `row_util.rounded` allows twice their figure and adds the rounding of
the output."""
import numpy as np

from oracle import dense_oracle as O

u = 2.0 ** -24


def half(dtype):
    """A rounding to the type, relative."""
    return 2.0 ** -8 if dtype == "bf16" else 0.0


def product(a, b, dtype, K):
    """Bound of a @ b computed by the kernels from exact operands."""
    s = np.abs(a) @ np.abs(b)
    return (1.1 * K + 16) * u * s + (2.0 ** -22 * s if dtype == "f32" else 0.0)


def act_bound(code, z, ez):
    """Bound of act(z) for z off by ez: |act'| is at most 1.13; Phi is within
    1.5e-7 and an exponential and a few roundings of it, e^-z within 4 u |z| + 4 u."""
    az = np.abs(z)
    if code == O.GELU:
        return 1.13 * ez + az * (1.5e-7 + 16 * u)
    if code == O.SILU:
        return 1.1 * ez + np.abs(O.act(code, z)) * (4 * u * np.minimum(az, 100.0) + 12 * u)
    return ez


def slope_bound(code, z):
    az = np.minimum(np.abs(z), 100.0)
    if code == O.GELU:
        # z phi(z): |z| e^(-z^2/2) is below 0.61, its exponent off by 4 u z^2
        return 1.5e-7 + 24 * u + az * np.exp(-0.5 * az * az) * (4 * u * az * az + 8 * u)
    if code == O.SILU:
        return (1.0 + az) * (4 * u * az + 16 * u) * np.exp(-np.maximum(0.0, az - 2.0)) + 8 * u
    return 0.0 * az


def linear_bounds(x, W, bias, code, residual, z, out, dtype):
    """(out, pre) bounds before the output's rounding."""
    ez = product(x, W, dtype, x.shape[1]) + (0.0 if bias is None else 2 * u * (np.abs(z)
                                                                             + np.abs(bias)))
    eo = act_bound(code, z, ez)
    if residual is not None:
        eo = eo + 2 * u * (np.abs(out) + np.abs(residual))
    return eo + u * np.abs(out), ez


def linear_grad_bounds(dout, x, W, pre, code, dz, dtype):
    """(dx, dW, db) bounds; dz is rounded to the type before the products."""
    n = x.shape[0]
    ed = np.zeros_like(dz) if code == O.NONE else (
        np.abs(dout) * slope_bound(code, pre) + 2 * u * np.abs(dz))
    er = ed + (half(dtype) * np.abs(dz) + 2.0 ** -133 if code not in (O.NONE, O.RELU) else 0.0)
    dx = er @ np.abs(W).T + product(dz, W.T, dtype, W.shape[1])
    dW = np.abs(x).T @ er + product(x.T, dz, dtype, n)
    return dx, dW, ed.sum(0) + (n + 8) * u * np.abs(dz).sum(0)


def xent_bounds(x, W, bias, ref, weight, dtype, lse_given=None):
    """dict of bounds of loss, lse (live rows), dx, dW, db.

    A logit is off by ez.  lse: the softmax's mean of ez, then at most 600 additions
    one after another (16 in a lane, four lanes, the tiles' joins), exponentials off
    by 4 u of their exponent and 4 u."""
    live, z, q, dz = ref["live"], ref["z"], ref["q"], ref["dz"]
    n, V = x.shape[0], W.shape[0]
    xl = x[live]
    ez = product(xl, W.T, dtype, x.shape[1])
    if bias is not None:
        ez = ez + 2 * u * (np.abs(np.where(np.isfinite(z), z, 0.0))
                           + np.abs(np.where(np.isfinite(bias), bias, 0.0)))
    lse = np.where(np.isfinite(ref["lse"][live]), ref["lse"][live], 0.0)
    far = np.where(np.isfinite(z), np.abs(z - lse[:, None]), 0.0)
    big = np.where(np.isfinite(z), np.abs(z), 0.0).max(1, initial=0.0)
    el = (q * (ez + 4 * u * far)).sum(1) + 600 * u + 4 * u * (np.abs(lse) + big)
    w = np.ones(n) if weight is None else weight
    at = np.take_along_axis(ez, ref["labels"][live][:, None], 1)[:, 0]
    zl = np.take_along_axis(np.where(np.isfinite(z), np.abs(z), 0.0),
                            ref["labels"][live][:, None], 1)[:, 0]
    elg = el if lse_given is None else u * np.abs(lse)
    eq = q * (ez + elg[:, None] + 6 * u * (far + np.abs(lse)[:, None]) + 8 * u) + 2.0 ** -126
    ed = np.abs(w[live])[:, None] * eq + 4 * u * np.abs(dz)
    er = ed + half(dtype) * np.abs(dz) + 2.0 ** -133
    dx = np.zeros_like(x)
    dx[live] = er @ np.abs(W) + product(dz, W, dtype, V)
    return dict(loss=el + at + 2 * u * (np.abs(lse) + zl), lse=el, dx=dx,
                dW=er.T @ np.abs(xl) + product(dz.T, xl, dtype, max(1, len(live))),
                db=ed.sum(0) + (n + 8) * u * np.abs(dz).sum(0))
