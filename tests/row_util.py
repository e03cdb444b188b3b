"""Helpers of the row operators' GPU tests: row tensors inside guarded buffers,
and error bounds derived from the kernels' arithmetic.

u = 2^-24 is the rounding unit of fp32; a bf16 output is rounded once more, by
at most 2^-8 of its magnitude (2^-133 below its normal range).  The bounds are
first-order; twice their figure is allowed throughout."""
import numpy as np
import torch

u = 2.0 ** -24
TDT = {"bf16": torch.bfloat16, "f32": torch.float32}
SENTINEL = 77.0


class Rows:
    """[n][C] rows in a buffer of sentinels: `extra` elements after each row,
    `off` elements before the first."""

    def __init__(self, n, C, dtype, extra=0, off=0, values=None):
        self.n, self.C, self.ld, self.off = n, C, C + extra, off
        self.buf = torch.full((off + max(n, 1) * self.ld + 16,), SENTINEL, dtype=TDT[dtype],
                              device="cuda")
        self.t = self.buf[off:off + max(n, 1) * self.ld].view(max(n, 1), self.ld)[:n, :C]
        if values is not None:
            self.t.copy_(torch.as_tensor(np.asarray(values, np.float32)))

    def get(self):
        return self.t.double().cpu().numpy()

    def check_guard(self, what=""):
        """Nothing outside the rows was written."""
        b = self.buf.clone()
        b[self.off:self.off + max(self.n, 1) * self.ld].view(max(self.n, 1),
                                                             self.ld)[:self.n, :self.C] = SENTINEL
        assert bool((b == SENTINEL).all()), f"{what}: written outside the rows"


def stored(a, dtype):
    """The values as the dtype holds them, in fp64."""
    return torch.as_tensor(np.asarray(a, np.float32)).to(TDT[dtype]).double().numpy()


def rounded(bound, ref, dtype):
    bound = 2.0 * np.asarray(bound) + 2.0 ** -140
    return bound + (2.0 ** -8 * np.abs(ref) + 2.0 ** -133 if dtype == "bf16" else 0.0)


def close(got, ref, bound, what=""):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), f"{what}: infinities"
    bad = ~(np.abs(np.where(inf, 0, got) - np.where(inf, 0, ref)) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        b = np.broadcast_to(bound, ref.shape)[i]
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside the bound; first at "
                             f"{i}: got {got[i]}, ref {ref[i]}, bound {b}")


# -- layer norm ---------------------------------------------------------------
# A thread adds at most 32 values of a row, then 6 lane steps, at most 16
# wavefronts and the product with 1/C (itself rounded twice): 64 roundings cover
# a row's sum.


def norm_bounds(x, gamma, beta, y, mean, rstd):
    """(y, mean, rstd) bounds."""
    dmu = 64 * u * np.abs(x).mean(1)
    rel = 0.5 * (72 * u + (dmu * rstd) ** 2) + 4 * u
    h = np.abs((x - mean[:, None]) * rstd[:, None])
    g = 1.0 if gamma is None else np.abs(gamma)
    b = 0.0 if beta is None else np.abs(beta)
    by = g * ((rstd * dmu)[:, None] + h * (rel + 4 * u)[:, None]) + 2 * u * (g * h + b)
    return by, dmu, rel * rstd


def norm_grad_bounds(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) bounds for the given mean and rstd."""
    n = x.shape[0]
    r = rstd[:, None]
    h = np.abs((x - mean[:, None]) * r)
    g = np.abs(dy if gamma is None else dy * gamma)
    mg, mgh = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    dx = r * (5 * u * g + 70 * u * mg + 80 * u * h * mgh)
    ady = np.abs(dy)
    return dx, (n + 8) * u * (ady * h).sum(0), (n + 2) * u * ady.sum(0)


# -- distillation -------------------------------------------------------------
# 2^((z - m) c): the difference, c (two roundings), the product and the
# hardware's exponential: 4 u of the exponent and 4 u of the value.  A sum of
# V such terms goes through at most 400 additions one after the other.


class DistillBounds:
    def __init__(self, z, ids, top, T, w, oracle):
        n, V = z.shape
        self.T, self.w = T, np.ones(n) if w is None else w
        p, lp, there, live = oracle.teacher(ids, top, V, T)
        q, lq, lse = oracle.student(z, T)
        with np.errstate(invalid="ignore"):
            m = z.max(1)
            m = np.where(np.isfinite(m), m, 0.0)
            a = np.where(q > 0, (m[:, None] - z) / T, 0.0)
            lns = np.where(np.isfinite(lse), np.abs(lse - m / T), 0.0)
            self.err_l = (q * 4 * u * a).sum(1) + (408 + 4 * (1 + lns)) * u
            lse = np.where(np.isfinite(lse), lse, 0.0)
            self.lse = self.err_l + 2 * u * (np.abs(m / T) + lns)
            e_lq = 6 * u * a + (self.err_l + 2 * u * lns)[:, None]
            b = np.where(p > 0, -lp, 0.0)
            e_lp = 6 * u * b + ((p * 4 * u * b).sum(1) + (ids.shape[1] + 20) * u)[:, None]
            at = np.where(there, ids, 0)
            d = np.where(p > 0, np.abs(lp - np.take_along_axis(lq, at, 1)), 0.0)
            d = np.where(np.isfinite(d), d, 0.0)
            terms = p * (e_lp + np.take_along_axis(e_lq, at, 1)
                         + (e_lp + (ids.shape[1] + 12) * u) * (d + 1))
            self.loss = T * T * np.where(there, terms, 0.0).sum(1)
            pt = np.zeros_like(q)
            np.add.at(pt, (np.repeat(np.arange(n), ids.shape[1]), at.reshape(-1)),
                      (p * (e_lp + (ids.shape[1] + 8) * u)).reshape(-1))
            step = q * (e_lq + 8 * u) + pt
            near = np.where(q > 0, np.abs(z / T - lse[:, None]), 0.0)
            back = q * ((self.lse + 3 * u * np.abs(lse))[:, None] + 6 * u * near + 8 * u) + pt
        f = (T * self.w)[:, None]
        # probabilities below the normal range may be flushed
        self.dz_step, self.dz_back = f * (step + 2.0 ** -126), f * (back + 2.0 ** -126)
