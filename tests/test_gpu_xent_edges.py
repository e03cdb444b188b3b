"""The cross entropy of a linear layer's logits where whole tiles of classes are masked by
their bias, against the 64-bit oracle, by every way to the gradients (logits formed again,
kept exponentials, kept logits)."""
import numpy as np
import pytest
import torch

from paper_2608_09388_amd import binding as shc
from tests.dense_util import xent_bounds
from tests.gpu_util import require_gpu
from tests.row_util import Rows, close, rounded
from tests.test_gpu_xent import Case, check, f32, wide

pytestmark = pytest.mark.gpu

N, V = 600, 700
WIDTHS = [40, 256, 768]  # bf16 keeps exponentials from 256 on, with db logits from 768 on


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def masked(C, dtype, mask, value, rest):
    """A case with `value` as the bias of masked classes, `rest` added to the others'; every
    label on a class that counts, but for row 3's."""
    c = Case(N, C, V, 0.0, 0, 0, dtype, seed=9)
    c.b = np.where(mask, value, rest + c.r.standard_normal(V)).astype(np.float32)
    free = np.flatnonzero(~mask)
    c.labels[:] = free[c.labels % len(free)]
    c.labels[3] = np.flatnonzero(mask)[0]
    return c


def bounds_of(c, ref, mask):
    """The masked classes have probability 0 and their logits' rounding reaches nothing but the
    loss of a label there."""
    return xent_bounds(c.x.get(), c.W.get(), wide(c.b),
                       dict(ref, z=np.where(mask, -np.inf, ref["z"])), wide(c.w), c.dtype)


def run_all(c):
    """(what, loss, lse or None, dx, dW, db or None) of every way to the gradients."""
    ids, bias, w = c.ids(), f32(c.b), f32(c.w)
    loss, lse = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    shc.linear_cross_entropy(c.x.t, c.W.t, ids, bias, loss, lse)
    for with_db in (True, False):
        for step in (True, False):
            dx, dW, db = c.grads()
            kw = dict(dx=dx.t, dW=dW.t, db=db.t[0] if with_db else None)
            if step:
                got = shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, w, bias, **kw)
            else:
                shc.linear_cross_entropy_backward(c.x.t, c.W.t, ids, lse, w, bias, **kw)
                got = loss
            yield (f"{'step' if step else 'backward'}{' with db ' if with_db else ' '}", got, lse,
                   dx, dW, db if with_db else None)


def check_masked(c, mask):
    ref = c.oracle()
    b = bounds_of(c, ref, mask)
    for what, loss, lse, dx, dW, db in run_all(c):
        close(loss.double().cpu().numpy(), ref["loss"], rounded(b["loss"], ref["loss"], "f32"),
              what + "loss")
        close(lse.double().cpu().numpy(), ref["lse"], rounded(b["lse"], ref["lse"], "f32"), "lse")
        if db is None:
            db = Rows(1, V, "f32", values=ref["db"][None])
        check(c, ref, b, dx, dW, db, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("rest", [0.0, -120.0, 120.0])
def test_tiles_of_nothing_but_minus_infinity(C, dtype, rest):
    """A log-sum far on either side of 0 beside tiles of probability 0 (from below -88.7 on e to
    its negative passes fp32)."""
    for mask in (np.arange(V) < 512, np.arange(V) >= 100, np.arange(V) // 128 % 2 == 1):
        check_masked(masked(C, dtype, mask, -np.inf, rest), mask)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_a_logit_that_is_not_a_number_beside_masked_tiles(C, dtype):
    """A NaN in another tile makes the results of the masked tiles' classes NaN too."""
    c = masked(C, dtype, np.arange(V) < 512, -np.inf, 0.0)
    c.b[600] = np.nan
    for what, loss, lse, dx, dW, db in run_all(c):
        for t in (loss, lse, dx.t, dW.t) + (() if db is None else (db.t,)):
            assert bool(torch.isnan(t).all()), what


FINITE = [-1e4, -1e8, -1e9, -1e10, -1e12, -1e18, -1e20, -1e30, float(np.finfo(np.float32).min)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("value", FINITE)
def test_tiles_of_finite_masks(C, dtype, value):
    """A finite number as a mask: probability 0 as with -inf, the loss of a label there finite."""
    for mask in (np.arange(V) < 512, np.arange(V) >= 100, np.arange(V) % 3 == 1):
        check_masked(masked(C, dtype, mask, value, 0.0), mask)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("value", FINITE)
def test_every_class_masked(C, dtype, value):
    """All classes at the mask's value.  u = 2^-24: lse and the logits are off by a rounding of
    their size each, loss by three, lse - z being rounded too, beside 1e-3 for all else; a
    probability stays within [0, 1] whatever these are, so that no dz passes the row's weight."""
    c = Case(N, C, V, 0.0, 0, 0, dtype)
    c.b = np.full(V, value, np.float32)
    ref = c.oracle()
    off = 4 * 2.0 ** -24 * abs(value) + 1e-3
    w = np.ones(N) if c.w is None else wide(c.w)
    W, x = np.abs(c.W.get()), np.abs(c.x.get())
    most_dx = w[:, None] * (W.sum(0)[None] + W[c.labels])
    most_dW = (w @ x)[None] + np.zeros((V, 1))
    for what, loss, lse, dx, dW, db in run_all(c):
        assert np.all(np.abs(loss.double().cpu().numpy() - ref["loss"]) <= off), what
        assert np.all(np.abs(lse.double().cpu().numpy() - ref["lse"]) <= off), what
        assert np.all(np.abs(dx.get()) <= 1.01 * most_dx), what
        assert np.all(np.abs(dW.get()) <= 1.01 * most_dW), what
        assert db is None or np.all(np.abs(db.get()) <= 1.01 * w.sum()), what
