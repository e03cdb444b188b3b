"""Layer norm where every group of lanes takes several rows one after the other,
in each arrangement of lanes, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import row_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu
from tests.row_util import Rows, close, norm_bounds, norm_grad_bounds, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def f32(a):
    return torch.as_tensor(a, dtype=torch.float32, device="cuda")


def wide(a):
    return np.asarray(a, np.float32).astype(np.float64)


# at most 1,024 workgroups of 256 lanes or of one row
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [
    (40003, 30), (40001, 60), (20001, 100), (9001, 250), (5003, 500), (5001, 760), (1101, 900),
    (4199, 1500), (1091, 1900), (2117, 2100), (1303, 3500), (1301, 5001), (1101, 7000),
    (1031, 9001), (1027, 16383),
])
def test_forward_of_many_rows(dtype, n, C):
    r = np.random.default_rng(n + C)
    x = r.standard_normal((n, C), np.float32) * np.exp(r.standard_normal((n, 1), np.float32))
    x += r.standard_normal((n, 1), np.float32)
    X, Y = Rows(n, C, dtype, 1, 0, x), Rows(n, C, dtype, 0, 1)
    gamma, beta = r.standard_normal(C), r.standard_normal(C)
    mean, rstd = Rows(1, n, "f32"), Rows(1, n, "f32")
    shc.layer_norm(X.t, f32(gamma), f32(beta), Y.t, mean.t[0], rstd.t[0])
    x, gamma, beta = X.get(), wide(gamma), wide(beta)
    ref, rm, rr = O.layer_norm(x, gamma, beta, float(np.float32(1e-5)))
    by, bm, br = norm_bounds(x, gamma, beta, ref, rm, rr)
    close(Y.get(), ref, rounded(by, ref, dtype), "y")
    close(mean.get()[0], rm, rounded(bm, rm, "f32"), "mean")
    close(rstd.get()[0], rr, rounded(br, rr, "f32"), "rstd")
    for t in (Y, mean, rstd):
        t.check_guard()


# at most 768 workgroups of 256 lanes, 512 or 256 of one row
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [
    (30001, 30), (30003, 60), (14001, 100), (9001, 250), (5003, 500), (2501, 760), (2201, 900),
    (2117, 1500), (2113, 2001), (2113, 2050), (1301, 3500), (1101, 5001), (601, 7000), (603, 8193),
    (599, 9001), (523, 16383),
])
def test_backward_of_many_rows(dtype, n, C):
    r = np.random.default_rng(n * 3 + C)
    x = 2 * r.standard_normal((n, C), np.float32) + r.standard_normal((n, 1), np.float32)
    X, dY = Rows(n, C, dtype, 0, 1, x), Rows(n, C, dtype, 1, 0, r.standard_normal((n, C)))
    gamma, x = r.standard_normal(C), X.get()
    mean = wide(x.mean(1))
    rstd = wide(1.0 / np.sqrt(x.var(1) + 1e-5))
    dx, dg, db = Rows(n, C, dtype, 2, 0), Rows(1, C, "f32"), Rows(1, C, "f32")
    shc.layer_norm_backward(dY.t, X.t, f32(gamma), f32(mean), f32(rstd), dx.t, dg.t[0], db.t[0])
    dy, gamma = dY.get(), wide(gamma)
    rx, rg, rb = O.layer_norm_backward(dy, x, gamma, mean, rstd)
    bx, bg, bb = norm_grad_bounds(dy, x, gamma, mean, rstd)
    close(dx.get(), rx, rounded(bx, rx, dtype), "dx")
    close(dg.get()[0], rg, rounded(bg, rg, "f32"), "dgamma")
    close(db.get()[0], rb, rounded(bb, rb, "f32"), "dbeta")
    for t in (dx, dg, db):
        t.check_guard()
