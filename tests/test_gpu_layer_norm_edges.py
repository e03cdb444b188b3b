"""Layer norm's gradient where the row's mean times 1/std passes fp32."""
import numpy as np
import pytest
import torch

from oracle import row_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu
from tests.row_util import TDT, Rows, close, norm_grad_bounds, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 5, 20, 130, 517, 1100, 2100, 4100, 9001, 16383])
def test_backward_of_constant_rows_of_large_values(dtype, C):
    """h is 0 throughout: dx = rstd (g - mean of g)."""
    r = np.random.default_rng(C)
    x = np.tile(np.array([[2.0 ** 123], [-2.0 ** 123], [3.0]]), (1, C))
    X, dy = Rows(3, C, dtype, 1, 0, x), Rows(3, C, dtype, 0, 1, r.standard_normal((3, C)))
    mean = X.get()[:, 0]
    rstd = np.full(3, np.float32(1e-5) ** -0.5, np.float32).astype(np.float64)
    dx, dg, db = Rows(3, C, dtype, 0, 0), Rows(1, C, "f32"), Rows(1, C, "f32")

    def f32(a):
        return torch.as_tensor(a, dtype=torch.float32, device="cuda")

    shc.layer_norm_backward(dy.t, X.t, None, f32(mean), f32(rstd), dx.t, dg.t[0], db.t[0])
    rx, rg, rb = O.layer_norm_backward(dy.get(), X.get(), None, mean, rstd)
    bx, bg, bb = norm_grad_bounds(dy.get(), X.get(), None, mean, rstd)
    close(dx.get(), rx, rounded(bx, rx, dtype), "dx")
    close(dg.get()[0], rg, rounded(bg, rg, "f32"), "dgamma")
    close(db.get()[0], rb, rounded(bb, rb, "f32"), "dbeta")
