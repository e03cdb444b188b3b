"""Distillation where values are far from the ordinary."""
import numpy as np
import pytest
import torch

from oracle import row_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu
from tests.row_util import TDT, DistillBounds, close, rounded

pytestmark = pytest.mark.gpu

LOWEST = {k: torch.finfo(t).min for k, t in TDT.items()}


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def run(z, ids, top, T=1.0, w=None):
    """(loss, lse, dz of the backward, the step's loss, its dz) in fp64."""
    n, V = z.shape
    lse = torch.empty(n, device="cuda")
    loss = shc.distill_top(z, ids, top, None, lse, T)
    dz = shc.distill_top_backward(z, ids, top, lse, w, None, T)
    loss2, dz2 = shc.distill_top_step(z, ids, top, w, None, None, T)
    return [t.double().cpu().numpy() for t in (loss, lse, dz, loss2, dz2)]


def entries(n, V, k, seed):
    """Entries in a row's first quarter."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn((n, V), generator=g, device="cuda")
    ids = torch.randint(0, V // 4, (n, k), generator=g, device="cuda", dtype=torch.int32)
    return z, ids, torch.randn((n, k), generator=g, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [600, 20000, 40000, 140001])
@pytest.mark.parametrize("n", [6, 300])
def test_nan_in_a_part_of_a_row(dtype, V, n):
    """Runs of columns longer than a part of a row that is cut up; the answer does
    not depend on the number of rows, and other rows' results stay."""
    z, ids, top = entries(n, V, 5, V)
    z = z.to(TDT[dtype])
    good = run(z, ids, top)
    z[1, V // 2:] = float("nan")
    z[2, V // 2:] = -float("inf")
    z[2, V - 1] = float("nan")               # nothing but -inf around it
    z[3] = float("nan")
    z[4, V // 2:] = torch.tensor(-1, dtype=torch.int32).view(torch.float32)  # sign bit set
    bad = run(z, ids, top)
    rows = [1, 2, 3, 4]
    keep = np.setdiff1d(np.arange(n), rows)
    for name, g, b in zip(("loss", "lse", "backward", "step's loss", "step"), good, bad):
        assert np.isnan(b[rows]).all(), name
        assert np.array_equal(g[keep], b[keep]), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 3000, 20000, 40000, 140001])
def test_nan_rows_with_entries_on_masked_logits(dtype, V):
    """In a row with a NaN, loss and gradient are NaN at entries on -inf too; without
    one they are +inf and -p there."""
    z, ids, top = entries(3, V, 4, V)
    z, ids = z.to(TDT[dtype]), torch.arange(4, dtype=torch.int32).repeat(3, 1).cuda()
    z[:, 2] = -float("inf")
    z[1, V - 1] = float("nan")
    z[2, V - 1] = float("inf")
    loss, lse, dz, loss2, dz2 = run(z, ids, top)
    p = torch.softmax(top[0].double(), 0)[2].item()
    for got in (dz, dz2):
        assert np.isnan(got[1:]).all()
        assert abs(got[0, 2] + p) <= 2.0 ** -8 * p
    assert loss[0] == loss2[0] == np.inf
    assert np.isnan(loss[1:]).all() and np.isnan(loss2[1:]).all()
    # no other entry in the row
    one = torch.full((3, 1), 2, dtype=torch.int32, device="cuda")
    loss, lse, dz, loss2, dz2 = run(z, one, top[:, :1].contiguous())
    for got in (loss, loss2):
        assert got[0] == np.inf and np.isnan(got[1:]).all()
    z[0] = -float("inf")                     # and no logit
    loss, lse, dz, loss2, dz2 = run(z, one, top[:, :1].contiguous())
    assert loss[0] == loss2[0] == np.inf and lse[0] == -np.inf
    for got in (dz, dz2):
        assert got[0, 2] == -1.0 and not np.delete(got[0], 2).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,k", [(9, 40, 4), (9, 200, 40), (9, 500, 9), (9, 1000, 5),
                                   (9, 2000, 5), (9, 4000, 5), (9, 9000, 20), (1600, 9000, 4),
                                   (1540, 4200, 5), (9, 33001, 6), (9, 140001, 200)])
def test_backward_of_rows_far_from_zero(dtype, n, V, k):
    """lse in 32 bits says nothing of the sum where the maximum is large: the
    backward is as near as the step is."""
    z, ids, top = entries(n, V, k, n + V)
    z *= 2
    for row, at in enumerate((0.0, 70.0, -900.0, 4000.0, -3e5, 1e6, 1e9)):
        z[row] += at
    z[7] = LOWEST[dtype]                     # masks that leave nothing
    z[8] = 6e4                               # equal logits
    z[3, V // 2:] = LOWEST[dtype]
    z = z.to(TDT[dtype])
    w = torch.rand(n, device="cuda") + 0.5
    dz = run(z[:9], ids[:9], top[:9], w=w[:9])[2] if n == 9 else run(z, ids, top, w=w)[2][:9]
    Z, I, t, W = (a[:9].double().cpu().numpy() for a in (z, ids, top, w))
    ref = O.distill(Z, I.astype(np.int64), t, 1.0, W)[2]
    b = DistillBounds(Z, I.astype(np.int64), t, 1.0, W, O)
    # row 0 is at 0, where lse keeps its digits; the others as the step's
    bound = np.concatenate([b.dz_back[:1], b.dz_step[1:]])
    if dtype == "bf16":                      # up to 1,024 the saved lse serves bf16
        bound[1:3] = b.dz_back[1:3]
    close(dz, ref, rounded(bound, ref, dtype), "backward")


@pytest.mark.parametrize("T", [0.01, 30.0])
@pytest.mark.parametrize("V", [300, 5000, 40000])
def test_backward_far_from_zero_at_other_temperatures(T, V):
    z, ids, top = entries(4, V, 6, V)
    z += torch.tensor([[0.0], [50.0], [-2000.0], [1e5]], device="cuda")
    dz = run(z, ids, top, T)[2]
    Z, I, t = (a.double().cpu().numpy() for a in (z, ids, top))
    T = float(np.float32(T))
    ref = O.distill(Z, I.astype(np.int64), t, T)[2]
    b = DistillBounds(Z, I.astype(np.int64), t, T, None, O)
    far = np.abs(Z.max(1, keepdims=True) / T) > 80
    bound = np.where(far, b.dz_step, b.dz_back)
    close(dz, ref, rounded(bound, ref, "f32"), "backward")


@pytest.mark.parametrize("T", [1e-25, 2e-20, 1e-12, 1e18])
@pytest.mark.parametrize("V", [30, 2000, 40000])
def test_loss_at_the_ends_of_the_temperatures(T, V):
    """T^2 leaves the range of fp32 long before T^2 times the sum does."""
    z, ids, top = entries(3, V, 5, V)
    loss, lse, dz, loss2, dz2 = run(z, ids, top, T)
    Z, I, t = (a.double().cpu().numpy() for a in (z, ids, top))
    T = float(np.float32(T))
    ref = O.distill(Z, I.astype(np.int64), t, T)[0]
    b = DistillBounds(Z, I.astype(np.int64), t, T, None, O)
    close(loss, ref, rounded(b.loss, ref, "f32"), "loss")
    close(loss2, ref, rounded(b.loss, ref, "f32"), "loss of the step")


def test_loss_of_equal_distributions_at_a_large_temperature():
    """T^2 is past fp32, T^2 times the rounding of the sum is not."""
    z, ids = torch.full((2, 1), 3.0, device="cuda"), torch.zeros((2, 1), device="cuda").int()
    T = float(np.float32(1e20))
    loss, lse, dz, loss2, dz2 = run(z, ids, z, T)
    b = DistillBounds(np.full((2, 1), 3.0), np.zeros((2, 1), np.int64), np.full((2, 1), 3.0), T,
                      None, O)
    for got in (loss, loss2):
        close(got, np.zeros(2), rounded(b.loss, np.zeros(2), "f32"), "loss")
