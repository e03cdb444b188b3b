"""Distillation from a teacher's top logits: loss, gradient and the fused step
against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import row_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu
from tests.row_util import DistillBounds, Rows, close, rounded

pytestmark = pytest.mark.gpu

LOWEST = {"f32": torch.finfo(torch.float32).min, "bf16": torch.finfo(torch.bfloat16).min}


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def case(r, n, V, k, masked):
    z = 2 * r.standard_normal((n, V))
    ids = r.integers(0, V, (n, k))
    top = 3 * r.standard_normal((n, k))
    np.put_along_axis(z, ids, top + 0.5 * r.standard_normal((n, k)), 1)
    if masked:
        z[r.random((n, V)) < 0.2] = -np.inf
        ids[r.random((n, k)) < 0.2] = -1
        ids[r.random((n, k)) < 0.05] = V
        top[r.random((n, k)) < 0.1] = -np.inf
        # no infinite loss here: entries keep a finite logit
        at = np.where((ids >= 0) & (ids < V), ids, 0)
        cur = np.take_along_axis(z, at, 1)
        np.put_along_axis(z, at, np.where(np.isfinite(cur), cur, 1.0), 1)
        if n > 2:
            ids[1] = -1                      # a padding row
    return z, ids, top


def run_all(z, ids, top, T, w, dtype, extra=0, off=0):
    n, V = z.shape
    Z = Rows(n, V, dtype, extra, off, z)
    di = torch.as_tensor(ids.astype(np.int32), device="cuda").contiguous()
    dt = torch.as_tensor(top.astype(np.float32), device="cuda").contiguous()
    dw = None if w is None else torch.as_tensor(w.astype(np.float32), device="cuda")
    loss, lse, loss2 = (Rows(1, n, "f32") for _ in range(3))
    dz, dz2 = (Rows(n, V, dtype, e, off) for e in (extra, 2 * extra))
    shc.distill_top(Z.t, di, dt, loss.t[0], lse.t[0], temperature=T)
    shc.distill_top_backward(Z.t, di, dt, lse.t[0], dw, dz.t, temperature=T)
    shc.distill_top_step(Z.t, di, dt, dw, loss2.t[0], dz2.t, temperature=T)
    for t in (loss, lse, loss2, dz, dz2):
        t.check_guard()
    return Z.get(), loss.get()[0], lse.get()[0], dz.get(), loss2.get()[0], dz2.get()


def check(z, ids, top, T, w, dtype, extra=0, off=0):
    Z, loss, lse, dz, loss2, dz2 = run_all(z, ids, top, T, w, dtype, extra, off)
    T = float(np.float32(T))
    w = None if w is None else w.astype(np.float32).astype(np.float64)
    top = top.astype(np.float32).astype(np.float64)
    rl, rlse, rdz = O.distill(Z, ids, top, T, w)
    b = DistillBounds(Z, ids, top, T, w, O)
    close(loss, rl, rounded(b.loss, rl, "f32"), "loss")
    close(loss2, rl, rounded(b.loss, rl, "f32"), "loss of the step")
    close(lse, rlse, rounded(b.lse, np.where(np.isfinite(rlse), rlse, 0), "f32"), "lse")
    close(dz, rdz, rounded(b.dz_back, rdz, dtype), "backward")
    close(dz2, rdz, rounded(b.dz_step, rdz, dtype), "step")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("n,V,k,T,extra,off", [
    (1, 1, 1, 1.0, 0, 0), (3, 2, 3, 2.0, 1, 1), (5, 9, 4, 0.5, 0, 0), (300, 16, 8, 1.0, 0, 0),
    (1000, 128, 8, 2.0, 0, 0), (65, 130, 64, 1.5, 3, 2), (40, 257, 256, 1.0, 0, 0),
    (33, 513, 5, 4.0, 0, 3), (17, 1000, 17, 1.0, 8, 8), (9, 2050, 64, 1.0, 0, 0),
    (7, 4099, 100, 2.0, 1, 1), (300, 4500, 3, 1.0, 0, 0), (2, 9000, 64, 3.0, 0, 0),
    (260, 8200, 20, 1.0, 5, 0), (257, 16500, 64, 1.0, 0, 1), (1, 33001, 50, 1.0, 0, 0),
    (258, 33001, 7, 1.5, 0, 0), (3, 70001, 64, 1.0, 1, 0), (256, 70001, 10, 1.0, 0, 0),
    (2, 140001, 64, 2.0, 0, 0), (256, 140001, 9, 1.0, 3, 0),
])
def test_against_the_oracle(dtype, masked, n, V, k, T, extra, off):
    r = np.random.default_rng(n + V)
    z, ids, top = case(r, n, V, k, masked)
    w = None if n % 3 == 0 else r.random(n) + 0.5
    check(z, ids, top, T, w, dtype, extra, off)


@pytest.mark.parametrize("V", [40, 700, 9000, 140001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_masks(dtype, V):
    """Rows of -inf, of the type's lowest value, of equal logits, and rows whose
    entries are all absent."""
    k = 4
    z = np.zeros((6, V))
    z[0] = -np.inf
    z[1] = LOWEST[dtype]
    z[2] = LOWEST[dtype]
    z[2, V // 2] = 3.0
    z[3, 1:] = -np.inf
    z[4] = 60000.0
    ids = np.tile(np.array([0, V // 2, V - 1, 2]), (6, 1))
    ids[5] = [-1, V, -7, 2 ** 30]
    top = np.tile(np.array([1.0, 2.0, 0.5, -np.inf]), (6, 1))
    Z, loss, lse, dz, loss2, dz2 = run_all(z, ids, top, 1.0, None, dtype)
    rl, rlse, rdz = O.distill(Z, ids, top, 1.0)
    for got in (loss, loss2):
        assert np.array_equal(np.isinf(got), np.isinf(rl))
        fin = np.isfinite(rl)
        assert np.allclose(got[fin], rl[fin], rtol=3e-6, atol=1e-6)
    assert rl[0] == np.inf and rl[5] == 0 and np.all(dz[5] == 0) and np.all(dz2[5] == 0)
    assert lse[0] == -np.inf and np.allclose(lse[1:], rlse[1:], rtol=3e-6)
    for got in (dz2, dz):
        tol = 2.0 ** -8 * np.abs(rdz) + 1e-6 if dtype == "bf16" else 1e-6
        # lse of rows 1, 4 is the logits' own size: its rounding is the
        # backward's whole error there
        rows = [0, 2, 3, 5] if got is dz else range(6)
        for i in rows:
            assert np.all(np.abs(got[i] - rdz[i]) <= (tol if np.isscalar(tol) else tol[i])), i
        assert np.all(np.isfinite(got))


@pytest.mark.parametrize("V", [40, 3000, 20000])
def test_a_bad_row_stays_alone(V):
    r = np.random.default_rng(V)
    z, ids, top = case(r, 12, V, 5, False)
    good = run_all(z, ids, top, 1.0, None, "f32")
    z[3, V // 3] = np.nan
    z[7, 0] = np.inf
    top[9, 2] = np.nan
    bad = run_all(z, ids, top, 1.0, None, "f32")
    keep = [i for i in range(12) if i not in (3, 7, 9)]
    for g, b in zip(good[1:], bad[1:]):
        assert np.array_equal(g[keep], b[keep])
    for loss in (bad[1], bad[4]):
        assert np.isnan(loss[[3, 7, 9]]).all()
    assert np.isnan(bad[5][3]).all()


@pytest.mark.parametrize("V", [64, 3000])
def test_entries_far_apart(V):
    """Teacher's probabilities down to the subnormal range and below add nothing,
    and no more."""
    r = np.random.default_rng(V)
    z = r.standard_normal((3, V))
    ids = np.stack([r.permutation(V)[:8] for _ in range(3)])
    top = np.array([[0, -1, -86.5, -87.3, -88, -95, -104, -300.0]] * 3)
    top[1, :2] = 0.0                     # a sum of two: the rest move down once more
    check(z, ids, top, 1.0, None, "f32")
    check(z, ids, top * 3, 3.0, None, "bf16")


def test_repeated_ids_share_their_probability():
    z = np.random.default_rng(0).standard_normal((2, 50))
    ids = np.array([[4, 4, 4, 9], [0, 49, 0, 49]])
    top = np.array([[1.0, 0.0, 2.0, 1.0], [0.0, 0.0, 0.0, 0.0]])
    check(z, ids, top, 1.0, None, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,k", [(40, 16), (40, 17), (300, 33), (300, 200), (1000, 129),
                                 (9000, 64), (33001, 256), (262145, 40), (300000, 256)])
def test_rows_with_and_without_repeated_ids(dtype, V, k):
    """Side by side: ids all different, one of them twice, ids that are equal in
    their low bits only, one id throughout, and absent ones between."""
    r = np.random.default_rng(V + k)
    z = 2 * r.standard_normal((7, V))
    ids = np.stack([r.permutation(V)[:k] for _ in range(7)])
    ids[1, k - 1] = ids[1, 0]
    ids[2, 1:4] = ids[2, 0]
    ids[3] = V - 1
    half = k // 2
    ids[4, half:2 * half] = (ids[4, :half] + 131072) % V
    ids[5, ::3] = -1
    ids[6, ::2] = V
    top = 3 * r.standard_normal((7, k))
    np.put_along_axis(z, np.where((ids >= 0) & (ids < V), ids, 0),
                      top + 0.5 * r.standard_normal((7, k)), 1)
    check(z, ids, top, 1.5, r.random(7) + 0.5, dtype)


@pytest.mark.parametrize("V", [20477, 20481, 32769, 41000, 53249, 65537])
def test_step_of_many_long_rows(V):
    r = np.random.default_rng(V)
    n = 512
    z, ids, top = case(r, n, V, 5, False)
    z, ids, top = z.astype(np.float32), ids.astype(np.int32), top.astype(np.float32)
    z[3, V // 2:] = LOWEST["f32"]
    z[5, :-1] = -np.inf
    ids[5], z[7] = -1, 1e6 + 20 * z[7]       # no entries; far from 0
    ids[9, 1:] = ids[9, 0]
    Z = torch.as_tensor(z, device="cuda")
    loss, dz = shc.distill_top_step(Z, torch.as_tensor(ids, device="cuda"),
                                    torch.as_tensor(top, device="cuda"))
    rows = np.array([0, 1, 3, 5, 7, 9, n - 1])
    z64, t64 = z[rows].astype(np.float64), top[rows].astype(np.float64)
    rl, _, rdz = O.distill(z64, ids[rows], t64, 1.0)
    b = DistillBounds(z64, ids[rows], t64, 1.0, None, O)
    close(loss.double().cpu().numpy()[rows], rl, rounded(b.loss, rl, "f32"), "loss")
    close(dz[torch.as_tensor(rows, device="cuda")].double().cpu().numpy(), rdz,
          rounded(b.dz_step, rdz, "f32"), "step")


@pytest.mark.parametrize("V", [28669, 28673, 32769, 40961, 53248, 65535, 65537])
def test_step_of_so_many_long_rows_that_registers_hold_them(V):
    n, k = 1000, 9
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    z = 2 * torch.randn((n, V), generator=g, device="cuda")
    ids = torch.randint(0, V, (n, k), generator=g, device="cuda", dtype=torch.int32)
    top = 3 * torch.randn((n, k), generator=g, device="cuda")
    z[3, V // 2:] = LOWEST["f32"]
    z[5, :-1] = -np.inf
    ids[5], z[7] = -1, 1e6 + 20 * z[7]       # no entries; far from 0
    ids[3] %= V // 2
    ids[9, 1:] = ids[9, 0]
    loss, dz = shc.distill_top_step(z, ids, top)
    rows = [0, 1, 3, 5, 7, 9, 511, n - 1]
    z64, t64 = z[rows].double().cpu().numpy(), top[rows].double().cpu().numpy()
    picked = ids[rows].cpu().numpy()
    rl, _, rdz = O.distill(z64, picked, t64, 1.0)
    b = DistillBounds(z64, picked, t64, 1.0, None, O)
    close(loss[rows].double().cpu().numpy(), rl, rounded(b.loss, rl, "f32"), "loss")
    close(dz[rows].double().cpu().numpy(), rdz, rounded(b.dz_step, rdz, "f32"), "step")


def test_backward_of_many_long_rows():
    r = np.random.default_rng(11)
    z, ids, top = case(r, 513, 9000, 20, True)
    check(z, ids, top, 1.0, None, "bf16")
    z, ids, top = case(r, 512, 4200, 40, False)
    check(z, ids, top, 1.0, None, "f32")
    z, ids, top = case(r, 1536, 4200, 40, True)
    check(z, ids, top, 1.0, None, "f32")
    z, ids, top = case(r, 1537, 8300, 20, False)
    check(z, ids, top, 1.0, None, "bf16")


def test_padding_rows_are_not_read():
    """A row without entries may hold anything."""
    z = np.zeros((4, 600))
    z[2] = np.nan
    ids = np.zeros((4, 3), np.int64)
    ids[2] = -1
    Z, loss, lse, dz, loss2, dz2 = run_all(z, ids, np.zeros((4, 3)), 1.0, None, "bf16")
    for a in (loss, lse, loss2, dz, dz2):
        assert np.all(np.isfinite(a)) and not a[2].any()


def test_no_rows_and_fewer_rows():
    z = torch.zeros((0, 64), device="cuda")
    loss, dz = shc.distill_top_step(z, torch.zeros((0, 4), dtype=torch.int32, device="cuda"),
                                    torch.zeros((0, 4), device="cuda"))
    assert loss.shape == (0,) and dz.shape == (0, 64)
    r = np.random.default_rng(1)
    z, ids, top = case(r, 300, 6000, 8, False)
    Z = torch.as_tensor(z, dtype=torch.float32, device="cuda")
    I = torch.as_tensor(ids, dtype=torch.int32, device="cuda")
    t = torch.as_tensor(top, dtype=torch.float32, device="cuda")
    loss, dz = torch.full((300,), 9.0, device="cuda"), torch.full((300, 6000), 9.0, device="cuda")
    call = shc.prepare_distill_top_step(Z, I, t, None, loss, dz)
    for n in (1, 5, 300):                    # few rows: cut into parts
        call(n)
        want = shc.distill_top_step(Z[:n], I[:n], t[:n])
        assert torch.equal(loss[:n], want[0]) and torch.equal(dz[:n], want[1])
        assert n == 300 or bool((dz[n:] == 9).all())


def test_rows_past_32_bit_offsets():
    n, ld = 300_000, 16000                   # 4.8e9 elements of bf16
    buf = torch.zeros((n, ld), dtype=torch.bfloat16, device="cuda")
    z, dz = buf[:, :40], buf[:, 100:140]
    z[-1, 3] = 2.0
    ids = torch.full((n, 2), -1, dtype=torch.int32, device="cuda")
    ids[-1] = torch.tensor([3, 5], device="cuda")
    top = torch.zeros((n, 2), device="cuda")
    loss, _ = shc.distill_top_step(z, ids, top, None, None, dz)
    want = O.distill(z[-1:].double().cpu().numpy(), ids[-1:].cpu().numpy(), np.zeros((1, 2)), 1.0)
    assert np.isclose(float(loss[-1]), want[0][0], rtol=1e-5) and not loss[:-1].any()
    assert np.allclose(dz[-1].double().cpu().numpy(), want[2][0], atol=2.0 ** -8)


def test_gradient_by_differences():
    r = np.random.default_rng(7)
    z, ids, top = case(r, 1, 60, 5, False)
    di = torch.as_tensor(ids, dtype=torch.int32, device="cuda")
    dt = torch.as_tensor(top, dtype=torch.float32, device="cuda")
    Z = torch.as_tensor(z, dtype=torch.float32, device="cuda")
    _, dz = shc.distill_top_step(Z, di, dt, temperature=2.0)
    h = 2.0 ** -5
    both = torch.cat([Z + h * torch.eye(60, device="cuda"), Z - h * torch.eye(60, device="cuda")])
    f = shc.distill_top(both, di.expand(120, 5).contiguous(), dt.expand(120, 5).contiguous(),
                        temperature=2.0).double()
    # h^2 / 6 of third derivatives below 1, and the loss's rounding over 2 h
    assert torch.allclose((f[:60] - f[60:]) / (2 * h), dz[0].double(), atol=5e-4)
