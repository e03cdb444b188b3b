"""The dense linear layer and its gradients against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import dense_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.dense_util import linear_bounds, linear_grad_bounds
from tests.gpu_util import require_gpu
from tests.row_util import TDT, Rows, close, rounded, stored

pytestmark = pytest.mark.gpu

# rows, Cin, Cout, elements after a row, elements before the first
SHAPES = [
    (1, 1, 1, 0, 0), (1, 64, 64, 0, 0), (2, 3, 5, 1, 1), (15, 16, 16, 0, 0), (16, 72, 264, 0, 0),
    (17, 33, 70, 3, 2), (64, 128, 48, 8, 8), (65, 256, 257, 0, 1), (100, 1000, 8, 0, 0),
    (129, 64, 128, 64, 0), (255, 40, 24, 0, 0), (300, 200, 520, 8, 0), (513, 130, 300, 6, 0),
    (1000, 16, 16, 0, 0), (3, 4099, 17, 0, 0), (40, 2048, 1030, 0, 0), (2, 5, 3000, 0, 0),
    (1025, 513, 63, 1, 3),
]
ACTS = [shc.SHC_ACT_NONE, shc.SHC_ACT_RELU, shc.SHC_ACT_GELU, shc.SHC_ACT_SILU]


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def f32(a):
    return None if a is None else torch.as_tensor(np.asarray(a, np.float32), device="cuda")


def wide(a):
    return None if a is None else np.asarray(a, np.float32).astype(np.float64)


class Case:
    def __init__(self, n, Cin, Cout, extra, off, dtype, seed=0):
        r = self.r = np.random.default_rng(seed + n + 3 * Cin + 7 * Cout)
        self.n, self.Cin, self.Cout, self.dtype, self.pad = n, Cin, Cout, dtype, (extra, off)
        self.x = self.rows(n, Cin)
        self.W = self.rows(Cin, Cout, Cin ** -0.5)
        self.b = r.standard_normal(Cout).astype(np.float32)

    def rows(self, n, C, scale=1.0):
        return Rows(n, C, self.dtype, *self.pad, self.r.standard_normal((n, C)) * scale)

    def out(self, n, C):
        return Rows(n, C, self.dtype, self.pad[0], self.pad[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dtype, shape):
    for act in ACTS:
        c = Case(*shape, dtype, act)
        bias = c.b if act % 2 == 0 else None
        res = c.rows(c.n, c.Cout) if act >= 2 else None
        out, pre = c.out(c.n, c.Cout), c.out(c.n, c.Cout) if act != 1 else None
        shc.linear(c.x.t, c.W.t, f32(bias), out.t, act, None if res is None else res.t,
                   None if pre is None else pre.t)
        rv = None if res is None else res.get()
        ref, z = O.linear(c.x.get(), c.W.get(), wide(bias), act, rv)
        bo, bz = linear_bounds(c.x.get(), c.W.get(), wide(bias), act, rv, z, ref, dtype)
        close(out.get(), ref, rounded(bo, ref, dtype), f"out, act {act}")
        out.check_guard()
        if pre is not None:
            close(pre.get(), z, rounded(bz, z, dtype), f"pre, act {act}")
            pre.check_guard()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dtype, shape):
    for act in ACTS:
        c = Case(*shape, dtype, act)
        dout, pre = c.rows(c.n, c.Cout), c.rows(c.n, c.Cout, 1.5)
        dx, dW, db = c.out(c.n, c.Cin), c.out(c.Cin, c.Cout), Rows(1, c.Cout, "f32")
        shc.linear_backward(dout.t, c.x.t, c.W.t, pre.t if act else None, dx.t, dW.t, db.t[0],
                            act)
        rx, rW, rb, dz = O.linear_backward(dout.get(), c.x.get(), c.W.get(), pre.get(), act)
        bx, bW, bb = linear_grad_bounds(dout.get(), c.x.get(), c.W.get(), pre.get(), act, dz,
                                        dtype)
        close(dx.get(), rx, rounded(bx, rx, dtype), f"dx, act {act}")
        close(dW.get(), rW, rounded(bW, rW, dtype), f"dW, act {act}")
        close(db.get()[0], rb, rounded(bb, rb, "f32"), f"db, act {act}")
        for t in (dx, dW, db):
            t.check_guard()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_residual_is_out(dtype):
    for n, Cin, Cout in ((300, 64, 200), (8, 4096, 72)):   # one launch; parts along Cin
        c = Case(n, Cin, Cout, 0, 0, dtype)
        out = c.rows(n, Cout)
        ref = shc.linear(c.x.t, c.W.t, f32(c.b), act=shc.SHC_ACT_GELU, residual=out.t.clone())
        shc.linear(c.x.t, c.W.t, f32(c.b), out.t, shc.SHC_ACT_GELU, residual=out.t)
        assert torch.equal(out.t, ref)
    with pytest.raises(shc.ShcError, match="another stride"):
        x = torch.zeros((2, 8), dtype=TDT[dtype], device="cuda")
        W = torch.zeros((8, 4), dtype=TDT[dtype], device="cuda")
        buf = torch.zeros(64, dtype=TDT[dtype], device="cuda")
        shc.linear(x, W, out=buf[:8].view(2, 4), residual=buf[:16].view(2, 8)[:, :4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_accumulate_and_parts_of_the_gradients(dtype):
    c = Case(200, 72, 136, 0, 0, dtype)
    dout, pre = c.rows(200, 136), c.rows(200, 136)
    dx, dW, db = c.out(200, 72), c.out(72, 136), Rows(1, 136, "f32")
    act = shc.SHC_ACT_SILU
    shc.linear_backward(dout.t, c.x.t, c.W.t, pre.t, dx.t, dW.t, db.t[0], act)
    for k in range(3):
        outs = [c.out(200, 72), c.out(72, 136), Rows(1, 136, "f32")]
        given = [o if i == k else None for i, o in enumerate(outs)]
        shc.linear_backward(dout.t, c.x.t, c.W.t, pre.t,
                            *[None if g is None else (g.t[0] if i == 2 else g.t)
                              for i, g in enumerate(given)], act)
        assert torch.equal(outs[k].t, (dx, dW, db)[k].t)
    old_W, old_b = c.rows(72, 136), Rows(1, 136, "f32", values=c.r.standard_normal((1, 136)))
    acc_W, acc_b = old_W.t.clone(), old_b.t.clone()
    shc.linear_backward(dout.t, c.x.t, c.W.t, pre.t, None, acc_W, acc_b[0], act, accumulate=True)
    rx, rW, rb, dz = O.linear_backward(dout.get(), c.x.get(), c.W.get(), pre.get(), act)
    _, bW, bb = linear_grad_bounds(dout.get(), c.x.get(), c.W.get(), pre.get(), act, dz, dtype)
    rW, rb = rW + old_W.get(), rb + old_b.get()[0]
    two = 2.0 ** -24
    close(acc_W.double().cpu().numpy(), rW, rounded(bW + two * np.abs(rW), rW, dtype), "dW")
    close(acc_b.double().cpu().numpy()[0], rb, rounded(bb + two * np.abs(rb), rb, "f32"), "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(dtype):
    x, d = (torch.zeros((0, c), dtype=TDT[dtype], device="cuda") for c in (16, 24))
    W = torch.ones((16, 24), dtype=TDT[dtype], device="cuda")
    assert shc.linear(x, W).shape == (0, 24)
    dW, db = torch.full_like(W, 3.0), torch.full((24,), 3.0, device="cuda")
    shc.linear_backward(d, x, W, dW=dW, db=db, accumulate=True)
    assert bool((dW == 3).all()) and bool((db == 3).all())
    shc.linear_backward(d, x, W, dW=dW, db=db)
    assert not bool(dW.any()) and not bool(db.any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_fewer_rows_than_prepared(dtype):
    """One prepared call and workspace at every count; rows behind the last are left alone."""
    c = Case(700, 520, 136, 0, 0, dtype)
    out = c.out(700, 136)
    call = shc.prepare_linear(c.x.t, c.W.t, f32(c.b), out.t, shc.SHC_ACT_RELU)
    dout, pre = c.rows(700, 136), c.rows(700, 136)
    dx, dW = c.out(700, 520), c.out(520, 136)
    back = shc.prepare_linear_backward(dout.t, c.x.t, c.W.t, pre.t, dx.t, dW.t, None,
                                       shc.SHC_ACT_RELU)
    for n in (700, 1, 16, 17, 129, 256, 400, 0):
        out.t.fill_(5.0)
        dx.t.fill_(5.0)
        call(n)
        back(n)
        assert bool((out.t[n:] == 5).all()) and bool((dx.t[n:] == 5).all())
        ref = shc.linear(c.x.t[:n], c.W.t, f32(c.b), act=shc.SHC_ACT_RELU)
        assert torch.equal(out.t[:n], ref)
        rW = torch.empty_like(dW.t)
        shc.linear_backward(dout.t[:n], c.x.t[:n], c.W.t, pre.t[:n], dW=rW, act=shc.SHC_ACT_RELU)
        assert torch.equal(dW.t, rW)
    with pytest.raises(ValueError, match="n_rows = 701"):
        call(701)


def test_values_that_three_terms_do_not_hold():
    """fp32: infinities, NaN, values of 2^104 and more and sums beyond 2^80 give what fp32
    arithmetic gives; the rest of the rows stay as near."""
    n, Cin, Cout = 300, 72, 140
    c = Case(n, Cin, Cout, 0, 0, "f32")
    x = c.x.get()
    plain = shc.linear(c.x.t, c.W.t).double().cpu().numpy()
    x[5, 3], x[70, 0], x[150, 71], x[299, 9] = np.inf, np.nan, 2.0 ** 120, 2.0 ** 90
    xt = f32(x)
    got = shc.linear(xt, c.W.t).double().cpu().numpy()
    W = c.W.get()
    assert np.array_equal(got[5], np.sign(W[3]) * np.inf) and np.isnan(got[70]).all()
    for r in (150, 299):
        ref = x[r] @ W
        assert np.all(np.abs(got[r] - ref) <= 2 * (Cin + 16) * 2.0 ** -24 * (np.abs(x[r]) @ np.abs(W)))
    rest = np.ones(n, bool)
    rest[[5, 70, 150, 299]] = False
    bound = linear_bounds(c.x.get(), W, None, 0, None, plain, plain, "f32")[0]
    close(got[rest], (c.x.get() @ W)[rest], rounded(bound, plain, "f32")[rest], "other rows")


@pytest.mark.parametrize("scale", [2.0 ** -140, 2.0 ** -100, 2.0 ** 60])
def test_fp32_range(scale):
    c = Case(65, 40, 48, 0, 0, "f32")
    x = stored(c.x.get() * scale, "f32")
    got = shc.linear(f32(x), c.W.t).double().cpu().numpy()
    ref = x @ c.W.get()
    bound = linear_bounds(x, c.W.get(), None, 0, None, ref, ref, "f32")[0]
    close(got, ref, rounded(bound, ref, "f32") + 2.0 ** -149, "out")


def test_activations_at_the_ends():
    z = np.array([[0.0, -0.0, 1e-30, -1e-30, 40.0, -40.0, 1e4, -1e4, 3e38, -3e38, 6.0, -6.0,
                   -13.0, 0.5, -0.5, 88.0]], np.float32)
    eye = torch.eye(16, device="cuda")
    for act in ACTS[1:]:
        got = shc.linear(f32(z), eye, act=act).double().cpu().numpy()
        ref = O.act(act, z.astype(np.float64))
        assert np.isfinite(got).all()
        assert np.all(np.abs(got - ref) <= 1.6e-7 * np.abs(z) + 1e-6 * np.abs(ref) + 1e-37)
        d = torch.empty((1, 16), device="cuda")
        shc.linear_backward(f32(np.ones_like(z)), f32(z), eye, f32(z), dx=d, act=act)
        ref = O.slope(act, z.astype(np.float64))
        assert np.all(np.abs(d.double().cpu().numpy() - ref) <= 2e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_bit_for_bit(dtype):
    c = Case(1000, 1024, 96, 0, 0, dtype)
    dout, pre = c.rows(1000, 96), c.rows(1000, 96)
    first = None
    for _ in range(3):
        out = shc.linear(c.x.t, c.W.t, f32(c.b), act=shc.SHC_ACT_GELU)
        dx, dW = torch.empty_like(c.x.t), torch.empty_like(c.W.t)
        db = torch.empty(96, device="cuda")
        shc.linear_backward(dout.t, c.x.t, c.W.t, pre.t, dx, dW, db, shc.SHC_ACT_GELU)
        now = (out, dx, dW, db)
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


def test_padding_behind_rows_is_not_read_into_sums():
    """NaN between the rows, and behind the last, reaches nothing."""
    for dtype in ("f32", "bf16"):
        for Cin, Cout, extra in ((40, 24, 8), (33, 70, 3), (72, 136, 64)):
            c = Case(70, Cin, Cout, extra, 0, dtype)
            x, W, d = c.x, c.W, c.rows(70, Cout)
            for t in (x, W, d):
                t.buf.masked_fill_(t.buf == 77.0, float("nan"))
            assert bool(torch.isfinite(shc.linear(x.t, W.t)).all())
            dx, dW = (torch.empty(s, dtype=TDT[dtype], device="cuda")
                      for s in ((70, Cin), (Cin, Cout)))
            shc.linear_backward(d.t, x.t, W.t, dx=dx, dW=dW)
            assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dW).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_activations_of_nan_and_infinities(dtype):
    """A NaN stays one, here too with ReLU; the gradient through it is not lost."""
    nan, inf = float("nan"), float("inf")
    z = torch.full((1, 8), 0.5, device="cuda", dtype=TDT[dtype])
    bias = torch.zeros(8, device="cuda")
    bias[1], bias[2], bias[3] = nan, inf, -inf
    eye = torch.eye(8, device="cuda", dtype=TDT[dtype])
    for act in ACTS:
        out = shc.linear(z, eye, bias, act=act)[0].tolist()
        assert math.isnan(out[1]) and out[2] == inf
        if act == shc.SHC_ACT_NONE:
            assert out[3] == -inf
        elif act == shc.SHC_ACT_RELU:
            assert out[3] == 0
        else:
            assert math.isnan(out[3])
        assert all(math.isfinite(out[k]) for k in (0, 4, 5, 6, 7))
    pre = z.clone()
    pre[0, 1], pre[0, 2] = nan, -inf
    dx = torch.empty_like(z)
    shc.linear_backward(torch.ones_like(z), z, eye, pre, dx=dx, act=shc.SHC_ACT_RELU)
    assert dx[0].tolist() == [1, 1, 0, 1, 1, 1, 1, 1]


@pytest.mark.parametrize("shape", [(3001, 3003, 210, 3, 0), (40, 6000, 12000, 0, 0),
                                   (9000, 1500, 130, 0, 2)])
def test_large_fp32(shape):
    """Products that are formed in three terms, forward and backward, and values that these do
    not hold: those rows and columns give what fp32 gives, no bit of the others changes."""
    n, Cin, Cout, extra, off = shape
    c = Case(n, Cin, Cout, extra, off, "f32")
    dout = c.rows(n, Cout)
    x, W, d = (t.get() for t in (c.x, c.W, dout))
    out = shc.linear(c.x.t, c.W.t, f32(c.b))
    dx, dW = torch.empty((n, Cin), device="cuda"), torch.empty((Cin, Cout), device="cuda")
    db = torch.empty(Cout, device="cuda")
    shc.linear_backward(dout.t, c.x.t, c.W.t, dx=dx, dW=dW, db=db)
    for got, ref, size, K in (
            (out, x @ W + c.b, np.abs(x) @ np.abs(W) + np.abs(c.b), Cin),
            (dx, d @ W.T, np.abs(d) @ np.abs(W).T, Cout),
            (dW, x.T @ d, np.abs(x).T @ np.abs(d), n), (db, d.sum(0), np.abs(d).sum(0), n)):
        off_by = np.abs(got.double().cpu().numpy() - ref)
        # a rounding of every sum, six products of terms, the one that is left out
        assert np.all(off_by <= (K + 16) * 2.0 ** -24 * size)
    c.x.t[7, 3], c.x.t[11, Cin - 1] = float("nan"), 2.0 ** 110
    again = shc.linear(c.x.t, c.W.t, f32(c.b))
    assert bool(torch.isnan(again[7]).all())
    ref = 2.0 ** 110 * W[Cin - 1]
    assert np.all(np.abs(again[11].double().cpu().numpy() - ref) <= 2.0 ** -22 * np.abs(ref) + 1e6)
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[7] = rest[11] = False
    assert torch.equal(again[rest], out[rest])
