"""The cross entropy of a linear layer's logits and its gradients against the 64-bit
oracle."""
import numpy as np
import pytest
import torch

from oracle import dense_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.dense_util import xent_bounds
from tests.gpu_util import require_gpu
from tests.row_util import TDT, Rows, close, rounded

pytestmark = pytest.mark.gpu

# rows, C, V, share of padding, elements after a row, elements before the first
SHAPES = [
    (1, 1, 1, 0.0, 0, 0), (1, 64, 1000, 0.0, 0, 0), (3, 5, 2, 0.0, 1, 1), (16, 72, 300, 0.3, 0, 0),
    (17, 33, 65, 0.0, 3, 2), (64, 128, 48, 0.5, 8, 8), (65, 256, 257, 0.0, 0, 1),
    (130, 16, 4000, 0.2, 0, 0), (129, 64, 512, 0.05, 64, 0), (300, 200, 520, 0.0, 8, 0),
    (513, 130, 300, 0.9, 6, 0), (1000, 40, 10, 0.1, 0, 0), (5, 1000, 70, 0.0, 0, 0),
    (700, 72, 1025, 0.33, 0, 0), (40, 8, 20000, 0.0, 0, 0), (257, 513, 63, 0.5, 1, 3),
    (300, 520, 1100, 0.3, 0, 0), (1300, 640, 136, 0.5, 8, 0), (2, 1024, 3001, 0.0, 0, 0),
    (2100, 24, 700, 0.1, 0, 0),
]


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def f32(a):
    return None if a is None else torch.as_tensor(np.asarray(a, np.float32), device="cuda")


def wide(a):
    return None if a is None else np.asarray(a, np.float32).astype(np.float64)


class Case:
    def __init__(self, n, C, V, ignored, extra, off, dtype, seed=0):
        r = self.r = np.random.default_rng(seed + n + 3 * C + 7 * V)
        self.n, self.C, self.V, self.dtype, self.pad = n, C, V, dtype, (extra, off)
        self.x = self.rows(n, C)
        self.W = self.rows(V, C, 2.0 * C ** -0.5)
        self.b = None if n % 2 else r.standard_normal(V).astype(np.float32)
        self.w = None if n % 3 == 0 else (r.random(n) + 0.5).astype(np.float32)
        self.labels = r.integers(0, V, n)
        self.labels[r.random(n) < ignored] = r.choice([-1, -100, V, V + 7, 2 ** 31 - 1])

    def rows(self, n, C, scale=1.0):
        return Rows(n, C, self.dtype, *self.pad, self.r.standard_normal((n, C)) * scale)

    def out(self, n, C):
        return Rows(n, C, self.dtype, *self.pad)

    def ids(self, kind="i64"):
        if kind == "i64":
            return torch.as_tensor(self.labels, device="cuda")
        pairs = torch.full((self.n, 2), -7, dtype=torch.int32, device="cuda")
        pairs[:, 1] = torch.as_tensor(self.labels.astype(np.int32), device="cuda")
        return pairs[:, 1]

    def oracle(self):
        ref = O.cross_entropy(self.x.get(), self.W.get(), self.labels, wide(self.b), wide(self.w))
        ref["labels"] = self.labels
        return ref

    def grads(self):
        return self.out(self.n, self.C), self.out(self.V, self.C), Rows(1, self.V, "f32")


def check(c, ref, bounds, dx, dW, db, what=""):
    close(dx.get(), ref["dx"], rounded(bounds["dx"], ref["dx"], c.dtype), what + "dx")
    close(dW.get(), ref["dW"], rounded(bounds["dW"], ref["dW"], c.dtype), what + "dW")
    close(db.get()[0], ref["db"], rounded(bounds["db"], ref["db"], "f32"), what + "db")
    for t in (dx, dW, db):
        t.check_guard(what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_all_three(dtype, shape):
    c = Case(*shape, dtype)
    ref = c.oracle()
    live = ref["live"]
    b = xent_bounds(c.x.get(), c.W.get(), wide(c.b), ref, wide(c.w), dtype)
    bias, w = f32(c.b), f32(c.w)
    loss, lse = Rows(1, c.n, "f32"), Rows(1, c.n, "f32")
    shc.linear_cross_entropy(c.x.t, c.W.t, c.ids(), bias, loss.t[0], lse.t[0])
    close(loss.get()[0][live], ref["loss"][live], rounded(b["loss"], ref["loss"][live], "f32"), "loss")
    close(lse.get()[0][live], ref["lse"][live], rounded(b["lse"], ref["lse"][live], "f32"), "lse")
    pad = np.setdiff1d(np.arange(c.n), live)
    assert not loss.get()[0][pad].any() and not lse.get()[0][pad].any()
    loss.check_guard(), lse.check_guard()
    dx, dW, db = c.grads()
    shc.linear_cross_entropy_backward(c.x.t, c.W.t, c.ids("i32"), lse.t[0], w, bias, dx.t, dW.t,
                                      db.t[0])
    check(c, ref, b, dx, dW, db, "backward ")
    assert not dx.get()[pad].any()
    dx, dW, db = c.grads()
    loss2 = Rows(1, c.n, "f32")
    shc.linear_cross_entropy_step(c.x.t, c.W.t, c.ids("i32"), w, bias, loss2.t[0], dx.t, dW.t,
                                  db.t[0])
    assert torch.equal(loss.t, loss2.t)
    check(c, ref, b, dx, dW, db, "step ")
    # without db the step may go another way
    dx, dW, _ = c.grads()
    shc.linear_cross_entropy_step(c.x.t, c.W.t, c.ids(), w, bias, loss2.t[0], dx.t, dW.t)
    assert torch.equal(loss.t, loss2.t)
    check(c, ref, b, dx, dW, db, "step without db ")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padding_may_hold_anything(dtype):
    """NaN and infinities in the rows of padding reach no result."""
    for n, C, V in ((70, 40, 100), (300, 72, 33)):
        c = Case(n, C, V, 0.5, 0, 0, dtype)
        ids = c.ids()
        pad = (ids < 0) | (ids >= V)
        want = [t.t for t in c.grads()]
        loss = shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, None, None, None, want[0],
                                             want[1], want[2][0])
        c.x.t[pad] = float("nan")
        c.x.t[torch.nonzero(pad)[0]] = float("inf")
        got = [t.t for t in c.grads()]
        loss2 = shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, None, None, None, got[0], got[1],
                                              got[2][0])
        assert torch.equal(loss, loss2) and all(torch.equal(a, b) for a, b in zip(want, got))
        assert not bool(got[0][pad].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_but_padding(dtype):
    c = Case(50, 24, 80, 0.0, 0, 0, dtype)
    ids = torch.full((50,), -100, device="cuda")
    c.x.t.fill_(float("nan"))
    old = [t.t.fill_(2.0) for t in c.grads()]
    loss = shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, None, None, None, old[0], old[1],
                                         old[2][0], accumulate=True)
    assert not bool(loss.any()) and not bool(old[0].any())
    assert bool((old[1] == 2).all()) and bool((old[2] == 2).all())
    shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, None, None, loss, old[0], old[1], old[2][0])
    assert not bool(old[1].any()) and not bool(old[2].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(dtype):
    x = torch.zeros((0, 24), dtype=TDT[dtype], device="cuda")
    W = torch.ones((80, 24), dtype=TDT[dtype], device="cuda")
    ids = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert shc.linear_cross_entropy(x, W, ids).shape == (0,)
    dW, db = torch.ones_like(W), torch.ones(80, device="cuda")
    shc.linear_cross_entropy_step(x, W, ids, dW=dW, db=db, accumulate=True)
    assert bool((dW == 1).all()) and bool((db == 1).all())
    shc.linear_cross_entropy_backward(x, W, ids, torch.zeros(0, device="cuda"), dW=dW, db=db)
    assert not bool(dW.any()) and not bool(db.any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("with_db", [True, False])
def test_masked_classes(dtype, with_db):
    """Classes of bias -inf: probability 0, a label there a loss of +inf, in a row of nothing
    else lse -inf; the type's lowest value as a mask stays finite."""
    c = Case(64, 40, 700, 0.0, 0, 0, dtype)
    low = float(np.finfo(np.float32).min)
    for mask in (np.arange(700) % 3 == 1, np.arange(700) < 690, np.ones(700, bool)):
        for value in (-np.inf, low):
            c.b = np.where(mask, value, c.r.standard_normal(700)).astype(np.float32)
            c.labels[:] = np.flatnonzero(~mask)[0] if not mask.all() else 4
            c.labels[3] = np.flatnonzero(mask)[0]
            ref = c.oracle()
            dx, dW, db = c.grads()
            loss = shc.linear_cross_entropy_step(
                c.x.t, c.W.t, c.ids(), f32(c.w), f32(c.b), None, dx.t, dW.t,
                db.t[0] if with_db else None)
            got = loss.double().cpu().numpy()
            assert np.array_equal(np.isinf(got), np.isinf(ref["loss"]))
            if value == low:
                continue
            b = xent_bounds(c.x.get(), c.W.get(), wide(c.b), ref, wide(c.w), dtype)
            if not with_db:
                db.t.copy_(f32(ref["db"][None]))
            check(c, ref, b, dx, dW, db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_row_that_is_not_a_number(dtype):
    c = Case(40, 24, 300, 0.0, 0, 0, dtype)
    want, _, _ = c.grads()
    loss = shc.linear_cross_entropy_step(c.x.t, c.W.t, c.ids(), None, None, None, want.t)
    for value in (float("nan"), float("inf")):
        c.x.t[7, 5] = value
        dx, dW, db = c.grads()
        got = shc.linear_cross_entropy_step(c.x.t, c.W.t, c.ids(), None, None, None, dx.t, dW.t,
                                            db.t[0])
        rest = torch.arange(40, device="cuda") != 7
        assert torch.equal(got[rest], loss[rest]) and bool(torch.isnan(got[7]))
        assert torch.equal(dx.t[rest], want.t[rest]) and bool(torch.isnan(dx.t[7]).all())
        assert bool(torch.isnan(db.t).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(dtype):
    """Logits of some thousand, one class far above the others."""
    c = Case(66, 40, 300, 0.0, 0, 0, dtype)
    c.x.t.mul_(300.0)
    ref = c.oracle()
    b = xent_bounds(c.x.get(), c.W.get(), wide(c.b), ref, wide(c.w), dtype)
    dx, dW, db = c.grads()
    loss = shc.linear_cross_entropy_step(c.x.t, c.W.t, c.ids(), f32(c.w), f32(c.b), None, dx.t,
                                         dW.t, db.t[0])
    close(loss.double().cpu().numpy(), ref["loss"], rounded(b["loss"], ref["loss"], "f32"), "loss")
    check(c, ref, b, dx, dW, db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_accumulate_and_parts(dtype):
    c = Case(130, 72, 200, 0.2, 0, 0, dtype)
    ids, w = c.ids(), f32(c.w)
    dx, dW, db = c.grads()
    shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, w, None, None, dx.t, dW.t, db.t[0])
    for k in range(3):
        outs = c.grads()
        given = [None, None, None]
        given[k] = outs[k].t[0] if k == 2 else outs[k].t
        lse = torch.empty(130, device="cuda")
        shc.linear_cross_entropy(c.x.t, c.W.t, ids, lse=lse)
        shc.linear_cross_entropy_backward(c.x.t, c.W.t, ids, lse, w, None, *given)
        assert torch.equal(outs[k].t, (dx, dW, db)[k].t)
    c.b = None
    ref = c.oracle()
    b = xent_bounds(c.x.get(), c.W.get(), None, ref, wide(c.w), dtype)
    old_W, old_b = c.rows(200, 72), Rows(1, 200, "f32", values=c.r.standard_normal((1, 200)))
    rW, rb = ref["dW"] + old_W.get(), ref["db"] + old_b.get()[0]
    shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, w, None, None, None, old_W.t, old_b.t[0],
                                  accumulate=True)
    close(old_W.get(), rW, rounded(b["dW"] + 2.0 ** -24 * np.abs(rW), rW, dtype), "dW")
    close(old_b.get()[0], rb, rounded(b["db"] + 2.0 ** -24 * np.abs(rb), rb, "f32"), "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_fewer_rows_than_prepared(dtype):
    c = Case(600, 72, 500, 0.3, 0, 0, dtype)
    ids = c.ids()
    loss = torch.empty(600, device="cuda")
    dx, dW, db = (t.t for t in c.grads())
    call = shc.prepare_linear_cross_entropy_step(c.x.t, c.W.t, None, ids, None, loss, dx, dW, db[0])
    for n in (600, 1, 16, 100, 257, 0):
        loss.fill_(5.0), dx.fill_(5.0)
        call(n)
        assert bool((loss[n:] == 5).all()) and bool((dx[n:] == 5).all())
        rx, rW, rb = (t.t for t in c.grads())
        ref = shc.linear_cross_entropy_step(c.x.t[:n], c.W.t, ids[:n], None, None, None, rx[:n],
                                            rW, rb[0])
        assert torch.equal(loss[:n], ref) and torch.equal(dx[:n], rx[:n])
        assert torch.equal(dW, rW) and torch.equal(db, rb)


def test_many_labels():
    """Labels over several blocks of the list, against a count of them."""
    n, C, V = 20001, 8, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((n, C), generator=g, device="cuda")
    W = torch.randn((V, C), generator=g, device="cuda")
    labels = torch.randint(-8, V + 8, (n,), generator=g, device="cuda")
    live = (labels >= 0) & (labels < V)
    loss = shc.linear_cross_entropy(x, W, labels)
    z = x.double() @ W.double().t()
    ref = torch.logsumexp(z, 1) - z.gather(1, labels.clamp(0, V - 1)[:, None])[:, 0]
    assert not bool(loss[~live].any())
    assert float((loss[live] - ref[live]).abs().max()) < 1e-5


@pytest.mark.parametrize("C", [16, 128])   # logits taken again, logits kept
def test_pieces_of_rows(C):
    """More pairs of row and class than a piece holds: the gradient of W over two pieces."""
    n, V = 300, (1 << 20) + 8
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((n, C), generator=g, device="cuda")
    W = torch.randn((V, C), generator=g, device="cuda") * (2.0 * C ** -0.5)
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty(V, device="cuda")
    old = torch.randn((V, C), generator=g, device="cuda") * 1e-3
    dW2 = old.clone()
    loss = shc.linear_cross_entropy_step(x, W, labels, None, None, None, dx, dW, db)
    shc.linear_cross_entropy_step(x, W, labels, None, None, loss, None, dW2, accumulate=True)
    z = x.double() @ W.double().t()
    lse = torch.logsumexp(z, 1)
    q = torch.exp(z - lse[:, None])
    q[torch.arange(n), labels] -= 1.0
    assert float((loss - (lse - z.gather(1, labels[:, None])[:, 0])).abs().max()) < 2e-5
    del z
    for got, ref in ((dx, q @ W.double()), (dW, q.t() @ x.double()), (db, q.sum(0)),
                     (dW2, q.t() @ x.double() + old.double())):
        assert float((got - ref).norm() / ref.norm()) < 2e-6


@pytest.mark.parametrize("shape", [(1, 448, 3456), (7, 448, 3456), (7, 72, 1000), (64, 128, 300),
                                   (3, 2048, 100), (33, 64, 5000)])
@pytest.mark.parametrize("with_db", [False, True])
def test_few_rows_in_bf16(shape, with_db):
    """Up to 64 rows dz is not rounded to bf16: gradients are off by their own rounding, half a
    step of 8 significand bits or 2^-8, by 2^-11 of the terms for exponentials kept in fp16 (half
    a step of 11 bits, 2^-11) and dz's second term (the rounding of what is at most 2^-8 of it,
    2^-16), and by fp32's sums.  (dz rounded once would be off by 2^-8 of the terms.)"""
    n, C, V = shape
    c = Case(n, C, V, 0.2 if n > 5 else 0.0, 0, 0, "bf16")
    ids, w = c.ids(), f32(c.w)
    x, W = c.x.get(), c.W.get()
    weight = np.ones(n) if c.w is None else wide(c.w)
    z = x @ W.T
    z -= z.max(1, keepdims=True)
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    y = ids.cpu().numpy()
    live = (y >= 0) & (y < V)
    dz = p.copy()
    dz[np.flatnonzero(live), y[live]] -= 1
    dz *= np.where(live, weight, 0)[:, None]
    # an fp32 logit is off by (C + 16) 2^-24 of its terms, lse by a few of its last bits, and
    # dz of its probability by as much; a kept exponential by 2^-40 of the row's largest
    off = ((C + 16) * 2.0 ** -24 * (np.abs(x) @ np.abs(W).T)).max() + 2.0 ** -18
    slack = weight.max() * (p * 2 * off + 2.0 ** -39) * live[:, None]
    for step in (False, True):
        dx, dW, db = c.grads()
        kw = dict(dx=dx.t, dW=dW.t, db=db.t[0] if with_db else None)
        if step:
            shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, w, **kw)
        else:
            lse = torch.empty(n, device="cuda")
            shc.linear_cross_entropy(c.x.t, c.W.t, ids, lse=lse)
            shc.linear_cross_entropy_backward(c.x.t, c.W.t, ids, lse, w, **kw)
        for got, ref, size, more in ((dx, dz @ W, np.abs(dz) @ np.abs(W), slack @ np.abs(W)),
                                     (dW, dz.T @ x, np.abs(dz).T @ np.abs(x), slack.T @ np.abs(x))):
            rest = 2.0 ** -11 + 2.0 ** -16 + (V + n) * 2.0 ** -24
            bound = 2.0 ** -8 * np.abs(ref) + rest * size + more
            assert np.all(np.abs(got.t.double().cpu().numpy() - ref) <= 1.01 * bound + 1e-30)


@pytest.mark.parametrize("n", [40, 70, 3000])
def test_weights_of_any_size(n):
    """The factor that dz in bf16 is formed with follows the largest weight of a row that counts:
    weights times a power of two give gradients times it, bit for bit; none, tiny, huge and
    infinite ones give what they say."""
    c = Case(n, 64, 96, 0.2, 0, 0, "bf16")
    ids = c.ids()
    w = torch.rand(n, generator=torch.Generator().manual_seed(3)).cuda() + 0.5
    w[c.labels >= 96] = float("inf")  # of padding
    w[c.labels < 0] = float("nan")

    def grads(weight):
        dx, dW, db = c.grads()
        shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, weight, dx=dx.t, dW=dW.t, db=db.t[0])
        return dx.t.clone(), dW.t.clone(), db.t.clone()

    first = grads(w)
    assert all(bool(torch.isfinite(g).all()) for g in first)
    for k in (-30, -1, 40):
        for a, b in zip(grads(w * 2.0 ** k), first):
            assert torch.equal(a, b * 2.0 ** k)
    assert all(bool((g == 0).all()) for g in grads(torch.zeros_like(w)))
    x, W = c.x.get(), c.W.get()
    dz = np.exp(x @ W.T)
    dz /= dz.sum(1, keepdims=True)
    live = (c.labels >= 0) & (c.labels < 96)
    dz[np.flatnonzero(live), c.labels[live]] -= 1
    dz = np.abs(dz * live[:, None])
    # what the terms of a gradient add up to: past 2^127 a sum of fp32 may pass its range on the
    # way, whatever it ends at
    terms = [torch.as_tensor(t, device="cuda") for t in
             (dz @ np.abs(W), dz.T @ np.abs(x), dz.sum(0)[None])]
    for size in (1e-42, 1e-38, 2e38):
        got = grads(torch.full_like(w, size))
        ref = grads(torch.ones_like(w))
        for a, b, t in zip(got, ref, terms):
            a, b = a.double(), b.double() * float(np.float32(size))
            fits = t * size < 2.0 ** 127
            assert bool(fits.any()) or size > 1
            slack = 2.0 ** -6 * b.abs().max() + 1e-40
            assert bool(((a - b).abs()[fits] <= slack).all())
    one = torch.ones_like(w)
    row = int(np.flatnonzero((c.labels >= 0) & (c.labels < 96))[0])
    one[row] = float("inf")
    rest = torch.arange(n, device="cuda") != row
    assert torch.equal(grads(one)[0][rest], grads(torch.ones_like(w))[0][rest])
