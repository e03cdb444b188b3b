"""The cross entropy's gradients in several pieces of rows, by every way to them, with row weights
and padding that leaves the last piece full, in part or empty, against 64 bits a chunk of classes
at a time; and gradients of few bf16 rows added to what the outputs hold."""
import numpy as np
import pytest
import torch

from paper_2608_09388_amd import binding as shc
from tests.dense_util import xent_bounds
from tests.gpu_util import require_gpu
from tests.row_util import Rows, close, rounded
from tests.test_gpu_xent import Case, f32, wide

pytestmark = pytest.mark.gpu

CHUNK = 1 << 16


@pytest.fixture(scope="module", autouse=True)
def dev():
    yield require_gpu()
    torch.cuda.empty_cache()


def inputs(n, C, V, dtype, live, seed):
    """live rows that count, at random places; the others' x holds NaN."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    x = torch.randn((n, C), generator=g, device="cuda").to(dt)
    W = torch.empty((V, C), dtype=dt, device="cuda").normal_(generator=g).mul_(2.0 * C ** -0.5)
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    pad = torch.randperm(n, generator=g, device="cuda")[live:]
    labels[pad] = -100
    x[pad] = float("nan")
    w = torch.rand(n, generator=g, device="cuda") + 0.5
    return x, W, labels, w


def check_chunks(x, W, labels, w, outs):
    """outs: list of (what, dx or None, dW, db or None, the value that dW and db held before, or
    None).  In the 2-norm of a row; the terms are those of a gradient's rounding, dz's, of kept
    exponentials (2^-11, and 2^-39 of a row's largest probability), of a logit's error for the
    probabilities, and of the sums: additions of 2^-24 after one another, a matrix instruction
    taking 16 products, in fp32 six times as many."""
    rows = torch.nonzero(labels >= 0)[:, 0]
    n, V, C = len(rows), W.shape[0], W.shape[1]
    xs, y, ws = x[rows].double(), labels[rows], w[rows].double()
    bf16 = x.dtype == torch.bfloat16
    u = 2.0 ** -24
    h, six = (2.0 ** -8, 1) if bf16 else (u, 6)

    def chunks():
        for v in range(0, V, CHUNK):
            c = W[v:v + CHUNK].double()
            z = xs @ c.t().contiguous()
            yield v, c, z, torch.nonzero((y >= v) & (y < v + len(c)))[:, 0]

    top = torch.full((n,), -1e300, dtype=torch.float64, device="cuda")
    total, off = torch.zeros_like(top), 0.0
    for v, c, z, mine in chunks():
        m = torch.maximum(top, z.amax(1))
        total = total * torch.exp(top - m) + torch.exp(z - m[:, None]).sum(1)
        top = m
        if n:
            off = max(off, float((xs.abs() @ c.abs().t().contiguous()).max()))
    lse = top + torch.log(total)
    off = (C + 16) * u * off + 2.0 ** -18
    terms = h + 2.0 ** -11 + 2 * off
    dx, size = torch.zeros_like(xs), torch.zeros_like(top)
    xn = xs.norm(dim=1)
    for v, c, z, mine in chunks():
        dz = torch.exp(z - lse[:, None])
        dz[mine, y[mine] - v] -= 1.0
        dz *= ws[:, None]
        dx += dz @ c
        slack = 2.0 ** -39 * ws[:, None]
        size += (dz.abs() + slack) @ c.norm(dim=1)
        dzt = dz.t().contiguous()
        rW, rs, rb = dzt @ xs, (dzt.abs() + slack.t()) @ xn, dz.sum(0)
        rbs = dz.abs().sum(0)
        sums = six * (n / 16 + 100) * u
        for what, _, dW, db, old in outs:
            got, ref = dW[v:v + CHUNK].double(), rW if old is None else rW + old
            err = (got - ref).norm(dim=1)
            bound = h * ref.norm(dim=1) + (terms + sums) * rs
            assert bool((err <= bound).all()), f"{what} dW, from class {v}"
            if db is not None:
                ref = rb if old is None else rb + old
                err = (db[v:v + CHUNK].double() - ref).abs()
                bound = (2 * off + (n + 100) * u) * rbs + 2 * u * ref.abs()
                assert bool((err <= bound).all()), f"{what} db, from class {v}"
    rest = labels < 0
    for what, got, _, _, _ in outs:
        if got is None:
            continue
        assert not bool(got[rest].any()), what
        err = (got[rows].double() - dx).norm(dim=1)
        bound = h * dx.norm(dim=1) + (terms + six * (V / 16 + 100) * u) * size
        assert bool((err <= bound).all()), (what, rows[err > bound].tolist())
    return lse, rows


@pytest.mark.parametrize("live", [300, 270, 256, 200, 0])
@pytest.mark.parametrize("C,dtype", [
    (16, "bf16"), (256, "bf16"), (768, "bf16"),   # logits again, exponentials, with db logits
    (16, "f32"), (128, "f32"),                    # logits again, logits
])
def test_pieces(C, dtype, live):
    n, V = 300, 1 << 22 if dtype == "bf16" else (1 << 20) + 8   # 256 rows to a piece
    x, W, labels, w = inputs(n, C, V, dtype, live, C + live)
    ws = torch.empty(shc.linear_cross_entropy_workspace(
        n, C, V, shc.SHC_BF16 if dtype == "bf16" else shc.SHC_F32), dtype=torch.uint8,
        device="cuda")
    ws.fill_(0xFF)  # NaN, whatever type is read
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    shc.linear_cross_entropy(x, W, labels, loss=loss, lse=lse, ws=ws)
    outs = []
    for what in ("step", "step without db", "step added", "backward"):
        added = what == "step added"
        dx = None if added else torch.full_like(x, 7.0)
        dW = torch.full_like(W, 0.25 if added else float("nan"))
        db = (None if what == "step without db" else
              torch.full((V,), 0.25 if added else float("nan"), device="cuda"))
        kw = dict(row_weight=w, dx=dx, dW=dW, db=db, accumulate=added, ws=ws)
        if what == "backward":
            shc.linear_cross_entropy_backward(x, W, labels, lse, **kw)
        else:
            again = shc.linear_cross_entropy_step(x, W, labels, **kw)
            assert float((again - loss).abs().max()) <= 1e-5
        outs.append((what, dx, dW, db, 0.25 if added else None))
    ref, rows = check_chunks(x, W, labels, w, outs)
    assert bool(((lse[rows] - ref).abs() <= 1e-4).all())
    assert not bool(lse[labels < 0].any()) and not bool(loss[labels < 0].any())


@pytest.mark.parametrize("n", [1, 7, 40, 64])
@pytest.mark.parametrize("C,V", [(72, 1000), (264, 333), (128, 5000)])
def test_few_rows_added(n, C, V):
    """Up to 64 rows of bf16, whose dz is two terms, with accumulate."""
    c = Case(n, C, V, 0.2 if n > 1 else 0.0, 0, 0, "bf16", seed=5)
    ids, w, bias = c.ids(), f32(c.w), f32(c.b)
    ref = c.oracle()
    b = xent_bounds(c.x.get(), c.W.get(), wide(c.b), ref, wide(c.w), "bf16")
    lse = torch.empty(n, device="cuda")
    shc.linear_cross_entropy(c.x.t, c.W.t, ids, bias, lse=lse)
    for step in (True, False):
        for with_db in (True, False):
            dW, db = c.rows(V, C), Rows(1, V, "f32", values=c.r.standard_normal((1, V)))
            dx = c.out(n, C)
            rW, rb = ref["dW"] + dW.get(), ref["db"] + db.get()[0]
            kw = dict(dx=dx.t, dW=dW.t, db=db.t[0] if with_db else None, accumulate=True)
            if step:
                shc.linear_cross_entropy_step(c.x.t, c.W.t, ids, w, bias, **kw)
            else:
                shc.linear_cross_entropy_backward(c.x.t, c.W.t, ids, lse, w, bias, **kw)
            close(dx.get(), ref["dx"], rounded(b["dx"], ref["dx"], "bf16"), "dx")
            close(dW.get(), rW, rounded(b["dW"] + 2.0 ** -24 * np.abs(rW), rW, "bf16"), "dW")
            if with_db:
                close(db.get()[0], rb, rounded(b["db"] + 2.0 ** -24 * np.abs(rb), rb, "f32"), "db")
