"""The norm of many gradients and their clipping against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import dense_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu
from tests.row_util import TDT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def make(sizes, seed=0, scale=1.0, off=0):
    r = np.random.default_rng(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = TDT["bf16" if (i + seed) % 2 else "f32"]
        buf = torch.as_tensor(r.standard_normal(n + off) * scale, device="cuda").to(dt)
        out.append(buf[off:])
    return out


def check(grads, outs, most):
    """u = 2^-24: the norm is rounded once from fp64, the factor's quotient and the product
    once each, a bf16 output once more (2^-8)."""
    norm, ref = O.clip([g.double().cpu().numpy() for g in grads], most)
    got = shc.grad_norm(grads)
    assert abs(float(got) - norm) <= 2.0 ** -23 * norm
    before = [g.clone() for g in grads]
    shc.clip_grads(grads, got, most, outs)
    for g, b, o, want in zip(grads, before, outs or grads, ref):
        if outs is not None:
            assert torch.equal(g, b)
        err = (2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0) + 4 * 2.0 ** -24
        o = o.double().cpu().numpy()
        assert np.all(np.abs(o - want) <= err * np.abs(want) + 2.0 ** -133)
        if norm <= most:
            assert np.array_equal(o, b.double().cpu().numpy())


SETS = [[1], [0, 7, 0], [3, 5, 8, 1000], [2047, 2048, 2049], [70001, 1, 300000],
        [17] * 127, [17] * 128, [17] * 129, list(range(300)), [3000000, 40]]


@pytest.mark.parametrize("sizes", SETS, ids=[f"{len(s)}x{max(s)}" for s in SETS])
@pytest.mark.parametrize("off", [0, 1])
def test_sets(sizes, off):
    for most in (0.01, 1e9):
        grads = make(sizes, len(sizes), 0.5, off)
        check(grads, None, most)
        grads = make(sizes, len(sizes), 0.5, off)
        check(grads, [torch.empty_like(g) for g in grads], most)


def test_nothing():
    assert float(shc.grad_norm([])) == 0.0
    shc.clip_grads([], torch.ones(1, device="cuda"), 1.0)
    z = [torch.zeros(100, device="cuda"), torch.zeros(0, device="cuda")]
    n = shc.grad_norm(z)
    shc.clip_grads(z, n, 0.0)
    assert float(n) == 0.0 and not bool(z[0].any())


def test_range():
    """Squares beyond fp32 and below it."""
    for scale in (1e30, 1e-30, 2.0 ** -140):
        g = [torch.full((1000,), scale, device="cuda"), torch.full((24,), scale, device="cuda")]
        want = math.sqrt(1024) * float(g[0][0].double())
        assert abs(float(shc.grad_norm(g)) - want) <= 2.0 ** -23 * want + 2.0 ** -149
    g = [torch.full((100,), 3e38, device="cuda")]
    n = shc.grad_norm(g)
    assert math.isinf(float(n))
    shc.clip_grads(g, n, 1.0)
    assert not bool(g[0].any())


def test_not_finite():
    g = [torch.ones(10, device="cuda"), torch.ones(70000, device="cuda")]
    g[1][69999] = float("inf")
    n = shc.grad_norm(g)
    out = [torch.empty_like(t) for t in g]
    shc.clip_grads(g, n, 1.0, out)
    assert math.isinf(float(n)) and not bool(out[0].any())
    assert bool(torch.isnan(out[1][69999])) and not bool(out[1][:69999].any())
    g[0][3] = float("nan")
    n = shc.grad_norm(g)
    shc.clip_grads(g, n, 1.0, out)
    assert math.isnan(float(n)) and all(bool(torch.isnan(o).all()) for o in out)


def test_max_norm_of_infinity_and_the_norm_itself():
    g = make([1000, 77])
    keep = [t.clone() for t in g]
    n = shc.grad_norm(g)
    for most in (float("inf"), float(n)):
        shc.clip_grads(g, n, most)
        assert all(torch.equal(a, b) for a, b in zip(g, keep))


def test_overlaps_are_refused():
    buf = torch.zeros(100, device="cuda")
    n = torch.ones(1, device="cuda")
    for grads, outs in (([buf[:60], buf[50:]], None), ([buf[:50]], [buf[1:51]]),
                        ([buf[:50], buf[50:]], [buf[50:], buf[:50]]), ([buf, buf], None),
                        ([buf[:10], buf[20:30]], [buf[40:50], buf[45:55]])):
        with pytest.raises(shc.ShcError, match="overlaps"):
            shc.clip_grads(grads, n, 1.0, outs)
    shc.clip_grads([buf[:50], buf[50:]], n, 1.0)
    twice = shc.grad_norm([n, n])
    assert abs(float(twice) - math.sqrt(2.0)) < 1e-6


def test_repeats_bit_for_bit():
    g = make([300000, 5, 123457], 4)
    a = shc.grad_norm(g)
    assert all(torch.equal(a, shc.grad_norm(g)) for _ in range(5))


def test_refusals():
    f = dict(device="cuda")
    n = torch.ones(1, **f)
    with pytest.raises(ValueError, match="contiguous"):
        shc.grad_norm([torch.ones((4, 4), **f).t()])
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        shc.grad_norm([torch.ones(4, **f).half()])
    with pytest.raises(ValueError, match="on the GPU"):
        shc.grad_norm([torch.ones(4)], norm=n)
    with pytest.raises(ValueError, match="outputs"):
        shc.clip_grads([n], n, 1.0, [])
    with pytest.raises(TypeError, match=r"outs\[0\]"):
        shc.clip_grads([torch.ones(4, **f)], n, 1.0, [torch.ones(4, **f).bfloat16()])
    with pytest.raises(ValueError, match="elements"):
        shc.clip_grads([torch.ones(4, **f)], n, 1.0, [torch.ones(5, **f)])
    for bad in (-1.0, float("nan")):
        with pytest.raises(shc.ShcError, match="max_norm"):
            shc.clip_grads([torch.ones(4, **f)], n, bad)
