"""The dense operators' oracle against PyTorch's functions and autograd in fp64 and
against difference quotients (CPU)."""
import numpy as np
import pytest
import torch

from oracle import dense_oracle as O

F = torch.nn.functional
ACTS = {O.NONE: lambda z: z, O.RELU: F.relu, O.GELU: F.gelu, O.SILU: F.silu}


@pytest.mark.parametrize("code", sorted(ACTS))
def test_linear(code):
    r = np.random.default_rng(code)
    x, W, b, res, dout = (r.standard_normal(s) for s in ((7, 5), (5, 6), 6, (7, 6), (7, 6)))
    tx, tW, tb, tr = (torch.tensor(a, requires_grad=True) for a in (x, W, b, res))
    z = tx @ tW + tb
    out = ACTS[code](z) + tr
    got, pre = O.linear(x, W, b, code, res)
    assert np.allclose(got, out.detach().numpy(), rtol=1e-12, atol=1e-13)
    assert np.allclose(pre, z.detach().numpy(), rtol=1e-12, atol=1e-13)
    out.backward(torch.tensor(dout))
    dx, dW, db, _ = O.linear_backward(dout, x, W, pre, code)
    for a, t in ((dx, tx), (dW, tW), (db, tb), (dout, tr)):
        assert np.allclose(a, t.grad.numpy(), rtol=1e-11, atol=1e-12)


@pytest.mark.parametrize("code", sorted(ACTS))
def test_linear_differences(code):
    r = np.random.default_rng(10 + code)
    x, W, b, dout = (r.standard_normal(s) for s in ((4, 3), (3, 5), 5, (4, 5)))
    _, pre = O.linear(x, W, b, code)
    dx, dW, db, _ = O.linear_backward(dout, x, W, pre, code)
    h = 1e-6
    for a, grad in ((x, dx), (W, dW), (b, db)):
        i = tuple(r.integers(0, s) for s in a.shape)
        was, side = a[i], []
        for step in (h, -h):
            a[i] = was + step
            side.append((O.linear(x, W, b, code)[0] * dout).sum())
        a[i] = was
        assert abs((side[0] - side[1]) / (2 * h) - grad[i]) < 1e-6 * (1 + abs(grad[i]))


def test_cross_entropy():
    r = np.random.default_rng(0)
    x, W, b, w = (r.standard_normal(s) for s in ((9, 4), (11, 4), 11, 9))
    labels = r.integers(0, 11, 9)
    labels[[1, 5]] = -100
    tx, tW, tb = (torch.tensor(a, requires_grad=True) for a in (x, W, b))
    loss = F.cross_entropy(tx @ tW.t() + tb, torch.tensor(labels), reduction="none")
    (loss * torch.tensor(w)).sum().backward()
    ref = O.cross_entropy(x, W, labels, b, w)
    assert np.allclose(ref["loss"], loss.detach().numpy(), rtol=1e-12, atol=1e-13)
    assert np.all(ref["loss"][[1, 5]] == 0) and np.all(ref["lse"][[1, 5]] == 0)
    for k, t in (("dx", tx), ("dW", tW), ("db", tb)):
        assert np.allclose(ref[k], t.grad.numpy(), rtol=1e-11, atol=1e-13), k


def test_cross_entropy_of_masked_classes():
    r = np.random.default_rng(1)
    x, W = r.standard_normal((3, 4)), r.standard_normal((6, 4))
    b = np.zeros(6)
    b[[1, 4]] = -np.inf
    ref = O.cross_entropy(x, W, [0, 1, 5], b)
    assert np.isfinite(ref["loss"][[0, 2]]).all() and ref["loss"][1] == np.inf
    assert np.all(ref["q"][:, [1, 4]] == 0) and np.isfinite(ref["dW"]).all()
    ref = O.cross_entropy(x, W, [0, 1, 5], np.full(6, -np.inf))
    assert np.all(np.isneginf(ref["lse"])) and np.all(ref["q"] == 0)


def test_clip():
    r = np.random.default_rng(2)
    g = [r.standard_normal(s) for s in (5, (3, 4), 0)]
    t = [torch.tensor(a) for a in g]
    norm, out = O.clip(g, 0.5)
    assert np.isclose(norm, float(torch.linalg.vector_norm(torch.cat([a.reshape(-1) for a in t]))))
    assert np.isclose(np.sqrt(sum((a * a).sum() for a in out)), 0.5)
    assert all(np.array_equal(a, b) for a, b in zip(O.clip(g, norm)[1], g))
