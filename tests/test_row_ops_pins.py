"""Pins of the row operators' oracle: library routines that reach the same
values by another route, closed forms, and every gradient against central
differences of its forward."""
import numpy as np
import pytest
import torch

from oracle import row_oracle as O


def rng(seed):
    return np.random.default_rng(seed)


def test_embed_against_torch():
    r = rng(1)
    E, ids = r.standard_normal((13, 5)), r.integers(0, 13, 29)
    want = torch.nn.functional.embedding(torch.from_numpy(ids), torch.from_numpy(E)).numpy() * 2.5
    assert np.array_equal(O.embed(E, ids, 2.5), want)
    add = r.standard_normal((29, 5))
    assert np.array_equal(O.embed(E, ids, 2.5, add), want + add)


def test_embed_without_a_row():
    E = np.ones((3, 2))
    out = O.embed(E, [-1, 0, 3, 2], 4.0, np.full((4, 2), 0.5))
    assert out[:, 0].tolist() == [0.5, 4.5, 0.5, 4.5]


def test_embed_backward_against_torch():
    r = rng(2)
    ids = r.integers(0, 7, 40)
    E = torch.from_numpy(r.standard_normal((7, 3))).requires_grad_()
    dY = r.standard_normal((40, 3))
    (torch.nn.functional.embedding(torch.from_numpy(ids), E, padding_idx=4) * 1.5).backward(
        torch.from_numpy(dY))
    assert np.allclose(O.embed_backward(dY, ids, 7, 1.5, 4), E.grad.numpy(), rtol=1e-13)
    assert not O.embed_backward(dY, ids, 7, 1.5, 4)[4].any()
    assert not O.embed_backward(dY, np.full(40, 9), 7).any()


def test_layer_norm_against_torch():
    r = rng(3)
    x, g, b = r.standard_normal((6, 17)) + 3.0, r.standard_normal(17), r.standard_normal(17)
    want = torch.nn.functional.layer_norm(torch.from_numpy(x), (17,), torch.from_numpy(g),
                                          torch.from_numpy(b), 1e-5).numpy()
    y, mean, rstd = O.layer_norm(x, g, b)
    assert np.allclose(y, want, rtol=1e-12, atol=1e-13)
    assert np.allclose(mean, x.mean(1)) and np.allclose(rstd, 1 / np.sqrt(x.var(1) + 1e-5))


def test_layer_norm_of_one_channel():
    y, mean, rstd = O.layer_norm(np.array([[7.0], [-2.0]]), np.array([3.0]), np.array([0.25]))
    assert y.tolist() == [[0.25], [0.25]] and mean.tolist() == [7.0, -2.0]
    assert np.allclose(rstd, 1e5 ** 0.5)


def differences(f, a, h=1e-5):
    """Central differences of the scalar f at a."""
    g = np.zeros_like(a)
    flat, out = a.reshape(-1), g.reshape(-1)
    for i in range(flat.size):
        keep = flat[i]
        flat[i] = keep + h
        up = f()
        flat[i] = keep - h
        out[i] = (up - f()) / (2 * h)
        flat[i] = keep
    return g


def test_layer_norm_backward_by_differences():
    r = rng(4)
    x, dy = r.standard_normal((3, 6)) * 2 + 1, r.standard_normal((3, 6))
    g, b = r.standard_normal(6), r.standard_normal(6)

    def f():
        return float((O.layer_norm(x, g, b)[0] * dy).sum())

    _, mean, rstd = O.layer_norm(x, g, b)
    dx, dg, db = O.layer_norm_backward(dy, x, g, mean, rstd)
    for got, a in ((dx, x), (dg, g), (db, b)):
        assert np.allclose(got, differences(f, a), rtol=1e-7, atol=1e-8)


def test_embed_backward_by_differences():
    r = rng(5)
    E, ids, dY = r.standard_normal((4, 3)), np.array([2, 0, 2, -1, 9]), r.standard_normal((5, 3))

    def f():
        return float((O.embed(E, ids, 0.75) * dY).sum())

    assert np.allclose(O.embed_backward(dY, ids, 4, 0.75), differences(f, E), atol=1e-9)


@pytest.mark.parametrize("T", [1.0, 2.0, 0.5])
def test_distill_of_a_whole_teacher_is_kl(T):
    """With every id present the loss is T^2 KL(teacher || student)."""
    r = rng(6)
    z, t = r.standard_normal((4, 9)), r.standard_normal((4, 9))
    ids = np.stack([r.permutation(9) for _ in range(4)])
    loss, lse, _ = O.distill(z, ids, np.take_along_axis(t, ids, 1), T)
    want = torch.nn.functional.kl_div(
        torch.log_softmax(torch.from_numpy(z) / T, 1), torch.log_softmax(torch.from_numpy(t) / T, 1),
        reduction="none", log_target=True).sum(1).numpy() * T * T
    assert np.allclose(loss, want, rtol=1e-11, atol=1e-13)
    assert np.allclose(lse, torch.logsumexp(torch.from_numpy(z) / T, 1).numpy())


def test_distill_of_one_entry_is_cross_entropy():
    r = rng(7)
    z, ids = r.standard_normal((5, 11)), r.integers(0, 11, (5, 1))
    loss, _, dz = O.distill(z, ids, r.standard_normal((5, 1)), 1.0)
    want = torch.nn.functional.cross_entropy(torch.from_numpy(z), torch.from_numpy(ids[:, 0]),
                                             reduction="none").numpy()
    assert np.allclose(loss, want, rtol=1e-12)
    q = torch.softmax(torch.from_numpy(z), 1).numpy()
    q[np.arange(5), ids[:, 0]] -= 1
    assert np.allclose(dz, q, atol=1e-14)


@pytest.mark.parametrize("T", [1.0, 3.0])
def test_distill_gradient_by_differences(T):
    r = rng(8)
    z = r.standard_normal((3, 7))
    ids = np.array([[1, 4, 1], [6, -1, 0], [-1, 8, -1]])     # repeated, absent, none
    top, w = r.standard_normal((3, 3)), np.array([0.5, 2.0, 1.0])

    def f():
        return float((O.distill(z, ids, top, T)[0] * w).sum())

    assert np.allclose(O.distill(z, ids, top, T, w)[2], differences(f, z), rtol=1e-7, atol=1e-8)


def test_distill_masks():
    inf = np.inf
    z = np.array([[0.0, -inf, 1.0], [-inf, -inf, -inf], [5.0, 5.0, 5.0]])
    ids = np.array([[0, 2], [0, 2], [-1, 3]])
    loss, lse, dz = O.distill(z, ids, np.array([[0.0, -inf], [1.0, 1.0], [1.0, 1.0]]), 1.0)
    assert np.isclose(loss[0], np.log(1 + np.e)) and loss[1] == inf and loss[2] == 0
    assert lse[1] == -inf and lse[2] == 0
    assert dz[1].tolist() == [-0.5, 0.0, -0.5] and not dz[2].any()
    assert dz[0, 1] == 0.0 and np.isclose(dz[0].sum(), 0.0)
