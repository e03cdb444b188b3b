"""The dense operators in a network's training step (LabelHead): its gradients against
autograd in 64 bits and against differences, and its edges."""
import numpy as np
import pytest
import torch

from paper_2608_09388_amd.label_head import LabelHead
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu
F = torch.nn.functional


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def setup(B=5, V=97, C=64, hidden=200, classes=331, blocks=2, dtype="f32", seed=3, p=0.3,
          max_norm=float("inf")):
    head = LabelHead(B, V, C, hidden, classes, blocks, max_norm, dtype, seed)
    r = np.random.default_rng(seed)
    x = torch.as_tensor(r.standard_normal((B * V, C)), device="cuda").to(head.S.dtype)
    mask = torch.as_tensor((r.random(B * V) < p).astype(np.uint8), device="cuda")
    n = head.compact(mask)
    labels = torch.as_tensor(r.integers(-60, classes + 20, max(n, 1)), device="cuda")[:n]
    return head, x, n, labels


def reference(head, x, n, labels):
    """(mean loss over the labelled rows, losses, gradients) in fp64 by autograd, the matrices
    as the layers read them."""
    p = {k: (head.weights[k] if k in head.weights else v).double().requires_grad_()
         for k, v in head.params.items()}
    at = head.coords[:n].long()
    h = x.double()[at[:, 0] * head.V + at[:, 1]] + head.scale * p["E"][at[:, 1]]
    y = F.layer_norm(h, (head.C,), p["gamma"], p["beta"], 1e-5)
    for k in range(head.blocks):
        y = y + F.gelu(y @ p[f"W1.{k}"] + p[f"b1.{k}"]) @ p[f"W2.{k}"] + p[f"b2.{k}"]
    live = (labels >= 0) & (labels < head.classes)
    losses = F.cross_entropy(y @ p["T"].t(), torch.where(live, labels, -100), reduction="none")
    mean = losses.sum() / live.sum()
    grads = dict(zip(p, torch.autograd.grad(mean, p.values())))
    return mean.detach(), losses.detach(), grads


def test_gradients_against_autograd():
    """fp32: a chain of seven products, each off by 1e-6 of its sums' magnitudes at most."""
    head, x, n, labels = setup()
    head.forward(x, n)
    only = head.losses(labels, n).clone()
    loss = head.backward(labels, n)
    assert torch.equal(only, loss)
    _, losses, want = reference(head, x, n, labels)
    assert float((loss - losses).abs().max()) <= 1e-5 * float(losses.abs().max())
    assert not bool(loss[(labels < 0) | (labels >= head.classes)].any())
    for k, w in want.items():
        err = float((head.grads[k] - w).abs().max())
        assert err <= 2e-5 * float(w.abs().max()), (k, err)
    norm = float(torch.sqrt(sum((w ** 2).sum() for w in want.values())))
    assert abs(float(head.norm) - norm) <= 1e-5 * norm


def test_gradients_in_bf16():
    """bf16: rows are rounded by 2^-8 at nine places on the way there and as many back, with
    independent signs (their root, 4.3, and as much for the sums of rounded rows); in the
    2-norm the figure is below 12 * 2^-8."""
    head, x, n, labels = setup(dtype="bf16", p=0.6)
    head.forward(x, n)
    head.backward(labels, n)
    _, _, want = reference(head, x, n, labels)
    for k, w in want.items():
        err = float((head.grads[k] - w).norm() / w.norm())
        assert err <= 12 * 2.0 ** -8, (k, err)


def test_gradients_against_differences():
    """Along a random direction of every parameter, the fp64 network's loss as the measure."""
    head, x, n, labels = setup(blocks=1, p=0.2)
    head.forward(x, n)
    head.backward(labels, n)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    for k, v in head.params.items():
        d = torch.randn(v.shape, generator=g, device="cuda")
        along = float((head.grads[k].double() * d.double()).sum())
        keep, side, h = v.clone(), [], 2.0 ** -10
        for s in (h, -h):
            v.copy_(keep + s * d)
            step = (v.double() - keep.double())
            head._refresh()
            side.append((float(reference(head, x, n, labels)[0]),
                         float((step * d.double()).sum() / (d.double() ** 2).sum())))
        v.copy_(keep)
        head._refresh()
        diff = (side[0][0] - side[1][0]) / (side[0][1] - side[1][1])
        size = float(head.grads[k].double().norm() * d.double().norm())
        assert abs(diff - along) <= 2e-3 * size, k


def test_clipping():
    head, x, n, labels = setup(max_norm=1e-3)
    head.forward(x, n)
    head.backward(labels, n)
    norm = torch.sqrt(sum((g.double() ** 2).sum() for g in head.grads.values()))
    assert float(head.norm) > 1e-3 and abs(float(norm) - 1e-3) <= 1e-8


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_run(dtype):
    head, x, n, labels = setup(dtype=dtype, max_norm=1.0)
    mask = torch.ones(head.B * head.V, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        loss = head.step(x, mask, lambda c: c[:, 1].long(), 0.1)
        assert loss.numel() == head.B * head.V and bool(torch.isfinite(loss).all())
    assert all(bool(torch.isfinite(v).all()) for v in head.params.values())


def test_no_active_row_and_no_label():
    head, x, n, labels = setup(p=0.0)
    assert n == 0 and head.forward(x, 0).shape[0] == 0
    assert head.backward(labels, 0).numel() == 0
    head, x, n, labels = setup()
    head.forward(x, n)
    loss = head.backward(torch.full_like(labels, -1), n)
    assert not bool(loss.any()) and float(head.norm) == 0.0
    assert not any(bool(g.any()) for g in head.grads.values())
