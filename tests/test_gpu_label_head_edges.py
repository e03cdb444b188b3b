"""What LabelHead says of a step: its gradients' norm without an active row, and the mean loss
over the rows that have a label."""
import pytest
import torch

from paper_2608_09388_amd import label_head
from tests.gpu_util import require_gpu
from tests.test_gpu_label_head import reference, setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def test_norm_of_no_active_row():
    head, x, n, labels = setup()
    head.norm.fill_(float("nan"))  # what fresh memory may hold
    loss = head.backward(labels[:0], 0)
    assert loss.numel() == 0 and float(head.norm) == 0.0
    head.forward(x, n)
    head.backward(labels, n)
    assert float(head.norm) > 0.0
    head.backward(labels[:0], 0)
    assert float(head.norm) == 0.0


def test_mean_loss_is_over_the_labelled_rows():
    head, x, n, labels = setup()
    head.forward(x, n)
    loss = head.backward(labels, n)
    live = (labels >= 0) & (labels < head.classes)
    assert 0 < int(live.sum()) < n
    mean, _, _ = reference(head, x, n, labels)
    assert abs(float(head.mean_loss(loss)) - float(mean)) <= 1e-5 * float(mean)
    loss = head.backward(torch.full_like(labels, -1), n)
    assert float(head.mean_loss(loss)) == 0.0
    loss = head.backward(labels[:0], 0)
    assert float(head.mean_loss(loss)) == 0.0


@pytest.mark.parametrize("classes", [1, 40])
def test_command_prints_that_mean(classes, monkeypatch, capsys):
    """One class: every labelled row's loss is 0; many: about the logarithm of their number, as
    the first step's logits are of the order of 1."""
    monkeypatch.setattr("sys.argv", ["label_head", "--bodies", "3", "--vertices", "200", "--channels",
                                     "64", "--hidden", "32", "--classes", str(classes), "--steps",
                                     "1"])
    seen = []
    step = label_head.LabelHead.step

    def watched(self, x, mask, labels, lr):
        loss = step(self, x, mask, labels, lr)
        y = labels(self.coords[:loss.numel()])
        live = (y >= 0) & (y < self.classes)
        assert int(live.sum()) < loss.numel()
        seen.append(float(loss[live].double().mean()))
        return loss

    monkeypatch.setattr(label_head.LabelHead, "step", watched)
    label_head.main()
    printed = float(capsys.readouterr().out.split("mean loss ")[1].split(",")[0])
    assert abs(printed - seen[0]) <= 1e-4
