"""What LabelHead says of a step: its gradients' norm without an active row."""
import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_label_head import setup

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
