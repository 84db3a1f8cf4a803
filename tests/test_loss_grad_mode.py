"""Autograd does not see the losses and the embedding: tensors that require a gradient are refused rather than taken for
constants (without a GPU: before anything else about the first tensor is checked)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino  # noqa: E402
from paper_2403_06988_gb300 import build as build_mod  # noqa: E402


@pytest.fixture(scope="module")
def calls():
    build_mod.build()
    d = Domino(-1)
    h, w, x = torch.zeros(3, 8), torch.zeros(4, 8), torch.zeros(3, 4)
    y, ids, f = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3)
    teacher = torch.zeros(3, 2)
    yield [(d.token_loss, (h, w, y), h), (d.token_loss_grad, (h, w, y, f, f), h), (d.distill_loss, (x, teacher, ids), x),
           (d.distill_grad, (x, teacher, ids, 1.0, f, f), x), (d.embed_grad, (y, h, 4), h)]
    d.close()


def test_refused_in_grad_mode_alone(calls):
    for call, args, over in calls:
        over.requires_grad_()
        with pytest.raises(RuntimeError, match="requires a gradient"):
            call(*args)
        with torch.no_grad(), pytest.raises(ValueError, match="device"):    # host tensors: the next check
            call(*args)
        over.requires_grad_(False)
        with pytest.raises(ValueError, match="device"):
            call(*args)
