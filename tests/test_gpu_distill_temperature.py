"""Temperatures of distill_loss and distill_grad: those whose square is no normal number are refused, near the
ends of the others the results are numbers."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import DominoError  # noqa: E402
from test_gpu_distill import d, inputs  # noqa: E402,F401


@pytest.mark.parametrize("tau", [3.5e-39, 1e-30, 1e-19, 2e19, 1e38])
def test_refused(d, tau):  # noqa: F811
    """log2(e) / tau overflows (the first), tau^2 overflows, or it loses the loss's bits."""
    x, t, ids, _, c = inputs(4, 100, 5)
    with pytest.raises(DominoError) as e:
        d.distill_loss(x, t, ids, tau)
    assert e.value.status == -1
    with pytest.raises(DominoError) as e:
        d.distill_grad(x, t, ids, tau, torch.zeros(4, device="cuda"), c)
    assert e.value.status == -1


@pytest.mark.parametrize("tau", [1.1e-19, 1.8e18])
def test_ends_of_the_range(d, tau):  # noqa: F811
    x, t, ids, _, c = inputs(4, 100, 5)
    loss, lse = d.distill_loss(x, t, ids, tau)
    dx = d.distill_grad(x, t, ids, tau, lse, c)
    for out in (loss, lse, dx):
        assert torch.isfinite(out).all()
