"""Tensors that require a gradient."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_token_loss import d, inputs  # noqa: E402,F401


def test_refused_where_autograd_would_lose_them(d):  # noqa: F811
    h, w, y, mask, c = inputs(8, 100, 24, density=0.5)
    w.requires_grad_()
    with pytest.raises(RuntimeError):
        d.token_loss(h, w, y, mask)
    with torch.no_grad():
        want = d.token_loss(h, w, y, mask)
    got = d.token_loss(h, w.detach(), y, mask)
    assert torch.equal(got[0], want[0])
    with pytest.raises(RuntimeError):
        d.embed(y.clamp(min=0), w)
    with pytest.raises(RuntimeError):
        d.token_loss_grad(h, w, y, want[1], c, mask)
