"""Masks are words of 32 bits: tensors of another type are refused, whatever their size."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_token_loss import d, inputs  # noqa: E402,F401


def test_a_mask_of_floats_is_refused(d):  # noqa: F811
    h, w, y, mask, c = inputs(8, 100, 24, density=0.5)
    loss, lse = d.token_loss(h, w, y, mask)
    bits = mask.view(torch.uint32)
    assert torch.equal(d.token_loss(h, w, y, bits)[1], lse)
    logits = (h.float() @ w.float().T).contiguous()
    ids = logits.topk(3, dim=1).indices.int()
    for bad in (mask.float(), mask.view(torch.float32)):
        with pytest.raises(TypeError):
            d.token_loss(h, w, y, bad)
        with pytest.raises(TypeError):
            d.token_loss_grad(h, w, y, lse, c, bad)
        with pytest.raises(TypeError):
            d.distill_loss(logits, logits[:, :3].contiguous(), ids, 1.0, bad)
