"""Outputs that the losses and the embedding make and that do not fit into memory."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_token_loss import d  # noqa: E402,F401


def test_out_of_memory_is_torchs(d, monkeypatch):  # noqa: F811
    """35 TB: the allocator refuses at once."""
    monkeypatch.setattr(type(d), "fill_byte", None)
    grad = torch.zeros(1, 1 << 20, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        d.embed_grad(torch.zeros(1, dtype=torch.int32, device="cuda"), grad, 1 << 24)
