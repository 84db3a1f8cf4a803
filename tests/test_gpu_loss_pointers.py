"""Pointers off their values' boundaries are refused before anything is launched; every pointer of every call in turn."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from test_gpu_token_loss import d  # noqa: E402,F401

# arguments after the handle: a letter is a pointer to values of its size (h: 2 bytes, w: 4)
CALLS = {
    "domino_token_loss": ("h", 8, "h", 8, 1, 4, 8, 100, "w", "w", "w", "w"),
    "domino_token_loss_grad": ("h", 8, "h", 8, 1, 4, 8, 100, "w", "w", "w", "w", "h", 8, "h", 8),
    "domino_distill_loss": ("h", 1, 4, 100, 100, "w", "w", 0, "w", 5, 1.0, "w", "w"),
    "domino_distill_grad": ("w", 0, 4, 100, 100, "w", "h", 1, "w", 5, 1.0, "w", "w", "w", 100),
    "domino_embed": ("w", 4, "h", 8, 1, 100, 8, 1.0, "h", 8),
    "domino_embed_grad": ("w", 4, "w", 8, 0, 100, 8, 1.0, 0, "w", 8),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_pointers_off_their_values(d, name):  # noqa: F811
    size = {"h": 2, "w": 4}
    spread = [torch.zeros(2000, device="cuda") for _ in CALLS[name]]
    plain = [x.data_ptr() if a in size else a for a, x in zip(CALLS[name], spread)]
    assert all(p % 4 == 0 for p, a in zip(plain, CALLS[name]) if a in size)
    for i, a in enumerate(CALLS[name]):
        for off in range(1, size.get(a, 1)):
            args = plain[:i] + [plain[i] + off] + plain[i + 1:]
            with pytest.raises(DominoError) as e:
                getattr(B, name)(d.h, *args)
            assert e.value.status == -1, (i, off)
    getattr(B, name)(d.h, *plain)
    torch.cuda.synchronize()
