"""The losses' and the embedding's entry points without a GPU: arguments are checked, host-only handles refuse."""
import pytest

from paper_2403_06988_gb300 import _binding as B
from paper_2403_06988_gb300 import build as build_mod

CALLS = {
    "domino_token_loss": (64, 8, 64, 8, 1, 4, 8, 100, None, 64, 64),
    "domino_token_loss_grad": (64, 8, 64, 8, 1, 4, 8, 100, None, 64, 64, 64, 64, 8, 64, 8),
    "domino_distill_loss": (64, 1, 4, 100, 100, None, 64, 0, 64, 5, 1.0, 64),
    "domino_distill_grad": (64, 1, 4, 100, 100, None, 64, 0, 64, 5, 1.0, 64, 64, 128, 100),
    "domino_embed": (64, 4, 64, 8, 1, 100, 8, 1.0, 64, 8),
    "domino_embed_grad": (64, 4, 64, 8, 1, 100, 8, 1.0, 0, 64, 8),
}


@pytest.fixture(scope="module")
def host_handle():
    build_mod.build()
    h = B.domino_create(-1)
    yield h
    B.domino_destroy(h)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_host_handle_refuses(host_handle, name):
    with pytest.raises(B.DominoError) as e:
        getattr(B, name)(host_handle, *CALLS[name], stream=0)
    assert e.value.status == -6


@pytest.mark.parametrize("name", sorted(CALLS))
def test_no_handle(host_handle, name):
    with pytest.raises(B.DominoError) as e:
        getattr(B, name)(None, *CALLS[name], stream=0)
    assert e.value.status == -1


def test_python_calls_refuse_without_a_device(host_handle):
    """The extension that Domino's methods go through loads without a GPU; host tensors and bad arguments are refused."""
    torch = pytest.importorskip("torch")
    from paper_2403_06988_gb300 import Domino
    d = Domino(-1)
    w, t = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        d.embed(t, w)
    with pytest.raises(ValueError):
        d.token_loss(w, w, t)
    with pytest.raises(TypeError):
        d.embed(3, w)
    with pytest.raises(TypeError):
        d.embed_grad(t, None, 4)
    d.close()
