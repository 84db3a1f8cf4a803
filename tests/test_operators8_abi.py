"""The entry points of the norm, of 8-bit operands and of the decode under penalties without a GPU: host-only handles refuse, and
so do the Python calls."""
import ctypes

import pytest

from paper_2403_06988_gb300 import _binding as B
from paper_2403_06988_gb300 import build as build_mod

CALLS = {
    "domino_norm": (64, 8, None, 0, 64, 1, 4, 8, 1e-6, 64, 8),
    "domino_norm8": (64, 8, None, 0, 64, 1, 4, 8, 1e-6, 64, 16, 64),
    "domino_norm_grad": (64, 8, 64, 64, 64, 8, None, 0, 1, 4, 8, 64, 8, 64),
    "domino_quantize8": (64, 8, 1, 4, 8, 1, 64, 16, 64),
    "domino_logits8": (64, 16, 64, 64, 16, 64, 4, 8, 100, 0, 64, 100),
    "domino_mask_logits_penalized": (64, 1, 4, 100, 100, B.penalties(), None, 64),
    "domino_mask_sample_penalized": (64, 1, 4, 100, 100, B.penalties(), None, 1.0, 0, 0, 64),
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


def test_penalties_layout():
    assert ctypes.sizeof(B.Penalties) == 72 and B.Penalties.history_len.offset == 64


def test_python_calls_refuse_without_a_device(host_handle):
    torch = pytest.importorskip("torch")
    from paper_2403_06988_gb300 import Domino
    d = Domino(-1)
    x, w, f = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4)
    q = torch.zeros(4, 16, dtype=torch.float8_e4m3fn)
    for call, args in ((d.norm, (x, w)), (d.norm8, (x, w)), (d.norm_grad, (x, w, f, x)), (d.quantize8, (x,)), (d.logits8, (q, f, q, f)),
                       (d.mask_logits_penalized, (x,)), (d.mask_sample_penalized, (x, 1.0, 0, 0))):
        with pytest.raises(ValueError, match="device"):
            call(*args)
        over = args[0]
        if over.dtype == torch.float32:
            over.requires_grad_()
            with pytest.raises(RuntimeError, match="requires a gradient"):
                call(*args)
            over.requires_grad_(False)
    with pytest.raises(TypeError):
        d.norm(3, w)
    with pytest.raises(TypeError):
        d.logits8(q, f, q, f, torch.float16)
    d.close()
