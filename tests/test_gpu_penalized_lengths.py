"""Lengths beside a history of no places: those that are not 0 are out of range, as beside any other history."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from test_gpu_norm import d  # noqa: E402,F401


@pytest.mark.parametrize("history", [False, True])
@pytest.mark.parametrize("lengths,bad", [((0, 0, 0), False), ((0, 1, 0), True), ((0, 0, -1), True), ((2 ** 31 - 1, 0, 0), True)])
def test_lengths_without_places(d, history, lengths, bad):  # noqa: F811
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(3, 700, generator=g, device="cuda")
    k = {"repetition": torch.full((3,), 1.5, device="cuda"), "bias_ids": torch.tensor([[5], [6], [-1]], dtype=torch.int32, device="cuda"),
         "bias_values": torch.full((3, 1), 2.0, device="cuda")}
    want = d.mask_logits_penalized(x, want_logprobs=True, **k)
    drawn = d.mask_sample_penalized(x, 0.9, 1, 2, **k)
    assert d.device_error() == 0
    k["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if history:
        k["history"] = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    got = d.mask_logits_penalized(x, want_logprobs=True, **k)
    assert d.device_error() == (B.DEVERR_BAD_TOKEN if bad else 0)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(d.mask_sample_penalized(x, 0.9, 1, 2, **k), drawn)
    assert d.device_error() == (B.DEVERR_BAD_TOKEN if bad else 0)
