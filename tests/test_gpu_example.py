"""examples/train_draft.py: the losses, their gradients and the embedding as a training program uses them together."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_and_distilling():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2403_06988_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("train_draft", os.path.join(ROOT, "examples", "train_draft.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, divergences, before, after = m.run(steps=30, batch=16, length=24)
    assert all(map(math.isfinite, losses + divergences))
    assert losses[-1] < losses[0] and divergences[-1] < divergences[0]
    assert min(divergences) >= -1e-3          # a divergence, to the rounding of its fp32 terms
    assert after > before
