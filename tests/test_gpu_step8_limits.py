"""The norm, 8-bit operands and the decode under penalties at the most tokens and at millions of short rows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from norm8_reference import Norm, assert_within, logits8  # noqa: E402
from test_gpu_logits8_rows import operands  # noqa: E402
from test_gpu_norm import check_codes, d, inputs  # noqa: E402,F401
from test_gpu_penalized import Case  # noqa: E402

MOST_TOKENS = 1 << 24


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_penalties_of_the_most_tokens(d, dtype):  # noqa: F811
    import oracle
    c = Case(2, MOST_TOKENS, 300, 20, dtype, seed=15, hot=False)
    c.check(d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args))
    x, m, _ = c.want()
    got = d.mask_sample_penalized(c.logits, 0.7, 11, 1 << 33, mask=c.mask, **c.args)
    assert (got.cpu().numpy() == oracle.mask_sample(x, m, 0.7, 11, 1 << 33)).all()


def test_logits_of_the_most_tokens(d):  # noqa: F811
    q, s, wq, ws = operands(3, MOST_TOKENS, 16)
    assert torch.equal(d.logits8(q, s, wq, ws).double(), logits8(q, s, wq, ws, torch.float32)[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_millions_of_rows(d, dtype):  # noqa: F811
    x, r, w, _, _ = inputs(3000001, 7, dtype)
    ref = Norm(x, w, r)
    y, h, rstd = d.norm(x, w, r)
    assert torch.equal(h, ref.sum)
    assert_within(rstd, ref.rstd, ref.tol["rstd"], "rstd")
    assert_within(y, ref.y, ref.tol["y"], "y")
    check_codes(*d.norm8(x, w, r)[:2], ref.y, ref.rel_y, 1, "norm8")
    check_codes(*d.quantize8(x), x.double(), 0.0, 1, "quantize8")
