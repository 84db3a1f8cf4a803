"""Numbers of rows whose tiles or chunks would pass 32 bits are refused before anything is launched."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from test_gpu_token_loss import d  # noqa: E402,F401

MOST = 2 ** 31 - 2 ** 20 - 1


@pytest.mark.parametrize("n", [MOST + 1, 2 ** 31 - 1])
def test_rows_beyond_the_limit_are_refused(d, n):  # noqa: F811
    x = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(64, dtype=torch.int32, device="cuda")
    f = torch.zeros(64, device="cuda")
    calls = [lambda: B.domino_embed_grad(d.h, t, n, x, 1, B.DTYPE_BF16, 4, 1, 1.0, 0, x, 1),
             lambda: B.domino_token_loss(d.h, x, 1, x, 1, B.DTYPE_BF16, n, 1, 4, None, t, f),
             lambda: B.domino_token_loss_grad(d.h, x, 1, x, 1, B.DTYPE_BF16, n, 1, 4, None, t, f, f, x, 1, x, 1)]
    for call in calls:
        with pytest.raises(DominoError) as e:
            call()
        assert e.value.status == -3
