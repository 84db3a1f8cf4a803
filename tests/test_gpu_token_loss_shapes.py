"""domino_token_loss and domino_token_loss_grad in the tile shapes that large calls take, over several k blocks (64 values
each) and, above 24 of them, with the logits summed in parts: several tiles a CTA, odd and even numbers of parts, a last part
of one block, rows off 16-byte boundaries and off 128-byte lines, with and without masks."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_token_loss import check, d, inputs  # noqa: E402,F401


# an even number of 128-row tiles, or rows off 128-byte lines: pairs of CTAs
@pytest.mark.parametrize("T,V,D", [(256, 20001, 512), (777, 9003, 1000), (256, 20001, 1600), (512, 20001, 3200),
                                   (260, 20100, 1700), (300, 20001, 1601)])
@pytest.mark.parametrize("density", [None, 0.02, 0.7])
def test_pairs(d, T, V, D, density):  # noqa: F811
    check(d, *inputs(T, V, D, density=density), f"{T} x {V} x {D}")


# an odd number of row tiles, rows on 128-byte lines: 256 columns a CTA
@pytest.mark.parametrize("T,V,D", [(300, 20001, 640), (100, 20001, 1600), (300, 20001, 3136), (260, 20100, 3200)])
@pytest.mark.parametrize("density", [None, 0.02, 0.7])
def test_wide_tiles(d, T, V, D, density):  # noqa: F811
    check(d, *inputs(T, V, D, density=density), f"{T} x {V} x {D}")


# few tiles: 64 columns a CTA
@pytest.mark.parametrize("T,V,D", [(40, 9001, 1600), (5, 3000, 3136), (130, 2001, 4100)])
@pytest.mark.parametrize("density", [None, 0.02, 0.7])
def test_narrow_tiles_in_parts(d, T, V, D, density):  # noqa: F811
    check(d, *inputs(T, V, D, density=density), f"{T} x {V} x {D}")
