"""domino_logits8 of many rows: pairs of row tiles whose second is beyond the last row, several groups of row tiles, and logits
whose offsets pass 2^31 values; whole numbers, exactly."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from norm8_reference import logits8  # noqa: E402
from test_gpu_norm import TYPES, d  # noqa: E402,F401


def operands(T, V, D):
    """Codes -8 .. 8 and scales that are powers of two: every sum is a whole number of steps, in fp32 without a rounding."""
    g = torch.Generator("cuda").manual_seed(T + V + D)
    wide, nb = -(-D // 16) * 16, -(-D // 128)
    q, wq = (torch.randint(-8, 9, (n, wide), generator=g, device="cuda").float().to(torch.float8_e4m3fn)[:, :D] for n in (T, V))
    s, ws = (2.0 ** torch.randint(-3, 3, (n, nb), generator=g, device="cuda").float() for n in (T, -(-V // 128)))
    return q, s, wq, ws


# 17 row tiles in pairs; 36 in pairs, three groups of 16 in narrow tiles, two groups of pairs, the second short
SIZES = [(2100, 3001, 130), (1921, 20000, 96), (4500, 200, 300), (4500, 1000, 96), (2049, 128, 40), (8321, 2000, 264)]


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_exactly(d, T, V, D, dtype):  # noqa: F811
    q, s, wq, ws = operands(T, V, D)
    want = logits8(q, s, wq, ws, torch.float32)[0].float().to(TYPES[dtype])     # fp32 holds it; one rounding to bf16
    assert torch.equal(d.logits8(q, s, wq, ws, TYPES[dtype]), want)
    base = torch.full((T * (V + 3) + 9,), 7.0, dtype=TYPES[dtype], device="cuda")
    out = base[5:5 + T * (V + 3)].view(T, V + 3)[:, :V]                          # off 16-byte boundaries
    d.logits8(q, s, wq, ws, out=out)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert (base == 7.0).all()


@pytest.mark.parametrize("pad", [0, 1])
def test_logits_beyond_32_bits(d, pad):  # noqa: F811
    """17000 x 128256: 2.18e9 logits; in copies of 32 rows (pad 0) and value by value."""
    T, V, D = 17000, 128256, 40
    q, s, wq, ws = operands(T, V, D)
    out = torch.full((T, V + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    d.logits8(q, s, wq, ws, out=out[:, :V])
    for lo in (0, 8300, 16640, T - 120):
        i = slice(lo, lo + 120)
        want = logits8(q[i], s[i], wq, ws, torch.float32)[0].float().bfloat16()
        assert torch.equal(out[i, :V], want), lo
    assert (out[:, V:] == 7.0).all()
    assert not (out[:, :V] == 7.0).all(1).any()                                  # no row is left as it was
