"""The norm, its gradient, 8-bit codes and logits of codes from their definitions, in 64 bits, and what fp32 arithmetic and
the results' rounding may make of them (`tol`, elementwise, derived below)."""
import torch

U = 2.0 ** -24          # half a step of fp32, relative
LEAST = 2.0 ** -100


def half(dtype):
    """A rounding's largest error, relative."""
    return torch.finfo(dtype).eps / 2


def additions(D):
    """A row's sum over D values: a thread adds at most 32 one after the other, or eight of each 4096, then five times
    over a warp's lanes and over at most 16 warps."""
    return max(32, -(-D // 4096) * 8) + 5 + 16


class Norm:
    """y, sum, rstd, and with dy dx and dweight, of float64 copies.  The norm is that of the rounded sum."""

    def __init__(self, x, weight, residual=None, eps=1e-6, dy=None, dsum=None):
        T, D = x.shape
        dtype = x.dtype
        self.sum = x if residual is None else (x.float() + residual.float()).to(dtype)     # exact: one addition, one rounding
        h, w = self.sum.double(), weight.double()
        self.rstd = ((h * h).mean(1) + eps) ** -0.5
        self.y = h * self.rstd[:, None] * w
        n = additions(D)
        # a sum of squares: each addition and each square a rounding, no cancellation; the quotient, eps, the root
        rel_rstd = ((n + 1) / 2 + 3) * U
        self.tol = {"rstd": self.rstd * rel_rstd}
        self.rel_y = rel_rstd + 2 * U                      # two products more
        self.tol["y"] = self.y.abs() * (self.rel_y + half(dtype)) + 1e-40
        if dy is None:
            return
        g = dy.double() * w
        c = (g * h).mean(1, keepdim=True)
        r = self.rstd[:, None]
        s = torch.zeros_like(h) if dsum is None else dsum.double()
        self.dx = r * (g - h * r * r * c) + s
        # every term's magnitude times the roundings it went through: the mean's additions, rstd's own (three times in
        # h r^3 c), a few products and differences
        size = r * (g.abs() + h.abs() * r * r * (g * h).abs().mean(1, keepdim=True)) + s.abs()
        self.tol["dx"] = self.dx.abs() * half(dtype) + size * (n + 3 * ((n + 1) / 2 + 3) + 10) * U + 1e-40
        terms = dy.double() * h * r
        self.dweight = terms.sum(0)
        # at least min(T, 152) strips of rows, at most 16 * 152 of them added 64 at a time and six times in halves; at most
        # dim / 2^10 fewer for long rows
        strips = max(1, min(T, 152 if D <= 8192 else 19))
        adds = -(-T // strips) + 16 * 152 // 64 + 1 + 6
        self.tol["dweight"] = self.dweight.abs() * half(dtype) + terms.abs().sum(0) * (adds + rel_rstd / U + 3) * U + 1e-40


class Codes:
    """scales, and v in units of them (`units`, what the codes round), of a float64 matrix known to `rel`."""

    def __init__(self, v, block, rel=0.0):
        R, D = v.shape
        nb, nr = -(-D // 128), -(-R // block)
        top = torch.zeros(nr, nb, dtype=torch.float64, device=v.device)
        for i in range(nb):
            most = v[:, i * 128:(i + 1) * 128].abs().amax(1)
            for j in range(0, R, block) if block > 1 else ():
                top[j // block, i] = most[j:j + block].max()
            if block == 1:
                top[:, i] = most
        self.scales = top.clamp(min=LEAST) / 448
        self.spread = self.scales.repeat_interleave(block, 0)[:R].repeat_interleave(128, 1)[:, :D]
        self.units = v / self.spread
        self.tol_scales = self.scales * (rel + 2 * U)
        # e4m3: half a step is 2^-4 of the value from 2^-6 on, below that 2^-10; the value's own error, and three roundings
        # of it and the scale (448 / a, the product; a's error enters again)
        step = torch.maximum(self.units.abs() * half(torch.float8_e4m3fn), torch.full_like(self.units, 2.0 ** -10))
        self.tol = step + self.units.abs() * (2 * rel + 4 * U)


def decode(codes):
    return codes.float().double()


def logits8(codes, scales, wcodes, wscales, dtype):
    """(logits, tol)."""
    (T, D), V = codes.shape, wcodes.shape[0]
    nb = -(-D // 128)
    out = torch.zeros(T, V, dtype=torch.float64, device=codes.device)
    size = torch.zeros_like(out)
    h, w = decode(codes), decode(wcodes)
    ws = wscales.double().repeat_interleave(128, 0)[:V]
    for b in range(nb):
        i = slice(128 * b, min(D, 128 * b + 128))
        c = scales.double()[:, b:b + 1] * ws[:, b][None]
        out += c * (h[:, i] @ w[:, i].T)
        size += c * (h[:, i].abs() @ w[:, i].abs().T)
    # a block's sum on the tensor cores: 128 products, exact, and its parts are each cut (not rounded) to no fewer than 24
    # bits of the largest; then a rounding of the scales' product and one for each block
    tol = size * (128 * 2 * U + (nb + 2) * U) + out.abs() * half(dtype) + 1e-40
    return out, tol


def assert_within(got, want, tol, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    if bad.any():
        i = int(torch.where(bad, (off - tol).nan_to_num(nan=float("inf")), torch.zeros_like(off)).reshape(-1).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; at {i} {float(got.reshape(-1)[i])} for "
                             f"{float(want.reshape(-1)[i])}, allowed {float(tol.reshape(-1)[i]):.3g}")
