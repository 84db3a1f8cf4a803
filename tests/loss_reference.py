"""Plain 64-bit definitions of the losses over the vocabulary and of the embedding's gradient (torch, any device), and
bounds on what fp32 sums and bf16 roundings may be off by, derived from the number formats."""
import torch

INF = float("inf")


def roundoff(dtype):
    """Largest relative error of one rounding to nearest: half of eps."""
    return torch.finfo(dtype).eps / 2


def unpack(mask, V):
    """[rows][W] int32 words -> bool [rows][V]."""
    bits = (mask[:, :, None] >> torch.arange(32, device=mask.device, dtype=torch.int32)) & 1
    return bits.reshape(mask.shape[0], -1)[:, :V].bool()


def pack(bits):
    rows, V = bits.shape
    W = (V + 31) // 32
    full = torch.zeros(rows, W * 32, dtype=torch.int64, device=bits.device)
    full[:, :V] = bits.long()
    words = (full.view(rows, W, 32) << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()


def logsumexp(x):
    top = x.max(1).values
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    return torch.log(torch.exp(x - top[:, None]).sum(1)) + top


class TokenLoss:
    """loss, lse, and with grad_loss dhidden and dweight, of float64 copies of the inputs; `tol`: by name, what the
    results may be off by, elementwise."""

    def __init__(self, hidden, weight, targets, mask=None, grad_loss=None):
        h, w, y = hidden.double(), weight.double(), targets.long()
        (T, D), V = h.shape, w.shape[0]
        x = h @ w.T
        if mask is not None:
            x = x.masked_fill(~unpack(mask, V), -INF)
        self.lse = logsumexp(x)
        given = (y >= 0) & (y < V)
        at = x.gather(1, y.clamp(0, V - 1)[:, None])[:, 0]
        self.loss = torch.where(at > -INF, self.lse - at, torch.full_like(at, INF))
        self.loss[~given] = 0.0
        # A logit is a sum of D products in fp32, 16 at a time: at most D / 16 + 16 roundings, each of at most one unit in
        # the last place (truncation) of the sum of magnitudes.  exp, the sums of exp (one rounding a merge) and the
        # logarithm: a few units in the last place of the result and of 1.
        size = float((h.abs() @ w.abs().T).max())
        tol_x = (D / 16 + 16) * 2.0 ** -23 * size
        self.tol = {"lse": tol_x + 2.0 ** -20 * (1 + self.lse.abs())}
        self.tol["loss"] = self.tol["lse"] + tol_x
        if grad_loss is None:
            return
        c = torch.where(given & (at > -INF), grad_loss.double(), torch.zeros_like(at))
        on = c != 0
        h = torch.where(on[:, None], h, torch.zeros_like(h))
        p = torch.exp(x - torch.where(torch.isinf(self.lse), torch.zeros_like(self.lse), self.lse)[:, None])
        hot = torch.zeros_like(p)
        hot[torch.arange(T, device=y.device), y.clamp(0, V - 1)] = 1.0
        p, hot = p * on[:, None], hot * on[:, None]
        G, size_G = c[:, None] * (p - hot), c.abs()[:, None] * (p + hot)
        # G: bf16's rounding, the logit's and lse's errors as relative ones of p; the products' sums in fp32 over V
        # or T as above; the result's rounding to bf16.  Results below bf16's normal numbers are off by 2^-133 at most,
        # terms below them by as much each.
        rel = roundoff(torch.bfloat16) + 2 * (tol_x + 2.0 ** -20 * float(1 + self.lse[on].abs().max() if on.any() else 1.0))
        self.dhidden, self.dweight = G @ w, G.T @ h
        for name, value, sizes, n in (("dhidden", self.dhidden, size_G @ w.abs(), V),
                                      ("dweight", self.dweight, size_G.T @ h.abs(), T)):
            self.tol[name] = (rel + (n / 16 + 16) * 2.0 ** -23) * sizes + roundoff(torch.bfloat16) * value.abs() + 2.0 ** -120


class Distill:
    """loss, lse and with grad_loss dlogits; `tol` as above.  scale: magnitude of the outputs' rounding."""

    def __init__(self, logits, teacher, ids, tau, mask=None, grad_loss=None):
        x = logits.double() / tau
        T, V = x.shape
        K = ids.shape[1]
        if mask is not None:
            x = x.masked_fill(~unpack(mask, V), -INF)
        self.lse = logsumexp(x)
        y = ids.long()
        on = (y >= 0) & (y < V)
        xs = x.gather(1, y.clamp(0, V - 1))
        on &= xs > -INF
        for k in range(1, K):     # of equal ids the first counts
            on[:, k] &= ~((y[:, :k] == y[:, k:k + 1]) & on[:, :k]).any(1)
        t = (teacher.double() / tau).masked_fill(~on, -INF)
        used = on.any(1)
        logp = t - torch.where(used, logsumexp(t), torch.zeros_like(self.lse))[:, None]
        p = torch.where(on, torch.exp(logp), torch.zeros_like(logp))
        lse = torch.where(torch.isinf(self.lse), torch.zeros_like(self.lse), self.lse)
        diff = torch.where(p > 0, logp - (xs - lse[:, None]), torch.zeros_like(p))
        self.loss = tau * tau * (p * diff).sum(1)
        # fp32: a scaled logit, its difference from the maximum, the exponential's argument and the sum's merges are each
        # within 2^-23 of their magnitudes (the largest scaled logit's), or of 1; a term's p is within 2^-20 (1 + its
        # argument) of itself.
        size = 1 + x[torch.isfinite(x)].abs().max() if torch.isfinite(x).any() else torch.tensor(1.0)
        size_t = 1 + t[torch.isfinite(t)].abs().max() if torch.isfinite(t).any() else torch.tensor(1.0)
        rel = float(2.0 ** -20 * (size + size_t))
        self.tol = {"lse": torch.full_like(self.lse, rel),
                    "loss": tau * tau * (rel * (2 + (p * diff.abs()).sum(1)) + rel * (p * logp.abs().nan_to_num(0, 0, 0)).sum(1))}
        if grad_loss is None:
            return
        c = torch.where(used, grad_loss.double() * tau, torch.zeros_like(self.lse))
        q = torch.exp(x - lse[:, None]) * used[:, None]
        g, size_g = q.clone(), q.clone()
        g.scatter_add_(1, y.clamp(0, V - 1), -p)
        size_g.scatter_add_(1, y.clamp(0, V - 1), p)
        self.dlogits = c[:, None] * g
        self.tol["dlogits"] = 2 * rel * c.abs()[:, None] * size_g + roundoff(logits.dtype) * self.dlogits.abs() + 2.0 ** -120


def embed_grad(tokens, grad, V, scale, into=None):
    """dweight and its tolerance, in float64."""
    t = tokens.long()
    on = (t >= 0) & (t < V)
    g = grad.double()[on] * scale
    dw = torch.zeros(V, grad.shape[1], dtype=torch.float64, device=grad.device).index_add_(0, t[on], g)
    size = torch.zeros_like(dw).index_add_(0, t[on], g.abs())
    if into is not None:
        dw, size = dw + into.double(), size + into.double().abs()
    n = int(torch.bincount(t[on], minlength=1).max()) if on.any() else 0
    # n additions in fp32, the scale, one rounding to the result's type
    return dw, (n + 4) * 2.0 ** -24 * size + roundoff(grad.dtype) * dw.abs() + 2.0 ** -133


def assert_within(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape, what
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(want), torch.isnan(got)), f"{what}: NaN in other places"
    odd = ~fin & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), f"{what}: infinities"
    off = ((got - want).abs() - tol)[fin]
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0, f"{what}: {int((off > 0).sum())} values off by up to {worst:.3g} more than the bound"
