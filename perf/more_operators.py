"""The operators between a model's last block and the masked decode, for serving in 8 bits and for training: what a user
has in hand before each call, the call, its plain form, the work it cannot do without and independent 64-bit results.

Kinds of call (`case["kind"]`):
  norm8       h = x + residual, its root-mean-square norm times a weight, in e4m3 with a scale for each 128 values
  norm_step   the norm in the stream's own type, and its gradient for h and the weight (a training step's part)
  quantize8   a matrix in e4m3 with a scale for each 1 x 128 (hidden states) or 128 x 128 values (a weight)
  logits8     hidden . weight^T of two such matrices: a step's logits
  penalized   greedy decode (argmax, log-sum-exp, log-probabilities) of logits under penalties for repeated tokens,
              biases and a grammar's mask

A stream has a few channels far larger than the others.  Tokens follow a 1/id distribution, as frequency-sorted
vocabularies give.  Masks are those of a decode step (bit t & 31 of word t >> 5): rows inside strings allow about 80 %
of the tokens, others 1 %, one of 50 nothing.  Histories are of different lengths, some empty; what stands behind a
row's length is not read.
"""
import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BLOCK = 128
MOST8 = 448.0          # the largest e4m3 value
LEAST = 2.0 ** -100    # a block's largest magnitude counts as this much at least


def listed():
    return [
        # the last norm of a small server's decode step, residual added: latency
        {"name": "norm8_decode_b32", "kind": "norm8", "T": 32, "D": 4096, "type": "bf16", "residual": True},
        # the same for a batch of prompts
        {"name": "norm8_prompts", "kind": "norm8", "T": 16384, "D": 4096, "type": "bf16", "residual": True},
        # training a small fp32 model on ragged texts, rows off 16-byte boundaries
        {"name": "norm_step_odd_f32", "kind": "norm_step", "T": 777, "D": 333, "type": "f32", "residual": True},
        # training a wide model
        {"name": "norm_step_wide", "kind": "norm_step", "T": 16384, "D": 4096, "type": "bf16", "residual": True},
        # hidden states that do not come from a norm of this library, odd sizes
        {"name": "quantize8_rows_odd", "kind": "quantize8", "R": 301, "D": 1001, "block": 1, "type": "bf16"},
        # a 128K vocabulary's weight, once when a model is loaded, or in each step that trained it
        {"name": "quantize8_weight", "kind": "quantize8", "R": 128256, "D": 4096, "block": 128, "type": "bf16"},
        # the logits of one sequence, 32K vocabulary: latency
        {"name": "logits8_b1_v32000", "kind": "logits8", "T": 1, "V": 32000, "D": 1024, "type": "f32"},
        # a server's decode step with a 128K vocabulary: one pass over the weight
        {"name": "logits8_b64_v128256", "kind": "logits8", "T": 64, "V": 128256, "D": 4096, "type": "f32"},
        # scoring whole texts; the largest
        {"name": "logits8_score", "kind": "logits8", "T": 2048, "V": 128256, "D": 4096, "type": "bf16"},
        # one chat with a short history: latency
        {"name": "penalized_b1", "kind": "penalized", "B": 1, "V": 32000, "L": 500, "bias": 16, "type": "f32",
         "mask": True, "logprobs": False},
        # a server's step, long histories
        {"name": "penalized_b256", "kind": "penalized", "B": 256, "V": 128256, "L": 4096, "bias": 64, "type": "bf16",
         "mask": True, "logprobs": False},
        # odd sizes: rows off 16-byte boundaries, log-probabilities for the user
        {"name": "penalized_odd_logprobs", "kind": "penalized", "B": 77, "V": 50001, "L": 1023, "bias": 7,
         "type": "bf16", "mask": True, "logprobs": True},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _round(rng, n, to):
    """Odd sizes, multiples of `to` and anything, a third each."""
    u = rng.random()
    return n | 1 if u < 0.33 else max(to, n // to * to) if u < 0.67 else n


def draw(rng):
    kind = rng.choice(["norm8", "norm_step", "quantize8", "logits8", "logits8", "penalized", "penalized"])
    dtype = rng.choice(["bf16", "f32"])
    if kind.startswith("norm"):
        D = _round(rng, _log(rng, 64, 8192), 64)
        T = min(_round(rng, _log(rng, 1, 16384), 64), 16384 * 4096 // D)
        return {"kind": kind, "T": T, "D": min(D, 8192), "type": dtype, "residual": rng.random() < 0.7}
    if kind == "quantize8":
        D = min(_round(rng, _log(rng, 64, 4096), 64), 4096)
        R = min(_round(rng, _log(rng, 1, 128256), 64), 128256 if dtype == "bf16" else 64128)
        return {"kind": kind, "R": R, "D": D, "block": rng.choice([1, 128]), "type": dtype}
    if kind == "logits8":
        V, D = _round(rng, _log(rng, 1000, 160000), 80), min(_round(rng, _log(rng, 64, 4096), 64), 4096)
        T = min(_round(rng, _log(rng, 1, 2048), 64), 2048, 2048 * 128256 // V)
        return {"kind": kind, "T": T, "V": V, "D": D, "type": dtype}
    V = _round(rng, _log(rng, 1000, 152064), 32)
    B = min(_round(rng, _log(rng, 1, 256), 8), 256, 256 * 128256 // V)
    return {"kind": kind, "B": B, "V": V, "L": _round(rng, _log(rng, 1, 8192), 64), "bias": rng.choice([0, _log(rng, 1, 300)]),
            "type": dtype, "mask": rng.random() < 0.8, "logprobs": rng.random() < 0.3}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 7919 + 23)


def _stream(T, D, dtype, g, size):
    x = torch.empty(T, D, dtype=dtype, device=DEV)
    loud = 1.0 + 30.0 * (torch.rand(D, generator=g, device=DEV) < 0.004)
    for lo in range(0, T, 16384):
        n = min(16384, T - lo)
        x[lo:lo + n] = torch.randn(n, D, generator=g, device=DEV) * (loud * size)
    return x


def _tokens(shape, V, g):
    """Token ids, P(id) falling as 1 / (id + 1)."""
    u = torch.rand(shape, generator=g, device=DEV, dtype=torch.float64)
    return ((V + 1.0) ** u - 1.0).long().clamp_(0, V - 1).int()


def _masks(B, V, g):
    """[B][W] packed masks."""
    W = (V + 31) // 32
    dense = (torch.rand(B, 1, generator=g, device=DEV) < 0.33).float() * 0.79 + 0.01
    bits = torch.rand(B, W * 32, generator=g, device=DEV) < dense
    bits[:, V:] = False
    bits[torch.rand(B, generator=g, device=DEV) < 0.02] = False
    words = (bits.view(B, W, 32).long() << torch.arange(32, device=DEV)).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()


def _rows16(R, D):
    """e4m3 [R][D], rows on 16-byte boundaries."""
    return torch.zeros(R, (D + 15) // 16 * 16, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)[:, :D]


def _in_blocks(x, rows):
    """x [R][D] (any float) with zeros up to whole blocks: [R / rows][rows][D / 128][128]."""
    R, D = x.shape
    x = torch.nn.functional.pad(x, (0, -D % BLOCK, 0, -R % rows))
    return x.view(x.shape[0] // rows, rows, x.shape[1] // BLOCK, BLOCK)


def _quantize(x, rows):
    """(codes, scales) of an fp32 matrix."""
    R, D = x.shape
    b = _in_blocks(x, rows)
    most = b.abs().amax((1, 3), keepdim=True).clamp(min=LEAST)
    q = (b * (MOST8 / most)).clamp(-MOST8, MOST8)
    q = q.view(b.shape[0] * rows, -1)[:R, :D].to(torch.float8_e4m3fn)
    return q, (most / MOST8).view(b.shape[0], b.shape[2])


def prepare(case, seed):
    g, s, kind = _generator(seed), dict(case), case["kind"]
    if kind.startswith("norm"):
        T, D, dtype = case["T"], case["D"], TYPES[case["type"]]
        s["x"] = _stream(T, D, dtype, g, 0.5)
        s["residual_rows"] = _stream(T, D, dtype, g, 2.0) if case["residual"] else None
        s["weight"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dtype)
        if kind == "norm_step":
            s["dy"] = (torch.randn(T, D, generator=g, device=DEV) * 1e-3).to(dtype)
            s["dsum"] = (torch.randn(T, D, generator=g, device=DEV) * 1e-3).to(dtype)
        return s
    if kind == "quantize8":
        s["x"] = _stream(case["R"], case["D"], TYPES[case["type"]], g, 0.02 if case["block"] == 128 else 1.0)
        return s
    if kind == "logits8":
        T, V, D = case["T"], case["V"], case["D"]
        s["q"], s["wq"] = _rows16(T, D), _rows16(V, D)
        q, s["scales"] = _quantize(_stream(T, D, torch.float32, g, 1.0), 1)
        s["q"].view(torch.uint8).copy_(q.view(torch.uint8))
        s["w_scales"] = torch.empty((V + 127) // 128, (D + 127) // 128, device=DEV)
        for lo in range(0, V, 16384):
            w = torch.randn(min(16384, V - lo), D, generator=g, device=DEV) * (2.0 / math.sqrt(D))
            q, sw = _quantize(w, 128)
            s["wq"][lo:lo + len(w)].view(torch.uint8).copy_(q.view(torch.uint8))
            s["w_scales"][lo // 128:lo // 128 + len(sw)] = sw
        return s
    B, V, L = case["B"], case["V"], case["L"]
    s["logits"] = (torch.randn(B, V, generator=g, device=DEV) * 3.0).to(TYPES[case["type"]])
    s["history"] = _tokens((B, L), V, g)
    s["lengths"] = torch.randint(0, L + 1, (B,), generator=g, device=DEV).int()
    s["prompt_lengths"] = (s["lengths"] * torch.rand(B, generator=g, device=DEV)).int()
    # some of a history's positions hold no token (padding on the left, pictures)
    s["history"][torch.rand(B, L, generator=g, device=DEV) < 0.02] = -1
    s["repetition"] = 1.0 + 0.3 * torch.rand(B, generator=g, device=DEV)
    s["presence"] = 0.5 * torch.rand(B, generator=g, device=DEV)
    s["frequency"] = 0.2 * torch.rand(B, generator=g, device=DEV)
    s["bias_ids"] = s["bias_values"] = None
    if case["bias"]:
        n = min(case["bias"], V)
        s["bias_ids"] = torch.stack([torch.randperm(V, generator=g, device=DEV)[:n] for _ in range(B)]).int()
        s["bias_ids"][torch.rand(B, n, generator=g, device=DEV) < 0.1] = -1
        s["bias_values"] = torch.randn(B, n, generator=g, device=DEV) * 5.0
        s["bias_values"][torch.rand(B, n, generator=g, device=DEV) < 0.1] = -math.inf      # banned
    s["mask_bits"] = _masks(B, V, g) if case["mask"] else None
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _handle():
    from paper_2403_06988_gb300 import Domino
    return Domino(0)


def _run_own(s):
    d, kind = _handle(), s["kind"]
    if kind == "norm8":
        q, scales, h = d.norm8(s["x"], s["weight"], s["residual_rows"], EPS)
        return {"q": q, "scales": scales, "sum": h}
    if kind == "norm_step":
        y, h, rstd = d.norm(s["x"], s["weight"], s["residual_rows"], EPS)
        dx, dw = d.norm_grad(h, s["weight"], rstd, s["dy"], s["dsum"])
        return {"y": y, "sum": h, "dx": dx, "dweight": dw}
    if kind == "quantize8":
        q, scales = d.quantize8(s["x"], s["block"])
        return {"q": q, "scales": scales}
    if kind == "logits8":
        return {"logits": d.logits8(s["q"], s["scales"], s["wq"], s["w_scales"], TYPES[s["type"]])}
    argmax, lse, logprobs = d.mask_logits_penalized(
        s["logits"], s["history"], s["lengths"], s["prompt_lengths"], s["repetition"], s["presence"], s["frequency"],
        s["bias_ids"], s["bias_values"], s["mask_bits"], want_logprobs=s["logprobs"])
    out = {"argmax": argmax, "lse": lse}
    return {**out, "logprobs": logprobs} if s["logprobs"] else out


def _plain_norm(s):
    x, r, w = s["x"], s["residual_rows"], s["weight"].float()
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    hf = h.float()
    rstd = 1.0 / torch.sqrt((hf * hf).mean(1) + EPS)
    y = hf * rstd[:, None] * w
    if s["kind"] == "norm8":
        q, scales = _quantize(y, 1)
        return {"q": q, "scales": scales, "sum": h}
    dy = s["dy"].float()
    g = w * dy
    c = (g * hf).mean(1) * rstd * rstd
    dx = rstd[:, None] * (g - hf * c[:, None]) + s["dsum"].float()
    dw = (dy * hf * rstd[:, None]).sum(0)
    return {"y": y.to(x.dtype), "sum": h, "dx": dx.to(x.dtype), "dweight": dw.to(x.dtype)}


def _scaled(q, scales, rows):
    R, D = q.shape
    b = _in_blocks(q.float(), rows) * scales[:, None, :, None]
    return b.view(b.shape[0] * rows, -1)[:R, :D]


def _plain_penalized(s):
    B, V, L = s["B"], s["V"], s["L"]
    x, t = s["logits"].float(), s["history"].long()
    at = torch.arange(L, device=DEV)[None]
    on = (t >= 0) & (at < s["lengths"][:, None])
    new = on & (at >= s["prompt_lengths"][:, None])
    t = t.clamp(min=0)
    seen = torch.zeros(B, V, device=DEV).scatter_add_(1, t, on.float())
    count = torch.zeros(B, V, device=DEV).scatter_add_(1, t, new.float())
    rep = s["repetition"][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][:, None] * count
    x = x - s["presence"][:, None] * (count > 0)
    if s["bias_ids"] is not None:
        ids = s["bias_ids"].long()
        bias = torch.zeros(B, V, device=DEV).scatter_add_(1, ids.clamp(min=0), torch.where(ids >= 0, s["bias_values"], 0.0))
        x = x + bias
    if s["mask_bits"] is not None:
        bits = (s["mask_bits"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        x = torch.where(bits.view(B, -1)[:, :V] != 0, x, -math.inf)
    m = x.amax(1, keepdim=True)
    least = torch.where(x == m, torch.arange(V, device=DEV)[None], V).amin(1)      # the lowest of equal ones
    ref = m.clamp(min=torch.finfo(x.dtype).min)
    lse = ref[:, 0] + (x - ref).exp().sum(1).log()
    none = m[:, 0] == -math.inf
    out = {"argmax": torch.where(none, -1, least).int(), "lse": lse.masked_fill(none, -math.inf)}
    if s["logprobs"]:
        out["logprobs"] = torch.where(x > -math.inf, x - lse[:, None], -math.inf)
    return out


def run(s):
    if own:
        return _run_own(s)
    if s["kind"].startswith("norm"):
        return _plain_norm(s)
    if s["kind"] == "quantize8":
        q, scales = _quantize(s["x"].float(), s["block"])
        return {"q": q, "scales": scales}
    if s["kind"] == "logits8":
        return {"logits": (_scaled(s["q"], s["scales"], 1) @ _scaled(s["wq"], s["w_scales"], 128).T).to(TYPES[s["type"]])}
    return _plain_penalized(s)


# ---------------------------------------------------------------------------
# work and 64-bit results
# ---------------------------------------------------------------------------
def _ceil(a, b):
    return -(-a // b)


def work(case):
    kind, size = case["kind"], 2 if case["type"] == "bf16" else 4
    if kind.startswith("norm"):
        T, D = case["T"], case["D"]
        read = T * D * size * (2 if case["residual"] else 1) + D * size
        total = T * D * size if case["residual"] else 0
        if kind == "norm8":
            return {"bytes": read + total + T * D + 4 * T * _ceil(D, BLOCK), "flops": 8 * T * D}
        # the gradient reads h and its two incoming gradients, writes one and the weight's
        return {"bytes": read + total + T * D * size + 4 * T * D * size + 2 * D * size + 8 * T, "flops": 17 * T * D}
    if kind == "quantize8":
        R, D = case["R"], case["D"]
        return {"bytes": R * D * (size + 1) + 4 * _ceil(R, case["block"]) * _ceil(D, BLOCK), "flops": 3 * R * D}
    if kind == "logits8":
        T, V, D = case["T"], case["V"], case["D"]
        scales = 4 * (T + _ceil(V, BLOCK)) * _ceil(D, BLOCK)
        return {"bytes": (T + V) * D + scales + T * V * size, "flops": 2 * T * V * D}
    B, V, L = case["B"], case["V"], case["L"]
    # half of a history's places are used on average
    return {"bytes": B * (V * size + (4 * _ceil(V, 32) if case["mask"] else 0) + 2 * L + 8 * case["bias"] + 28) +
            (4 * B * V if case["logprobs"] else 0), "flops": 4 * B * V}


def _exact_codes(y, rows):
    """y in units of its block's scale, before the rounding to 8 bits, and the scales."""
    R, D = y.shape
    cols, lines = torch.arange(D, device=DEV) // BLOCK, torch.arange(R, device=DEV) // rows
    scales = torch.empty(_ceil(R, rows), _ceil(D, BLOCK), dtype=torch.float64, device=DEV)
    for j in range(scales.shape[1]):
        top = y[:, j * BLOCK:(j + 1) * BLOCK].abs().max(dim=1).values
        for_rows = torch.zeros(len(scales), dtype=torch.float64, device=DEV)
        scales[:, j] = for_rows.scatter_reduce(0, lines, top, "amax").clamp(min=LEAST) / MOST8
    return torch.cat([y[lo:lo + 8192] / scales[lines[lo:lo + 8192]][:, cols] for lo in range(0, R, 8192)]), scales


def _exact_penalized(s):
    B, V = s["B"], s["V"]
    rows, best, lse = [], [], []
    words = None if s["mask_bits"] is None else np.ascontiguousarray(s["mask_bits"].cpu().numpy()).view(np.uint8)
    hist, length, prompt = (s[k].cpu().numpy() for k in ("history", "lengths", "prompt_lengths"))
    rep, pres, freq = (s[k].double().cpu().numpy() for k in ("repetition", "presence", "frequency"))
    bias = None if s["bias_ids"] is None else (s["bias_ids"].cpu().numpy(), s["bias_values"].double().cpu().numpy())
    for b in range(B):
        x = s["logits"][b].double().cpu().numpy()
        for upto, counted in ((0, False), (prompt[b], True)):
            ids, n = np.unique(hist[b, upto:length[b]], return_counts=True)
            keep = ids >= 0
            ids, n = ids[keep], n[keep]
            if counted:
                x[ids] -= freq[b] * n + pres[b]
            else:
                x[ids] = np.where(x[ids] > 0, x[ids] / rep[b], x[ids] * rep[b])
        if bias is not None:
            on = bias[0][b] >= 0
            x[bias[0][b][on]] += bias[1][b][on]
        if words is not None:
            x[np.unpackbits(words[b], bitorder="little")[:V] == 0] = -np.inf
        top = x.max()
        z = -np.inf if np.isinf(top) else top + math.log(np.exp(x - top).sum())
        lse.append(z)
        if s["logprobs"]:
            rows.append(np.where(np.isinf(x), -np.inf, x - (0.0 if np.isinf(z) else z)))
    out = {"argmax": None, "lse": torch.tensor(lse, dtype=torch.float64)}      # near ties fall by the 32-bit values
    return {**out, "logprobs": torch.from_numpy(np.stack(rows))} if s["logprobs"] else out


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind.startswith("norm"):
        x, w = s["x"].double(), s["weight"].double()
        total = x if s["residual_rows"] is None else x + s["residual_rows"].double()
        h = total.to(s["x"].dtype).double()            # the norm is that of the rounded sum
        power = torch.einsum("td,td->t", h, h) / case["D"] + EPS
        y = torch.einsum("td,t,d->td", h, power.rsqrt(), w)
        if kind == "norm8":
            q, scales = _exact_codes(y, 1)
            return {"q": q, "scales": scales, "sum": total}
        dy = s["dy"].double()
        # d y / d h = diag(w) rstd - (w h) h^T rstd^3 / D
        along = torch.einsum("td,td,d->t", dy, h, w) / (case["D"] * power ** 1.5)
        dx = torch.einsum("td,d,t->td", dy, w, power.rsqrt()) - along[:, None] * h + s["dsum"].double()
        return {"y": y, "sum": total, "dx": dx, "dweight": torch.einsum("td,td,t->d", dy, h, power.rsqrt())}
    if kind == "quantize8":
        q, scales = _exact_codes(s["x"].double(), case["block"])
        return {"q": q, "scales": scales}
    if kind == "logits8":
        T, V, D = case["T"], case["V"], case["D"]
        h, out = s["q"].double(), torch.empty(T, V, dtype=torch.float64, device=DEV)
        cols = torch.arange(D, device=DEV) // BLOCK
        h *= s["scales"].double()[:, cols]
        for lo in range(0, V, 16384):
            hi = min(V, lo + 16384)
            lines = torch.arange(lo, hi, device=DEV) // 128
            w = s["wq"][lo:hi].double() * s["w_scales"].double()[lines][:, cols]
            out[:, lo:hi] = torch.einsum("td,vd->tv", h, w)
        return {"logits": out}
    return _exact_penalized(s)
