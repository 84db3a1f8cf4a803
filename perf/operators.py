"""The operators at a model's two vocabulary-sized ends, for training and distilling a model whose answers a grammar
constrains: what a user has in hand before each call, the call, its plain form, the work it cannot do without and
independent 64-bit results.

Kinds of call (`case["kind"]`):
  loss          the cross entropy of target tokens under softmax(hidden . weight^T) over the tokens that a mask allows:
                per row the loss and the log-sum-exp (scoring given tokens, evaluation)
  loss_step     the same and its gradient for the hidden states and the weight (a training step's end)
  distill       Kullback-Leibler divergence of a teacher's top logits from a student's masked softmax
  distill_step  the same and its gradient for the student's logits
  embed         the scaled rows of an embedding table for a list of tokens
  embed_grad    the gradient of that table

Masks are those of a decode step (bit t & 31 of word t >> 5): rows inside strings allow about 80 % of the tokens,
others 1 %.  Tokens follow a 1/id distribution, as frequency-sorted vocabularies give.  Targets below 0 are positions
without a target (a prompt, padding); a token below 0 (a row that has ended) embeds as zeros and has no gradient; a
teacher's list may end early (ids below 0).  Rows whose mask excludes the target have an infinite loss and no gradient.
"""
import functools
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the log-probability of one token, 32K vocabulary: latency
        {"name": "loss_row_v32000", "kind": "loss", "T": 1, "V": 32000, "D": 1024, "mask": True},
        # scoring a batch of positions under a grammar's masks with a 128K vocabulary: one pass over the weight
        {"name": "loss_score_v128256", "kind": "loss", "T": 256, "V": 128256, "D": 4096, "mask": True},
        # fine-tuning on short ragged texts, a vocabulary and a width that divide by nothing much
        {"name": "loss_step_ragged", "kind": "loss_step", "T": 777, "V": 32003, "D": 1000, "mask": True},
        # training a narrow draft model for speculation: few products per logit
        {"name": "loss_step_draft", "kind": "loss_step", "T": 1024, "V": 128256, "D": 512, "mask": True},
        # the largest: a training step of a wide model, no masks (the grammar comes in later)
        {"name": "loss_step_wide", "kind": "loss_step", "T": 4096, "V": 128256, "D": 4096, "mask": False},
        # agreement of a draft model with its target at a small server's batch, fp32 logits
        {"name": "distill_f32_b32", "kind": "distill", "T": 32, "V": 32000, "K": 16, "type": "f32", "tau": 1.0,
         "mask": True},
        # distilling a draft model from stored top logits
        {"name": "distill_step_v128256", "kind": "distill_step", "T": 2048, "V": 128256, "K": 64, "type": "bf16",
         "tau": 2.0, "mask": False},
        # the same under masks, odd sizes: rows off 16-byte boundaries
        {"name": "distill_step_odd", "kind": "distill_step", "T": 301, "V": 50001, "K": 33, "type": "bf16",
         "tau": 1.5, "mask": True},
        # the tokens that a decode step chose, into the next step: latency
        {"name": "embed_decode_b32", "kind": "embed", "N": 32, "V": 128256, "D": 4096, "type": "bf16"},
        # a batch of prompts
        {"name": "embed_prompts", "kind": "embed", "N": 16384, "V": 128256, "D": 4096, "type": "bf16"},
        # the table's gradient for a small fp32 model of odd width
        {"name": "embed_grad_odd_f32", "kind": "embed_grad", "N": 2500, "V": 32003, "D": 333, "type": "f32"},
        # the table's gradient for a large batch: a few tokens carry a tenth of the rows each
        {"name": "embed_grad_v128256", "kind": "embed_grad", "N": 16384, "V": 128256, "D": 4096, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _round(rng, n, to):
    """Odd sizes, multiples of `to` and anything, a third each."""
    u = rng.random()
    return n | 1 if u < 0.33 else max(to, n // to * to) if u < 0.67 else n


def draw(rng):
    kind = rng.choice(["loss", "loss_step", "loss_step", "distill", "distill_step", "embed", "embed_grad"])
    V = _round(rng, _log(rng, 1000, 160000), 80)
    if kind.startswith("loss"):
        T, D = _round(rng, _log(rng, 1, 4096), 80), _round(rng, _log(rng, 64, 4096), 80)
        T = min(T, 4096 if rng.random() < 0.5 else 4095)
        most = 4096 * 128256 * 4096 // 4
        return {"kind": kind, "T": max(1, min(T, most // (V * D))), "V": V, "D": min(D, 4096),
                "mask": rng.random() < 0.6}
    if kind.startswith("distill"):
        T = min(_round(rng, _log(rng, 1, 2048), 80), 2048 * 128256 // V)
        return {"kind": kind, "T": T, "V": V, "K": _log(rng, 1, 256), "type": rng.choice(["bf16", "f32"]),
                "tau": rng.choice([0.7, 1.0, 2.0, 4.0]), "mask": rng.random() < 0.6}
    N, D = _round(rng, _log(rng, 1, 16384), 64), _round(rng, _log(rng, 64, 4096), 80)
    V = min(V, 128256)
    return {"kind": kind, "N": min(N, 16384), "V": V, "D": min(D, 4096), "type": rng.choice(["bf16", "f32"])}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _tokens(n, V, g):
    """Token ids, P(id) falling as 1 / (id + 1)."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    return ((V + 1.0) ** u - 1.0).long().clamp_(0, V - 1).int()


def _masks(T, V, keep, g):
    """[T][W] packed masks: a third of the rows allow 80 % of the tokens, the others 1 %; `keep` [T][k] tokens (below 0:
    none) are allowed, but in one row of 50, which allows nothing."""
    W = (V + 31) // 32
    dense = (torch.rand(T, 1, generator=g, device=DEV) < 0.33).float() * 0.79 + 0.01
    place = (torch.arange(32, device=DEV, dtype=torch.int64))
    out = torch.zeros(T, W, dtype=torch.int32, device=DEV)
    nothing = torch.rand(T, generator=g, device=DEV) < 0.02
    for lo in range(0, T, 512):
        n = min(512, T - lo)
        bits = torch.rand(n, W * 32, generator=g, device=DEV) < dense[lo:lo + n]
        k = keep[lo:lo + n].long()
        bits.scatter_(1, k.clamp(min=0), (k >= 0) | bits.gather(1, k.clamp(min=0)))
        bits[:, V:] = False
        bits[nothing[lo:lo + n]] = False
        words = (bits.view(n, W, 32).long() << place).sum(-1)
        out[lo:lo + n] = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
    return out


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 17)
    s, V = dict(case), case["V"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    if case["kind"].startswith("loss"):
        T, D = case["T"], case["D"]
        weight = torch.empty(V, D, dtype=torch.bfloat16, device=DEV)
        for lo in range(0, V, 16384):
            n = min(16384, V - lo)
            weight[lo:lo + n] = normal(n, D) * (2.0 / math.sqrt(D))
        targets = _tokens(T, V, g)
        # hidden states of a model that has learnt something: the target's logit is raised by up to 10
        lift = torch.rand(T, 1, generator=g, device=DEV) * 2.5
        s["hidden"] = (normal(T, D) + lift * weight[targets.long()].float()).bfloat16()
        if T > 1:
            targets[torch.rand(T, generator=g, device=DEV) < 0.1] = -1
        s["weight"], s["targets"] = weight, targets
        s["mask_bits"] = _masks(T, V, targets[:, None], g) if case["mask"] else None
        # weights of the rows' losses: the mean over the batch, texts weighted a little differently
        s["grad_loss"] = (0.5 + torch.rand(T, generator=g, device=DEV)) / T
        return s
    if case["kind"].startswith("distill"):
        T, K = case["T"], case["K"]
        s["logits"] = torch.empty(T, V, dtype=TYPES[case["type"]], device=DEV)
        s["teacher"] = torch.empty(T, K, dtype=torch.float32, device=DEV)
        s["ids"] = torch.empty(T, K, dtype=torch.int32, device=DEV)
        for lo in range(0, T, 512):
            n = min(512, T - lo)
            x = normal(n, V) * 3.0
            s["logits"][lo:lo + n] = x
            top, ids = (x + normal(n, V) * 1.5).topk(K, dim=1)
            s["teacher"][lo:lo + n], s["ids"][lo:lo + n] = top, ids
        # lists cut at a share of the teacher's mass end early
        length = torch.randint(1, 2 * K + 1, (T, 1), generator=g, device=DEV)
        s["ids"].masked_fill_(torch.arange(K, device=DEV)[None] >= length, -1)
        s["mask_bits"] = _masks(T, V, s["ids"][:, ::2], g) if case["mask"] else None
        s["grad_loss"] = (0.5 + torch.rand(T, generator=g, device=DEV)) / T
        return s
    N, D = case["N"], case["D"]
    s["tokens"] = _tokens(N, V, g)
    if N > 8:
        s["tokens"][torch.rand(N, generator=g, device=DEV) < 0.03] = -1
    s["scale"] = math.sqrt(D)
    if case["kind"] == "embed":
        s["weight"] = (normal(V, D) / math.sqrt(D)).to(TYPES[case["type"]])
    else:
        s["grad"] = (normal(N, D) * 1e-3).to(TYPES[case["type"]])
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
    if kind.startswith("loss"):
        loss, lse = d.token_loss(s["hidden"], s["weight"], s["targets"], s["mask_bits"])
        if kind == "loss":
            return {"loss": loss, "lse": lse}
        dh, dw = d.token_loss_grad(s["hidden"], s["weight"], s["targets"], lse, s["grad_loss"], s["mask_bits"])
        return {"loss": loss, "lse": lse, "dhidden": dh, "dweight": dw}
    if kind.startswith("distill"):
        loss, lse = d.distill_loss(s["logits"], s["teacher"], s["ids"], s["tau"], s["mask_bits"])
        if kind == "distill":
            return {"loss": loss, "lse": lse}
        dl = d.distill_grad(s["logits"], s["teacher"], s["ids"], s["tau"], lse, s["grad_loss"], s["mask_bits"])
        return {"loss": loss, "lse": lse, "dlogits": dl}
    if kind == "embed":
        return {"out": d.embed(s["tokens"], s["weight"], s["scale"])}
    return {"dweight": d.embed_grad(s["tokens"], s["grad"], s["V"], s["scale"])}


def _allowed(mask_bits, V):
    bits = (mask_bits[:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
    return bits.view(mask_bits.shape[0], -1)[:, :V] != 0


def _lse(x):
    m = x.amax(1, keepdim=True).clamp(min=torch.finfo(x.dtype).min)
    return m[:, 0] + (x - m).exp().sum(1).log()


def _plain_loss(s):
    h, w, y = s["hidden"].float(), s["weight"].float(), s["targets"].long()
    x = h @ w.T
    if s["mask_bits"] is not None:
        x = x.masked_fill(~_allowed(s["mask_bits"], s["V"]), -math.inf)
    lse = _lse(x)
    xy = x.gather(1, y.clamp(min=0)[:, None])[:, 0]
    out = xy > -math.inf
    loss = torch.where(out, lse - xy, math.inf).where(y >= 0, 0.0)
    if s["kind"] == "loss":
        return {"loss": loss, "lse": lse}
    c = torch.where(out & (y >= 0), s["grad_loss"], 0.0)
    p = (x - lse.clamp(min=torch.finfo(x.dtype).min)[:, None]).exp()
    p[torch.arange(len(y), device=DEV), y.clamp(min=0)] -= 1.0
    p *= c[:, None]
    return {"loss": loss, "lse": lse, "dhidden": (p @ w).bfloat16(), "dweight": (p.T @ h).bfloat16()}


def _plain_distill(s):
    tau, ids = s["tau"], s["ids"].long()
    x = s["logits"].float() / tau
    on = ids >= 0
    if s["mask_bits"] is not None:
        x = x.masked_fill(~_allowed(s["mask_bits"], s["V"]), -math.inf)
    lse = _lse(x)
    xs = x.gather(1, ids.clamp(min=0))
    on = on & (xs > -math.inf)
    t = (s["teacher"] / tau).masked_fill(~on, -math.inf)
    any_on = on.any(1)
    logp = t - _lse(t).clamp(min=torch.finfo(x.dtype).min)[:, None]
    p = logp.exp()
    terms = torch.where(on, p * (logp - (xs - lse[:, None])), 0.0)
    loss = tau * tau * terms.sum(1)
    if s["kind"] == "distill":
        return {"loss": loss, "lse": lse}
    c = torch.where(any_on, s["grad_loss"] * tau, 0.0)
    q = (x - lse.clamp(min=torch.finfo(x.dtype).min)[:, None]).exp()
    q.scatter_add_(1, ids.clamp(min=0), torch.where(on, -p, 0.0))
    return {"loss": loss, "lse": lse, "dlogits": (q * c[:, None]).to(s["logits"].dtype)}


def run(s):
    if own:
        return _run_own(s)
    if s["kind"].startswith("loss"):
        return _plain_loss(s)
    if s["kind"].startswith("distill"):
        return _plain_distill(s)
    t = s["tokens"].long()
    if s["kind"] == "embed":
        w = s["weight"]
        return {"out": torch.where((t >= 0)[:, None], w[t.clamp(min=0)].float() * s["scale"], 0.0).to(w.dtype)}
    grad = torch.where((t >= 0)[:, None], s["grad"].float() * s["scale"], 0.0)
    dw = torch.zeros(s["V"], s["D"], device=DEV).index_add_(0, t.clamp(min=0), grad)
    return {"dweight": dw.to(s["grad"].dtype)}


# ---------------------------------------------------------------------------
# work and 64-bit results
# ---------------------------------------------------------------------------
def work(case):
    V, kind = case["V"], case["kind"]
    W = (V + 31) // 32
    if kind.startswith("loss"):
        T, D = case["T"], case["D"]
        once = 2 * T * D + 2 * V * D + 4 * T + (4 * T * W if case["mask"] else 0) + 8 * T
        if kind == "loss":
            return {"bytes": once, "flops": 2 * T * V * D}
        return {"bytes": once + 4 * T + 2 * T * D + 2 * V * D, "flops": 6 * T * V * D}
    if kind.startswith("distill"):
        T, K, size = case["T"], case["K"], 2 if case["type"] == "bf16" else 4
        once = T * V * size + 8 * T * K + (4 * T * W if case["mask"] else 0) + 8 * T
        return {"bytes": once + (T * V * size + 4 * T if kind == "distill_step" else 0),
                "flops": T * V * (4 if kind == "distill" else 8)}
    N, D, size = case["N"], case["D"], 2 if case["type"] == "bf16" else 4
    if kind == "embed":   # a token's row is read once however often it comes
        rows = sum(1.0 - (1.0 - math.log((i + 2) / (i + 1)) / math.log(V + 1)) ** N for i in range(V))
        return {"bytes": 4 * N + (rows + N) * D * size, "flops": N * D}
    return {"bytes": 4 * N + (N + V) * D * size, "flops": N * D}


def _exact_lse(x):
    """log(sum(exp)) of each row in 64 bits; -inf where nothing is allowed."""
    top = x.max(dim=1).values
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    return torch.log(torch.exp(x - top[:, None]).sum(dim=1)) + top


def _exact_bits(mask_bits, lo, hi, V):
    words = np.ascontiguousarray(mask_bits[lo:hi].cpu().numpy()).view("<u4").view(np.uint8)
    bits = np.unpackbits(words.reshape(hi - lo, -1), axis=1, bitorder="little")[:, :V]
    return torch.from_numpy(bits).to(DEV).bool()


def exact(case, seed):
    kind, V = case["kind"], case["V"]
    if kind.startswith("loss") and case["T"] * V * case["D"] * (1 if kind == "loss" else 3) > 1e12:
        return None
    s = prepare(case, seed)
    if kind.startswith("loss"):
        T, D = case["T"], case["D"]
        w, loss, lse = s["weight"].double(), [], []
        dh, dw = [], torch.zeros(V, D, dtype=torch.float64, device=DEV) if kind == "loss_step" else None
        for lo in range(0, T, 256):
            hi = min(T, lo + 256)
            h, y = s["hidden"][lo:hi].double(), s["targets"][lo:hi].cpu().numpy()
            x = torch.einsum("td,vd->tv", h, w)
            if s["mask_bits"] is not None:
                x[~_exact_bits(s["mask_bits"], lo, hi, V)] = -math.inf
            z = _exact_lse(x)
            lse.append(z)
            grads = torch.zeros_like(x)
            for i, t in enumerate(y):
                if t < 0:
                    loss.append(0.0)
                    continue
                at = float(x[i, int(t)])
                loss.append(math.inf if at == -math.inf else float(z[i]) - at)
                if at != -math.inf and dw is not None:
                    row = torch.exp(x[i] - z[i])
                    row[int(t)] -= 1.0
                    grads[i] = row * float(s["grad_loss"][lo + i].double())
            if dw is not None:
                dh.append(torch.einsum("tv,vd->td", grads, w))
                dw += torch.einsum("tv,td->vd", grads, h)
        got = {"loss": torch.tensor(loss, dtype=torch.float64), "lse": torch.cat(lse)}
        return got if dw is None else {**got, "dhidden": torch.cat(dh), "dweight": dw}
    if kind.startswith("distill"):
        T, K, tau, loss, lse, dl = case["T"], case["K"], float(case["tau"]), [], [], []
        teacher, ids = s["teacher"].double().cpu().numpy(), s["ids"].cpu().numpy()
        for lo in range(0, T, 256):
            hi = min(T, lo + 256)
            x = s["logits"][lo:hi].double() / tau
            if s["mask_bits"] is not None:
                x[~_exact_bits(s["mask_bits"], lo, hi, V)] = -math.inf
            z = _exact_lse(x)
            lse.append(z)
            picked = x.gather(1, torch.from_numpy(np.maximum(ids[lo:hi], 0)).long().to(DEV)).cpu().numpy()
            zs, p = z.cpu().numpy(), np.zeros((hi - lo, K))
            for i in range(hi - lo):
                on = np.flatnonzero((ids[lo + i] >= 0) & np.isfinite(picked[i]))
                if not len(on):
                    loss.append(0.0)
                    continue
                t = teacher[lo + i, on] / tau
                logp = t - (np.log(np.exp(t - t.max()).sum()) + t.max())
                p[i, on] = np.exp(logp)
                loss.append(tau * tau * float((p[i, on] * (logp - picked[i, on] + zs[i])).sum()))
            if kind == "distill_step":
                q = torch.exp(x - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
                for k in range(K):
                    at = torch.from_numpy(np.maximum(ids[lo:hi, k], 0)).long().to(DEV)
                    q[torch.arange(hi - lo, device=DEV), at] -= torch.from_numpy(p[:, k]).to(DEV)
                used = torch.from_numpy(p.sum(1) > 0).to(DEV)
                dl.append(q * (s["grad_loss"][lo:hi].double() * tau * used)[:, None])
        got = {"loss": torch.tensor(loss, dtype=torch.float64), "lse": torch.cat(lse)}
        return got if kind == "distill" else {**got, "dlogits": torch.cat(dl)}
    N, D, ids = case["N"], case["D"], s["tokens"].cpu().numpy()
    if kind == "embed":
        out = torch.zeros(N, D, dtype=torch.float64, device=DEV)
        on = torch.from_numpy(np.flatnonzero(ids >= 0)).to(DEV)
        out[on] = s["weight"][s["tokens"].long()[on]].double() * s["scale"]
        return {"out": out}
    dw = torch.zeros(case["V"], D, dtype=torch.float64, device=DEV)
    order = np.argsort(ids, kind="stable")
    uniq, first = np.unique(ids[order], return_index=True)
    sums = torch.zeros(N + 1, D, dtype=torch.float64, device=DEV)
    sums[1:] = torch.cumsum(s["grad"][torch.from_numpy(order).to(DEV)].double(), dim=0)
    ends = np.append(first[1:], N)
    rows = (sums[torch.from_numpy(ends).to(DEV)] - sums[torch.from_numpy(first).to(DEV)]) * s["scale"]
    keep = np.flatnonzero(uniq >= 0)
    dw[torch.from_numpy(uniq[keep]).long().to(DEV)] = rows[torch.from_numpy(keep).to(DEV)]
    return {"dweight": dw}
