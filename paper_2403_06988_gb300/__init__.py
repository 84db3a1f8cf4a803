"""DOMINO constrained decoding hot path on GB300 (sm_103a).

The compute lives in libdomino.so (C ABI in include/domino.h, kernels in
csrc/).  `_binding` exposes every entry point under its C name; `Domino`
below is a thin holder of one handle that allocates output tensors with torch
and forwards to those entry points.  There is no CPU fallback: without a
built libdomino.so the binding raises ImportError, and compute calls on a
handle created without a GPU raise DominoError(E_NO_DEVICE).
"""
from __future__ import annotations

from typing import Optional, Tuple

from . import _binding as B
from ._binding import DominoError, DTYPE_BF16, DTYPE_F32  # noqa: F401


_T = None        # torch, and its types' codes, once a method below has been called
_CODES = {}


def _torch():
    global _T
    if _T is None:
        import torch
        _CODES.update({torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32})
        _T = torch
    return _T


def _matrix(x, device, what):
    """(rows, columns, elements from a row to the next, type code) of a matrix of contiguous rows on `device`."""
    if x.dim() != 2:
        raise ValueError(f"{what}: a matrix expected, not {tuple(x.shape)}")
    rows, cols = x.shape
    step, one = x.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{what} rows must be contiguous")
    code = _CODES.get(x.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32 or bfloat16")
    if x.get_device() != device:
        raise ValueError(f"{what} must be on the handle's device")
    return rows, cols, step if rows > 1 else cols, code


def _like(x, device, what, rows, cols, code):
    """Elements from a row of x to the next; x is a matrix of this shape and type."""
    got = _matrix(x, device, what)
    if got[0] != rows or got[1] != cols:
        raise ValueError(f"{what}: shape {(rows, cols)} expected, not {got[:2]}")
    if got[3] != code:
        raise TypeError(f"{what} must be of the inputs' type")
    return got[2]


def _words(x, device, dtype, n, what):
    """The address of n contiguous values of a 4-byte type."""
    if x.dtype is not dtype:
        raise TypeError(f"{what} must be {dtype}")
    if x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous values expected, not {tuple(x.shape)}")
    if x.get_device() != device:
        raise ValueError(f"{what} must be on the handle's device")
    return x.data_ptr()


def _mask_words(mask, device, rows, n_tokens):
    if mask is None:
        return None
    if mask.shape != (rows, (n_tokens + 31) >> 5) or mask.element_size() != 4 or not mask.is_contiguous():
        raise ValueError("mask: one contiguous row of ceil(n_tokens / 32) 32-bit words per row expected")
    if mask.get_device() != device:
        raise ValueError("mask must be on the handle's device")
    return mask.data_ptr()


class Domino:
    """One library handle: a vocabulary plus a scanner (+ bracket rules).

    fill_byte: None (default), or a byte value that every output buffer this
    holder allocates is filled with before the call that writes it.  A word a
    kernel leaves unwritten then keeps that pattern (0xAB bytes, say) instead
    of whatever the allocator handed back, so an exact comparison catches it.
    A debugging aid; it costs one fill per output.
    """

    fill_byte: Optional[int] = None

    def __init__(self, device: int = 0):
        self.device = device
        self.h = B.domino_create(device)

    def close(self):
        if self.h:
            B.domino_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- loads ---------------------------------------------------------------
    def load_vocab(self, vocab) -> None:
        B.domino_load_vocab(self.h, vocab.data, vocab.offsets, vocab.n_tokens, vocab.eos_id)

    def load_automaton(self, a) -> None:
        B.domino_load_automaton(self.h, a.delta, a.n_states, a.live, a.accepting, a.start, a.rules, None,
                                a.max_depth)

    @staticmethod
    def from_parts(automaton, vocab, device: int = 0) -> "Domino":
        d = Domino(device)
        d.load_vocab(vocab)
        d.load_automaton(automaton)
        return d

    def info(self) -> dict:
        return B.domino_get_info(self.h)

    def _empty(self, shape, dtype, device):
        import torch
        t = torch.empty(shape, dtype=dtype, device=device)
        if self.fill_byte is not None and t.numel():
            t.view(torch.uint8).fill_(self.fill_byte)
        return t

    # -- compute (torch tensors on this handle's device) -----------------------
    def step_mask(self, states, stacks=None, want_next: bool = False, out_mask=None, out_next=None,
                  stream=None):
        import torch
        b = states.shape[0]
        mask, nxt = out_mask, out_next
        if mask is None or (want_next and nxt is None):
            V, W = B.sizes(self.h)
            if mask is None:
                mask = self._empty((b, W), torch.int32, states.device)
            if want_next and nxt is None:
                nxt = self._empty((b, V), torch.int32, states.device)
        B.domino_step_mask(self.h, states, stacks, b, mask, nxt, stream)
        return mask, nxt

    def step_decode(self, states, stacks, logits, want_logprobs: bool = False, advance: bool = False, out_mask=None,
                    stream=None):
        """Mask step fused with the masked greedy decode: returns (mask, argmax, lse, logprobs or None).
        advance: states (and stacks) are then updated in place by the decoded tokens."""
        import torch
        b = states.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if dtype == DTYPE_F32 and logits.dtype != torch.float32:
            raise TypeError("logits must be float32 or bfloat16")
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        dev = states.device
        mask, lp = out_mask, None
        if mask is None or want_logprobs:
            V, W = B.sizes(self.h)
            if mask is None:
                mask = self._empty((b, W), torch.int32, dev)
            if want_logprobs:
                lp = self._empty((b, V), torch.float32, dev)
        argmax = self._empty(b, torch.int32, dev)
        lse = self._empty(b, torch.float32, dev)
        B.domino_step_decode(self.h, states, stacks, b, logits.data_ptr(), dtype, logits.stride(0), mask, argmax, lse,
                             lp, states if advance else None, stacks if advance else None, stream)
        return mask, argmax, lse, lp

    def precompute_table(self, want_next: bool = True, want_mask: bool = True, stream=None):
        import torch
        info = self.info()
        dev = f"cuda:{self.device}"
        nxt = self._empty((info["n_states"], info["n_tokens"]), torch.int32, dev) if want_next else None
        mask = self._empty((info["n_states"], info["n_words"]), torch.int32, dev) if want_mask else None
        B.domino_precompute_table(self.h, nxt, mask, stream)
        return nxt, mask

    def mask_logits(self, logits, mask, want_lse: bool = True, want_logprobs: bool = False, n_tokens: Optional[int]
                    = None, out=None, stream=None) -> Tuple:
        import torch
        b = logits.shape[0]
        if n_tokens is None and want_logprobs and (out is None or out[2] is None):
            n_tokens = B.sizes(self.h)[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if dtype == DTYPE_F32 and logits.dtype != torch.float32:
            raise TypeError("logits must be float32 or bfloat16")
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        argmax, lse, lp = out if out is not None else (None, None, None)
        if argmax is None:
            argmax = self._empty(b, torch.int32, logits.device)
        if want_lse and lse is None:
            lse = self._empty(b, torch.float32, logits.device)
        if want_logprobs and lp is None:
            lp = self._empty((b, n_tokens), torch.float32, logits.device)
        B.domino_mask_logits(self.h, logits.data_ptr(), dtype, b, logits.stride(0), mask, argmax,
                             lse if want_lse else None, lp if want_logprobs else None, stream)
        return argmax, (lse if want_lse else None), (lp if want_logprobs else None)

    def advance(self, states, stacks, tokens, states_out=None, stacks_out=None, stream=None):
        b = states.shape[0]
        so = states if states_out is None else states_out
        wo = stacks if stacks_out is None else stacks_out
        B.domino_advance(self.h, states, stacks, tokens, b, so, wo, stream)
        return so, wo

    def mask_sample(self, logits, mask, temperature: float, seed: int, offset: int, stream=None):
        """Gumbel-max draw per row from softmax(logits / T) over the allowed tokens (-1: none allowed)."""
        import torch
        b = logits.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        tokens = self._empty(b, torch.int32, logits.device)
        B.domino_mask_sample(self.h, logits, dtype, b, logits.stride(0), mask, temperature, seed, offset, tokens,
                             stream)
        return tokens

    def opportunistic_step(self, logits, states, stacks=None, stream=None):
        """Greedy tokens via opportunistic masking; returns (tokens, number of fallback rows as a tensor)."""
        import torch
        b = logits.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        W = B.sizes(self.h)[1]
        scratch = self._empty((b, W), torch.int32, logits.device)
        tokens = self._empty(b, torch.int32, logits.device)
        n_fb = torch.zeros(1, dtype=torch.int32, device=logits.device)
        B.domino_opportunistic_step(self.h, logits, dtype, b, logits.stride(0), states, stacks, scratch, tokens, n_fb,
                                    stream)
        return tokens, n_fb

    def mask_logits_table(self, logits, table_mask, states, want_lse: bool = True, want_logprobs: bool = False,
                          stream=None) -> Tuple:
        """Table-driven mask + decode: row b's mask is table_mask[states[b]] (DFA only)."""
        import torch
        b = logits.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        argmax = self._empty(b, torch.int32, logits.device)
        lse = self._empty(b, torch.float32, logits.device) if want_lse else None
        lp = self._empty((b, B.sizes(self.h)[0]), torch.float32, logits.device) if want_logprobs else None
        B.domino_mask_logits_table(self.h, logits, dtype, b, logits.stride(0), table_mask, states, argmax, lse, lp,
                                   stream)
        return argmax, lse, lp

    def advance_table(self, table_next, states, tokens, states_out=None, stream=None):
        """Table-driven update: states_out[b] = table_next[states[b], tokens[b]] (DFA only)."""
        so = states if states_out is None else states_out
        B.domino_advance_table(self.h, table_next, states, tokens, states.shape[0], so, stream)
        return so

    # -- losses over the vocabulary, the embedding (no loaded vocabulary needed) -----
    # These methods call the library themselves: of a small call's time, the host's
    # is the larger part.
    def _new(self, shape, dtype, device):
        return _T.empty(shape, dtype=dtype, device=device) if self.fill_byte is None else self._empty(shape, dtype, device)

    def _floats(self, out, i, n, like, what):
        """out[i], or a new fp32 tensor of n values, and its address."""
        x = None if out is None else out[i]
        if x is None:
            x = self._new(n, _T.float32, like.device)
            return x, x.data_ptr()
        return x, _words(x, self.device, _T.float32, n, what)

    def _raw(self, stream):
        """The cudaStream_t of `stream`, or of the handle's device's current one."""
        return _T._C._cuda_getCurrentRawStream(self.device) if stream is None else B._stream(stream)

    def _loss_inputs(self, hidden, weight, targets, mask):
        torch, dev = _torch(), self.device
        rows, dim, hs, code = _matrix(hidden, dev, "hidden")
        V, wd, ws, wcode = _matrix(weight, dev, "weight")
        if wd != dim:
            raise ValueError(f"weight: {dim} columns expected, not {wd}")
        if wcode != code:
            raise TypeError("weight must be of hidden's type")
        return (self.h, hidden.data_ptr(), hs, weight.data_ptr(), ws, code, rows, dim, V,
                _mask_words(mask, dev, rows, V), _words(targets, dev, torch.int32, rows, "targets"))

    def token_loss(self, hidden, weight, targets, mask=None, out=None, stream=None) -> Tuple:
        """Cross entropy of `targets` under the masked softmax of hidden @ weight.T, the logits never kept: (loss,
        lse), fp32 [rows].  hidden [rows, dim], weight [n_tokens, dim] bf16; targets int32 (below 0: none); mask as
        step_mask's or None.  out: (loss, lse) to write to."""
        args = self._loss_inputs(hidden, weight, targets, mask)
        loss, pl = self._floats(out, 0, args[6], hidden, "loss")
        lse, pz = self._floats(out, 1, args[6], hidden, "lse")
        rc = B.lib().domino_token_loss(*args, pl, pz, self._raw(stream))
        if rc:
            B._check("domino_token_loss", rc)
        return loss, lse

    def token_loss_grad(self, hidden, weight, targets, lse, grad_loss, mask=None, out=None, stream=None) -> Tuple:
        """(dhidden, dweight) of sum(grad_loss * loss), lse as token_loss returned it; in the inputs' type."""
        args = self._loss_inputs(hidden, weight, targets, mask)
        code, rows, dim, V = args[5:9]
        dh, dw = out if out is not None else (None, None)
        hs = ws = dim
        if dh is None:
            dh = self._new((rows, dim), hidden.dtype, hidden.device)
        else:
            hs = _like(dh, self.device, "dhidden", rows, dim, code)
        if dw is None:
            dw = self._new((V, dim), weight.dtype, weight.device)
        else:
            ws = _like(dw, self.device, "dweight", V, dim, code)
        rc = B.lib().domino_token_loss_grad(*args, _words(lse, self.device, _T.float32, rows, "lse"),
                                            _words(grad_loss, self.device, _T.float32, rows, "grad_loss"),
                                            dh.data_ptr(), hs, dw.data_ptr(), ws, self._raw(stream))
        if rc:
            B._check("domino_token_loss_grad", rc)
        return dh, dw

    def _distill_inputs(self, logits, teacher, ids, temperature, mask):
        torch, dev = _torch(), self.device
        rows, V, step, code = _matrix(logits, dev, "logits")
        trows, k, tstep, tcode = _matrix(teacher, dev, "teacher")
        if trows != rows or tstep != k:
            raise ValueError(f"teacher: {rows} contiguous rows expected")
        if ids.shape != teacher.shape:
            raise ValueError("ids must have the teacher's shape")
        return (self.h, logits.data_ptr(), code, rows, step, V, _mask_words(mask, dev, rows, V), teacher.data_ptr(),
                tcode, _words(ids, dev, torch.int32, rows * k, "ids"), k, temperature)

    def distill_loss(self, logits, teacher, ids, temperature: float = 1.0, mask=None, out=None, stream=None) -> Tuple:
        """Divergence of the teacher's top logits (teacher, ids [rows, k]; ids below 0: no entry) from the masked
        softmax of logits / temperature, times temperature^2: (loss, lse), fp32 [rows]."""
        args = self._distill_inputs(logits, teacher, ids, temperature, mask)
        loss, pl = self._floats(out, 0, args[3], logits, "loss")
        lse, pz = self._floats(out, 1, args[3], logits, "lse")
        rc = B.lib().domino_distill_loss(*args, pl, pz, self._raw(stream))
        if rc:
            B._check("domino_distill_loss", rc)
        return loss, lse

    def distill_grad(self, logits, teacher, ids, temperature: float, lse, grad_loss, mask=None, out=None, stream=None):
        """d sum(grad_loss * loss) / d logits, in the logits' type; out may be `logits` itself."""
        args = self._distill_inputs(logits, teacher, ids, temperature, mask)
        rows, V = args[3], args[5]
        step = V
        if out is None:
            out = self._new((rows, V), logits.dtype, logits.device)
        else:
            step = _like(out, self.device, "out", rows, V, args[2])
        rc = B.lib().domino_distill_grad(*args, _words(lse, self.device, _T.float32, rows, "lse"),
                                         _words(grad_loss, self.device, _T.float32, rows, "grad_loss"),
                                         out.data_ptr(), step, self._raw(stream))
        if rc:
            B._check("domino_distill_grad", rc)
        return out

    def embed(self, tokens, weight, scale: float = 1.0, out=None, stream=None):
        """scale * weight[tokens], zeros for tokens below 0: [n, dim] of the weight's type."""
        torch, dev = _torch(), self.device
        V, dim, ws, code = _matrix(weight, dev, "weight")
        n = tokens.numel()
        pt = _words(tokens, dev, torch.int32, n, "tokens")
        step = dim
        if out is None:
            out = self._new((n, dim), weight.dtype, weight.device)
        else:
            step = _like(out, dev, "out", n, dim, code)
        rc = B.lib().domino_embed(self.h, pt, n, weight.data_ptr(), ws, code, V, dim, scale, out.data_ptr(), step,
                                  self._raw(stream))
        if rc:
            B._check("domino_embed", rc)
        return out

    def embed_grad(self, tokens, grad, n_tokens: int, scale: float = 1.0, into=None, stream=None):
        """Gradient of the table [n_tokens, dim]: scale * the sums of grad's rows by token.  into: a gradient that the
        sums are added to (the loss's, for a table that is its weight too)."""
        torch, dev = _torch(), self.device
        n, dim, gs, code = _matrix(grad, dev, "grad")
        pt = _words(tokens, dev, torch.int32, n, "tokens")
        dw, step = into, dim
        if dw is None:
            dw = self._new((n_tokens, dim), grad.dtype, grad.device)
        else:
            step = _like(dw, dev, "into", n_tokens, dim, code)
        rc = B.lib().domino_embed_grad(self.h, pt, n, grad.data_ptr(), gs, code, n_tokens, dim, scale,
                                       0 if into is None else 1, dw.data_ptr(), step, self._raw(stream))
        if rc:
            B._check("domino_embed_grad", rc)
        return dw

    def device_error(self, stream=None) -> int:
        return B.domino_get_device_error(self.h, stream)
