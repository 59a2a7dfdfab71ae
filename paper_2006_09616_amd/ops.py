"""Operators of a transformer's training step that store nothing their
backward pass can make again (the C ABI of include/dtr_ops.h).

``attention``        capped, biased, masked attention with grouped heads
``dropout_add``      dropout from a counter-based generator, plus a residual
``token_logprobs``   log probabilities of given tokens, entropy, alternatives

All three run on the current stream of their inputs' device, are
differentiable through ``torch.autograd`` and give the same bits each time
they are run on the same inputs, so that a rematerialized call replaces the
one that was dropped.  The kernels are in ``libdtrsim.so``; there is no
fallback: on anything but a GPU the calls raise.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import NamedTuple, Optional

import torch

from . import dtr

HEADER = os.path.join(os.path.dirname(dtr.HERE), "include", "dtr_ops.h")
TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
TOP_MAX = 32
MAX_STRIDE = 1 << 26


class _Attn(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("type", "batch", "q_len", "k_len", "q_heads", "k_heads", "head_dim", "causal")] + \
               [("scale", C.c_float), ("cap", C.c_float)] + \
               [(n, C.c_void_p) for n in ("slopes", "prefix", "docs", "lengths", "starts")]


class _Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("position", C.c_int64), ("head", C.c_int64)]


_ready = False


def lib():
    """The HIP library with the operators' signatures set (raises if it has not been built)."""
    global _ready
    L = dtr.lib()
    if not _ready:
        vp, i32, i64, sz, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_uint64
        L.dtr_attn_workspace_bytes.argtypes = [vp, i32, vp]
        L.dtr_attn_forward.argtypes = [vp] * 8 + [sz, vp]
        L.dtr_attn_backward.argtypes = [vp] * 12 + [sz, vp]
        L.dtr_dropout_add.argtypes = [i32, i64, i64, vp, i64, vp, i64, vp, i64, C.c_double, u64, u64, vp]
        L.dtr_logprobs_workspace_bytes.argtypes = [i32, i64, i64, i32, vp]
        L.dtr_logprobs_forward.argtypes = [i32, i64, i64, i32, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.dtr_logprobs_backward.argtypes = [i32, i64, i64, i32, vp, i64] + [vp] * 8 + [i64, vp]
        for f in ("dtr_attn_workspace_bytes", "dtr_attn_forward", "dtr_attn_backward", "dtr_dropout_add",
                  "dtr_logprobs_workspace_bytes", "dtr_logprobs_forward", "dtr_logprobs_backward"):
            getattr(L, f).restype = C.c_int
        _ready = True
    return L


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _workspace(n: int, device) -> Optional[torch.Tensor]:
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _on_gpu(name: str, t: torch.Tensor):
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}: the operators run on a GPU")


def _int32(name: str, t, shape, device):
    """A tensor of whole numbers for the kernels (int32, contiguous)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.is_floating_point() or t.is_complex() or t.dtype == torch.bool:
        raise TypeError(f"{name} must be a tensor of whole numbers")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the inputs are on {device}")
    if t.dtype == torch.int64:
        t = t.clamp(-2 ** 31, 2 ** 31 - 1)               # what int32 cannot hold stays out of range
    return t.to(torch.int32).contiguous()


# ---- attention -------------------------------------------------------------------

def _rows(t: torch.Tensor) -> torch.Tensor:
    """t itself where its rows can be read in 16-byte pieces, else a copy."""
    ok = t.numel() == 0 or (t.stride(3) == 1 and t.data_ptr() % 16 == 0 and
                            all(t.stride(d) % 8 == 0 or t.shape[d] == 1 for d in range(3)) and
                            (t.stride(1) < MAX_STRIDE or t.shape[1] == 1))
    return t if ok else t.contiguous()


def _heads(t: torch.Tensor) -> _Heads:
    return _Heads(t.data_ptr(), *(t.stride(d) if t.shape[d] > 1 else 0 for d in range(3)))


def _like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _record(q, k, opts) -> _Attn:
    return _Attn(TYPES[q.dtype], q.shape[0], q.shape[1], k.shape[1], q.shape[2], k.shape[2], q.shape[3],
                 int(opts["causal"]), opts["scale"], opts["cap"],
                 *(_ptr(opts[n]) for n in ("slopes", "prefix", "docs", "lengths", "starts")))


def _attn_forward(q, k, v, opts, want_lse: bool, want_rest: bool = False):
    L = lib()
    with torch.cuda.device(q.device):
        q, k, v = _rows(q), _rows(k), _rows(v)
        rec = _record(q, k, opts)
        out = _like(q)
        lse = torch.empty(q.shape[0], q.shape[2], q.shape[1], dtype=torch.float32, device=q.device) if want_lse else None
        rest = _like(q) if want_rest else None
        n = C.c_size_t(0)
        dtr._check(L.dtr_attn_workspace_bytes(C.byref(rec), 0, C.byref(n)))
        ws = _workspace(n.value, q.device)
        dtr._check(L.dtr_attn_forward(C.byref(rec), C.byref(_heads(q)), C.byref(_heads(k)), C.byref(_heads(v)),
                                      C.byref(_heads(out)), _ptr(rest), _ptr(lse), _ptr(ws), n.value, _stream(q.device)))
    return out, lse, rest


def _attn_backward(q, k, v, out, rest, lse, dout, opts):
    L = lib()
    with torch.cuda.device(q.device):
        q, k, v, out, dout = _rows(q), _rows(k), _rows(v), _rows(out), _rows(dout)
        rec = _record(q, k, opts)
        dq, dk, dv = _like(q), _like(k), _like(v)
        n = C.c_size_t(0)
        dtr._check(L.dtr_attn_workspace_bytes(C.byref(rec), 1, C.byref(n)))
        ws = _workspace(n.value, q.device)
        dtr._check(L.dtr_attn_backward(C.byref(rec), *(C.byref(_heads(t)) for t in (q, k, v, out)), _ptr(rest), _ptr(lse),
                                       *(C.byref(_heads(t)) for t in (dout, dq, dk, dv)), _ptr(ws), n.value,
                                       _stream(q.device)))
    return dq, dk, dv


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, opts):
        out, lse, rest = _attn_forward(q, k, v, opts, True, True)
        ctx.save_for_backward(q, k, v, out, lse, rest)
        ctx.opts = opts
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, _):
        q, k, v, out, lse, rest = ctx.saved_tensors
        return (*_attn_backward(q, k, v, out, rest, lse, dout, ctx.opts), None)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, scale: Optional[float] = None, cap: float = 0.0,
              slopes: Optional[torch.Tensor] = None, causal: bool = False, prefix: Optional[torch.Tensor] = None,
              docs: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
              starts: Optional[torch.Tensor] = None, return_lse: bool = False):
    """Attention of ``q`` [B, Sq, Hq, D] over ``k``, ``v`` [B, Sk, Hk, D] (bf16
    or fp16; Hq a multiple of Hk; D a multiple of 8 up to 128), any strides.

    scale    of the scores, default 1 / sqrt(D)
    cap      scores become cap * tanh(score / cap); 0: they stay
    slopes   [Hq] 32-bit: a bias of -slopes[h] * |distance| (a constant: no
             gradient)
    causal   a query at position p sees keys 0 .. p
    prefix   [B]: keys before prefix[b] are seen by every query (with causal)
    docs     [B, Sk]: a query sees the keys of its own document only
    lengths  [B]: keys from lengths[b] on are masked and not read
    starts   [B]: position of the first query, default Sk - Sq (the queries
             are the last key slots).  For new tokens of requests of unequal
             lengths: lengths - Sq.

    Returns ``out`` like q (contiguous); with ``return_lse`` also the log-sum-
    exp of each row's scores [B, Hq, Sq] (32-bit, no gradient).  Queries that
    see no key give zeros and minus infinity.  Rows that do not start at
    multiples of 16 bytes are copied first."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dim() != 4:
            raise ValueError(f"{name} has {t.dim()} dimensions, expected [batch, length, heads, head size]")
        _on_gpu(name, t)
    if q.dtype not in (torch.bfloat16, torch.float16) or k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError(f"q, k and v are {q.dtype}, {k.dtype} and {v.dtype}, expected one of bfloat16 and float16")
    if k.device != q.device or v.device != q.device:
        raise ValueError("q, k and v are on different devices")
    B, Sq, Hq, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        raise ValueError(f"shapes {tuple(q.shape)}, {tuple(k.shape)} and {tuple(v.shape)} do not belong together")
    Sk, Hk = k.shape[1], k.shape[2]
    if slopes is not None:
        if tuple(slopes.shape) != (Hq,) or slopes.device != q.device:
            raise ValueError(f"slopes must be [{Hq}] on {q.device}")
        slopes = slopes.detach().float().contiguous()
    opts = dict(scale=float(scale) if scale is not None else 1.0 / math.sqrt(D) if D else 1.0, cap=float(cap),
                slopes=slopes, causal=bool(causal), prefix=_int32("prefix", prefix, (B,), q.device),
                docs=_int32("docs", docs, (B, Sk), q.device), lengths=_int32("lengths", lengths, (B,), q.device),
                starts=_int32("starts", starts, (B,), q.device))
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad):
        out, lse = _Attention.apply(q, k, v, opts)
    else:
        out, lse, _ = _attn_forward(q, k, v, opts, return_lse)
    return (out, lse) if return_lse else out


# ---- dropout -----------------------------------------------------------------------

def _as_rows(t: torch.Tensor):
    """(rows, cols, row stride) of a tensor whose elements are evenly spaced
    rows of contiguous columns, or None."""
    if t.is_contiguous():
        return 1, t.numel(), t.numel()
    if t.dim() < 2 or t.stride(-1) != 1 and t.shape[-1] != 1:
        return None
    rows, stride = 1, None
    for d in range(t.dim() - 2, -1, -1):
        if t.shape[d] == 1:
            continue
        if stride is None:
            stride = t.stride(d)
        elif t.stride(d) != stride * rows:
            return None
        rows *= t.shape[d]
    return rows, t.shape[-1], t.shape[-1] if stride is None else stride


def _dropout(x, residual, p, seed, offset):
    L = lib()
    with torch.cuda.device(x.device):
        shapes = [_as_rows(x), _as_rows(residual) if residual is not None else None]
        # rows of columns as they lie, if both inputs have the same ones; else copies
        if shapes[0] is None or (residual is not None and (shapes[1] is None or shapes[0][:2] != shapes[1][:2])):
            x = x.contiguous()
            residual = residual.contiguous() if residual is not None else None
            shapes = [_as_rows(x), _as_rows(residual) if residual is not None else None]
        rows, cols, xs = shapes[0]
        out = _like(x)
        dtr._check(L.dtr_dropout_add(TYPES[x.dtype], rows, cols, x.data_ptr(), xs, _ptr(residual),
                                     shapes[1][2] if residual is not None else 0, out.data_ptr(), cols, p,
                                     seed & (2 ** 64 - 1), offset & (2 ** 64 - 1), _stream(x.device)))
    return out


class _DropoutAdd(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, offset):
        ctx.call = (p, seed, offset)
        return _dropout(x, residual, p, seed, offset)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        dx = _dropout(dout, None, *ctx.call) if ctx.needs_input_grad[0] else None
        return dx, dout if ctx.needs_input_grad[1] else None, None, None, None


def dropout_add(x: torch.Tensor, residual: Optional[torch.Tensor] = None, *, p: float, seed: int,
                offset: int = 0) -> torch.Tensor:
    """``residual + dropout(x)``: elements are dropped with probability p and
    the others divided by 1 - p; one rounding at the end.  bf16, fp16 or fp32.

    The mask is a function of (seed, offset) and of the element's number in
    row-major order of x's shape, not of its strides; it is never stored, and
    the backward pass makes it again.  A call on n elements uses the draws
    offset .. offset + (n + 1) // 2 - 1: calls that share a seed take offsets
    that far apart."""
    _on_gpu("x", x)
    if x.dtype not in TYPES:
        raise TypeError(f"x is {x.dtype}, expected bfloat16, float16 or float32")
    if residual is not None:
        if residual.shape != x.shape or residual.dtype != x.dtype or residual.device != x.device:
            raise ValueError(f"residual is {tuple(residual.shape)} {residual.dtype} on {residual.device}, "
                             f"x is {tuple(x.shape)} {x.dtype} on {x.device}")
    p = float(p)
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"probability {p} is not within 0..1")
    seed, offset = int(seed), int(offset)
    if torch.is_grad_enabled() and (x.requires_grad or (residual is not None and residual.requires_grad)):
        return _DropoutAdd.apply(x, residual, p, seed, offset)
    return _dropout(x, residual, p, seed, offset)


# ---- log probabilities ----------------------------------------------------------------

class TokenLogprobs(NamedTuple):
    logp: torch.Tensor
    entropy: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]


def _logprobs_forward(x, tokens, top):
    L = lib()
    T, V = x.shape
    with torch.cuda.device(x.device):
        logp, entropy, lse = (torch.empty(T, dtype=torch.float32, device=x.device) for _ in range(3))
        top_logp = torch.empty(T, top, dtype=torch.float32, device=x.device) if top else None
        top_ids = torch.empty(T, top, dtype=torch.int64, device=x.device) if top else None
        n = C.c_size_t(0)
        dtr._check(L.dtr_logprobs_workspace_bytes(TYPES[x.dtype], T, V, top, C.byref(n)))
        ws = _workspace(n.value, x.device)
        dtr._check(L.dtr_logprobs_forward(TYPES[x.dtype], T, V, top, x.data_ptr(), x.stride(0), tokens.data_ptr(),
                                          logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), _ptr(top_logp),
                                          _ptr(top_ids), _ptr(ws), n.value, _stream(x.device)))
    return logp, entropy, lse, top_logp, top_ids


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, tokens, top):
        logp, entropy, lse, top_logp, top_ids = _logprobs_forward(x, tokens, top)
        ctx.save_for_backward(x, tokens, entropy, lse, top_ids)
        ctx.top = top
        ctx.set_materialize_grads(False)
        if top:
            ctx.mark_non_differentiable(top_ids)
            return logp, entropy, top_logp, top_ids
        return logp, entropy

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp, dentropy, dtop=None, _=None):
        x, tokens, entropy, lse, top_ids = ctx.saved_tensors
        T, V = x.shape
        dlogp, dentropy, dtop = (g.float().contiguous() if g is not None else None for g in (dlogp, dentropy, dtop))
        with torch.cuda.device(x.device):
            dx = _like(x)
            dtr._check(lib().dtr_logprobs_backward(
                TYPES[x.dtype], T, V, ctx.top, x.data_ptr(), x.stride(0), tokens.data_ptr(), entropy.data_ptr(),
                lse.data_ptr(), _ptr(top_ids), _ptr(dlogp), _ptr(dentropy), _ptr(dtop), dx.data_ptr(), V,
                _stream(x.device)))
        return dx, None, None


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, *, top: int = 0) -> TokenLogprobs:
    """Log probabilities of ``tokens`` [...] under ``logits`` [..., V] (bf16,
    fp16 or fp32), the entropy of each row, and its ``top`` likeliest columns
    with their log probabilities (largest first, the lower column among
    equals; at most 32).  Outputs are 32-bit, top_ids 64-bit.

    A negative token means none: its logp is 0 and has no gradient; a token
    beyond the vocabulary gives NaN.  logp, entropy and top_logp are
    differentiable; the softmax is made again in the backward pass."""
    _on_gpu("logits", logits)
    if logits.dtype not in TYPES:
        raise TypeError(f"logits are {logits.dtype}, expected bfloat16, float16 or float32")
    if logits.dim() < 1 or tokens.shape != logits.shape[:-1]:
        raise ValueError(f"tokens are {tuple(tokens.shape)}, logits {tuple(logits.shape)}")
    if tokens.is_floating_point() or tokens.is_complex() or tokens.dtype == torch.bool:
        raise TypeError("tokens must be whole numbers")
    if tokens.device != logits.device:
        raise ValueError(f"tokens are on {tokens.device}, logits on {logits.device}")
    lead, V, top = logits.shape[:-1], logits.shape[-1], int(top)
    if V == 0:
        raise ValueError("the vocabulary is empty")
    if not 0 <= top <= min(TOP_MAX, V):
        raise ValueError(f"{top} alternatives of a vocabulary of {V} (at most {TOP_MAX})")
    x = logits.reshape(-1, V)
    if x.stride(1) != 1 and V > 1:
        x = x.contiguous()
    tok = tokens.reshape(-1).to(torch.int64).contiguous()
    if torch.is_grad_enabled() and x.requires_grad:
        r = _TokenLogprobs.apply(x, tok, top)
        logp, entropy, top_logp, top_ids = r if top else (*r, None, None)
    else:
        logp, entropy, _, top_logp, top_ids = _logprobs_forward(x, tok, top)
    return TokenLogprobs(logp.view(lead), entropy.view(lead), top_logp.view(*lead, top) if top else None,
                         top_ids.view(*lead, top) if top else None)
