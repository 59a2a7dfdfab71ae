"""Operators of a transformer's training step that store nothing their
backward pass can make again.

``attention``        capped, biased, masked attention with grouped heads
``dropout_add``      dropout from a counter-based generator, plus a residual
``token_logprobs``   log probabilities of given tokens, entropy, alternatives

All three run on the current stream of their inputs' device, are
differentiable (once: with create_graph the gradients raise when they are
differentiated again) through ``torch.autograd`` and give the same bits each
time they are run on the same inputs, so that a rematerialized call replaces
the one that was dropped.  The kernels are in ``libdtrsim.so`` behind the C ABI
of include/dtr_ops.h; ``_ops.so`` puts torch tensors through it.  There is no
fallback: on anything but a GPU the calls raise.

Errors: ValueError and TypeError for tensors that do not fit together,
``dtr.DtrError`` for what the C ABI refuses, and NotImplementedError for
forward-mode differentiation and ``torch.jit.trace``.
"""
from __future__ import annotations

import os
from operator import index
from typing import NamedTuple, Optional

import torch

from . import dtr

HEADER = os.path.join(os.path.dirname(dtr.HERE), "include", "dtr_ops.h")
BINDING = os.path.join(dtr.HERE, "_ops.so")
TOP_MAX = 32

_binding = None


def lib():
    """The binding (raises if it or the HIP library has not been built)."""
    global _binding
    if _binding is None:
        dtr.lib()
        if not os.path.exists(BINDING):
            raise RuntimeError(f"{BINDING} is missing: build it with __graft_entry__.build()")
        from . import _ops
        _binding = _ops
    return _binding


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, scale: Optional[float] = None, cap: float = 0.0,
              slopes: Optional[torch.Tensor] = None, causal: bool = False, prefix: Optional[torch.Tensor] = None,
              docs: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
              starts: Optional[torch.Tensor] = None, return_lse: bool = False):
    """Attention of ``q`` [B, Sq, Hq, D] over ``k``, ``v`` [B, Sk, Hk, D] (bf16
    or fp16; Hq a multiple of Hk; D a multiple of 8 up to 128), any strides.

    scale    of the scores, default 1 / sqrt(D)
    cap      scores become cap * tanh(score / cap); 0: they stay
    slopes   [Hq]: a bias of -slopes[h] * |distance| (a constant: no gradient)
    causal   a query at position p sees keys 0 .. p
    prefix   [B]: keys before prefix[b] are seen by every query (with causal)
    docs     [B, Sk], of at most 32 bits: a query sees the keys of its own
             document only
    lengths  [B]: keys from lengths[b] on are masked and not read
    starts   [B]: position of the first query, default Sk - Sq (the queries
             are the last key slots).  For new tokens of requests of unequal
             lengths: lengths - Sq.

    Returns ``out`` like q (contiguous); with ``return_lse`` also the log-sum-
    exp of each row's scores [B, Hq, Sq] (32-bit, no gradient).  Queries that
    see no key give zeros and minus infinity.  Rows that do not start at
    multiples of 16 bytes are copied first."""
    out, lse = (_binding or lib()).attention(q, k, v, scale, cap, slopes, causal, prefix, docs, lengths, starts, return_lse)
    return (out, lse) if return_lse else out


def dropout_add(x: torch.Tensor, residual: Optional[torch.Tensor] = None, *, p: float, seed: int,
                offset: int = 0) -> torch.Tensor:
    """``residual + dropout(x)``: elements are dropped with probability p and
    the others divided by 1 - p; one rounding at the end.  bf16, fp16 or fp32.

    The mask is a function of (seed, offset) and of the element's number in
    row-major order of x's shape, not of its strides; it is never stored, and
    the backward pass makes it again.  A call on n elements uses the draws
    offset .. offset + (n + 1) // 2 - 1: calls that share a seed take offsets
    that far apart.  seed and offset count modulo 2^64."""
    m = 0xFFFFFFFFFFFFFFFF
    return (_binding or lib()).dropout_add(x, residual, p, index(seed) & m, index(offset) & m)


class TokenLogprobs(NamedTuple):
    logp: torch.Tensor
    entropy: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, *, top: int = 0) -> TokenLogprobs:
    """Log probabilities of ``tokens`` [...] under ``logits`` [..., V] (bf16,
    fp16 or fp32), the entropy of each row, and its ``top`` likeliest columns
    with their log probabilities (largest first, the lower column among
    equals; at most 32).  Outputs are 32-bit, top_ids 64-bit.

    A negative token means none: its logp is 0 and has no gradient; a token
    beyond the vocabulary gives NaN.  logp, entropy and top_logp are
    differentiable; the softmax is made again in the backward pass."""
    return TokenLogprobs(*(_binding or lib()).token_logprobs(logits, tokens, top))
