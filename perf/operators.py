"""The operators of a transformer's training step and answers, as cases that can be timed and compared.

Three operators: attention (capped scores, distance bias, document, prefix and
causal masks, grouped heads), dropout from a counter-based generator with the
residual sum, and log probabilities of given tokens with entropy and top
alternatives.  ``run`` is one pass through one of them: a training step's
forward and backward, or a forward alone.

``own`` chooses what computes a pass: the framework's kernels
(``paper_2006_09616_amd.ops``), or plain torch operations in 32 bits, rounded
once at the end.  ``exact`` gives the same outputs from the definitions in 64
bits.

A case is a dict.  For attention (op "attention"):
  mode       "train" (out, dq, dk, dv) or "forward" (out)
  B, Sq, Sk  requests, queries and key slots of each
  Hq, Hkv, D heads of the queries, heads of the keys, size of a head
  type       "bf16" or "fp16"
  layout     "separate" (one [B, S, H, D] tensor each), "heads" ([B, H, S, D]
             seen as [B, S, H, D]) or "packed" (views of one projection)
  cap        scores go through cap * tanh(score / cap); 0: they do not
  slopes     a bias of -slope[head] * |distance|
  causal     keys after the query's position are masked
  prefix     each request has a prefix that every query sees
  docs       documents packed in the sequence (0: one, without a mask)
  lengths    keys of each request from this share of Sk on (1.0: all Sk)
For dropout: rows, cols, type, p, residual.  For logprobs: mode "train" or
"score", T rows, V columns, type, top, masked (share of the vocabulary at
minus infinity).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- cases -------------------------------------------------------------------

def _attention(name, mode, B, Sq, Sk, Hq, Hkv, D, type="bf16", layout="separate", cap=0.0, slopes=False, causal=False,
               prefix=False, docs=0, lengths=1.0):
    c = dict(op="attention", mode=mode, B=B, Sq=Sq, Sk=Sk, Hq=Hq, Hkv=Hkv, D=D, type=type, layout=layout, cap=cap,
             slopes=slopes, causal=causal, prefix=prefix, docs=docs, lengths=lengths)
    return dict(name=name, **c) if name else c


def _dropout(name, rows, cols, type="bf16", p=0.1, residual=True):
    c = dict(op="dropout", rows=rows, cols=cols, type=type, p=p, residual=residual)
    return dict(name=name, **c) if name else c


def _logprobs(name, mode, T, V, type="bf16", top=0, masked=0.0):
    c = dict(op="logprobs", mode=mode, T=T, V=V, type=type, top=top, masked=masked)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one request's next token over a short cache: the smallest call, latency is all of it
        _attention("decode one", "forward", 1, 1, 512, 12, 12, 64, lengths=0.5),
        # the next token of many requests over long caches of unequal length: the cache's bytes
        _attention("decode batch", "forward", 32, 1, 16384, 32, 8, 128, layout="heads", cap=30.0, causal=True, lengths=0.5),
        # a handful of drafted tokens checked at once, odd sizes, few requests: split over the keys
        _attention("decode draft", "forward", 3, 5, 30011, 24, 4, 96, type="fp16", slopes=True, causal=True, lengths=0.7),
        # a layer of the encoder that the framework's transformer program describes (hidden 768, 12 heads, 512
        # tokens, batch 8, 2-byte elements), requests padded, a distance bias in place of learned positions
        _attention("encoder step", "train", 8, 512, 512, 12, 12, 64, type="fp16", layout="packed", slopes=True,
                   lengths=0.4),
        # a long packed sequence of a language model's training: documents, causal, capped, shared key heads
        _attention("packed documents step", "train", 1, 8192, 8192, 16, 4, 128, cap=50.0, causal=True, docs=3),
        # long causal sequences with every key in sight: the largest amount of arithmetic
        _attention("long causal step", "train", 4, 4096, 4096, 16, 16, 128, layout="packed", causal=True),
        # prompts with a prefix seen from both sides, odd lengths and head size: answers' first pass
        _attention("prefix prompt", "forward", 2, 2731, 2731, 20, 5, 80, cap=30.0, causal=True, prefix=True, lengths=0.6),
        # the residual sum of the encoder layer, forward and backward
        _dropout("dropout encoder", 8 * 512, 768, type="fp16", p=0.1),
        # the same of a large batch: memory traffic only
        _dropout("dropout large", 32768, 8192, p=0.15),
        # one answer's next tokens with their alternatives: few rows, a long vocabulary
        _logprobs("logprobs answer", "score", 4, 50021, type="fp32", top=8, masked=0.05),
        # the loss of a training step and its gradient
        _logprobs("logprobs step", "train", 4096, 32000),
        # answers scored afterwards: every token's log probability, entropy and alternatives
        _logprobs("logprobs score", "score", 8192, 100003, top=20),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "train", "train", "forward", "dropout", "logprobs", "logprobs"])
    t16 = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "dropout":
        cols = _log_uniform(rng, 1, 16384)
        rows = _log_uniform(rng, 1, max(1, min(65536, 200_000_000 // cols)))
        return _dropout(None, rows, cols, rng.choice(["bf16", "fp16", "fp32"]), round(rng.uniform(0.0, 0.6), 3),
                        rng.random() < 0.7)
    if kind == "logprobs":
        V = _log_uniform(rng, 100, 200_000)
        T = _log_uniform(rng, 1, max(1, min(16384, 250_000_000 // V)))
        mode = rng.choice(["train", "score"])
        return _logprobs(None, mode, T, V, rng.choice(["bf16", "fp16", "fp32"]),
                         0 if mode == "train" else rng.choice([0, 1, 5, rng.randint(1, 32)]),
                         rng.choice([0.0, 0.0, 0.1]))
    Hkv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 4, 6])
    D = rng.choice([64, 64, 128, 128, 8 * rng.randint(4, 16)])
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    slopes = rng.random() < 0.4
    layout = rng.choice(["separate", "heads", "packed"])
    if kind == "decode":
        Sk, B = _log_uniform(rng, 1, 40000), _log_uniform(rng, 1, 48)
        B = max(1, min(B, 400_000_000 // (Sk * Hkv * D)))
        Sq = min(Sk, rng.choice([1, 1, 1, 2, rng.randint(1, 8)]))
        return _attention(None, "forward", B, Sq, Sk, Hkv * group, Hkv, D, t16, layout if layout != "packed" else "heads",
                          cap, slopes, True, False, 0, rng.choice([1.0, 0.3, 0.8]))
    S = _log_uniform(rng, 4, 8192)
    B = max(1, min(_log_uniform(rng, 1, 64), 800_000_000 // (S * S * Hkv * group)))
    while B * S * S * Hkv * group > 1_000_000_000:
        S = S * 3 // 4
    causal = rng.random() < 0.7
    docs = rng.choice([0, 0, 0, rng.randint(2, 9)]) if S >= 64 else 0
    return _attention(None, kind, B, S, S, Hkv * group, Hkv, D, t16, layout, cap, slopes, causal,
                      causal and rng.random() < 0.3, docs, rng.choice([1.0, 0.5]) if not docs else 1.0)


# ---- inputs ------------------------------------------------------------------

def _prepare_attention(c, g, dev):
    B, Sq, Sk, Hq, Hkv, D, dt = c["B"], c["Sq"], c["Sk"], c["Hq"], c["Hkv"], c["D"], TYPES[c["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=dt)

    if c["layout"] == "packed":
        qkv = normal(B, Sq, Hq + 2 * Hkv, D)
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    elif c["layout"] == "heads":
        q, k, v = (normal(B, h, s, D).transpose(1, 2) for h, s in ((Hq, Sq), (Hkv, Sk), (Hkv, Sk)))
    else:
        q, k, v = normal(B, Sq, Hq, D), normal(B, Sk, Hkv, D), normal(B, Sk, Hkv, D)
    if c["cap"]:
        q.mul_(2.5)                                       # scores that a cap is there for
    st = dict(q=q, k=k, v=v, slopes=None, prefix=None, docs=None, lengths=None, starts=None)

    def whole(lo, hi, shape):
        return torch.randint(lo, hi + 1, shape, generator=g, device=dev, dtype=torch.int32)

    if c["slopes"]:                                       # a geometric range over the heads
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=dev, dtype=torch.float32) / Hq)
    if c["lengths"] < 1.0:
        st["lengths"] = whole(max(Sq if Sq < Sk else 1, int(c["lengths"] * Sk)), Sk, (B,))
        if Sq < Sk:                                       # the queries are the last tokens of each request
            st["starts"] = st["lengths"] - Sq
    if c["prefix"]:
        st["prefix"] = whole(0, Sk // 2, (B,))
    if c["docs"]:
        cuts = whole(1, Sk - 1, (B, c["docs"] - 1)).long()
        ends = torch.zeros(B, Sk, dtype=torch.int32, device=dev)
        ends.scatter_add_(1, cuts, torch.ones_like(cuts, dtype=torch.int32))
        st["docs"] = torch.cumsum(ends, 1).to(torch.int32)
    if c["mode"] == "train":
        st["dout"] = normal(B, Sq, Hq, D) * 0.1
        for n in "qkv":
            st[n] = st[n].detach().requires_grad_()
    return st


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    if case["op"] == "attention":
        st = _prepare_attention(case, g, dev)
    elif case["op"] == "dropout":
        shape, dt = (case["rows"], case["cols"]), TYPES[case["type"]]
        x, r, dout = (torch.randn(shape, generator=g, device=dev, dtype=dt) for _ in range(3))
        st = dict(x=x.requires_grad_(), residual=r if case["residual"] else None, dout=dout,
                  seed=(seed * 0x5851F42D4C957F2D + 1) & 0x7FFFFFFFFFFFFFFF, offset=(seed % 1000) * 12345)
    else:
        T, V = case["T"], case["V"]
        x = torch.randn(T, V, generator=g, device=dev, dtype=TYPES[case["type"]]) * 2
        tokens = torch.randint(0, V, (T,), generator=g, device=dev)
        if case["masked"]:
            x.masked_fill_(torch.rand(V, generator=g, device=dev) < case["masked"], -math.inf)
        st = dict(x=x, tokens=tokens)
        if case["mode"] == "train":
            tokens.masked_fill_(torch.rand(T, generator=g, device=dev) < 0.1, -1)      # rows without a token
            st["x"].requires_grad_()
            st["dlogp"] = torch.randn(T, generator=g, device=dev) / T
            st["dentropy"] = torch.full((T,), 0.01 / T, device=dev)
    st["case"] = case
    return st


# ---- a pass ------------------------------------------------------------------

def _own(st):
    from paper_2006_09616_amd import ops
    c = st["case"]
    if c["op"] == "attention":
        out = ops.attention(st["q"], st["k"], st["v"], cap=c["cap"], slopes=st["slopes"], causal=c["causal"],
                            prefix=st["prefix"], docs=st["docs"], lengths=st["lengths"], starts=st["starts"])
        if c["mode"] == "forward":
            return {"out": out}
        dq, dk, dv = torch.autograd.grad(out, (st["q"], st["k"], st["v"]), st["dout"])
        return {"out": out.detach(), "dq": dq, "dk": dk, "dv": dv}
    if c["op"] == "dropout":
        out = ops.dropout_add(st["x"], st["residual"], p=c["p"], seed=st["seed"], offset=st["offset"])
        dx, = torch.autograd.grad(out, (st["x"],), st["dout"])
        return {"out": out.detach(), "dx": dx}
    r = ops.token_logprobs(st["x"], st["tokens"], top=c["top"])
    if c["mode"] == "score":
        res = {"logp": r.logp, "entropy": r.entropy}
        return {**res, "top_logp": r.top_logp, "top_ids": r.top_ids} if c["top"] else res
    dx, = torch.autograd.grad((r.logp, r.entropy), (st["x"],), (st["dlogp"], st["dentropy"]))
    return {"logp": r.logp.detach(), "entropy": r.entropy.detach(), "dx": dx}


def _allowed(c, st, dev):
    """Which key each query sees, [B, 1 or Sq, Sk] (None: every key), and the positions of the queries."""
    Sq, Sk = c["Sq"], c["Sk"]
    pos = torch.arange(Sq, device=dev)[None] + (st["starts"][:, None].long() if st["starts"] is not None else Sk - Sq)
    key = torch.arange(Sk, device=dev)
    ok = None
    if c["causal"]:
        ok = key[None, None] <= pos[:, :, None]
        if st["prefix"] is not None:
            ok = ok | (key[None, None] < st["prefix"][:, None, None])
    if st["lengths"] is not None:
        inside = key[None, None] < st["lengths"][:, None, None]
        ok = inside if ok is None else ok & inside
    if st["docs"] is not None:
        docs = st["docs"]
        same = torch.gather(docs, 1, pos.expand(docs.shape[0], Sq))[:, :, None] == docs[:, None]
        ok = same if ok is None else ok & same
    return ok, pos


def _plain_attention(st):
    c = st["case"]
    B, Sq, Sk, Hq, Hkv, D = (c[n] for n in ("B", "Sq", "Sk", "Hq", "Hkv", "D"))
    G, dt = Hq // Hkv, TYPES[c["type"]]
    scale = 1.0 / math.sqrt(D)

    def heads(x, h):                                     # [B, S, h, D] -> [B, Hkv, (h / Hkv) * S, D]
        return x.detach().float().permute(0, 2, 1, 3).reshape(B, Hkv, h // Hkv * x.shape[1], D).contiguous()

    def back(x, h):
        return x.view(B, h, -1, D).permute(0, 2, 1, 3).to(dt).contiguous()

    q, k, v = heads(st["q"], Hq), heads(st["k"], Hkv), heads(st["v"], Hkv)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(B, Hq, Sq, Sk)
    t = None
    if c["cap"]:
        t = torch.tanh(s / c["cap"])
        s = t * c["cap"]
        if c["mode"] == "forward":
            t = None
    ok, pos = _allowed(c, st, q.device)
    if st["slopes"] is not None:
        dist = (pos[:, :, None] - torch.arange(Sk, device=q.device)).abs().float()
        s.sub_(st["slopes"][None, :, None, None] * dist[:, None])
    if ok is not None:
        s.masked_fill_(~ok[:, None], -math.inf)
    m = s.amax(3, keepdim=True)
    s.sub_(torch.where(torch.isinf(m), torch.zeros_like(m), m)).exp_()
    total = s.sum(3, keepdim=True)
    P = s.div_(torch.where(total == 0, torch.ones_like(total), total)).view(B, Hkv, G * Sq, Sk)
    out = torch.matmul(P, v)
    if c["mode"] == "forward":
        return {"out": back(out, Hq)}
    do = heads(st["dout"], Hq)
    dv = torch.matmul(P.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds.sub_((do * out).sum(3, keepdim=True)).mul_(P)
    if t is not None:
        ds.mul_(1 - (t * t).view(B, Hkv, G * Sq, Sk))
    ds.mul_(scale)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    return {"out": back(out, Hq), "dq": back(dq, Hq), "dk": back(dk, Hkv), "dv": back(dv, Hkv)}


GAMMA = 0x9E3779B97F4A7C15
MIX1, MIX2 = 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def _signed(x):
    x &= (1 << 64) - 1
    return x - (1 << 64) if x >> 63 else x


def _mix(z):
    m = (1 << 64) - 1
    z = ((z ^ (z >> 30)) * MIX1) & m
    z = ((z ^ (z >> 27)) * MIX2) & m
    return z ^ (z >> 31)


def _plain_dropout(st):
    c, x = st["case"], st["x"].detach()
    n = x.numel()
    z = torch.arange((n + 1) // 2, device=x.device).add_(st["offset"])
    z.mul_(_signed(GAMMA)).add_(_signed(_mix((st["seed"] + GAMMA) & ((1 << 64) - 1))))
    z.bitwise_xor_((z >> 30) & ((1 << 34) - 1)).mul_(_signed(MIX1))
    z.bitwise_xor_((z >> 27) & ((1 << 37) - 1)).mul_(_signed(MIX2))
    z.bitwise_xor_((z >> 31) & ((1 << 33) - 1))
    u = torch.stack((z & 0xFFFFFFFF, (z >> 32) & 0xFFFFFFFF), 1).view(-1)[:n].view(x.shape)
    keep = u >= int(c["p"] * 4294967296.0)
    inv = 1.0 / (1.0 - c["p"])
    out = torch.where(keep, x.float() * inv, torch.zeros((), device=x.device))
    if st["residual"] is not None:
        out = out + st["residual"].float()
    dx = torch.where(keep, st["dout"].float() * inv, torch.zeros((), device=x.device))
    return {"out": out.to(x.dtype), "dx": dx.to(x.dtype)}


def _plain_logprobs(st):
    c, x = st["case"], st["x"].detach().float()
    tok = st["tokens"]
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    p = e.div_(total)
    entropy = lse - torch.where(p > 0, p * x, torch.zeros((), device=x.device)).sum(1)
    at = torch.gather(x, 1, tok.clamp_min(0)[:, None])[:, 0]
    logp = torch.where(tok >= 0, at - lse, torch.zeros_like(lse))
    if c["mode"] == "score":
        res = {"logp": logp, "entropy": entropy}
        if c["top"]:
            column = torch.arange(c["V"], device=x.device)
            values, ids = [], []
            left = x.clone()
            for _ in range(c["top"]):                    # the largest left, the lowest index among equals
                best = left.amax(1, keepdim=True)
                first = torch.where(left == best, column, c["V"]).amin(1, keepdim=True)
                values.append(best[:, 0] - lse)
                ids.append(first[:, 0])
                left.scatter_(1, first, -math.inf)
            res.update(top_logp=torch.stack(values, 1), top_ids=torch.stack(ids, 1))
        return res
    g = torch.where(tok >= 0, st["dlogp"], torch.zeros_like(st["dlogp"]))
    logs = torch.where(p > 0, x - lse[:, None] + entropy[:, None], torch.zeros((), device=x.device))
    dx = -p * (g[:, None] + st["dentropy"][:, None] * logs)
    dx.scatter_add_(1, tok.clamp_min(0)[:, None], g[:, None])
    return {"logp": logp, "entropy": entropy, "dx": dx.to(st["x"].dtype)}


def run(state):
    if own:
        return _own(state)
    return {"attention": _plain_attention, "dropout": _plain_dropout, "logprobs": _plain_logprobs}[state["case"]["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------

def work(case):
    size = 4 if case["type"] == "fp32" else 2
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * size * (5 if case["residual"] else 4), "flops": 3.0 * n}
    if case["op"] == "logprobs":
        n, T = case["T"] * case["V"], case["T"]
        if case["mode"] == "train":
            return {"bytes": 2.0 * n * size + 24 * T, "flops": 12.0 * n}
        return {"bytes": float(n * size + T * (16 + 12 * case["top"])), "flops": 6.0 * n}
    B, Sq, Sk, Hq, Hkv, D = (case[n] for n in ("B", "Sq", "Sk", "Hq", "Hkv", "D"))
    share = (1 + case["lengths"]) / 2                    # the mean of lengths drawn evenly
    keys = Sk * share
    if case["causal"] and Sq > Sk // 2:                  # a triangle (cut off at the length) and what the prefix adds
        pairs = Sk * Sk * (share - share * share / 2 + (1 / 24 if case["prefix"] else 0))
        if case["docs"]:                                 # the mean sum of squares of pieces cut at random
            pairs *= 2 / (case["docs"] + 1)
    else:
        pairs = Sq * keys * (2 / (case["docs"] + 1) if case["docs"] else 1)
    q, kv = B * Sq * Hq * D * size, 2 * B * keys * Hkv * D * size
    if case["mode"] == "train":
        return {"bytes": 4.0 * q + 2 * kv, "flops": 14.0 * B * Hq * D * pairs}
    return {"bytes": 2.0 * q + kv, "flops": 4.0 * B * Hq * D * pairs}


# ---- the definitions in 64 bits ---------------------------------------------------

def _exact_attention(c, st):
    """One query head of one request at a time: the sums of the definition, row by row of the score matrix."""
    B, Sq, Sk, Hq, Hkv, D = (c[n] for n in ("B", "Sq", "Sk", "Hq", "Hkv", "D"))
    G, train = Hq // Hkv, c["mode"] == "train"
    q, k, v = (st[n].detach().double() for n in "qkv")
    out = torch.zeros_like(q)
    if train:
        do = st["dout"].double()
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    j = torch.arange(Sk, device=q.device)
    for b in range(B):
        first = int(st["starts"][b]) if st["starts"] is not None else Sk - Sq
        length = int(st["lengths"][b]) if st["lengths"] is not None else Sk
        i = torch.arange(first, first + Sq, device=q.device)[:, None]
        hidden = (j >= length).expand(Sq, Sk)
        if c["causal"]:
            late = j > i
            if st["prefix"] is not None:
                late = late & (j >= int(st["prefix"][b]))
            hidden = hidden | late
        if st["docs"] is not None:
            hidden = hidden | (st["docs"][b][i] != st["docs"][b][None])
        for h in range(Hq):
            kk, vv = k[b, :, h // G].contiguous(), v[b, :, h // G].contiguous()
            qq = q[b, :, h].contiguous()
            raw = qq @ kk.t().contiguous() / math.sqrt(D)
            s = raw
            if c["cap"]:
                s = c["cap"] * torch.tanh(raw / c["cap"])
                slope_of_cap = 1 - (s / c["cap"]) ** 2
            if st["slopes"] is not None:
                s = s - float(st["slopes"][h]) * (i - j).abs()
            s = s.masked_fill(hidden, -math.inf)
            lse = torch.logsumexp(s, 1, keepdim=True)
            p = torch.exp(s - lse).masked_fill(hidden, 0.0)
            out[b, :, h] = p @ vv
            if train:
                g = do[b, :, h].contiguous()
                gp = g @ vv.t().contiguous()
                gs = p * (gp - (p * gp).sum(1, keepdim=True))
                if c["cap"]:
                    gs = gs * slope_of_cap
                gs = gs / math.sqrt(D)
                dq[b, :, h] = gs @ kk
                dk[b, :, h // G] += gs.t().contiguous() @ qq
                dv[b, :, h // G] += p.t().contiguous() @ g
    return {"out": out, "dq": dq, "dk": dk, "dv": dv} if train else {"out": out}


def _exact_dropout(c, st):
    x = st["x"].detach()
    n = x.numel()
    with np.errstate(over="ignore"):
        key = np.uint64(st["seed"]) + np.uint64(GAMMA)
        key = (key ^ (key >> np.uint64(30))) * np.uint64(MIX1)
        key = (key ^ (key >> np.uint64(27))) * np.uint64(MIX2)
        key = key ^ (key >> np.uint64(31))
        u = np.empty(n + n % 2, np.uint32)
        step = 1 << 24
        for lo in range(0, (n + 1) // 2, step):
            hi = min(lo + step, (n + 1) // 2)
            z = np.arange(lo, hi, dtype=np.uint64)
            z += np.uint64(st["offset"])
            z *= np.uint64(GAMMA)
            z += key
            z ^= z >> np.uint64(30)
            z *= np.uint64(MIX1)
            z ^= z >> np.uint64(27)
            z *= np.uint64(MIX2)
            z ^= z >> np.uint64(31)
            u[2 * lo:2 * hi] = z.astype("<u8").view("<u4")
    keep = torch.from_numpy(u[:n] >= np.uint64(math.floor(c["p"] * 2.0 ** 32))).to(x.device).view(x.shape)
    part = keep.double() / (1 - c["p"])
    out = x.double() * part
    if st["residual"] is not None:
        out += st["residual"].double()
    return {"out": out, "dx": st["dout"].double() * part}


def _exact_logprobs(c, st):
    rows = []
    for lo in range(0, c["T"], 1024):
        x = st["x"].detach()[lo:lo + 1024].double()
        tok = st["tokens"][lo:lo + 1024]
        logq = x - torch.logsumexp(x, 1, keepdim=True)
        q = torch.exp(logq)
        given = tok >= 0
        finite = torch.where(q > 0, logq, 0.0)
        entropy = -(q * finite).sum(1)
        one = torch.zeros_like(x)
        one.scatter_(1, tok.clamp_min(0)[:, None], given.double()[:, None])
        r = {"logp": torch.where(given, torch.gather(logq, 1, tok.clamp_min(0)[:, None])[:, 0], 0.0), "entropy": entropy}
        if c["mode"] == "train":
            g = torch.where(given, st["dlogp"][lo:lo + 1024].double(), 0.0)[:, None]
            dh = st["dentropy"][lo:lo + 1024].double()[:, None]
            r["dx"] = g * (one - q) - dh * q * (finite + entropy[:, None])
        elif c["top"]:
            order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :c["top"]]
            r["top_logp"], r["top_ids"] = torch.gather(logq, 1, order), order
        rows.append(r)
    return {n: torch.cat([r[n] for r in rows]) for n in rows[0]}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attention":
        # the score matrices in 64 bits, several passes over each
        if case["B"] * case["Hq"] * case["Sq"] * case["Sk"] > 1.2e9 or case["B"] * case["Hq"] > 1100:
            return None
        return _exact_attention(case, st)
    return {"dropout": _exact_dropout, "logprobs": _exact_logprobs}[case["op"]](case, st)
