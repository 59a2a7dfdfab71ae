"""The operators on the GPU against their definitions in 64 bits.

Tolerances are bounds, element by element, derived from what the kernels
round: u is the unit roundoff of the tensors' type (2^-8 bf16, 2^-11 fp16,
2^-24 fp32), every sum and statistic is held in 32 bits, and probabilities and
score gradients are rounded to the tensors' type once, before a product."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}       # half the smallest fp16 step
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2006_09616_amd import ops as O
    O.lib()
    return O


# ---- attention --------------------------------------------------------------------

def definition(q, k, v, do, scale, cap, slopes, causal, prefix, docs, lengths, starts):
    """out, lse, dq, dk, dv in 64 bits and, for each, the bound of what the
    kernels' roundings come to."""
    u, tiny = U[q.dtype], TINY[q.dtype]
    q, k, v, do = (t.detach().double().cpu() for t in (q, k, v, do))
    B, Sq, Hq, D = q.shape
    Sk, Hk = k.shape[1], k.shape[2]
    res = {n: torch.zeros_like(t) for n, t in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    tol = {n: torch.zeros_like(t) for n, t in res.items()}
    res["lse"] = torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64)
    tol["lse"] = torch.zeros(B, Hq, Sq, dtype=torch.float64)
    j = torch.arange(Sk)[None]
    for b in range(B):
        p = (torch.arange(Sq) + (int(starts[b]) if starts is not None else Sk - Sq))[:, None]
        seen = (j < (int(lengths[b]) if lengths is not None else Sk)).expand(Sq, Sk).clone()
        if causal:
            seen &= (j <= p) | (j < (int(prefix[b]) if prefix is not None else 0))
        if docs is not None:
            d = docs[b].cpu()
            inside = (p >= 0) & (p < Sk)
            seen &= inside & (d[p.clamp(0, max(Sk - 1, 0))] == d[None])
        for h in range(Hq):
            Q, G = q[b, :, h], do[b, :, h]
            K, V = k[b, :, h // (Hq // Hk)].clone(), v[b, :, h // (Hq // Hk)].clone()
            unseen = ~seen.any(0)
            K[unseen] = 0                                 # values that no query sees may be anything
            V[unseen] = 0
            r = scale * Q @ K.T
            mag = scale * Q.abs() @ K.abs().T
            s, dc = r, torch.ones_like(r)
            if cap:
                t = torch.tanh(r / cap)
                s, dc = cap * t, 1 - t * t
            dist = (p - j).abs().double()
            sl = float(slopes[h]) if slopes is not None else 0.0
            s = (s - sl * dist).masked_fill(~seen, -math.inf)
            L = torch.logsumexp(s, 1, keepdim=True) if Sk else torch.full((Sq, 1), -math.inf, dtype=torch.float64)
            empty = ~seen.any(1, keepdim=True)
            P = torch.where(seen, torch.exp(s - L), 0.0)
            # relative error of a probability that 32-bit scores and statistics leave: the product's sum
            # over D, tanh and exp2 to a few units of 2^-24, and the sum over Sk
            e = (2.0 ** -20 * (1 + mag) + cap * 2.0 ** -20 + sl * dist * 2.0 ** -22 + 2.0 ** -24 * s.abs().nan_to_num(0, 0, 0) * 8)
            e = torch.where(seen, e, 0.0)
            e = e + (P * e).sum(1, keepdim=True) + 2.0 ** -22 * math.sqrt(Sk + 1)
            out = P @ V
            # p is rounded relative to the running maximum, so that P = 1 is at least 2^-25 of it away
            et = u * P + e * P + tiny * seen
            t_out = et @ V.abs() + u * out.abs() + tiny
            g = h // (Hq // Hk)
            res["out"][b, :, h], tol["out"][b, :, h] = out, t_out
            res["lse"][b, h] = L[:, 0]
            tol["lse"][b, h] = torch.where(empty[:, 0], 0.0, (P * e).sum(1) + 2.0 ** -20 * (1 + L[:, 0].abs().nan_to_num(0, 0, 0)))
            dP = G @ V.T
            Dl = (G * out).sum(1, keepdim=True)
            dS = P * (dP - Dl)
            t_D = (G.abs() * t_out).sum(1, keepdim=True) + 2.0 ** -21 * (G * out).abs().sum(1, keepdim=True)
            t_dS = (u + e) * dS.abs() + P * (t_D + 2.0 ** -20 * (G.abs() @ V.abs().T)) + tiny * seen
            if cap:
                t_dS = t_dS * dc + dS.abs() * 2.0 ** -19 * (1 + mag / cap)
                dS = dS * dc
            t_P = (u + e) * P + tiny * seen
            res["dq"][b, :, h] = scale * dS @ K
            tol["dq"][b, :, h] = scale * t_dS @ K.abs() + u * res["dq"][b, :, h].abs() + tiny
            res["dk"][b, :, g] += scale * dS.T @ Q
            tol["dk"][b, :, g] += scale * t_dS.T @ Q.abs()
            res["dv"][b, :, g] += P.T @ G
            tol["dv"][b, :, g] += t_P.T @ G.abs()
    for n in ("dk", "dv"):
        tol[n] += u * res[n].abs() + tiny
    return res, tol


def close(got, want, tol, label):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, label
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{label}: infinities differ"
    bad = ~((got - want).abs() <= tol) & ~inf
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{label}: {int(bad.sum())} of {bad.numel()} off, first {i}: {float(got[i])} for "
                             f"{float(want[i])} +- {float(tol[i])}")


def inputs(B, Sq, Sk, Hq, Hk, D, dtype, layout="separate", seed=0, gain=1.0):
    g = torch.Generator().manual_seed(seed * 7919 + Sq * 131 + Sk * 17 + D)

    def normal(*shape, a=1.0):
        return (torch.randn(*shape, generator=g) * a).to(dtype).cuda()

    if layout == "packed":
        x = normal(B, Sq, Hq + 2 * Hk, D)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hk], x[:, :, Hq + Hk:]
    elif layout == "heads":
        q, k, v = (normal(B, h, s, D).transpose(1, 2) for h, s in ((Hq, Sq), (Hk, Sk), (Hk, Sk)))
    elif layout == "offset":                             # rows at odd multiples of 2 bytes: copied
        q, k, v = (normal(B, s, h, D + 3)[..., 1:D + 1] for h, s in ((Hq, Sq), (Hk, Sk), (Hk, Sk)))
    elif layout == "time":                               # [S, B, H, D]
        q, k, v = (normal(s, B, h, D).transpose(0, 1) for h, s in ((Hq, Sq), (Hk, Sk), (Hk, Sk)))
    else:
        q, k, v = normal(B, Sq, Hq, D), normal(B, Sk, Hk, D), normal(B, Sk, Hk, D)
    q, k, v = (t.detach().requires_grad_() for t in (q * gain if gain != 1.0 else q, k, v))
    return q, k, v, normal(B, Sq, Hq, D, a=0.25)


def check(ops, q, k, v, do, label, scale=None, cap=0.0, slopes=None, causal=False, prefix=None, docs=None, lengths=None,
          starts=None, backward=True):
    print(label, flush=True)
    scale_ = scale if scale is not None else q.shape[3] ** -0.5
    dev = [t.cuda() if t is not None else None for t in (slopes, prefix, docs, lengths, starts)]
    kw = dict(scale=scale, cap=cap, slopes=dev[0], causal=causal, prefix=dev[1], docs=dev[2], lengths=dev[3], starts=dev[4])
    want, tol = definition(q, k, v, do, scale_, cap, slopes, causal, prefix, docs, lengths, starts)
    if not backward:
        with torch.no_grad():
            out, lse = ops.attention(q, k, v, return_lse=True, **kw)
        close(out, want["out"], tol["out"], label + " out")
        close(lse, want["lse"], tol["lse"], label + " lse")
        return
    out, lse = ops.attention(q, k, v, return_lse=True, **kw)
    close(out, want["out"], tol["out"], label + " out")
    close(lse, want["lse"], tol["lse"], label + " lse")
    grads = torch.autograd.grad(out, (q, k, v), do)
    for n, t in zip(("dq", "dk", "dv"), grads):
        close(t, want[n], tol[n], f"{label} {n}")


LENGTHS = [(1, 1), (1, 2), (2, 1), (3, 5), (31, 31), (32, 33), (33, 32), (64, 64), (65, 63), (127, 129), (128, 128),
           (130, 257), (200, 77)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_lengths(ops, dtype, causal):
    for i, (Sq, Sk) in enumerate(LENGTHS):
        q, k, v, do = inputs(2, Sq, Sk, 4, 2, 64, dtype, seed=i)
        check(ops, q, k, v, do, f"{dtype} causal {causal} {Sq} {Sk}", causal=causal)


@pytest.mark.parametrize("D", [8, 16, 24, 40, 56, 64, 72, 80, 96, 104, 128])
def test_attention_head_sizes(ops, D):
    for i, (dtype, cap) in enumerate(((BF, 0.0), (FP, 5.0))):
        q, k, v, do = inputs(1, 70, 70, 3, 1, D, dtype, seed=i, gain=2.0)
        check(ops, q, k, v, do, f"head size {D} {dtype}", cap=cap, causal=True, slopes=torch.tensor([0.5, 0.1, 0.0]))


@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (6, 2), (5, 5), (8, 1), (48, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_grouped_heads(ops, heads, D):
    Hq, Hk = heads
    q, k, v, do = inputs(2, 37, 90, Hq, Hk, D, BF, seed=Hq)
    check(ops, q, k, v, do, f"heads {heads} {D}", causal=True, cap=20.0)


@pytest.mark.parametrize("layout", ["packed", "heads", "offset", "time"])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_attention_layouts(ops, layout, dtype):
    q, k, v, do = inputs(3, 75, 75, 4, 2, 64, dtype, layout)
    check(ops, q, k, v, do, f"layout {layout}", causal=True)
    # the output's gradient in an order of its own
    do = do.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    check(ops, q, k, v, do, f"layout {layout}, gradient by heads", causal=False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 3.0, 50.0])
@pytest.mark.parametrize("bias", [False, True])
def test_attention_scores(ops, D, cap, bias):
    slopes = torch.tensor([1.0, 0.25, 0.01, 0.0]) if bias else None
    for causal in (False, True):
        q, k, v, do = inputs(1, 150, 150, 4, 2, D, BF, gain=4.0, seed=int(cap))
        check(ops, q, k, v, do, f"cap {cap} bias {bias} causal {causal} {D}", cap=cap, slopes=slopes, causal=causal)
    q, k, v, do = inputs(1, 40, 190, 4, 2, D, FP, seed=int(cap))
    check(ops, q, k, v, do, f"scale, cap {cap} bias {bias} {D}", cap=cap, slopes=slopes, scale=0.37)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attention_masks(ops, dtype):
    i32 = torch.int32
    # prefixes: none, inside a tile, at a tile's end, beyond the keys, negative
    q, k, v, do = inputs(5, 140, 140, 2, 1, 64, dtype)
    check(ops, q, k, v, do, "prefix", causal=True, prefix=torch.tensor([0, 37, 128, 500, -4], dtype=i32))
    # lengths: none, one key, inside a tile, all, beyond the slots (clamped), negative (clamped)
    q, k, v, do = inputs(6, 70, 130, 2, 1, 64, dtype)
    for causal in (False, True):
        check(ops, q, k, v, do, f"lengths causal {causal}", causal=causal,
              lengths=torch.tensor([0, 1, 67, 130, 999, -3], dtype=i32).clamp(0, 130))
    # positions before the first key, across it, after the last key
    q, k, v, do = inputs(4, 70, 130, 2, 1, 64, dtype)
    check(ops, q, k, v, do, "starts", causal=True, starts=torch.tensor([-200, -30, 64, 300], dtype=i32),
          slopes=torch.tensor([0.3, 0.02]))
    # documents: packed, of one token, in any order, positions outside the keys
    docs = torch.zeros(4, 200, dtype=i32)
    docs[0, 64:] = 1
    docs[1] = torch.arange(200) // 7
    docs[2] = torch.arange(200)
    docs[3] = torch.randint(0, 3, (200,), generator=torch.Generator().manual_seed(3)).to(i32) - 1
    q, k, v, do = inputs(4, 200, 200, 4, 2, 64, dtype)
    for causal in (False, True):
        check(ops, q, k, v, do, f"documents causal {causal}", causal=causal, docs=docs)
    q, k, v, do = inputs(4, 90, 200, 4, 2, 64, dtype)
    check(ops, q, k, v, do, "documents, positions outside", docs=docs, starts=torch.tensor([-20, 150, 0, 250], dtype=i32))
    check(ops, q, k, v, do, "all masks", causal=True, docs=docs, prefix=torch.tensor([10, 100, 3, 0], dtype=i32),
          lengths=torch.tensor([180, 101, 200, 64], dtype=i32), starts=torch.tensor([100, 90, 110, 0], dtype=i32), cap=8.0,
          slopes=torch.tensor([0.1, 0.2, 0.0, 1.0]))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_long_documents(ops, dtype, D):
    """Many tiles, most of them skipped."""
    S = 1500
    docs = (torch.arange(S)[None] // 190).to(torch.int32)
    q, k, v, do = inputs(1, S, S, 2, 1, D, dtype)
    check(ops, q, k, v, do, f"long documents {D}", causal=True, docs=docs, cap=30.0)


@pytest.mark.parametrize("dtype,D,group", [(BF, 64, 1), (FP, 64, 4), (BF, 128, 8), (FP, 80, 6), (BF, 96, 3)])
def test_attention_few_tokens(ops, dtype, D, group):
    """New tokens over caches: one to nine queries, keys split over workgroups and joined."""
    for i, (B, Sq, Sk) in enumerate(((1, 1, 1), (2, 1, 63), (1, 1, 700), (3, 1, 2049), (2, 5, 3000), (1, 9, 5003), (5, 2, 517))):
        q, k, v, do = inputs(B, Sq, Sk, 2 * group, 2, D, dtype, "heads" if i % 2 else "separate", seed=i)
        lengths = torch.tensor([max(Sq, Sk - 37 * b * (Sk // 150)) for b in range(B)], dtype=torch.int32)
        if B > 2:
            lengths[1] = 0
        check(ops, q, k, v, do, f"few tokens {B} {Sq} {Sk} {D}", causal=True, lengths=lengths, starts=lengths - Sq,
              cap=15.0 if i % 3 == 0 else 0.0, slopes=torch.rand(2 * group) if i % 2 else None, backward=False)
    q, k, v, do = inputs(2, 100, 2500, group, 1, D, dtype)
    check(ops, q, k, v, do, f"split with more rows {D}", causal=False, backward=False)


def test_attention_nothing_beyond_the_length(ops):
    """NaN and infinities in the padding of a cache."""
    q, k, v, do = inputs(2, 30, 300, 2, 1, 64, BF)
    lengths = torch.tensor([77, 0], dtype=torch.int32)
    for b in range(2):
        k.data[b, int(lengths[b]):] = float("nan")
        v.data[b, int(lengths[b]):] = float("inf")
    check(ops, q, k, v, do, "padding", lengths=lengths)
    check(ops, q, k, v, do, "padding, split", lengths=lengths, backward=False)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Sq,Sk", [(150, 150), (20, 150), (7, 150), (150, 1300)])
def test_attention_infinities_and_nan_of_other_queries(ops, dtype, D, Sq, Sk):
    """Keys and values that are not numbers reach the queries that see them,
    and no others, also where both are worked on together."""
    q, k, v, do = inputs(1, Sq, Sk, 2, 1, D, dtype)
    a, b, c = Sk - Sq // 3 * 2, Sk - Sq // 3 - 1, Sk - 1  # seen by about two thirds, one third and one of the queries
    want, tol = definition(q, k, v, do, D ** -0.5, 0.0, None, True, None, None, None, None)
    clean = v.detach().clone()
    clean[0, a, 0, 3] = clean[0, b, 0, 5] = 0             # only these columns change
    want, tol = definition(q, k, clean, do, D ** -0.5, 0.0, None, True, None, None, None, None)
    v.data[0, a, 0, 3] = float("nan")
    v.data[0, b, 0, 5] = float("-inf")
    k.data[0, c] = float("nan")
    out = ops.attention(q, k, v, causal=True)
    with torch.no_grad():
        assert torch.equal(ops.attention(q, k, v, causal=True).nan_to_num(7, 8, 9), out.detach().nan_to_num(7, 8, 9))
    got = out.detach().cpu().double()
    pos = torch.arange(Sq) + Sk - Sq
    assert torch.isnan(got[0, pos >= c]).all()
    assert torch.isnan(got[0, pos >= a][:, :, 3]).all()
    assert (got[0, (pos >= b) & (pos < c)][:, :, 5] == -math.inf).all()
    ok = torch.ones_like(got, dtype=torch.bool)
    ok[0, pos >= c] = False
    ok[0, pos >= a, :, 3] = False
    ok[0, pos >= b, :, 5] = False
    assert torch.isfinite(got[ok]).all()
    assert ((got - want["out"]).abs() <= tol["out"])[ok].all()
    dq, = torch.autograd.grad(out, q, do)
    rows = pos < a
    assert ((dq.cpu().double() - want["dq"]).abs() <= tol["dq"])[0, rows].all()
    assert torch.isnan(dq[0, (pos >= a).cuda()]).any(-1).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_attention_a_document_of_nan(ops, dtype, D):
    """A document of nothing but NaN leaves the others' outputs and gradients alone."""
    S = 200
    docs = torch.zeros(1, S, dtype=torch.int32)
    docs[0, 40:75] = 1
    docs[0, 130:190:2] = 1
    bad = (docs[0] == 1)
    for causal in (False, True):
        q, k, v, do = inputs(1, S, S, 4, 2, D, dtype)
        kw = dict(scale=D ** -0.5, cap=0.0, slopes=None, causal=causal, prefix=None, docs=docs, lengths=None, starts=None)
        want, tol = definition(q, k, v, do, *kw.values())
        for t in (q, k, v, do):
            t.data[:, bad.cuda()] = float("nan")
        out = ops.attention(q, k, v, causal=causal, docs=docs.cuda())
        grads = torch.autograd.grad(out, (q, k, v), do)
        for n, t in zip(("out", "dq", "dk", "dv"), (out.detach(), *grads)):
            t = t.cpu().double()
            assert torch.isnan(t[:, bad]).all(), n
            close(t[:, ~bad], want[n][:, ~bad], tol[n][:, ~bad], f"{n} causal {causal}")


def test_attention_gradient_alone_is_not_a_number(ops):
    """A NaN in the output's gradient of one query reaches the values and keys that it sees only."""
    q, k, v, do = inputs(1, 160, 160, 2, 2, 64, BF)
    want, tol = definition(q, k, v, torch.cat([do[:, :70], torch.zeros_like(do[:, 70:71]), do[:, 71:]], 1), 0.125, 0.0, None,
                           True, None, None, None, None)
    do.data[:, 70] = float("nan")
    dq, dk, dv = torch.autograd.grad(ops.attention(q, k, v, causal=True), (q, k, v), do)
    assert torch.isnan(dv[:, :71]).all() and torch.isnan(dk[:, :71]).all() and torch.isnan(dq[:, 70]).all()
    close(dv[:, 71:], want["dv"][:, 71:], tol["dv"][:, 71:], "dv")
    close(dk[:, 71:], want["dk"][:, 71:], tol["dk"][:, 71:], "dk")
    keep = torch.arange(160) != 70
    close(dq[:, keep.cuda()], want["dq"][:, keep], tol["dq"][:, keep], "dq")


def test_attention_lengths_out_of_range(ops):
    """Lengths beyond the key slots count as all of them, negative ones as none."""
    q, k, v, do = inputs(2, 20, 90, 2, 1, 64, FP)
    with torch.no_grad():
        for bad, good in (([1000, -7], [90, 0]), ([2 ** 31 - 1, -2 ** 31], [90, 0])):
            a = ops.attention(q, k, v, lengths=torch.tensor(bad, dtype=torch.int64).cuda())
            b = ops.attention(q, k, v, lengths=torch.tensor(good, dtype=torch.int32).cuda())
            assert torch.equal(a, b)
        far = ops.attention(q, k, v, causal=True, starts=torch.tensor([2 ** 40, -2 ** 40]).cuda())
        assert torch.equal(far[0], ops.attention(q, k, v)[0]) and not far[1].any()


def test_attention_empty(ops):
    dev = "cuda"
    for B, Sq, Sk in ((0, 4, 4), (2, 0, 5), (2, 5, 0), (1, 0, 0)):
        q = torch.randn(B, Sq, 4, 64, device=dev, dtype=BF, requires_grad=True)
        k, v = (torch.randn(B, Sk, 2, 64, device=dev, dtype=BF, requires_grad=True) for _ in range(2))
        out, lse = ops.attention(q, k, v, return_lse=True)
        assert out.shape == q.shape and not out.any()
        assert (lse == -math.inf).all()
        for t, g in zip((q, k, v), torch.autograd.grad(out, (q, k, v), torch.ones_like(out))):
            assert g.shape == t.shape and not g.any()


def test_attention_shared_inputs(ops):
    """Gradients of keys that are broadcast over the batch and of one tensor used three times."""
    q, k, v, do = inputs(3, 50, 50, 4, 2, 64, BF)
    k1, v1 = k.detach()[:1].requires_grad_(), v.detach()[:1].requires_grad_()
    ke, ve = k1.expand(3, -1, -1, -1), v1.expand(3, -1, -1, -1)
    want, tol = definition(q, ke, ve, do, 0.125, 0.0, None, True, None, None, None, None)
    out = ops.attention(q, ke, ve, causal=True)
    dk, dv = torch.autograd.grad(out, (k1, v1), do)
    # the sum over the batch is torch's, in bf16: at most a rounding of each partial sum
    for n, g in (("dk", dk), ("dv", dv)):
        close(g, want[n].sum(0, keepdim=True), tol[n].sum(0, keepdim=True) + 3 * U[BF] * want[n].abs().sum(0, keepdim=True), n)
    x = torch.randn(2, 33, 3, 64, device="cuda", dtype=BF, requires_grad=True)
    out = ops.attention(x, x, x)
    g, = torch.autograd.grad(out, x, torch.ones_like(out))
    want, tol = definition(x, x, x, torch.ones_like(out), 0.125, 0.0, None, False, None, None, None, None)
    total = want["dq"] + want["dk"] + want["dv"]
    size = want["dq"].abs() + want["dk"].abs() + want["dv"].abs()
    close(g, total, tol["dq"] + tol["dk"] + tol["dv"] + 3 * U[BF] * size, "one tensor")


def test_attention_differences(ops):
    """The gradient against central differences of the forward pass, along
    random directions.  In fp16 with n queries the forward's rounding, u |out|,
    limits a difference: it is summed over the outputs as independent errors
    (six standard deviations), and the third derivative's term is h^2."""
    g = torch.Generator().manual_seed(5)
    B, S, H, D = 1, 40, 2, 64
    base = [torch.randn(B, S, H, D, generator=g).half() for _ in range(3)]
    w = torch.randn(B, S, H, D, generator=g)
    kw = dict(cap=4.0, slopes=torch.tensor([0.2, 0.05]).cuda(), causal=True, scale=0.125)
    leaves = [t.cuda().requires_grad_() for t in base]
    out = ops.attention(*leaves, **kw)
    grads = torch.autograd.grad(out, leaves, w.half().cuda())
    w16 = w.half().double()
    h = 2.0 ** -4
    for i in range(3):
        d = torch.sign(torch.randn(B, S, H, D, generator=g))

        def at(step):
            x = [t.clone() for t in base]
            x[i] = (x[i].double() + step * d).half()
            o = ops.attention(*[t.cuda() for t in x], **kw).double().cpu()
            return (o * w16).sum().item(), o, x[i].double()

        fp, op, xp = at(h)
        fm, om, xm = at(-h)
        exact_step = (xp - xm)                            # what the rounded inputs really moved by
        slope = (fp - fm)
        want = (grads[i].double().cpu() * exact_step).sum().item()
        noise = 6 * U[FP] * math.sqrt(((op.abs() * w16) ** 2).sum().item() * 2) + \
            6 * U[FP] * 2 * math.sqrt(((grads[i].double().cpu() * exact_step) ** 2).sum().item())
        curve = 4 * h * h * (grads[i].double().cpu().abs() * exact_step.abs()).sum().item()
        assert abs(slope - want) <= noise + curve, (i, slope, want, noise, curve)


def test_attention_same_bits(ops):
    """A replay gives the same bits, on another stream and within a graph too."""
    q, k, v, do = inputs(2, 300, 300, 4, 2, 128, BF)
    kw = dict(causal=True, cap=20.0, docs=(torch.arange(300)[None] // 110).expand(2, -1).to(torch.int32).cuda())

    def once():
        out = ops.attention(q, k, v, **kw)
        return (out.detach(), *torch.autograd.grad(out, (q, k, v), do))

    first = once()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = once()
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    qs, ks, vs = q.detach()[:, :3].contiguous(), k.detach(), v.detach()
    eager = ops.attention(qs, ks, vs, causal=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ops.attention(qs, ks, vs, causal=True)
    for i in range(3):
        qs.mul_(1.5)
        want = ops.attention(qs, ks, vs, causal=True)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want), i
    assert eager.shape == held.shape


# ---- dropout --------------------------------------------------------------------------

def kept(n, p, seed, offset):
    with np.errstate(over="ignore"):
        def mix(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            return z ^ (z >> np.uint64(31))

        G = np.uint64(0x9E3779B97F4A7C15)
        key = mix(np.array([seed % 2 ** 64], np.uint64) + G)
        z = mix(key + G * (np.arange((n + 1) // 2, dtype=np.uint64) + np.uint64(offset % 2 ** 64)))
        u = z.astype("<u8").view("<u4")[:n]
    return torch.from_numpy(u.astype(np.int64) >= math.floor(p * 2.0 ** 32))


SHAPES = [(1,), (7,), (8,), (2, 3), (1, 2049), (5, 16), (33, 1000), (3, 7, 40), (257, 255), (4, 1)]


@pytest.mark.parametrize("dtype", [BF, FP, F32])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.97, 1.0])
def test_dropout(ops, dtype, p):
    for i, shape in enumerate(SHAPES):
        seed, offset = (-1, 2 ** 64 - 3, 12345678901234567)[i % 3], (0, 5, 2 ** 63 + 11)[i % 3]
        g = torch.Generator().manual_seed(i)
        x, r, do = (torch.randn(shape, generator=g).to(dtype).cuda() for _ in range(3))
        n = x.numel()
        keep = kept(n, p, seed, offset).view(shape)
        x.requires_grad_()
        inv = 1 / (1 - p) if p < 1 else 0.0
        for res in (None, r):
            out = ops.dropout_add(x, res, p=p, seed=seed, offset=offset)
            want = x.detach().double().cpu() * keep * inv
            size = want.abs()
            if res is not None:
                want, size = want + r.double().cpu(), size + r.double().cpu().abs()
            close(out, want, U[dtype] * want.abs() + 2.0 ** -22 * size + TINY[dtype], f"dropout {shape} {p}")
            dx, = torch.autograd.grad(out, x, do)
            want = do.double().cpu() * keep * inv
            close(dx, want, U[dtype] * want.abs() + 2.0 ** -22 * want.abs() + TINY[dtype], f"dx {shape} {p}")
            assert torch.equal((dx != 0).cpu(), keep & (do.cpu() != 0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_dropout_strides(ops, dtype):
    """The mask goes by the element's number, not by the strides."""
    base = torch.randn(40, 64, device="cuda", dtype=dtype)
    keep = kept(40 * 64, 0.3, 9, 4).view(40, 64).cuda()
    views = {"plain": base, "rows apart": torch.randn(40, 80, device="cuda", dtype=dtype)[:, 8:72],
             "odd rows": torch.randn(40, 67, device="cuda", dtype=dtype)[:, 3:],
             "transposed": torch.randn(64, 40, device="cuda", dtype=dtype).t(),
             "broadcast": torch.randn(1, 64, device="cuda", dtype=dtype).expand(40, 64),
             "backwards in pairs": torch.randn(20, 2, 64, device="cuda", dtype=dtype).transpose(0, 1).reshape(40, 64)}
    for name, x in views.items():
        for rname, r in views.items():
            out = ops.dropout_add(x, r, p=0.3, seed=9, offset=4)
            part = torch.where(keep, x.double() / 0.7, 0.0)
            want = part + r.double()
            close(out, want.cpu(), (U[dtype] * want.abs() + 2.0 ** -22 * (part.abs() + r.double().abs())).cpu(), name + rname)
    three = torch.randn(5, 8, 96, device="cuda", dtype=dtype)[:, :, :64]
    out = ops.dropout_add(three, p=0.3, seed=9, offset=4)
    assert torch.equal(out != 0, keep.view(5, 8, 64) & (three != 0))


def test_dropout_drops_anything(ops):
    """Dropped infinities and NaN leave nothing; kept ones stay; residuals pass."""
    n = 4096
    keep = kept(n, 0.5, 1, 0).cuda()
    x = torch.full((n,), float("nan"), device="cuda", dtype=BF)
    x[::2] = float("inf")
    out = ops.dropout_add(x, p=0.5, seed=1)
    assert (out[~keep] == 0).all() and not torch.isfinite(out[keep]).any()
    assert (ops.dropout_add(x, p=1.0, seed=1) == 0).all()
    r = torch.randn(n, device="cuda", dtype=BF, requires_grad=True)
    out = ops.dropout_add(torch.zeros_like(r), r, p=0.5, seed=1)
    assert torch.equal(out, r)
    assert torch.equal(torch.autograd.grad(out, r, torch.ones_like(r))[0], torch.ones_like(r))
    assert ops.dropout_add(torch.empty(0, 5, device="cuda"), p=0.5, seed=1).shape == (0, 5)


def test_more_than_the_caches_hold(ops):
    """Rows in and out of more than 256 MiB: the same bits as a few of the rows by themselves."""
    torch.manual_seed(3)
    x = torch.randn(8200, 8203, device="cuda", dtype=torch.bfloat16)
    for t in (x, x[:, :8200], x[:, 3:8195]):                    # one long row, rows of odd and of even addresses
        whole, few = (ops.dropout_add(u, u, p=0.1, seed=5) for u in (t, t[:70]))
        assert torch.equal(whole[:70], few)
        big, small = t.detach().requires_grad_(), t[:70].detach().requires_grad_()
        ids = torch.randint(0, t.shape[1], (8200,), device="cuda")
        a, b = ops.token_logprobs(big, ids), ops.token_logprobs(small, ids[:70])
        (a.logp.sum() + a.entropy.sum()).backward()
        (b.logp.sum() + b.entropy.sum()).backward()
        torch.testing.assert_close(a.logp[:70], b.logp, rtol=2 ** -20, atol=2 ** -20)   # few rows are split further
        torch.testing.assert_close(big.grad[:70].float(), small.grad.float(), rtol=2 ** -7, atol=2 ** -30)


def test_offsets_beyond_32_bits(ops):
    """Rows so far apart that their offsets pass 2^31 elements: the bits of the same rows laid together."""
    step = 2 ** 23 + 8
    flat = torch.empty(300 * step, device="cuda", dtype=BF)
    assert flat.numel() > 2 ** 31
    torch.manual_seed(4)

    def spread(t, at):                                   # [300, columns] into rows `step` apart
        view = flat[at:].as_strided(t.shape, (step, 1))
        view.copy_(t)
        return view

    k, v = torch.randn(300, 64, device="cuda", dtype=BF), torch.randn(300, 64, device="cuda", dtype=BF)
    far = [spread(k, 0)[None, :, None], spread(v, 64)[None, :, None]]
    for Sq in (1, 300):
        q = torch.randn(1, Sq, 4, 64, device="cuda", dtype=BF)
        results = []
        for kk, vv in (far, [k[None, :, None], v[None, :, None]]):
            ins = [t.detach().requires_grad_() for t in (q, kk, vv)]
            out = ops.attention(*ins, causal=True)
            results.append([out, *torch.autograd.grad(out, ins, q)])
        for a, b in zip(*results):
            assert torch.equal(a, b), Sq
    x, ids = torch.randn(300, 1000, device="cuda", dtype=BF), torch.arange(300, device="cuda")
    results = []
    for t in (spread(x, 128), x):
        t = t.detach().requires_grad_()
        r = ops.token_logprobs(t, ids, top=3)
        results.append([*r, *torch.autograd.grad((r.logp.sum(), r.top_logp.sum()), t)])
    for a, b in zip(*results):
        torch.testing.assert_close(a, b, rtol=2 ** -7 if a.dtype == BF else 2 ** -20, atol=2 ** -20)  # sums in another order
    del flat, far, results, t, r, a, b, kk, vv, ins, out
    n = 2 ** 32
    long = torch.ones(n + 64, device="cuda", dtype=BF)
    out = ops.dropout_add(long, p=0.5, seed=11)
    assert torch.equal(out[n - 64:], ops.dropout_add(long[n - 64:], p=0.5, seed=11, offset=(n - 64) // 2))
    assert torch.equal(out[:64], ops.dropout_add(long[:64], p=0.5, seed=11))


def test_dropout_parts_make_the_whole(ops):
    """Calls whose offsets follow one another draw what one call draws."""
    x = torch.randn(1000, 64, device="cuda", dtype=BF)
    whole = ops.dropout_add(x, p=0.2, seed=77, offset=100)
    first, rest = ops.dropout_add(x[:300], p=0.2, seed=77, offset=100), ops.dropout_add(x[300:], p=0.2, seed=77,
                                                                                     offset=100 + 300 * 32)
    assert torch.equal(whole, torch.cat([first, rest]))
    share = (whole == 0).double().mean().item()          # 64000 draws: six standard deviations are 0.0095
    assert abs(share - 0.2) < 0.0095
    assert not torch.equal(whole == 0, ops.dropout_add(x, p=0.2, seed=78, offset=100) == 0)


# ---- log probabilities ----------------------------------------------------------------------

def logprobs_definition(x, tok, top, dlogp, dent, dtop):
    u, tiny = U[x.dtype], TINY[x.dtype]
    x, tok = x.detach().double().cpu(), tok.cpu()
    T, V = x.shape
    L = torch.logsumexp(x, 1)
    nothing = L == -math.inf
    logq = torch.where(nothing[:, None], -math.inf, x - L[:, None])
    q = torch.exp(logq)
    fin = torch.where(q > 0, logq, 0.0)
    H = -(q * fin).sum(1)
    has, over = tok >= 0, tok >= V
    at = torch.gather(logq, 1, tok.clamp(0, V - 1)[:, None])[:, 0]
    logp = torch.where(has, at, 0.0)
    # 32-bit sums: a lane adds up to V / 64 terms, six joins; exp2 of an argument rounded to 2^-24 of itself
    rel = 2.0 ** -24 * (V / 64 + 40 + 4 * (q * fin.abs()).sum(1))
    mag = x.masked_fill(torch.isinf(x), 0).abs().amax(1) + L.abs().nan_to_num(0, 0, 0)
    tol = dict(logp=rel + 2.0 ** -22 * mag, entropy=rel * (1 + H.abs() * 2) + 2.0 ** -22 * (1 + H.abs()) + 2.0 ** -21 * mag)
    res = dict(logp=logp, entropy=torch.where(nothing, 0.0, H))
    G = torch.where(has, dlogp.double().cpu(), 0.0) if dlogp is not None else torch.zeros(T, dtype=torch.float64)
    dx = torch.zeros_like(x)
    dx.scatter_add_(1, tok.clamp(0, V - 1)[:, None], torch.where(over, 0.0, G)[:, None])
    total = G.clone()
    size = G.abs()
    if top:
        order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :top]
        res["top_ids"] = order
        res["top_logp"] = torch.gather(logq, 1, order)
        tol["top_logp"] = tol["logp"][:, None].expand(T, top)
        if dtop is not None:
            dx.scatter_add_(1, order, dtop.double().cpu())
            total = total + dtop.double().cpu().sum(1)
            size = size + dtop.double().cpu().abs().sum(1)
    dh = dent.double().cpu() if dent is not None else torch.zeros(T, dtype=torch.float64)
    inner = total[:, None] + dh[:, None] * (fin + H[:, None])
    dx = dx - q * inner
    dx[nothing] = 0
    e = (rel + 2.0 ** -22 * mag)[:, None] * 4 + 2.0 ** -22 * fin.abs()
    tol["dx"] = u * dx.abs() + q * (e * (size[:, None] + dh.abs()[:, None] * (1 + fin.abs() + H[:, None].abs()))) + \
        2.0 ** -21 * size[:, None] * (dx != 0) * q.clamp_min(2.0 ** -30) + 2.0 ** -22 * dx.abs() + tiny
    res["dx"] = dx
    return res, tol


def check_logprobs(ops, x, tok, top, label, dtop_too=True):
    print(label, flush=True)
    T, V = x.shape
    g = torch.Generator().manual_seed(T + V)
    dlogp, dent = torch.randn(T, generator=g).cuda(), torch.randn(T, generator=g).cuda()
    dtop = torch.randn(T, top, generator=g).cuda() if top else None
    want, tol = logprobs_definition(x, tok, top, dlogp, dent, dtop)
    with torch.no_grad():
        plain = ops.token_logprobs(x, tok, top=top)
    x = x.detach().requires_grad_()
    r = ops.token_logprobs(x, tok, top=top)
    assert torch.equal(r.logp, plain.logp) and torch.equal(r.entropy, plain.entropy)
    close(r.logp, want["logp"], tol["logp"], label + " logp")
    close(r.entropy, want["entropy"], tol["entropy"], label + " entropy")
    outs, grads = [r.logp, r.entropy], [dlogp, dent]
    if top:
        assert torch.equal(r.top_ids.cpu(), want["top_ids"]), label
        close(r.top_logp, want["top_logp"], tol["top_logp"], label + " top")
        outs.append(r.top_logp)
        grads.append(dtop)
    dx, = torch.autograd.grad(outs, x, grads)
    close(dx, want["dx"], tol["dx"], label + " dx")


VOCABS = [1, 2, 7, 8, 9, 63, 64, 65, 255, 512, 513, 2047, 2048, 2051, 4100, 8191, 8192, 8203, 30011]


@pytest.mark.parametrize("dtype", [BF, FP, F32])
def test_logprobs_sizes(ops, dtype):
    for V in VOCABS:
        for T in ((1, 5) if V > 600 else (1, 9)):
            g = torch.Generator().manual_seed(V * 10 + T)
            x = (torch.randn(T, V, generator=g) * 3).to(dtype).cuda()
            tok = torch.randint(0, V, (T,), generator=g).cuda()
            tok[T // 2] = -100 if T > 1 else 0
            check_logprobs(ops, x, tok, min(V, 0 if V % 2 else 5), f"{dtype} T {T} V {V}")


@pytest.mark.parametrize("dtype", [BF, FP, F32])
@pytest.mark.parametrize("T,V,top", [(1030, 1000, 20), (1024, 1000, 7), (3, 40002, 5), (128, 24576, 2), (129, 24580, 0)])
def test_logprobs_rows(ops, dtype, T, V, top):
    """Numbers of rows about the limits of what works on a row."""
    g = torch.Generator().manual_seed(T)
    x = (torch.randn(T, V, generator=g) * 3).to(dtype).cuda()
    tok = torch.randint(0, V, (T,), generator=g).cuda()
    check_logprobs(ops, x, tok, top, f"{dtype} T {T} V {V}")


@pytest.mark.parametrize("top", [1, 2, 20, 32])
@pytest.mark.parametrize("order", ["random", "rising", "falling", "equal", "two values"])
def test_logprobs_alternatives(ops, top, order):
    """Orders that make every element a candidate, and ties."""
    for T, V in ((3, 300), (2, 5000), (300, 9001), (1, 70001)):
        if order == "random":
            x = torch.randn(T, V, generator=torch.Generator().manual_seed(V))
        elif order == "equal":
            x = torch.full((T, V), 0.5)
        elif order == "two values":
            x = torch.randint(0, 2, (T, V), generator=torch.Generator().manual_seed(V)).float()
        else:
            x = torch.arange(V).float().expand(T, V) * (2.0 ** -10) * (1 if order == "rising" else -1)
        tok = torch.arange(T) % V
        x = x.contiguous().to(F32 if V != 9001 else BF).cuda()
        with torch.no_grad():
            r = ops.token_logprobs(x, tok.cuda(), top=top)
        want = torch.sort(x.cpu(), dim=1, descending=True, stable=True)[1][:, :top]
        assert torch.equal(r.top_ids.cpu(), want), (T, V)


def test_logprobs_masked_vocabulary(ops):
    for dtype in (BF, F32):
        for T, V in ((6, 100), (6, 5000), (3, 20011)):
            x = torch.randn(T, V, generator=torch.Generator().manual_seed(1)).to(dtype)
            x[0] = -math.inf                              # nothing left
            x[1, 3:] = -math.inf                          # fewer than the alternatives
            x[2, ::2] = -math.inf
            if T > 3:
                x[3] = torch.finfo(dtype).min             # the type's lowest value everywhere
                x[4, 1:] = torch.finfo(dtype).min
                x[5] = 88.0
            tok = torch.tensor([5, 1, 3, 7, 0, -1][:T])
            check_logprobs(ops, x.cuda(), tok.cuda(), 6, f"masked {dtype} {V}")


def test_logprobs_not_numbers(ops):
    for T, V in ((4, 90), (4, 6001)):
        x = torch.randn(T, V).cuda()
        x[0, 3] = math.nan
        x[1, V - 1] = math.inf
        x[2] = math.nan
        tok = torch.tensor([1, 2, 3, V], device="cuda")
        r = ops.token_logprobs(x.requires_grad_(), tok, top=4)
        for n in (r.logp, r.entropy, r.top_logp[:, 0]):
            assert torch.isnan(n[:3]).all()
        assert torch.isnan(r.logp[3]) and torch.isfinite(r.entropy[3])
        assert ((r.top_ids >= 0) & (r.top_ids < V)).all()
        dx, = torch.autograd.grad(r.logp.sum(), x)
        assert torch.isnan(dx).any(1).all()


def test_logprobs_strides(ops):
    wide = torch.randn(6, 7000, device="cuda", dtype=BF)
    tok = torch.tensor([0, 5, 6, -1, 9, 3000], device="cuda")
    check_logprobs(ops, wide[:, 5:5006], tok, 3, "columns of a wider table")
    check_logprobs(ops, wide[::2, :4096], tok[::2], 3, "every other row")
    check_logprobs(ops, wide[:1].expand(6, 7000), tok, 2, "one row for all")
    check_logprobs(ops, torch.randn(5000, 6, device="cuda").t(), tok, 2, "transposed")
    x = torch.randn(2, 3, 5001, device="cuda")
    r = ops.token_logprobs(x, tok.view(2, 3), top=2)
    assert r.logp.shape == (2, 3) and r.top_ids.shape == (2, 3, 2)
    flat = ops.token_logprobs(x.view(6, 5001), tok, top=2)
    assert torch.equal(flat.logp, r.logp.view(-1)) and torch.equal(flat.top_ids, r.top_ids.view(6, 2))
    empty = ops.token_logprobs(x[:0], tok.view(2, 3)[:0])
    assert empty.logp.shape == (0, 3)


def test_logprobs_one_gradient_at_a_time(ops):
    x = torch.randn(5, 3000, device="cuda", requires_grad=True)
    tok = torch.arange(5, device="cuda")
    r = ops.token_logprobs(x, tok, top=2)
    z = torch.log_softmax(x.double(), 1)
    for got, want in ((r.logp.sum(), z[torch.arange(5), tok].sum()), (r.entropy.sum(), -(z.exp() * z).sum()),
                      (r.top_logp.sum(), z.topk(2, dim=1)[0].sum())):
        a, = torch.autograd.grad(got, x, retain_graph=True)
        b, = torch.autograd.grad(want, x, retain_graph=True)
        assert (a.double() - b.double()).abs().max() < 2.0 ** -18


def test_logprobs_differences(ops):
    """Against central differences in 64 bits of the definition, along a direction, and of the operator itself."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(4, 2500, generator=g).cuda().requires_grad_()
    d = torch.randn(4, 2500, generator=g).cuda()
    tok = torch.tensor([3, 4, 5, -1], device="cuda")
    w = torch.tensor([1.0, -2.0, 0.5, 3.0], device="cuda")
    r = ops.token_logprobs(x, tok)
    dx, = torch.autograd.grad((r.logp, r.entropy), x, (w, 0.3 * w))
    h = 2.0 ** -6
    with torch.no_grad():
        ends = []
        for s in (h, -h):
            y = ops.token_logprobs(x + s * d, tok)
            ends.append((y.logp.double() * w).sum() + 0.3 * (y.entropy.double() * w).sum())
    slope = ((ends[0] - ends[1]) / (2 * h)).item()
    # 32-bit results of magnitude 10 differ by 2^-21 at most, divided by 2 h; the cubic term is of the order h^2
    assert abs(slope - (dx.double() * d.double()).sum().item()) < 8 * 10 * 2.0 ** -21 / (2 * h) * 6.5 + 8 * h * h


def test_logprobs_graph(ops):
    x = torch.randn(2, 60000, device="cuda", dtype=BF)
    tok = torch.tensor([1, 2], device="cuda")
    ops.token_logprobs(x, tok, top=5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ops.token_logprobs(x, tok, top=5)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        want = ops.token_logprobs(x, tok, top=5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)


# ---- refusals ------------------------------------------------------------------------------

def test_refusals(ops):
    q = torch.randn(2, 5, 4, 64, device="cuda", dtype=BF)
    k = torch.randn(2, 7, 2, 64, device="cuda", dtype=BF)
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (lambda: ops.attention(q[0], k, k), lambda: ops.attention(q, k, k[:, :6]),
                lambda: ops.attention(q, k[..., :56], k[..., :56]), lambda: ops.attention(q, k, k, lengths=n[:1]),
                lambda: ops.attention(q, k, k, docs=torch.zeros(2, 5, dtype=torch.int32, device="cuda")),
                lambda: ops.attention(q, k, k, starts=n.cpu()), lambda: ops.attention(q, k, k, slopes=torch.zeros(3).cuda()),
                lambda: ops.attention(q.cpu(), k.cpu(), k.cpu()),
                lambda: ops.dropout_add(q, q[:1], p=0.1, seed=0), lambda: ops.dropout_add(q, p=1.5, seed=0),
                lambda: ops.dropout_add(q, p=float("nan"), seed=0), lambda: ops.dropout_add(q.cpu(), p=0.1, seed=0),
                lambda: ops.token_logprobs(q, n), lambda: ops.token_logprobs(q[0, 0], n.new_zeros(4).long(), top=65),
                lambda: ops.token_logprobs(q[:, :, 0, :0], n.new_zeros(2, 5).long())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ops.attention(q.float(), k.float(), k.float()), lambda: ops.attention(q, k.half(), k.half()),
                lambda: ops.attention(q, k, k, lengths=n.float()), lambda: ops.dropout_add(q.double(), p=0.1, seed=0),
                lambda: ops.token_logprobs(q[0, 0], torch.zeros(4, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    from paper_2006_09616_amd.dtr import DtrError
    for bad, why in ((lambda: ops.attention(q[:, :, :3], k, k), "multiple of 2 key heads"),
                     (lambda: ops.attention(q[..., :60], k[..., :60], k[..., :60]), "multiple of 8"),
                     (lambda: ops.attention(q, k, k, prefix=n), "causal"), (lambda: ops.attention(q, k, k, cap=-1.0), "cap"),
                     (lambda: ops.attention(q, k, k, scale=0.0), "scale"),
                     (lambda: ops.attention(q, k, k, scale=float("inf")), "scale")):
        with pytest.raises(DtrError) as e:
            bad()
        assert why in str(e.value)


@pytest.mark.parametrize("dtype,D", [(BF, 64), (FP, 96), (BF, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_few_tokens_with_documents(ops, dtype, D, causal):
    """Few rows a key head within documents: lengths that end before the queries' document, lengths of zero,
    positions outside the key slots, keys that no query sees and that are not numbers; whole and split over the keys."""
    i32 = torch.int32
    for i, (Sq, Sk, size) in enumerate(((1, 128, 64), (5, 150, 40), (3, 3000, 700), (8, 2050, 64))):
        B = 5
        docs = (torch.arange(Sk) // size).to(i32).expand(B, -1).contiguous()   # the same numbers in every request
        docs[4] = torch.randint(0, 3, (Sk,), generator=torch.Generator().manual_seed(i)).to(i32)
        short = Sk // size * size - size                  # ends before the last document
        lengths = torch.tensor([Sk, 0, max(short // 2, 1), short, Sk], dtype=i32)
        outside = torch.tensor([-40, Sk + 60, -1, Sk - 1, 7], dtype=i32)
        for name, kw in (("lengths", dict(lengths=lengths)), ("positions outside", dict(starts=outside)),
                         ("both", dict(lengths=lengths, starts=outside))):
            q, k, v, do = inputs(B, Sq, Sk, 4, 2, D, dtype, "heads" if i % 2 else "separate", seed=i)
            start = kw.get("starts", torch.full((B,), Sk - Sq, dtype=i32))
            for b in range(B):                            # what no query sees may be anything
                p = torch.arange(Sq) + int(start[b])
                p = p[(p >= 0) & (p < Sk)]
                seen = (docs[b][p][:, None] == docs[b][None]) & (not causal or torch.arange(Sk)[None] <= p[:, None])
                seen &= torch.arange(Sk)[None] < int(kw.get("lengths", torch.full((B,), Sk))[b])
                hidden = ~seen.any(0).cuda()
                k.data[b, hidden] = float("nan")
                v.data[b, hidden] = float("-inf")
            check(ops, q, k, v, do, f"few tokens, documents, {name} {Sq} {Sk} {D} causal {causal}", causal=causal, docs=docs,
                  cap=15.0 if i == 1 else 0.0, backward=False, **kw)


@pytest.mark.parametrize("dtype,D", [(BF, 64), (FP, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradient_of_queries_outside_the_slots(ops, dtype, D, causal):
    """With documents a query outside the key slots sees nothing: whatever its gradient is, keys and values get
    none of it."""
    Sq, Sk = 150, 130
    docs = torch.zeros(2, Sk, dtype=torch.int32)
    docs[1, 60:] = 4
    starts = torch.tensor([-30, 55], dtype=torch.int32)
    q, k, v, do = inputs(2, Sq, Sk, 4, 2, D, dtype)
    pos = torch.arange(Sq)[None] + starts[:, None]
    outside = ((pos < 0) | (pos >= Sk)).cuda()
    do = torch.where(outside[:, :, None, None], torch.zeros_like(do), do)
    want, tol = definition(q, k, v, do, D ** -0.5, 0.0, None, causal, None, docs, None, starts)
    for bad in (math.nan, math.inf):
        g = do.clone()
        g[outside] = bad
        out = ops.attention(q, k, v, causal=causal, docs=docs.cuda(), starts=starts.cuda())
        for n, t in zip(("dq", "dk", "dv"), torch.autograd.grad(out, (q, k, v), g)):
            close(t, want[n], tol[n], f"{n} {bad}")


@pytest.mark.parametrize("dtype,D", [(BF, 64), (FP, 96), (BF, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients_of_keys_that_nobody_sees(ops, dtype, D, causal):
    """Keys within the length that no query sees may be anything and get gradients of zero, also where the queries
    end within a tile."""
    i32 = torch.int32
    docs = torch.stack([torch.arange(130) // 40, torch.arange(130) % 3]).to(i32)
    for name, Sq, kw in (("documents", 5, dict(docs=docs)), ("documents", 70, dict(docs=docs)),
                         ("starts", 20, dict(starts=torch.tensor([0, 45], dtype=i32))),
                         ("both", 33, dict(docs=docs, starts=torch.tensor([3, 60], dtype=i32)))):
        q, k, v, do = inputs(2, Sq, 130, 4, 2, D, dtype)
        for b in range(2):
            p = torch.arange(Sq) + int(kw["starts"][b] if "starts" in kw else 130 - Sq)
            seen = torch.ones(Sq, 130, dtype=torch.bool)
            if "docs" in kw:
                seen &= docs[b][p][:, None] == docs[b][None]
            if causal:
                seen &= torch.arange(130)[None] <= p[:, None]
            hidden = ~seen.any(0).cuda()
            k.data[b, hidden] = float("nan")
            v.data[b, hidden] = float("inf")
        check(ops, q, k, v, do, f"nobody sees, {name} {Sq} {D} causal {causal}", causal=causal, **kw)


@pytest.mark.parametrize("cap", [1e-39, 200.0, 1e3, 1e4, 1e5, 1e7, 1e30, 3e38])
@pytest.mark.parametrize("dtype,D", [(BF, 64), (FP, 64), (FP, 96), (FP, 128)])
def test_attention_any_cap(ops, cap, dtype, D):
    """Scores keep their digits under any cap: the bound is that of scores without one (a large cap hardly changes
    them, and where scores reach the cap the bound for it is taken).  Terms below the least normal number of 32 bits,
    2^-126, may count as zero: 150 of at most 4 times that."""
    least = 2.0 ** -116
    for i, (Sq, Sk, gain) in enumerate(((150, 150, 1.0), (4, 700, 1.0), (150, 150, 30.0 if cap <= 200 or cap > 1e3 else 8.0))):
        slopes = torch.tensor([0.5, 0.1, 0.0, 0.01]) if i == 1 or D == 96 else None
        q, k, v, do = inputs(2, Sq, Sk, 4, 2, D, dtype, seed=i, gain=gain)
        q.data[0, 1] = 0                                  # scores of exactly zero
        kw = dict(scale=D ** -0.5, slopes=slopes, causal=True, prefix=None, docs=None, lengths=None, starts=None)
        rest = [kw[n] for n in ("slopes", "causal", "prefix", "docs", "lengths", "starts")]
        want, tol = definition(q, k, v, do, D ** -0.5, cap, *rest)
        if cap >= 1e3:
            _, tol = definition(q, k, v, do, D ** -0.5, 0.0, *rest)
        dev = {n: t.cuda() if torch.is_tensor(t) else t for n, t in kw.items()}
        out, lse = ops.attention(q, k, v, cap=cap, return_lse=True, **dev)
        close(out, want["out"], tol["out"], f"cap {cap} out {i}")
        close(lse, want["lse"], tol["lse"], f"cap {cap} lse {i}")
        for n, t in zip(("dq", "dk", "dv"), torch.autograd.grad(out, (q, k, v), do)):
            close(t, want[n], tol[n] + least, f"cap {cap} {n} {i}")


def whole_sums(q, k, v, do, cap):
    """Gradients of one head without masks in 64 bits, and the root of the squares of the terms of each."""
    scale = q.shape[3] ** -0.5
    q, k, v, do = (t.detach()[0, :, 0].double().cpu() for t in (q, k, v, do))
    s, dc = scale * q @ k.T, 1.0
    if cap:
        t = torch.tanh(s / cap)
        s, dc = cap * t, 1 - t * t
    P = torch.softmax(s, 1)
    dP = do @ v.T
    dS = P * (dP - (P * dP).sum(1, keepdim=True)) * dc * scale
    return {"dq": dS @ k, "dk": dS.T @ q, "dv": P.T @ do, "dq noise": ((dS ** 2) @ (k ** 2)).sqrt(),
            "dk noise": ((dS.T ** 2) @ (q ** 2)).sqrt()}


@pytest.mark.parametrize("size", [1e-1, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("cap", [0.0, 10.0])
def test_attention_small_gradients_in_fp16(ops, size, cap):
    """fp16 gradients of a long row lose what rounding them once takes, and what rounding the score gradients by
    u = 2^-11 each takes (independent errors: their root of squares, at two standard deviations of the largest
    rounding), however small the output's gradient is."""
    S, D = 6000, 128
    q, k, v, do = inputs(1, S, S, 1, 1, D, FP)
    do.mul_(size / 0.25)
    want = whole_sums(q, k, v, do, cap)
    out = ops.attention(q, k, v, cap=cap)
    grads = dict(zip(("dq", "dk", "dv"), torch.autograd.grad(out, (q, k, v), do)))
    for n in ("dq", "dk"):
        exact, noise = want[n], want[n + " noise"]
        least = (exact.half().double() - exact).norm()
        err = (grads[n][0, :, 0].double().cpu() - exact).norm()
        assert err <= 1.1 * least + 2 * U[FP] * noise.norm(), (n, float(err), float(least), float(U[FP] * noise.norm()))


def test_attention_large_gradients_in_fp16(ops):
    """Score gradients beyond fp16's range whose products are within it."""
    q, k, v, do = inputs(2, 40, 4, 2, 1, 128, FP)
    v.data.mul_(8)
    do.mul_(900 / 0.25)
    out = ops.attention(q, k, v)
    got = torch.autograd.grad(out, (q, k, v), do)
    want, tol = definition(q, k, v, do, 128 ** -0.5, 0.0, None, False, None, None, None, None)
    sizes = {n: want[n].abs().max().item() for n in ("dq", "dk", "dv")}
    assert max(sizes.values()) < 65000, sizes
    for n, t in zip(("dq", "dk", "dv"), got):
        close(t, want[n], tol[n], n)


@pytest.mark.parametrize("T,V", [(2, 300), (3, 5000), (2, 40000), (200, 40000)])
def test_logprobs_zeros_of_both_signs(ops, T, V):
    """Minus zero equals zero: the lower column first, in rows read whole and in parts."""
    g = torch.Generator().manual_seed(V)
    x = torch.full((T, V), -1.0)
    at = torch.randint(0, V, (T, 60), generator=g)
    x.scatter_(1, at, torch.where(torch.rand(T, 60, generator=g) < 0.5, 0.0, -0.0))
    for dtype in (F32, BF):
        with torch.no_grad():
            r = ops.token_logprobs(x.to(dtype).cuda(), torch.zeros(T, dtype=torch.long, device="cuda"), top=12)
        want = torch.sort(x + 0.0, dim=1, descending=True, stable=True)[1][:, :12]
        assert torch.equal(r.top_ids.cpu(), want), dtype


def test_attention_document_numbers(ops):
    """Documents are told apart by all bits of their numbers: 8 to 32 bits are taken, 64 refused."""
    q, k, v, _ = inputs(1, 6, 6, 2, 1, 64, BF)
    q, k, v = (t.detach() for t in (q, k, v))
    docs = torch.tensor([[0, 0, 1, 1, 2, 2]], device="cuda")
    want = ops.attention(q, k, v, docs=docs.to(torch.int32))
    for t in (torch.int16, torch.int8, torch.uint8):
        assert torch.equal(ops.attention(q, k, v, docs=docs.to(t)), want)
    ends = torch.tensor([[-2 ** 31, -2 ** 31, -1, -1, 2 ** 31 - 1, 2 ** 31 - 1]], device="cuda")
    assert torch.equal(ops.attention(q, k, v, docs=ends.to(torch.int32)), want)
    for bad in (docs + 2 ** 40, docs):
        with pytest.raises(TypeError, match="docs"):
            ops.attention(q, k, v, docs=bad)
    with pytest.raises(TypeError, match="docs"):
        ops.attention(q, k, v, docs=docs.float())


@pytest.mark.parametrize("dtype,D", [(BF, 64), (FP, 96), (BF, 128)])
@pytest.mark.parametrize("what", ["key", "query"])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_attention_gradients_of_infinite_scores(ops, dtype, D, what, cap):
    """An infinite component of a key or query that a cap, or a probability of zero, makes finite: gradients that
    come out finite are those of the definition, also where a mask cuts through the tile."""
    S = 200
    q, k, v, do = inputs(1, S, S, 2, 1, D, dtype)
    at = 130                                             # within a tile that the causal mask cuts
    q.data[..., 3] = q[..., 3].abs() + 0.5
    k.data[..., 3] = k[..., 3].abs() + 0.5
    if what == "key":
        k.data[0, at, 0, 3] = -math.inf
    else:
        if not cap:
            return                                       # its row is not a number throughout
        q.data[0, at, :, 3] = math.inf
    want, _ = definition(q, k, v, do, D ** -0.5, cap, None, True, None, None, None, None)
    big = [t.detach().clone().clamp(-300, 300).requires_grad_() for t in (q, k)]      # scores whose size bounds the errors
    _, tol = definition(*big, v, do, D ** -0.5, cap, None, True, None, None, None, None)
    out = ops.attention(q, k, v, cap=cap, causal=True)
    grads = torch.autograd.grad(out, (q, k, v), do)
    close(out, want["out"], tol["out"], "out")
    for n, t in zip(("dq", "dk", "dv"), grads):
        t = t.double().cpu()
        both = torch.isfinite(t) & torch.isfinite(want[n])
        bad = both & ~((t - want[n]).abs() <= tol[n])
        assert not bad.any(), (n, bad.nonzero()[:4], t[bad][:4], want[n][bad][:4], tol[n][bad][:4])
        # queries before the key, and keys after the query, do not meet it (above, theirs is 0 x infinity)
        free, meet = (slice(0, at), slice(at, S)) if n == "dq" else (slice(at + 1, S), slice(0, at + 1))
        assert not (torch.isfinite(t) & ~torch.isfinite(want[n]))[:, meet].any(), n
        assert torch.isfinite(t[:, free]).all(), n


def test_gradients_of_gradients_are_refused(ops):
    """With create_graph the gradients can be used, and refuse to be differentiated again rather than count as
    constants."""
    q, k, v, do = inputs(1, 9, 9, 2, 1, 64, BF)
    x = torch.randn(3, 50, device="cuda", requires_grad=True)
    tok = torch.tensor([1, 2, 3], device="cuda")
    plain = torch.autograd.grad(ops.attention(q, k, v), (q, k, v), do)
    for gdo in (do, do.clone().requires_grad_()):
        for i, t in enumerate((q, k, v)):
            g, = torch.autograd.grad(ops.attention(q, k, v), t, gdo, create_graph=True)
            assert torch.equal(g, plain[i]) and g.requires_grad
            with pytest.raises(RuntimeError, match="not differentiable"):
                torch.autograd.grad((g * g).sum() + (q * q).sum() + (k * k).sum() + (v * v).sum(), t)
    for part in ("logp", "entropy", "top_logp"):
        g, = torch.autograd.grad(getattr(ops.token_logprobs(x, tok, top=2), part).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="not differentiable"):
            ((x * x).sum() + (g * g).sum()).backward()
    # the gradient of dropout does not depend on its input; on the output's gradient it does
    y = torch.randn(64, device="cuda", requires_grad=True)
    w = torch.randn(64, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(ops.dropout_add(y, p=0.5, seed=1), y, torch.ones_like(y), create_graph=True)
    (y.sum() + g.sum() * 0).backward() if g.requires_grad else y.sum().backward()
    assert torch.equal(y.grad, torch.ones_like(y))
    g, = torch.autograd.grad(ops.dropout_add(y, p=0.5, seed=1), y, w, create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable"):
        torch.autograd.grad(g.sum() + w.sum(), w)


def test_tangents_are_refused(ops):
    """Forward-mode differentiation is not supported: it raises rather than lose the tangent."""
    import torch.autograd.forward_ad as fw
    q, k, v, _ = (t.detach() for t in inputs(1, 9, 9, 2, 1, 64, BF))
    x = torch.randn(3, 50, device="cuda")
    tok = torch.tensor([1, 2, 3], device="cuda")
    slopes = torch.rand(2, device="cuda")
    with fw.dual_level():
        def dual(t):
            return fw.make_dual(t, torch.ones_like(t))

        for call in (lambda: ops.attention(dual(q), k, v), lambda: ops.attention(q, dual(k), v), lambda: ops.attention(q, k, dual(v)),
                     lambda: ops.attention(q, k, v, slopes=dual(slopes)), lambda: ops.dropout_add(dual(x), p=0.1, seed=1),
                     lambda: ops.dropout_add(x, dual(x), p=0.1, seed=1), lambda: ops.token_logprobs(dual(x), tok)):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call()
        assert torch.equal(ops.dropout_add(x, p=0.1, seed=1), ops.dropout_add(x.clone(), p=0.1, seed=1))


def test_recorded_calls_are_refused(ops):
    """torch.jit.trace would record the outputs' allocation without the kernels that fill them."""
    q = torch.randn(1, 5, 2, 64, device="cuda", dtype=BF)
    x = torch.randn(3, 50, device="cuda")
    tok = torch.tensor([1, 2, 3], device="cuda")
    for call, arg in ((lambda t: ops.attention(t, t, t), q), (lambda t: ops.dropout_add(t, p=0.1, seed=1), x),
                      (lambda t: ops.token_logprobs(t, tok).logp, x)):
        with pytest.raises(NotImplementedError, match="trace"):
            torch.jit.trace(call, arg, check_trace=False)


def test_logprobs_scaled_in_place(ops):
    """Outputs are tensors of their own: log probabilities may be changed in place before the backward pass."""
    tok = torch.tensor([1, -1, 3, 4], device="cuda")
    w = torch.tensor([1.0, 0.0, 2.0, -1.0], device="cuda")
    for T, V in ((4, 60), (4, 50000)):
        x = torch.randn(T, V, device="cuda", requires_grad=True)
        r = ops.token_logprobs(x, tok, top=3)
        want, = torch.autograd.grad((r.logp * w).sum() + r.entropy.sum() + (2 * r.top_logp).sum(), x)
        r = ops.token_logprobs(x, tok, top=3)
        r.logp.mul_(w)
        r.top_logp.mul_(2)
        got, = torch.autograd.grad(r.logp.sum() + r.entropy.sum() + r.top_logp.sum(), x)
        assert torch.equal(got, want)
        r = ops.token_logprobs(x, tok)
        with torch.no_grad():
            r.logp.detach().mul_(w)                       # nothing that the backward pass needs
        torch.autograd.grad(r.logp.sum() + r.entropy.sum(), x)
        r = ops.token_logprobs(x, tok)
        for t in (r.logp, r.entropy):
            assert t._base is None and t.untyped_storage().nbytes() == 4 * T


def test_refusals_of_a_backward_pass(ops):
    """What the C ABI refuses raises DtrError from a backward pass too: here the gradient of keys that lie by heads,
    whose contiguous positions are too far apart."""
    from paper_2006_09616_amd.dtr import DtrError
    H = 2 ** 18
    q = torch.zeros(1, 1, H, 64, device="cuda", dtype=BF, requires_grad=True)
    k = torch.zeros(1, H, 2, 64, device="cuda", dtype=BF).transpose(1, 2)
    out = ops.attention(q, k, k)
    for _ in range(2):
        with pytest.raises(DtrError, match="positions of dk") as e:
            torch.autograd.grad(out, q, torch.ones_like(out), retain_graph=True)
        assert e.value.code < 0


def test_dropout_seeds_of_any_integer_type(ops):
    x = torch.randn(100, device="cuda")
    want = ops.dropout_add(x, p=0.5, seed=12345, offset=7)
    assert torch.equal(ops.dropout_add(x, p=0.5, seed=np.int64(12345), offset=np.int32(7)), want)
    assert torch.equal(ops.dropout_add(x, p=0.5, seed=np.int64(-1)), ops.dropout_add(x, p=0.5, seed=2 ** 64 - 1))
    for bad in (1.5, "7", None):
        with pytest.raises(TypeError):
            ops.dropout_add(x, p=0.5, seed=bad)


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients_beside_rows_that_see_nothing(ops, causal):
    """Large gradients of queries that see nothing leave the bits of the others' as they are."""
    Sq, Sk = 150, 130
    docs = torch.zeros(2, Sk, dtype=torch.int32, device="cuda")
    docs[1, 60:] = 4
    starts = torch.tensor([-30, 55], dtype=torch.int32, device="cuda")
    pos = torch.arange(Sq, device="cuda")[None] + starts[:, None]
    outside = (pos < 0) | (pos >= Sk)
    q, k, v, do = inputs(2, Sq, Sk, 4, 2, 64, FP)
    do.mul_(2.0 ** -12)
    results = []
    for other in (0.0, 60000.0):
        do[outside] = other
        out = ops.attention(q, k, v, causal=causal, docs=docs, starts=starts)
        results.append(torch.autograd.grad(out, (q, k, v), do))
    for n, a, b in zip(("dq", "dk", "dv"), *results):
        assert torch.equal(a, b), n


@pytest.mark.parametrize("shape", [(1, 1, 1, 120), (2, 37, 2, 64)])
def test_attention_contiguous_rows_at_odd_addresses(ops, shape):
    """Tensors that are contiguous but do not start at a multiple of 16 bytes are copied, too."""
    def odd(t):
        flat = torch.empty(t.numel() + 1, device="cuda", dtype=t.dtype)
        flat[1:] = t.detach().reshape(-1)
        return flat[1:].view(t.shape)

    B, S, H, D = shape
    q, k, v, do = inputs(B, S, S, H, H, D, BF)
    want = ops.attention(q, k, v, causal=True)
    want = [want, *torch.autograd.grad(want, (q, k, v), do)]
    ins = [odd(t).requires_grad_() for t in (q, k, v)]
    assert ins[0].is_contiguous() and ins[0].data_ptr() % 16
    out = ops.attention(*ins, causal=True)
    for a, b in zip((out, *torch.autograd.grad(out, ins, odd(do))), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Sq", [1, 64])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("high", [9.0, 15.2, 19.0])
def test_attention_small_probabilities_in_fp16(ops, Sq, D, high):
    """Many keys beside one of a high score and no value: their probabilities are rounded by u = 2^-11 of themselves
    and so is the output, though e^-19 is below fp16's range; two u are left for sums, score and exponential."""
    Sk = 20000
    q = torch.zeros(1, Sq, 1, D, device="cuda", dtype=FP)
    k = torch.zeros(1, Sk, 1, D, device="cuda", dtype=FP)
    v = torch.ones(1, Sk, 1, D, device="cuda", dtype=FP)
    q[..., 0], k[:, 77, :, 0], v[:, 77] = high, 1.0, 0.0
    do = torch.full_like(q, 1000.0)
    score = float(q[0, 0, 0, 0])
    small = math.exp(-score) / (1 + (Sk - 1) * math.exp(-score))
    for t in (q, k, v):
        t.requires_grad_()
    out = ops.attention(q, k, v, scale=1.0)
    want = (Sk - 1) * small
    assert (out.double() - want).abs().max() <= 4 * U[FP] * want, (out.max().item(), out.min().item(), want)
    dv, = torch.autograd.grad(out, v, do)
    others = torch.arange(Sk, device="cuda") != 77
    want = Sq * 1000.0 * small
    assert (dv[:, others].double() - want).abs().max() <= 4 * U[FP] * want + 2 * TINY[FP], (dv[:, others].max().item(), want)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attention_training_step_in_a_graph(ops, dtype):
    """Forward and backward pass captured, and replayed on other numbers with eager work in between."""
    q, k, v, do = inputs(2, 200, 200, 4, 2, 64, dtype)
    docs = (torch.arange(200)[None] // 70).expand(2, -1).to(torch.int32).cuda()

    def step():
        out = ops.attention(q, k, v, causal=True, docs=docs, cap=20.0)
        return (out.detach(), *torch.autograd.grad(out, (q, k, v), do))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        with torch.no_grad():
            for t in (q, k, v, do):
                t.mul_(0.5 if i % 2 else -1.5)
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), i
