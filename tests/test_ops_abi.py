"""C ABI of the operators (include/dtr_ops.h): exports, layouts and what is
refused before anything is launched (no GPU needed)."""
import ctypes as C
import math
import re

import pytest

from paper_2006_09616_amd import dtr as D
from paper_2006_09616_amd import ops


class Attn(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("type", "batch", "q_len", "k_len", "q_heads", "k_heads", "head_dim", "causal")] + \
               [("scale", C.c_float), ("cap", C.c_float)] + \
               [(n, C.c_void_p) for n in ("slopes", "prefix", "docs", "lengths", "starts")]


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("position", C.c_int64), ("head", C.c_int64)]


@pytest.fixture(scope="module")
def lib():
    L = D.lib()
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.dtr_attn_workspace_bytes.argtypes = [vp, i32, vp]
    L.dtr_attn_forward.argtypes = [vp] * 8 + [sz, vp]
    L.dtr_attn_backward.argtypes = [vp] * 12 + [sz, vp]
    L.dtr_dropout_add.argtypes = [i32, i64, i64, vp, i64, vp, i64, vp, i64, C.c_double, C.c_uint64, C.c_uint64, vp]
    L.dtr_logprobs_workspace_bytes.argtypes = [i32, i64, i64, i32, vp]
    L.dtr_logprobs_forward.argtypes = [i32, i64, i64, i32, vp, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dtr_logprobs_backward.argtypes = [i32, i64, i64, i32, vp, i64] + [vp] * 8 + [i64, vp]
    return L


def refused(rc, why):
    assert rc == D.DTR_EINVAL
    assert why in D.dtr_sim_last_error()


def attn(**kw):
    a = dict(type=0, batch=2, q_len=8, k_len=16, q_heads=4, k_heads=2, head_dim=64, causal=0, scale=0.125, cap=0.0)
    a.update(kw)
    return Attn(**a)


def test_every_declared_function_is_exported(lib):
    text = open(ops.HEADER).read()
    names = set(re.findall(r"^int (dtr_\w+)\(", text, re.M))
    assert len(names) == 7
    for n in names:
        assert hasattr(lib, n), n


def test_record_layouts_match_the_header():
    text = open(ops.HEADER).read()
    body = text[text.index("typedef struct {"):text.index("} dtr_attn;")]
    names = [n.strip(" *") for line in re.findall(r"^\s+(?:const )?(?:int32_t|float) ([^;]+);", body, re.M) for n in line.split(",")]
    assert names == [n for n, _ in Attn._fields_]
    assert C.sizeof(Attn) == 80 and C.sizeof(Heads) == 32


def test_binding_loads_without_a_gpu():
    assert {"attention", "dropout_add", "token_logprobs"} <= set(dir(ops.lib()))
    import torch
    with pytest.raises(ValueError, match="run on a GPU"):
        ops.attention(*(torch.zeros(1, 2, 2, 8, dtype=torch.bfloat16) for _ in range(3)))
    with pytest.raises(ValueError, match="run on a GPU"):
        ops.dropout_add(torch.zeros(3), p=0.5, seed=1)
    with pytest.raises(ValueError, match="run on a GPU"):
        ops.token_logprobs(torch.zeros(2, 3), torch.zeros(2, dtype=torch.long))


@pytest.mark.parametrize("change,why", [
    (dict(type=2), "neither bf16 nor fp16"), (dict(batch=-1), "batch"), (dict(q_len=-1), "lengths"),
    (dict(k_len=2 ** 24 + 1), "lengths"), (dict(k_heads=3), "multiple of 3 key heads"), (dict(k_heads=0), "key heads"),
    (dict(head_dim=0), "head size"), (dict(head_dim=60), "head size"), (dict(head_dim=136), "head size"),
    (dict(causal=2), "causal"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"),
    (dict(scale=math.inf), "scale"), (dict(cap=-1.0), "cap"), (dict(cap=math.nan), "cap"), (dict(prefix=256), "causal"),
    (dict(batch=2 ** 20, q_len=2 ** 20), "too many")])
def test_attention_records_refused(lib, change, why):
    n = C.c_size_t(0)
    refused(lib.dtr_attn_workspace_bytes(C.byref(attn(**change)), 0, C.byref(n)), why)


def test_attention_arguments_refused(lib):
    n = C.c_size_t(0)
    refused(lib.dtr_attn_workspace_bytes(None, 0, C.byref(n)), "null")
    refused(lib.dtr_attn_workspace_bytes(C.byref(attn()), 0, None), "null bytes")
    a = attn(docs=4096)
    assert lib.dtr_attn_workspace_bytes(C.byref(a), 1, C.byref(n)) == D.DTR_OK and n.value > 0
    q, k, o = Heads(4096, 2048, 256, 64), Heads(4096, 2048, 128, 64), Heads(4096, 2048, 256, 64)

    def forward(q=q, k=k, v=k, o=o, ws=4096, given=n.value, rest=None, a=a):
        return lib.dtr_attn_forward(C.byref(a), *(C.byref(t) if t else None for t in (q, k, v, o)), rest, None, ws, given, None)

    refused(forward(q=None), "null q")
    refused(forward(v=Heads(None, 2048, 128, 64)), "null v")
    refused(forward(k=Heads(4098, 2048, 128, 64)), "rows of k do not start")
    refused(forward(k=Heads(4096, 2048, 132, 64)), "rows of k do not start")
    refused(forward(k=Heads(4096, 2048, 2 ** 24, 64)), "elements apart")
    refused(forward(k=Heads(4096, -2048, 128, 64)), "negative stride")
    refused(forward(o=Heads(4096, 2048, 0, 64)), "overlaps")
    refused(forward(ws=None), "null workspace")
    refused(forward(ws=4100), "aligned")
    refused(forward(given=0), "too small")
    refused(forward(rest=4100), "rest")
    g = Heads(4096, 2048, 256, 64)
    assert lib.dtr_attn_backward(C.byref(a), C.byref(q), C.byref(k), C.byref(k), C.byref(o), None, None, C.byref(g), C.byref(g),
                                 C.byref(k), C.byref(k), 4096, 1 << 30, None) == D.DTR_EINVAL
    assert "null lse" in D.dtr_sim_last_error()
    empty = attn(batch=0)
    none = Heads(None, 0, 0, 0)
    assert forward(none, none, none, none, None, 0, a=empty) == D.DTR_OK


def test_dropout_arguments_refused(lib):
    def call(type=0, rows=2, cols=8, x=4096, xs=8, r=None, rs=8, out=8192, os=8, p=0.5):
        return lib.dtr_dropout_add(type, rows, cols, x, xs, r, rs, out, os, p, 1, 0, None)

    for kw, why in ((dict(type=3), "type"), (dict(rows=-1), "elements"), (dict(cols=2 ** 48), "elements"), (dict(p=-0.1), "probability"),
                    (dict(p=1.01), "probability"), (dict(p=math.nan), "probability"), (dict(x=None), "null x"),
                    (dict(out=None), "null out"), (dict(xs=-1), "strides"), (dict(os=7), "strides"), (dict(x=4097), "addresses"),
                    (dict(r=4097), "addresses")):
        refused(call(**kw), why)
    assert call(rows=0, x=None) == D.DTR_OK


def test_logprobs_arguments_refused(lib):
    n = C.c_size_t(0)
    for kw, why in (((5, 2, 8, 0), "type"), ((0, -1, 8, 0), "rows"), ((0, 2 ** 24, 8, 0), "rows"), ((0, 2, 0, 0), "vocabulary"),
                    ((0, 2, 8, 9), "alternatives"), ((0, 2, 100, 33), "alternatives"), ((0, 2, 8, -1), "alternatives")):
        refused(lib.dtr_logprobs_workspace_bytes(*kw, C.byref(n)), why)
    assert lib.dtr_logprobs_workspace_bytes(0, 1, 100000, 5, C.byref(n)) == D.DTR_OK and n.value > 0
    p = 4096

    def call(x=p, stride=100000, tok=p, top=5, ids=p, ws=p, given=n.value):
        return lib.dtr_logprobs_forward(0, 1, 100000, top, x, stride, tok, p, p, p, p, ids, ws, given, None)

    refused(call(x=None), "null")
    refused(call(tok=None), "null")
    refused(call(ids=None), "null")
    refused(call(x=4097), "aligned")
    refused(call(stride=-1), "stride")
    refused(call(ws=None), "null workspace")
    refused(call(given=1), "too small")
    refused(lib.dtr_logprobs_backward(0, 2, 8, 0, p, 8, p, p, p, None, p, p, None, None, 8, None), "null")
    refused(lib.dtr_logprobs_backward(0, 2, 8, 0, p, 8, p, p, p, None, p, p, None, p, 7, None), "strides")
    assert lib.dtr_logprobs_forward(0, 0, 8, 0, None, 8, None, None, None, None, None, None, None, 0, None) == D.DTR_OK


def test_build_finds_scratch_memory():
    from paper_2006_09616_amd import build as B
    lines = ["/x/attention.hip:9:1: remark: Function Name: first [-Rpass-analysis=kernel-resource-usage]",
             "/x/attention.hip:9:1: remark:     ScratchSize [bytes/lane]: 0 [-Rpass-analysis=kernel-resource-usage]",
             "/x/attention.hip:12:1: remark: Function Name: second [-Rpass-analysis=kernel-resource-usage]",
             "/x/attention.hip:12:1: remark:     ScratchSize [bytes/lane]: 164 [-Rpass-analysis=kernel-resource-usage]",
             "/x/replay.hip:5:1: remark:     ScratchSize [bytes/lane]: 48 [-Rpass-analysis=kernel-resource-usage]"]
    assert B.scratch_of(lines, "attention.hip") == ["second: ScratchSize [bytes/lane]: 164"]
    assert B.scratch_of(lines[:2], "attention.hip") == []
