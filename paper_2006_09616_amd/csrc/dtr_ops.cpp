// dtr_ops.cpp -- host side of include/dtr_ops.h: checks of arguments, launch
// plans and workspaces.  Nothing here allocates or throws; a call is checked
// in full before its first launch.
#include "../../include/dtr_ops.h"

#include <algorithm>
#include <cmath>

#include "host.h"
#include "ops.h"

using dtrhost::align_up;
using dtrhost::fail;
using namespace dtrops;

namespace {

constexpr int32_t MAX_LEN = 1 << 24;
constexpr int64_t MAX_STRIDE = int64_t(1) << 24; // between positions: 64 of them within 2^31 bytes
constexpr int64_t MAX_ROWS = int64_t(1) << 31;
constexpr int64_t MAX_GROUPS = int64_t(1) << 24;   // workgroups of a launch: 2^32 work items

int check_attn(const dtr_attn *a)
{
    if (!a) return fail(DTR_EINVAL, "null attention");
    if (a->type != DTR_BF16 && a->type != DTR_FP16)
        return fail(DTR_EINVAL, "attention: type %d is neither bf16 nor fp16", a->type);
    if (a->batch < 0) return fail(DTR_EINVAL, "attention: batch %d", a->batch);
    if (a->q_len < 0 || a->q_len > MAX_LEN || a->k_len < 0 || a->k_len > MAX_LEN)
        return fail(DTR_EINVAL, "attention: lengths %d and %d are not within 0..2^24", a->q_len, a->k_len);
    if (a->k_heads < 1 || a->q_heads < 1 || a->q_heads % a->k_heads)
        return fail(DTR_EINVAL, "attention: %d query heads are not a multiple of %d key heads", a->q_heads, a->k_heads);
    if (a->head_dim < 8 || a->head_dim > 128 || a->head_dim % 8)
        return fail(DTR_EINVAL, "attention: head size %d is not a multiple of 8 within 8..128", a->head_dim);
    if (a->causal != 0 && a->causal != 1) return fail(DTR_EINVAL, "attention: causal %d", a->causal);
    if (!(a->scale > 0) || !std::isfinite(a->scale)) return fail(DTR_EINVAL, "attention: scale %g", (double)a->scale);
    if (!(a->cap >= 0) || !std::isfinite(a->cap)) return fail(DTR_EINVAL, "attention: cap %g", (double)a->cap);
    if (a->prefix && !a->causal) return fail(DTR_EINVAL, "attention: a prefix needs the causal mask");
    const int64_t rows = (int64_t)a->q_len * (a->q_heads / a->k_heads);
    const int64_t units = (int64_t)a->batch * a->k_heads;
    // grids have one workgroup per row tile (or key tile) and part of the keys
    if (rows >= MAX_ROWS || units >= MAX_ROWS ||
        units * std::max<int64_t>(rows / ROW_TILE + 1, a->k_len / KEY_TILE + 1) >= MAX_GROUPS)
        return fail(DTR_EINVAL, "attention: %lld rows of %lld key heads are too many", (long long)rows, (long long)units);
    return DTR_OK;
}

int check_heads(const char *name, const dtr_heads *t, const dtr_attn *a, bool output)
{
    if (!t) return fail(DTR_EINVAL, "attention: null %s", name);
    const bool of_q = name[0] == 'q' || name[0] == 'o' || (name[0] == 'd' && (name[1] == 'q' || name[1] == 'o'));
    const int64_t len = of_q ? a->q_len : a->k_len, heads = of_q ? a->q_heads : a->k_heads;
    if (a->batch == 0 || len == 0) return DTR_OK;
    if (!t->data) return fail(DTR_EINVAL, "attention: null %s", name);
    if ((uintptr_t)t->data % 16 || t->batch % 8 || t->position % 8 || t->head % 8)
        return fail(DTR_EINVAL, "attention: rows of %s do not start at multiples of 16 bytes", name);
    if (len > 1 && t->position >= MAX_STRIDE)
        return fail(DTR_EINVAL, "attention: positions of %s are %lld elements apart", name, (long long)t->position);
    if (t->batch < 0 || t->position < 0 || t->head < 0) return fail(DTR_EINVAL, "attention: negative stride of %s", name);
    if (output && ((a->batch > 1 && t->batch == 0) || (len > 1 && t->position == 0) || (heads > 1 && t->head == 0)))
        return fail(DTR_EINVAL, "attention: %s overlaps itself", name);
    return DTR_OK;
}

struct Plan {
    int32_t splits, parts, chunks;
    size_t docs, part_out, part_stat, part_grad, row_stat, value_magnitude, row_magnitude, total;
};

// Parts that the keys are split into.  One part per row tile leaves most of
// the 256 compute units idle where there are few rows; each part costs a
// partial result (32-bit, written and read again) and the join's launch.
//   Few rows: two workgroups are resident on each compute unit.  Up to 128
// units, parts for one round of them (12 units of 30011 keys: 33 us with 504
// workgroups, 39 with 696); beyond, where lengths are many and unequal, for
// two (256 units of 8192 to 16384 keys: 287 us with 1024, 319 with 512).  A
// part has 128 keys at least (8 units of 4096 keys: 11 us; 15 with 512 keys,
// 14 with 64), and 512 keys are one part (7.9 us; 8.5 in four).
//   Others: parts for two rounds of one workgroup, 256 keys at least (33 rows
// of 8 units, 4096 keys: 14 us; 17 with 384), and 1024 keys are one part (1024
// rows of 8 units: 18 us, in four parts 23; 2048 keys in parts: 30 against 31).
int32_t splits_for(int64_t units, int64_t rows, int64_t k_len)
{
    const bool few = rows <= FEW_ROWS;
    const int64_t groups = std::max<int64_t>(few ? units : units * ((rows + ROW_TILE - 1) / ROW_TILE), 1);
    const int64_t want = few ? (groups <= 128 ? 512 : 1024) / groups : groups >= 256 ? 1 : (512 + groups - 1) / groups;
    if (k_len <= (few ? 512 : 1024)) return 1;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min(want, k_len / (few ? 128 : 256)), 256));
}

// Parts that the rows are cut into for dK and dV.  A key block's work ranges
// from none to all rows under a causal mask or with documents, so that a card
// of 256 compute units wants several blocks for each; the 32-bit partial sums
// and their join are the price.  8192 tokens in three documents, 4 key heads,
// 256 blocks: 651 us at 1536 workgroups with the join, 679 at 1024, 778 at
// 768, 731 at 2048.  A part of fewer than 512 rows does not pay: 8 x 12 heads
// of 512 tokens, 36 us in one part, 52 in two.
int32_t parts_for(int64_t blocks, int64_t rows)
{
    if (blocks >= 1024) return 1;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((1536 + blocks - 1) / std::max<int64_t>(blocks, 1), rows / 512), 16));
}

Plan make_plan(const dtr_attn *a, bool backward)
{
    Plan p{};
    const int64_t group = a->q_heads / a->k_heads, rows = a->q_len * group;
    const int64_t units = (int64_t)a->batch * a->k_heads, key_tiles = (a->k_len + KEY_TILE - 1) / KEY_TILE;
    p.splits = backward ? 1 : splits_for(units, rows, a->k_len);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    };
    if (a->docs) p.docs = take(sizeof(int2) * a->batch * key_tiles);
    if (p.splits > 1) {
        p.part_out = take(sizeof(float) * p.splits * units * rows * a->head_dim);
        p.part_stat = take(sizeof(float2) * p.splits * units * rows);
    }
    p.parts = 1;
    if (backward) {
        p.parts = parts_for(units * ((a->k_len + GRAD_KEYS - 1) / GRAD_KEYS), rows);
        p.row_stat = take(sizeof(float2) * units * rows);
        if (a->type == DTR_FP16) {
            // two workgroups a compute unit to read all of v: 64 units of 4096 keys 13 us,
            // 27 with a quarter of them and 13 with four times as many; 96 units of 512 keys
            // 4.6, 6.5 and 5.4
            p.chunks = (int32_t)std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(units, 1), 64));
            p.value_magnitude = take(sizeof(float) * units * p.chunks);
            p.row_magnitude = take(sizeof(float) * units * ((rows + ROW_TILE - 1) / ROW_TILE) * 4);
        }
        if (p.parts > 1) p.part_grad = take(sizeof(float) * 2 * p.parts * units * a->k_len * a->head_dim);
    }
    p.total = at;
    return p;
}

Heads of(const dtr_heads *t) { return t ? Heads{(char *)t->data, t->batch, t->position, t->head} : Heads{}; }

// what both passes need, and the backward pass besides
AttnGradArgs make_args(const dtr_attn *a, const Plan &p, char *ws)
{
    AttnGradArgs k{};
    k.batch = a->batch;
    k.q_len = a->q_len;
    k.k_len = a->k_len;
    k.k_heads = a->k_heads;
    k.group = a->q_heads / a->k_heads;
    k.head_dim = a->head_dim;
    k.causal = a->causal;
    k.scale = a->scale;
    k.cap = a->cap;
    k.slopes = a->slopes;
    k.prefix = a->prefix;
    k.docs = a->docs;
    k.lengths = a->lengths;
    k.starts = a->starts;
    k.rows = (int32_t)((int64_t)a->q_len * k.group);
    k.splits = p.splits;
    k.parts = p.parts;
    k.part_grad = (float *)(ws + p.part_grad);
    k.key_tiles = (a->k_len + KEY_TILE - 1) / KEY_TILE;
    k.doc_tiles = (int2 *)(ws + p.docs);
    k.part_out = (float *)(ws + p.part_out);
    k.part_stat = (float2 *)(ws + p.part_stat);
    k.row_stat = (float2 *)(ws + p.row_stat);
    k.chunks = p.chunks;
    k.value_magnitude = (float *)(ws + p.value_magnitude);
    k.row_magnitude = (float *)(ws + p.row_magnitude);
    return k;
}

int check_workspace(const void *ws, size_t given, size_t needed)
{
    if (!needed) return DTR_OK;
    if (!ws) return fail(DTR_EINVAL, "null workspace, %zu bytes needed", needed);
    if ((uintptr_t)ws % dtrhost::ALIGN) return fail(DTR_EINVAL, "workspace must be 256-byte aligned");
    if (given < needed) return fail(DTR_EINVAL, "workspace too small: %zu bytes given, %zu needed", given, needed);
    return DTR_OK;
}

int launched(hipError_t e, const char *what)
{
    return e == hipSuccess ? DTR_OK : fail(DTR_EHIP, "%s: %s", what, hipGetErrorString(e));
}

bool known_type(int32_t type) { return type == DTR_BF16 || type == DTR_FP16 || type == DTR_FP32; }

uint64_t mix64(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

int check_logprobs(int32_t type, int64_t rows, int64_t vocab, int32_t top)
{
    if (!known_type(type)) return fail(DTR_EINVAL, "log probabilities: unknown type %d", type);
    if (rows < 0 || rows >= MAX_GROUPS) return fail(DTR_EINVAL, "log probabilities: %lld rows", (long long)rows);
    if (vocab < 1 || vocab >= MAX_ROWS) return fail(DTR_EINVAL, "log probabilities: vocabulary of %lld", (long long)vocab);
    if (top < 0 || top > DTR_TOP_MAX || top > vocab)
        return fail(DTR_EINVAL, "log probabilities: %d alternatives of a vocabulary of %lld (at most %d)", top,
                    (long long)vocab, DTR_TOP_MAX);
    return DTR_OK;
}

// Parts of a row read by workgroups of their own: one workgroup a row leaves
// the card idle where there are few rows.  A part has at least 4096 columns,
// and a row 64 parts at most.  64 rows of 131072, 32 bits: 9.8 us, in one part
// 22; of 32768: 6.8 and 8.0; of 16384: 6.3 and 5.7.  255 rows of 65536: 17 and
// 14.
int32_t logprob_splits(int64_t rows, int64_t vocab)
{
    if (rows > 128 || vocab < 24576) return 1;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((512 + rows - 1) / rows, 64), vocab / 4096));
}

}  // namespace

extern "C" {

int dtr_attn_workspace_bytes(const dtr_attn *attn, int32_t backward, size_t *bytes)
{
    if (!bytes) return fail(DTR_EINVAL, "null bytes");
    if (int rc = check_attn(attn)) return rc;
    *bytes = make_plan(attn, backward != 0).total;
    return DTR_OK;
}

int dtr_attn_forward(const dtr_attn *attn, const dtr_heads *q, const dtr_heads *k, const dtr_heads *v,
                     const dtr_heads *out, void *rest, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_attn(attn)) return rc;
    if (int rc = check_heads("q", q, attn, false)) return rc;
    if (int rc = check_heads("k", k, attn, false)) return rc;
    if (int rc = check_heads("v", v, attn, false)) return rc;
    if (int rc = check_heads("out", out, attn, true)) return rc;
    const Plan p = make_plan(attn, false);
    if (int rc = check_workspace(workspace, workspace_bytes, p.total)) return rc;
    if (attn->batch == 0 || attn->q_len == 0) return DTR_OK;
    AttnArgs a = make_args(attn, p, (char *)workspace);
    a.q = of(q);
    a.k = of(k);
    a.v = of(v);
    a.out = of(out);
    if ((uintptr_t)rest % 16) return fail(DTR_EINVAL, "attention: rest is not 16-byte aligned");
    a.rest = (char *)rest;
    a.lse = lse;
    return launched(launch_attn_forward(a, attn->type, (hipStream_t)stream), "attention forward");
}

int dtr_attn_backward(const dtr_attn *attn, const dtr_heads *q, const dtr_heads *k, const dtr_heads *v,
                      const dtr_heads *out, const void *rest, const float *lse, const dtr_heads *dout,
                      const dtr_heads *dq, const dtr_heads *dk, const dtr_heads *dv, void *workspace,
                      size_t workspace_bytes, void *stream)
{
    if (int rc = check_attn(attn)) return rc;
    if (int rc = check_heads("q", q, attn, false)) return rc;
    if (int rc = check_heads("k", k, attn, false)) return rc;
    if (int rc = check_heads("v", v, attn, false)) return rc;
    if (int rc = check_heads("out", out, attn, false)) return rc;
    if (int rc = check_heads("dout", dout, attn, false)) return rc;
    if (int rc = check_heads("dq", dq, attn, true)) return rc;
    if (int rc = check_heads("dk", dk, attn, true)) return rc;
    if (int rc = check_heads("dv", dv, attn, true)) return rc;
    const Plan p = make_plan(attn, true);
    if (int rc = check_workspace(workspace, workspace_bytes, p.total)) return rc;
    if (attn->batch == 0 || (attn->q_len == 0 && attn->k_len == 0)) return DTR_OK;
    if (!lse && attn->q_len) return fail(DTR_EINVAL, "attention: null lse");
    AttnGradArgs a = make_args(attn, p, (char *)workspace);
    a.q = of(q);
    a.k = of(k);
    a.v = of(v);
    a.out = of(out);
    if ((uintptr_t)rest % 16) return fail(DTR_EINVAL, "attention: rest is not 16-byte aligned");
    a.rest = (char *)rest;
    a.dout = of(dout);
    a.dq = of(dq);
    a.dk = of(dk);
    a.dv = of(dv);
    a.lse = const_cast<float *>(lse);
    return launched(launch_attn_backward(a, attn->type, (hipStream_t)stream), "attention backward");
}

int dtr_dropout_add(int32_t type, int64_t rows, int64_t cols, const void *x, int64_t x_stride, const void *residual,
                    int64_t residual_stride, void *out, int64_t out_stride, double p, uint64_t seed, uint64_t offset,
                    void *stream)
{
    if (!known_type(type)) return fail(DTR_EINVAL, "dropout: unknown type %d", type);
    if (rows < 0 || cols < 0 || rows >= MAX_ROWS || (cols && rows > (int64_t(1) << 48) / cols))
        return fail(DTR_EINVAL, "dropout: %lld x %lld elements", (long long)rows, (long long)cols);
    if (!(p >= 0 && p <= 1)) return fail(DTR_EINVAL, "dropout: probability %g is not within 0..1", p);
    if (rows == 0 || cols == 0) return DTR_OK;
    if (!x || !out) return fail(DTR_EINVAL, "dropout: null %s", x ? "out" : "x");
    if (x_stride < 0 || residual_stride < 0 || (rows > 1 && out_stride < cols))
        return fail(DTR_EINVAL, "dropout: row strides %lld, %lld, %lld of %lld columns", (long long)x_stride,
                    (long long)residual_stride, (long long)out_stride, (long long)cols);
    const int64_t size = type == DTR_FP32 ? 4 : 2;
    if ((uintptr_t)x % size || (uintptr_t)out % size || (residual && (uintptr_t)residual % size))
        return fail(DTR_EINVAL, "dropout: addresses are not multiples of the element size");
    DropArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.residual = residual;
    a.out = out;
    a.x_stride = x_stride;
    a.r_stride = residual ? residual_stride : 0;
    a.o_stride = out_stride;
    if (rows == 1 || (x_stride == cols && out_stride == cols && (!residual || residual_stride == cols))) {
        a.cols = rows * cols;                       // one long row
        a.rows = 1;
        a.x_stride = a.r_stride = a.o_stride = 0;
    }
    a.vector = (uintptr_t)x % 16 == 0 && (uintptr_t)out % 16 == 0 && (uintptr_t)residual % 16 == 0 &&
               (a.rows == 1 || (cols % 8 == 0 && a.x_stride % 8 == 0 && a.r_stride % 8 == 0 && a.o_stride % 8 == 0));
    a.key = mix64(seed + 0x9E3779B97F4A7C15ull);
    a.offset = offset;
    a.threshold = (uint64_t)std::floor(p * 4294967296.0);
    a.inv = p < 1 ? (float)(1.0 / (1.0 - p)) : 0.0f;
    return launched(launch_dropout(a, type, (hipStream_t)stream), "dropout");
}

int dtr_logprobs_workspace_bytes(int32_t type, int64_t rows, int64_t vocab, int32_t top, size_t *bytes)
{
    if (!bytes) return fail(DTR_EINVAL, "null bytes");
    if (int rc = check_logprobs(type, rows, vocab, top)) return rc;
    const int32_t s = logprob_splits(rows, vocab);
    *bytes = s > 1 ? align_up(sizeof(float) * 4 * rows * s) + align_up(sizeof(float2) * rows * s * top) : 0;
    return DTR_OK;
}

int dtr_logprobs_forward(int32_t type, int64_t rows, int64_t vocab, int32_t top, const void *logits, int64_t stride,
                         const int64_t *tokens, float *logp, float *entropy, float *lse, float *top_logp,
                         int64_t *top_ids, void *workspace, size_t workspace_bytes, void *stream)
{
    size_t needed = 0;
    if (int rc = dtr_logprobs_workspace_bytes(type, rows, vocab, top, &needed)) return rc;
    if (rows == 0) return DTR_OK;
    if (!logits || !tokens || !logp || !entropy || !lse || (top && (!top_logp || !top_ids)))
        return fail(DTR_EINVAL, "log probabilities: null argument");
    const int64_t size = type == DTR_FP32 ? 4 : 2;
    if ((uintptr_t)logits % size) return fail(DTR_EINVAL, "log probabilities: logits are not aligned to their elements");
    if (stride < 0) return fail(DTR_EINVAL, "log probabilities: row stride %lld", (long long)stride);
    if (int rc = check_workspace(workspace, workspace_bytes, needed)) return rc;
    LogpArgs a{};
    a.rows = rows;
    a.vocab = vocab;
    a.stride = stride;
    a.top = top;
    a.splits = logprob_splits(rows, vocab);
    a.x = logits;
    a.tokens = tokens;
    a.logp = logp;
    a.entropy = entropy;
    a.lse = lse;
    a.top_logp = top_logp;
    a.top_ids = top_ids;
    a.part = (float *)workspace;
    a.part_top = (float2 *)((char *)workspace + align_up(sizeof(float) * 4 * rows * a.splits));
    return launched(launch_logprobs(a, type, (hipStream_t)stream), "log probabilities");
}

int dtr_logprobs_backward(int32_t type, int64_t rows, int64_t vocab, int32_t top, const void *logits, int64_t stride,
                          const int64_t *tokens, const float *entropy, const float *lse, const int64_t *top_ids,
                          const float *dlogp, const float *dentropy, const float *dtop_logp, void *dlogits,
                          int64_t dstride, void *stream)
{
    if (int rc = check_logprobs(type, rows, vocab, top)) return rc;
    if (rows == 0) return DTR_OK;
    if (!logits || !tokens || !entropy || !lse || !dlogits || (top && dtop_logp && !top_ids))
        return fail(DTR_EINVAL, "log probabilities: null argument");
    const int64_t size = type == DTR_FP32 ? 4 : 2;
    if ((uintptr_t)logits % size || (uintptr_t)dlogits % size)
        return fail(DTR_EINVAL, "log probabilities: logits or gradient are not aligned to their elements");
    if (stride < 0 || (rows > 1 && dstride < vocab))
        return fail(DTR_EINVAL, "log probabilities: row strides %lld and %lld", (long long)stride, (long long)dstride);
    LogpGradArgs a{};
    a.rows = rows;
    a.vocab = vocab;
    a.stride = stride;
    a.dstride = dstride;
    a.top = dtop_logp ? top : 0;
    a.x = logits;
    a.tokens = tokens;
    a.top_ids = top_ids;
    a.entropy = entropy;
    a.lse = lse;
    a.dlogp = dlogp;
    a.dentropy = dentropy;
    a.dtop = dtop_logp;
    a.dx = dlogits;
    return launched(launch_logprobs_grad(a, type, (hipStream_t)stream), "log probabilities' gradient");
}

}  // extern "C"
