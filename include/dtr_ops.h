/*
 * dtr_ops.h -- C ABI of the operators of a transformer's training step that
 * store nothing their backward pass can make again, for AMD Instinct MI355X
 * (gfx950).
 *
 * Rematerialization (include/dtr_sim.h simulates its policies) trades stored
 * tensors for recomputation between operators.  The operators here do the
 * same within one operator, for the three tensors that a transformer step
 * stores at sizes out of proportion to its activations: the probabilities of
 * an attention (queries x keys), the mask of a dropout, and the softmax of a
 * loss (tokens x vocabulary).  None of them uses atomics on results: the same
 * call on the same inputs gives the same bits, as recomputation assumes.
 *
 * Conventions (as in dtr_sim.h):
 *   - every tensor is device memory, owned by the caller; nothing is kept
 *     after the call's work on `stream` (a hipStream_t as void*) has run;
 *   - calls are asynchronous, allocate nothing and may be captured in a graph;
 *   - the workspace is caller-owned device memory of at least the size that
 *     the matching _workspace_bytes call gives (256-byte aligned; NULL where
 *     that is 0);
 *   - functions return DTR_OK or a negative DTR_E* code; dtr_sim_last_error()
 *     has the message.  Numbers in device memory (lengths, tokens, ...) cannot
 *     be checked by the host; the kernels clamp them, as said below.
 */
#ifndef DTR_OPS_H
#define DTR_OPS_H

#include "dtr_sim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define DTR_BF16 0
#define DTR_FP16 1
#define DTR_FP32 2

/* ---- attention ---------------------------------------------------------------
 * For request b, query i at position p = starts[b] + i, query head h and its
 * key head g = h / (q_heads / k_heads), over keys j:
 *   c  = scale q.k                            (cap == 0)
 *   c  = cap tanh(scale q.k / cap)            (cap > 0)
 *   s  = c - slopes[h] |p - j|
 *   j is seen  iff  j < lengths[b]
 *              and  (not causal, or j <= p, or j < prefix[b])
 *              and  (no docs, or 0 <= p < k_len and docs[b][p] == docs[b][j])
 *   out = sum over seen j of softmax(s)_j v_j,  lse = log sum exp s.
 * A query that sees no key has out = 0, lse = -infinity and adds nothing to
 * any gradient.  Sums and softmax statistics are held in 32 bits; the
 * probabilities (and, backward, the gradients of the scores) are rounded to
 * the inputs' type for the matrix instructions, in fp16 times powers of two
 * that keep them within its range.
 * Keys from lengths[b] on are not read (values there may be anything).
 * Infinities and NaN reach the queries that see them and no others.  Gradients
 * of a query that has an infinite component, or sees a key with one, may be
 * NaN where a cap or a probability of zero makes them finite.
 */
typedef struct {
    int32_t type;               /* DTR_BF16 or DTR_FP16                               */
    int32_t batch;              /* requests, >= 0                                     */
    int32_t q_len, k_len;       /* queries and key slots of each, 0 .. 2^24           */
    int32_t q_heads, k_heads;   /* q_heads a multiple of k_heads                      */
    int32_t head_dim;           /* a multiple of 8, 8 .. 128                          */
    int32_t causal;             /* 0 or 1                                             */
    float scale;                /* > 0, finite                                        */
    float cap;                  /* 0 (none) or > 0, finite                            */
    const float *slopes;        /* [q_heads], or NULL: no bias                        */
    const int32_t *prefix;      /* [batch], or NULL; needs causal                     */
    const int32_t *docs;        /* [batch][k_len] document of each position, or NULL  */
    const int32_t *lengths;     /* [batch], or NULL: k_len; clamped to 0 .. k_len     */
    const int32_t *starts;      /* [batch], or NULL: k_len - q_len; clamped to
                                   -2^24 .. 2^24                                      */
} dtr_attn;

/* A tensor [batch][position][head][head_dim]: strides in elements, the last
 * dimension contiguous; data 16-byte aligned and strides multiples of 8,
 * that of positions below 2^24.  Input strides may be 0 (broadcast). */
typedef struct {
    void *data;
    int64_t batch, position, head;
} dtr_heads;

int dtr_attn_workspace_bytes(const dtr_attn *attn, int32_t backward, size_t *bytes);

/* out like q; lse [batch][q_heads][q_len] 32-bit, NULL if no backward follows.
 * rest [batch][q_len][q_heads][head_dim] (contiguous, the inputs' type; or
 * NULL) receives what the rounding took from out.  With it the backward pass
 * knows out . dout, which it subtracts from every score gradient of a row, to
 * twice the digits; without it dq and dk lose about a third of a bit. */
int dtr_attn_forward(const dtr_attn *attn, const dtr_heads *q, const dtr_heads *k, const dtr_heads *v,
                     const dtr_heads *out, void *rest, float *lse, void *workspace, size_t workspace_bytes,
                     void *stream);

/* Gradients dq, dk, dv of the forward pass that gave out, rest (or NULL) and lse. */
int dtr_attn_backward(const dtr_attn *attn, const dtr_heads *q, const dtr_heads *k, const dtr_heads *v,
                      const dtr_heads *out, const void *rest, const float *lse, const dtr_heads *dout,
                      const dtr_heads *dq, const dtr_heads *dk, const dtr_heads *dv,
                      void *workspace, size_t workspace_bytes, void *stream);

/* ---- dropout with the residual sum ---------------------------------------------
 * out[r][c] = residual[r][c] + (kept ? x[r][c] / (1 - p) : 0), computed in 32
 * bits and rounded once.  The mask is a function of (seed, offset) and the
 * element's number e = r cols + c alone, whatever the strides:
 *   mix(z): z = (z ^ z >> 30) 0xBF58476D1CE4E5B9, z = (z ^ z >> 27)
 *           0x94D049BB133111EB, z ^ z >> 31  (the SplitMix64 finaliser)
 *   draw(n) = mix(mix(seed + G) + G n),  G = 0x9E3779B97F4A7C15, modulo 2^64
 *   u = the low (e even) or high (e odd) 32 bits of draw(offset + e / 2)
 *   kept  iff  u >= floor(p 2^32)
 * The backward pass of x is the same call on the output's gradient with
 * residual NULL.  A call of n elements uses the draws offset ..
 * offset + (n + 1) / 2 - 1.
 * x, residual (or NULL) and out are [rows][cols] with row strides in elements
 * and contiguous columns; out may be x or residual itself.
 */
int dtr_dropout_add(int32_t type, int64_t rows, int64_t cols, const void *x, int64_t x_stride,
                    const void *residual, int64_t residual_stride, void *out, int64_t out_stride,
                    double p, uint64_t seed, uint64_t offset, void *stream);

/* ---- log probabilities of given tokens -------------------------------------------
 * For each row t of logits x [rows][vocab] (row stride in elements, contiguous
 * columns; bf16, fp16 or fp32), with L = log sum exp x:
 *   logp[t]    = x[token] - L;  0 if tokens[t] < 0 (no token);  NaN if
 *                tokens[t] >= vocab
 *   entropy[t] = L - sum softmax(x) x   (minus infinity in x counts as 0)
 *   top_logp[t][0..top-1], top_ids[t][0..top-1]: the largest x - L and their
 *                columns, largest first, the lower column among equals
 * All outputs are 32-bit but top_ids (64-bit); lse [rows] is L, for the
 * backward pass.  A row of nothing but minus infinity has lse = -infinity,
 * entropy 0, logp and top_logp -infinity (logp 0 without a token) and a zero
 * gradient.  A row with a NaN (or plus infinity) has NaN lse, logp, entropy
 * and top_logp; its top_ids are columns, in no particular order.
 */
#define DTR_TOP_MAX 32

int dtr_logprobs_workspace_bytes(int32_t type, int64_t rows, int64_t vocab, int32_t top, size_t *bytes);

int dtr_logprobs_forward(int32_t type, int64_t rows, int64_t vocab, int32_t top, const void *logits,
                         int64_t stride, const int64_t *tokens, float *logp, float *entropy, float *lse,
                         float *top_logp, int64_t *top_ids, void *workspace, size_t workspace_bytes,
                         void *stream);

/* Gradient of the logits: with G = dlogp + sum_k dtop_logp (dlogp taken as 0
 * where tokens[t] < 0), p = softmax(x), H = entropy,
 *   dx_v = dlogp [v = token] + sum_k dtop_logp_k [v = top_ids_k] - G p_v
 *          - dentropy p_v (log p_v + H).
 * dlogp, dentropy and dtop_logp (with top_ids) may each be NULL: zero.  With
 * dlogp, the gradient of a row whose token is >= vocab is NaN. */
int dtr_logprobs_backward(int32_t type, int64_t rows, int64_t vocab, int32_t top, const void *logits,
                          int64_t stride, const int64_t *tokens, const float *entropy, const float *lse,
                          const int64_t *top_ids, const float *dlogp, const float *dentropy,
                          const float *dtop_logp, void *dlogits, int64_t dstride, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DTR_OPS_H */
