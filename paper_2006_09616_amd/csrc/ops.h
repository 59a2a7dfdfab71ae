// ops.h -- what the host file (dtr_ops.cpp) and the kernels of the operators
// (attention.hip, rows.hip) share: argument records, launch plans and the
// launchers.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace dtrops {

constexpr int KEY_TILE = 64;      // keys of a tile of the attention kernels
constexpr int ROW_TILE = 128;     // rows (queries x heads of a group) of a workgroup
constexpr int FEW_ROWS = 32;      // rows of a key head that the kernel for few rows takes
constexpr int GRAD_KEYS = 128;    // keys of a workgroup that sums dK and dV
constexpr int SEGS = 4;           // wavefronts of a workgroup of the log-probability kernel

struct Heads {                    // [batch][position][head][head_dim], strides in elements
    char *data;
    int64_t batch, position, head;
};

struct AttnArgs {
    int32_t batch, q_len, k_len, k_heads, group, head_dim, causal;
    float scale, cap;
    const float *slopes;
    const int32_t *prefix, *docs, *lengths, *starts;
    Heads q, k, v, out;
    char *rest;                   // [batch][q_len][q_heads][head_dim] what rounding took from out, or NULL
    float *lse;                   // [batch][q_heads][q_len]
    int32_t rows;                 // q_len * group: rows of one key head, row = query * group + head of the group
    int32_t splits;               // parts that the keys are split into (forward)
    int32_t key_tiles;            // ceil(k_len / KEY_TILE)
    int2 *doc_tiles;              // [batch][key_tiles] smallest and largest document of each tile
    float *part_out;              // [splits][batch][k_heads][rows][head_dim] (splits > 1)
    float2 *part_stat;            // [splits][batch][k_heads][rows] maximum and sum
};

// What the backward pass needs besides; apart, as the smallest forward calls
// notice the size of their arguments.
struct AttnGradArgs : AttnArgs {
    Heads dout, dq, dk, dv;
    int32_t parts;                // parts that the rows are cut into (dK and dV)
    float *part_grad;             // [parts][2][batch][k_heads][k_len][head_dim] (parts > 1)
    float2 *row_stat;             // [batch][q_heads][q_len] log2-sum-exp2 and out . dout
    int32_t chunks;               // of a key head's values, whose largest numbers are looked for (fp16)
    float *value_magnitude;       // [batch][k_heads][chunks] largest finite number of v
    float *row_magnitude;         // [batch][k_heads][row tiles][4] of dout, 32 rows each
};

struct LogpArgs {
    int64_t rows, vocab, stride;
    int32_t top, splits;
    const void *x;
    const int64_t *tokens;
    float *logp, *entropy, *lse, *top_logp;
    int64_t *top_ids;
    float *part;                  // [rows][splits][4] maximum, sum, weighted sum, the token's logit
    float2 *part_top;             // [rows][splits][top] value, column (as bits)
};

struct LogpGradArgs {
    int64_t rows, vocab, stride, dstride;
    int32_t top;
    const void *x;
    const int64_t *tokens, *top_ids;
    const float *entropy, *lse, *dlogp, *dentropy, *dtop;
    void *dx;
};

struct DropArgs {
    int64_t rows, cols, x_stride, r_stride, o_stride;
    const void *x, *residual;
    void *out;
    uint64_t key, offset, threshold;
    float inv;
    int32_t vector;               // groups of 8 elements start at multiples of 16 bytes
};

hipError_t launch_attn_forward(const AttnArgs &a, int type, hipStream_t st);
hipError_t launch_attn_backward(const AttnGradArgs &a, int type, hipStream_t st);
hipError_t launch_logprobs(const LogpArgs &a, int type, hipStream_t st);
hipError_t launch_logprobs_grad(const LogpGradArgs &a, int type, hipStream_t st);
hipError_t launch_dropout(const DropArgs &a, int type, hipStream_t st);

}  // namespace dtrops
