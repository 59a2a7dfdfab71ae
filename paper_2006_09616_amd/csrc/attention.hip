// attention.hip -- attention whose probabilities are never stored: forward,
// backward, and the join of parts where the keys are split.
//
// All three products use the 32x32x16 matrix instruction with the operands
// ordered so that the probabilities never change lanes.  Forward: S^T = K Q^T
// leaves one query per lane (column lane % 32) and 16 of 32 keys in its
// registers, so a row's maximum and sum are a reduction over registers and one
// exchange with lane ^ 32.  O^T = V^T P^T takes those registers as they are:
// a product may run over its keys in any order, so V^T is read (transposed,
// from LDS) in the order in which the lane holds its keys.  Backward does the
// same with the roles of queries and keys exchanged where needed.
#include "ops.h"

namespace dtrops {
namespace {

constexpr int WAVE = 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.402823466e+38f;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

struct Bf16 {
    using raw = __bf16;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static __device__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static constexpr float p_gain = 1.0f;
};
// Backward probabilities of long rows are below the smallest normal number
// of fp16; 2^6 keeps six more bits of them (they are at most 1).
struct Fp16 {
    using raw = _Float16;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static __device__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static constexpr float p_gain = 64.0f;
};

// eight numbers rounded to the inputs' type: an operand of the next product
template <typename T> __device__ __forceinline__ s16x8 rounded(const float *p)
{
    typename T::v8 v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (typename T::raw)p[i];
    return __builtin_bit_cast(s16x8, v);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// the other half's value: lane ^ 32
__device__ __forceinline__ float other_half(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// tanh(x) = 1 - 2 / (1 + exp(2 x)), with x2 = 2 log2(e) x
__device__ __forceinline__ float tanh_of(float x2) { return 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + exp2_(x2)); }

// A tile in LDS: rows of PITCH 16-bit elements as chunks of 16 bytes, chunk c
// of row r at c ^ swizzle(r).  Reads of a row's chunk by 16 consecutive rows,
// and of four chunks by four consecutive rows (the transposed reads), then
// fall on distinct banks.
template <int NB> struct Tile {
    static constexpr int PITCH = NB <= 2 ? 64 : 128, CHUNKS = PITCH / 8;
    static __device__ int swizzle(int r)
    {
        return CHUNKS == 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    }
    static __device__ int at(int r, int chunk) { return r * PITCH + ((chunk ^ swizzle(r)) << 3); }      // in elements

    // operand of rows: row lane % 32, elements 16 s + 8 (lane / 32) ..
    static __device__ s16x8 row_operand(const short *tile, int row, int s)
    {
        const int lane = threadIdx.x % WAVE;
        return *(const s16x8 *)(tile + at(row, 2 * s + lane / 32));
    }
    // operand of columns: column 32 d + lane % 32, over the rows row0 + 4 (lane / 32) + {0..3, 8..11}
    static __device__ s16x8 column_operand(short *tile, int row0, int d)
    {
        const int lane = threadIdx.x % WAVE, j = lane % 16, blk = lane / 16;
        const int r = row0 + 4 * (blk >> 1) + j / 4, chunk = 4 * d + 2 * (blk & 1) + (j % 4) / 2, off = (j & 1) * 4;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + at(r, chunk) + off));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + at(r + 8, chunk) + off));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// ROWS rows of a tensor on their way to LDS, 256 threads; rows from `end` on
// and columns from head_dim on are zero.
template <int NB, int ROWS> struct Staged {
    using L = Tile<NB>;
    static constexpr int N = ROWS * L::CHUNKS / 256;
    uint4 r[N];
    __device__ void load(const char *base, int64_t stride, int row0, int end, int head_dim)
    {
        const int c = threadIdx.x % L::CHUNKS;
#pragma unroll
        for (int n = 0; n < N; n++) {
            const int row = row0 + threadIdx.x / L::CHUNKS + n * (256 / L::CHUNKS);
            r[n] = row < end && c * 8 < head_dim ? *(const uint4 *)(base + ((int64_t)row * stride + c * 8) * 2)
                                                 : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ void store(short *tile) const
    {
        const int c = threadIdx.x % L::CHUNKS;
#pragma unroll
        for (int n = 0; n < N; n++) *(uint4 *)(tile + L::at(threadIdx.x / L::CHUNKS + n * (256 / L::CHUNKS), c)) = r[n];
    }
};

// Rows of one key head in packed order: row = query * group + head of the
// group, so that a tile holds the group's heads of few queries and reads the
// keys once for all of them.
struct Unit {
    int b, g, start, len, prefix;
    const int *docs;
    const int2 *doc_tiles;
    __device__ Unit(const AttnArgs &a, int unit)
    {
        b = unit / a.k_heads;
        g = unit % a.k_heads;
        start = a.starts ? min(max(a.starts[b], -(1 << 24)), 1 << 24) : a.k_len - a.q_len;
        len = a.lengths ? min(max(a.lengths[b], 0), a.k_len) : a.k_len;
        prefix = a.prefix ? a.prefix[b] : 0;
        docs = a.docs ? a.docs + (int64_t)b * a.k_len : nullptr;
        doc_tiles = a.doc_tiles + (int64_t)b * a.key_tiles;
    }
    // keys from here on are masked for a query at position p
    __device__ int end(const AttnArgs &a, int p) const { return a.causal ? min(len, max(p + 1, prefix)) : len; }
};

// 64-bit offsets from the base, in bytes of 16-bit elements
__device__ __forceinline__ const char *head_base(const Heads &t, int b, int head)
{
    return t.data + (b * t.batch + head * t.head) * 2;
}

// Workgroups go round the 8 dies; neighbours in `unit` share keys, so each die
// gets a contiguous range.
__device__ __forceinline__ int spread(int id, int n)
{
    const int per = n / 8, rest = n % 8, x = id % 8, i = id / 8;
    return x * per + min(x, rest) + i;
}

__global__ void __launch_bounds__(64) doc_tiles_kernel(AttnArgs a)
{
    const int tile = blockIdx.x, b = blockIdx.y, j = tile * KEY_TILE + threadIdx.x;
    for (int bb = b; bb < a.batch; bb += gridDim.y) {
        const int d = a.docs[(int64_t)bb * a.k_len + min(j, a.k_len - 1)];
        int lo = d, hi = d;
#pragma unroll
        for (int s = 1; s < WAVE; s *= 2) {
            lo = min(lo, __shfl_xor(lo, s));
            hi = max(hi, __shfl_xor(hi, s));
        }
        if (threadIdx.x == 0) a.doc_tiles[(int64_t)bb * a.key_tiles + tile] = make_int2(lo, hi);
    }
}

// ---- forward -----------------------------------------------------------------
// A workgroup has 128 rows, a wavefront 32, and walks over tiles of 64 keys.

template <typename T, int NB, bool CAP>
__global__ void __launch_bounds__(256, 2) forward_kernel(AttnArgs a)
{
    using L = Tile<NB>;
    using R = typename T::raw;
    __shared__ __align__(16) short ks[KEY_TILE * L::PITCH], vs[KEY_TILE * L::PITCH];
    __shared__ int range[4];                            // first and last active tile, least and greatest document

    const int row_tiles = (a.rows + ROW_TILE - 1) / ROW_TILE;
    const int units = a.batch * a.k_heads;
    int id = spread(blockIdx.x, gridDim.x);
    const int split = id % a.splits;
    id /= a.splits;
    const Unit u(a, id / row_tiles);
    const int tile_row = (row_tiles - 1 - id % row_tiles) * ROW_TILE;      // the longest first under a causal mask
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, hi = lane / 32;

    const int row = tile_row + wave * 32 + lane % 32;
    const int crow = min(row, a.rows - 1);
    const int query = crow / a.group, head = u.g * a.group + crow % a.group;
    const int pos = u.start + query;
    const int p_first = u.start + tile_row / a.group, p_last = u.start + min(tile_row + ROW_TILE - 1, a.rows - 1) / a.group;
    const bool has_doc = !u.docs || (pos >= 0 && pos < a.k_len);
    const int doc = u.docs && has_doc ? u.docs[pos] : 0;
    const int row_end = has_doc ? u.end(a, pos) : 0;

    // tiles that any row of the workgroup may see
    int t0 = 0, t1 = (u.end(a, p_last) + KEY_TILE - 1) / KEY_TILE, doc_lo = 0, doc_hi = 0;
    bool one_doc = true;
    if (u.docs) {
        if (threadIdx.x == 0) {
            range[0] = INT32_MAX;
            range[1] = -1;
            range[2] = INT32_MAX;
            range[3] = INT32_MIN;
        }
        __syncthreads();
        if (has_doc) {
            atomicMin(&range[2], doc);
            atomicMax(&range[3], doc);
        }
        one_doc = __syncthreads_and(has_doc);
        doc_lo = range[2];
        doc_hi = range[3];
        for (int t = threadIdx.x; t < t1; t += 256) {
            const int2 d = u.doc_tiles[t];
            if (d.x <= doc_hi && d.y >= doc_lo) {
                atomicMin(&range[0], t);
                atomicMax(&range[1], t);
            }
        }
        __syncthreads();
        t0 = range[0];
        t1 = range[1] + 1;
        one_doc = one_doc && doc_lo == doc_hi;
    }
    if (a.splits > 1) {                                  // this part's tiles
        const int n = max(t1 - t0, 0), per = (n + a.splits - 1) / a.splits;
        t0 = min(t0, t1) + per * split;
        t1 = min(t0 + per, t1);
    }

    s16x8 q[2 * NB];
    {
        const char *qp = head_base(a.q, u.b, head) + query * a.q.position * 2;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++) {
            const int d = 16 * s + 8 * hi;
            q[s] = d < a.head_dim ? *(const s16x8 *)(qp + d * 2) : s16x8{};
        }
    }
    const float slope2 = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
    const float scale2 = CAP ? 2.0f * LOG2E * a.scale / a.cap : a.scale * LOG2E, cap2 = a.cap * LOG2E;

    f32x16 o[NB] = {};
    float m = LOWEST, l = 0;
    const char *kb = head_base(a.k, u.b, u.g), *vb = head_base(a.v, u.b, u.g);

    for (int t = t0; t < t1; t++) {
        const int j0 = t * KEY_TILE;
        bool in_doc = true;
        if (u.docs) {
            const int2 d = u.doc_tiles[t];
            if (d.x > doc_hi || d.y < doc_lo) continue;
            in_doc = one_doc && d.x == d.y;
        }
        Staged<NB, KEY_TILE> sk, sv;
        sk.load(kb, a.k.position, j0, u.len, a.head_dim);
        sv.load(vb, a.v.position, j0, u.len, a.head_dim);
        __syncthreads();
        sk.store(ks);
        sv.store(vs);
        __syncthreads();
        const bool whole = in_doc && j0 + KEY_TILE <= u.end(a, p_first);

        f32x16 s[2] = {};
#pragma unroll
        for (int kbk = 0; kbk < 2; kbk++)
#pragma unroll
            for (int st = 0; st < 2 * NB; st++)
                s[kbk] = T::mfma(L::row_operand(ks, 32 * kbk + lane % 32, st), q[st], s[kbk]);

        float x[32];
        const float pf = (float)(pos - j0 - 4 * hi);
        float most = LOWEST;
#pragma unroll
        for (int i = 0; i < 32; i++) {
            const int c = 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4;          // key j0 + 4 hi + c
            float v = s[i / 16][i % 16] * scale2;
            if (CAP) v = cap2 * tanh_of(v);
            if (a.slopes) v -= slope2 * fabsf(pf - (float)c);
            x[i] = v;
        }
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 32; i++) {
                const int j = j0 + 4 * hi + 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4;
                bool seen = j < row_end;
                if (u.docs) seen = seen && u.docs[min(j, a.k_len - 1)] == doc;
                x[i] = seen ? x[i] : -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < 32; i++) most = fmaxf(most, x[i]);
        most = fmaxf(most, other_half(most));
        const float m_new = fmaxf(m, most);
        const float f = exp2_(m - m_new);
        m = m_new;
        l *= f;
#pragma unroll
        for (int d = 0; d < NB; d++) o[d] *= f;
#pragma unroll
        for (int i = 0; i < 32; i++) {
            x[i] = exp2_(x[i] - m);
            l += x[i];
        }
#pragma unroll
        for (int kc = 0; kc < 4; kc++) {
            const s16x8 p = rounded<T>(x + 8 * kc);
#pragma unroll
            for (int d = 0; d < NB; d++) o[d] = T::mfma(L::column_operand(vs, 16 * kc, d), p, o[d]);
        }
    }
    l += other_half(l);
    if (row >= a.rows) return;
    const bool nothing = l == 0;
    if (a.splits > 1) {
        const int64_t at = ((int64_t)split * units + u.b * a.k_heads + u.g) * a.rows + row;
        float *po = a.part_out + at * a.head_dim;
#pragma unroll
        for (int d = 0; d < NB; d++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int col = 32 * d + 8 * e + 4 * hi;
                if (col < a.head_dim) *(f32x4 *)(po + col) = f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
            }
        if (hi == 0) a.part_stat[at] = make_float2(m, l);
        return;
    }
    const float inv = nothing ? 0.0f : 1.0f / l;
    char *op = a.out.data + (u.b * a.out.batch + head * a.out.head + query * a.out.position) * 2;
#pragma unroll
    for (int d = 0; d < NB; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int col = 32 * d + 8 * e + 4 * hi;
            typedef R r4 __attribute__((ext_vector_type(4)));
            r4 v;
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = (R)(nothing ? 0.0f : o[d][4 * e + i] * inv);
            if (col < a.head_dim) *(r4 *)(op + col * 2) = v;
        }
    if (a.lse && hi == 0)
        a.lse[((int64_t)u.b * a.k_heads * a.group + head) * a.q_len + query] =
            nothing ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// Joins the parts of a row: 8 rows a workgroup, 32 lanes a row, 4 columns each.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(AttnArgs a)
{
    using R = typename T::raw;
    const int64_t units = (int64_t)a.batch * a.k_heads, n = units * a.rows;
    const int64_t r = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (r >= n) return;
    const int c = threadIdx.x % 32 * 4;
    float m = LOWEST, l = 0;
    for (int s = 0; s < a.splits; s++) m = fmaxf(m, a.part_stat[s * n + r].x);
    f32x4 o = {};
    for (int s = 0; s < a.splits; s++) {
        const float2 st = a.part_stat[s * n + r];
        const float f = exp2_(st.x - m);
        l += st.y * f;
        if (c < a.head_dim) o += *(const f32x4 *)(a.part_out + (s * n + r) * a.head_dim + c) * f;
    }
    const bool nothing = l == 0;
    const int64_t unit = r / a.rows;
    const int row = (int)(r % a.rows), b = (int)(unit / a.k_heads), g = (int)(unit % a.k_heads);
    const int query = row / a.group, head = g * a.group + row % a.group;
    if (c < a.head_dim) {
        typedef R r4 __attribute__((ext_vector_type(4)));
        r4 v;
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = (R)(nothing ? 0.0f : o[i] / l);
        *(r4 *)(a.out.data + (b * a.out.batch + head * a.out.head + query * a.out.position + c) * 2) = v;
    }
    if (a.lse && c == 0)
        a.lse[((int64_t)b * a.k_heads * a.group + head) * a.q_len + query] =
            nothing ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// ---- backward ------------------------------------------------------------------
// With L = log-sum-exp and D = out . dout of each row:
//   P = exp(s - L), dP = dout V^T, dS = P (dP - D) (1 - tanh^2)
//   dV = P^T dout, dK = scale dS^T Q, dQ = scale dS K
// Scores are made again from Q and K in both kernels below: one owns rows and
// sums dQ over the keys, the other owns keys and sums dK and dV over the rows
// of all heads of the group.  Seven products instead of five, but every sum
// has one owner and a fixed order: no atomics, the same bits each time.

// log2-sum-exp2 (plus infinity for a row that sees nothing, so that its P is 0) and D
template <typename T>
__global__ void __launch_bounds__(256) row_stat_kernel(AttnArgs a)
{
    using R = typename T::raw;
    typedef R r8 __attribute__((ext_vector_type(8)));
    const int64_t n = (int64_t)a.batch * a.k_heads * a.rows;
    const int64_t r = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    if (r >= n) return;
    const int64_t unit = r / a.rows;
    const int row = (int)(r % a.rows), b = (int)(unit / a.k_heads), g = (int)(unit % a.k_heads);
    const int query = row / a.group, head = g * a.group + row % a.group, c = threadIdx.x % 16 * 8;
    float sum = 0;
    if (c < a.head_dim) {
        const r8 x = *(const r8 *)(head_base(a.out, b, head) + (query * a.out.position + c) * 2);
        const r8 y = *(const r8 *)(head_base(a.dout, b, head) + (query * a.dout.position + c) * 2);
#pragma unroll
        for (int i = 0; i < 8; i++) sum += (float)x[i] * (float)y[i];
    }
#pragma unroll
    for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
    if (c == 0) {
        const float lse = a.lse[((int64_t)b * a.k_heads * a.group + head) * a.q_len + query];
        a.row_stat[r] = make_float2(lse == -INFINITY ? INFINITY : lse * LOG2E, sum);
    }
}

template <typename T, int NB, bool CAP>
__global__ void __launch_bounds__(256, 2) dq_kernel(AttnArgs a)
{
    using L = Tile<NB>;
    using R = typename T::raw;
    __shared__ __align__(16) short ks[KEY_TILE * L::PITCH], vs[KEY_TILE * L::PITCH];
    __shared__ int range[4];

    const int row_tiles = (a.rows + ROW_TILE - 1) / ROW_TILE;
    const int id = spread(blockIdx.x, gridDim.x);
    const Unit u(a, id / row_tiles);
    const int tile_row = (row_tiles - 1 - id % row_tiles) * ROW_TILE;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, hi = lane / 32;
    const int row = tile_row + wave * 32 + lane % 32, crow = min(row, a.rows - 1);
    const int query = crow / a.group, head = u.g * a.group + crow % a.group;
    const int pos = u.start + query;
    const int p_first = u.start + tile_row / a.group, p_last = u.start + min(tile_row + ROW_TILE - 1, a.rows - 1) / a.group;
    const bool has_doc = !u.docs || (pos >= 0 && pos < a.k_len);
    const int doc = u.docs && has_doc ? u.docs[pos] : 0;
    const int row_end = has_doc ? u.end(a, pos) : 0;

    int t0 = 0, t1 = (u.end(a, p_last) + KEY_TILE - 1) / KEY_TILE, doc_lo = 0, doc_hi = 0;
    bool one_doc = true;
    if (u.docs) {
        if (threadIdx.x == 0) {
            range[0] = INT32_MAX;
            range[1] = -1;
            range[2] = INT32_MAX;
            range[3] = INT32_MIN;
        }
        __syncthreads();
        if (has_doc) {
            atomicMin(&range[2], doc);
            atomicMax(&range[3], doc);
        }
        one_doc = __syncthreads_and(has_doc);
        doc_lo = range[2];
        doc_hi = range[3];
        for (int t = threadIdx.x; t < t1; t += 256) {
            const int2 d = u.doc_tiles[t];
            if (d.x <= doc_hi && d.y >= doc_lo) {
                atomicMin(&range[0], t);
                atomicMax(&range[1], t);
            }
        }
        __syncthreads();
        t0 = range[0];
        t1 = range[1] + 1;
        one_doc = one_doc && doc_lo == doc_hi;
    }

    s16x8 q[2 * NB], g[2 * NB];
    {
        const char *qp = head_base(a.q, u.b, head) + query * a.q.position * 2;
        const char *gp = head_base(a.dout, u.b, head) + query * a.dout.position * 2;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++) {
            const int d = 16 * s + 8 * hi;
            q[s] = d < a.head_dim ? *(const s16x8 *)(qp + d * 2) : s16x8{};
            g[s] = d < a.head_dim ? *(const s16x8 *)(gp + d * 2) : s16x8{};
        }
    }
    const float2 stat = a.row_stat[(int64_t)(u.b * a.k_heads + u.g) * a.rows + crow];
    const float slope2 = a.slopes ? a.slopes[head] * LOG2E : 0.0f;
    const float scale2 = CAP ? 2.0f * LOG2E * a.scale / a.cap : a.scale * LOG2E, cap2 = a.cap * LOG2E;
    f32x16 dq[NB] = {};
    const char *kb = head_base(a.k, u.b, u.g), *vb = head_base(a.v, u.b, u.g);

    for (int t = t0; t < t1; t++) {
        const int j0 = t * KEY_TILE;
        bool in_doc = true;
        if (u.docs) {
            const int2 d = u.doc_tiles[t];
            if (d.x > doc_hi || d.y < doc_lo) continue;
            in_doc = one_doc && d.x == d.y;
        }
        Staged<NB, KEY_TILE> sk, sv;
        sk.load(kb, a.k.position, j0, u.len, a.head_dim);
        sv.load(vb, a.v.position, j0, u.len, a.head_dim);
        __syncthreads();
        sk.store(ks);
        sv.store(vs);
        __syncthreads();
        const bool whole = in_doc && j0 + KEY_TILE <= u.end(a, p_first);
#pragma unroll
        for (int kbk = 0; kbk < 2; kbk++) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int st = 0; st < 2 * NB; st++) {
                s = T::mfma(L::row_operand(ks, 32 * kbk + lane % 32, st), q[st], s);
                dp = T::mfma(L::row_operand(vs, 32 * kbk + lane % 32, st), g[st], dp);
            }
            float x[16];
            const float pf = (float)(pos - j0 - 32 * kbk - 4 * hi);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int c = 8 * (i / 4) + i % 4;
                float v = s[i] * scale2, dcap = 1.0f;
                if (CAP) {
                    const float th = tanh_of(v);
                    v = cap2 * th;
                    dcap = 1.0f - th * th;
                }
                if (a.slopes) v -= slope2 * fabsf(pf - (float)c);
                x[i] = exp2_(v - stat.x) * (dp[i] - stat.y) * dcap;
            }
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int j = j0 + 32 * kbk + 4 * hi + 8 * (i / 4) + i % 4;
                    bool seen = j < row_end;
                    if (u.docs) seen = seen && u.docs[min(j, a.k_len - 1)] == doc;
                    x[i] = seen ? x[i] : 0.0f;
                }
            }
#pragma unroll
            for (int kc = 0; kc < 2; kc++) {
                const s16x8 p = rounded<T>(x + 8 * kc);
#pragma unroll
                for (int d = 0; d < NB; d++) dq[d] = T::mfma(L::column_operand(ks, 32 * kbk + 16 * kc, d), p, dq[d]);
            }
        }
    }
    if (row >= a.rows) return;
    char *op = a.dq.data + (u.b * a.dq.batch + head * a.dq.head + query * a.dq.position) * 2;
#pragma unroll
    for (int d = 0; d < NB; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int col = 32 * d + 8 * e + 4 * hi;
            typedef R r4 __attribute__((ext_vector_type(4)));
            r4 v;
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = (R)(dq[d][4 * e + i] * a.scale);
            if (col < a.head_dim) *(r4 *)(op + col * 2) = v;
        }
}

constexpr int GRAD_KEYS = 128;    // keys of a workgroup
constexpr int GRAD_ROWS = 32;     // rows of a step

template <typename T, int NB, bool CAP>
__global__ void __launch_bounds__(256, 1) dkv_kernel(AttnArgs a)
{
    using L = Tile<NB>;
    using R = typename T::raw;
    __shared__ __align__(16) short qs[GRAD_ROWS * L::PITCH], gs[GRAD_ROWS * L::PITCH];
    __shared__ __align__(16) float lse2[GRAD_ROWS], delta[GRAD_ROWS], slopes2[GRAD_ROWS], posf[GRAD_ROWS];
    __shared__ __align__(16) int end[GRAD_ROWS], rdoc[GRAD_ROWS];

    const int key_blocks = (a.k_len + GRAD_KEYS - 1) / GRAD_KEYS;
    const int id = spread(blockIdx.x, gridDim.x);
    const Unit u(a, id / key_blocks);
    const int j0 = id % key_blocks * GRAD_KEYS;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, hi = lane / 32;
    const int key = j0 + wave * 32 + lane % 32;

    s16x8 kf[2 * NB], vf[2 * NB];
    {
        const char *kp = head_base(a.k, u.b, u.g) + key * a.k.position * 2;
        const char *vp = head_base(a.v, u.b, u.g) + key * a.v.position * 2;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++) {
            const int d = 16 * s + 8 * hi;
            const bool in = key < u.len && d < a.head_dim;
            kf[s] = in ? *(const s16x8 *)(kp + d * 2) : s16x8{};
            vf[s] = in ? *(const s16x8 *)(vp + d * 2) : s16x8{};
        }
    }
    const int kdoc = u.docs ? u.docs[min(key, a.k_len - 1)] : 0;
    const float scale2 = CAP ? 2.0f * LOG2E * a.scale / a.cap : a.scale * LOG2E, cap2 = a.cap * LOG2E;
    f32x16 dk[NB] = {}, dv[NB] = {};

    // rows that may see any of the keys
    int r0 = 0, r1 = j0 < u.len ? a.rows : 0, doc_lo = 0, doc_hi = 0;
    if (a.causal && j0 >= u.prefix) r0 = (int)min((int64_t)max(j0 - u.start, 0) * a.group, (int64_t)a.rows) / GRAD_ROWS * GRAD_ROWS;
    if (u.docs) {
        const int2 d0 = u.doc_tiles[j0 / KEY_TILE], d1 = u.doc_tiles[min(j0 / KEY_TILE + 1, a.key_tiles - 1)];
        doc_lo = min(d0.x, d1.x);
        doc_hi = max(d0.y, d1.y);
    }
    const float2 *stats = a.row_stat + (int64_t)(u.b * a.k_heads + u.g) * a.rows;

    for (int rr = r0; rr < r1; rr += GRAD_ROWS) {
        const int p_first = u.start + rr / a.group, p_last = u.start + min(rr + GRAD_ROWS - 1, a.rows - 1) / a.group;
        bool in_doc = true;
        if (u.docs) {
            if (p_last < 0 || p_first >= a.k_len) continue;
            const int2 d0 = u.doc_tiles[max(p_first, 0) / KEY_TILE], d1 = u.doc_tiles[min(p_last, a.k_len - 1) / KEY_TILE];
            bool overlap = false;
            int lo = min(d0.x, d1.x), hi2 = max(d0.y, d1.y);
            for (int t = max(p_first, 0) / KEY_TILE + 1; t < min(p_last, a.k_len - 1) / KEY_TILE; t++) {
                const int2 d = u.doc_tiles[t];
                lo = min(lo, d.x);
                hi2 = max(hi2, d.y);
            }
            overlap = lo <= doc_hi && hi2 >= doc_lo;
            if (!overlap) continue;
            in_doc = lo == hi2 && doc_lo == doc_hi && p_first >= 0 && p_last < a.k_len;
        }
        __syncthreads();
        {
            constexpr int N = GRAD_ROWS * L::CHUNKS / 256;
            const int c = threadIdx.x % L::CHUNKS;
#pragma unroll
            for (int n = 0; n < N; n++) {
                const int i = threadIdx.x / L::CHUNKS + n * (256 / L::CHUNKS), r = rr + i;
                const int query = r / a.group, head = u.g * a.group + r % a.group;
                uint4 x = make_uint4(0, 0, 0, 0), y = x;
                if (r < a.rows && c * 8 < a.head_dim) {
                    x = *(const uint4 *)(head_base(a.q, u.b, head) + (query * a.q.position + c * 8) * 2);
                    y = *(const uint4 *)(head_base(a.dout, u.b, head) + (query * a.dout.position + c * 8) * 2);
                }
                *(uint4 *)(qs + L::at(i, c)) = x;
                *(uint4 *)(gs + L::at(i, c)) = y;
            }
            if (threadIdx.x < GRAD_ROWS) {
                const int i = threadIdx.x, r = rr + i, query = r / a.group, pos = u.start + query;
                const bool in = r < a.rows, has_doc = !u.docs || (pos >= 0 && pos < a.k_len);
                const float2 st = in ? stats[r] : make_float2(INFINITY, 0.0f);
                lse2[i] = st.x;
                delta[i] = st.y / T::p_gain;
                slopes2[i] = a.slopes && in ? a.slopes[u.g * a.group + r % a.group] * LOG2E : 0.0f;
                posf[i] = (float)pos;
                end[i] = in && has_doc ? u.end(a, pos) : 0;
                rdoc[i] = in && u.docs && has_doc ? u.docs[pos] : 0;
            }
        }
        __syncthreads();
        const bool whole = in_doc && j0 + GRAD_KEYS <= u.end(a, p_first);

        f32x16 s = {}, dp = {};
#pragma unroll
        for (int st = 0; st < 2 * NB; st++) {
            s = T::mfma(L::row_operand(qs, lane % 32, st), kf[st], s);
            dp = T::mfma(L::row_operand(gs, lane % 32, st), vf[st], dp);
        }
        float p[16], ds[16];
        const float keyf = (float)key;
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int r = 8 * (i / 4) + 4 * hi + i % 4;
            float v = s[i] * scale2, dcap = 1.0f;
            if (CAP) {
                const float th = tanh_of(v);
                v = cap2 * th;
                dcap = 1.0f - th * th;
            }
            if (a.slopes) v -= slopes2[r] * fabsf(posf[r] - keyf);
            p[i] = exp2_(v - lse2[r]) * T::p_gain;
            ds[i] = p[i] * (dp[i] * (1.0f / T::p_gain) - delta[r]) * dcap;
        }
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int r = 8 * (i / 4) + 4 * hi + i % 4;
                bool seen = key < end[r];
                if (u.docs) seen = seen && rdoc[r] == kdoc;
                p[i] = seen ? p[i] : 0.0f;
                ds[i] = seen ? ds[i] : 0.0f;
            }
        }
#pragma unroll
        for (int kc = 0; kc < 2; kc++) {
            const s16x8 pr = rounded<T>(p + 8 * kc), dr = rounded<T>(ds + 8 * kc);
#pragma unroll
            for (int d = 0; d < NB; d++) {
                dv[d] = T::mfma(L::column_operand(gs, 16 * kc, d), pr, dv[d]);
                dk[d] = T::mfma(L::column_operand(qs, 16 * kc, d), dr, dk[d]);
            }
        }
    }
    if (key >= a.k_len) return;
    char *kp = a.dk.data + (u.b * a.dk.batch + u.g * a.dk.head + key * a.dk.position) * 2;
    char *vp = a.dv.data + (u.b * a.dv.batch + u.g * a.dv.head + key * a.dv.position) * 2;
#pragma unroll
    for (int d = 0; d < NB; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int col = 32 * d + 8 * e + 4 * hi;
            typedef R r4 __attribute__((ext_vector_type(4)));
            r4 x, y;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[i] = (R)(dk[d][4 * e + i] * a.scale);
                y[i] = (R)(dv[d][4 * e + i] * (1.0f / T::p_gain));
            }
            if (col < a.head_dim) {
                *(r4 *)(kp + col * 2) = x;
                *(r4 *)(vp + col * 2) = y;
            }
        }
}

hipError_t doc_tiles(const AttnArgs &a, hipStream_t st)
{
    if (!a.docs || !a.key_tiles) return hipSuccess;
    doc_tiles_kernel<<<dim3(a.key_tiles, a.batch < 32768 ? a.batch : 32768), 64, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T, int NB, bool CAP> hipError_t forward_sized(const AttnArgs &a, hipStream_t st)
{
    const int64_t units = (int64_t)a.batch * a.k_heads;
    const unsigned n = (unsigned)(units * ((a.rows + ROW_TILE - 1) / ROW_TILE) * a.splits);
    forward_kernel<T, NB, CAP><<<n, 256, 0, st>>>(a);
    if (a.splits > 1) {
        if (hipError_t e = hipGetLastError()) return e;
        join_kernel<T><<<(unsigned)((units * a.rows + 7) / 8), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

template <typename T, int NB, bool CAP> hipError_t backward_sized(const AttnArgs &a, hipStream_t st)
{
    const int64_t units = (int64_t)a.batch * a.k_heads;
    if (a.rows) {
        row_stat_kernel<T><<<(unsigned)((units * a.rows + 15) / 16), 256, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        dq_kernel<T, NB, CAP><<<(unsigned)(units * ((a.rows + ROW_TILE - 1) / ROW_TILE)), 256, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (a.k_len) dkv_kernel<T, NB, CAP><<<(unsigned)(units * ((a.k_len + GRAD_KEYS - 1) / GRAD_KEYS)), 256, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t forward_typed(const AttnArgs &a, hipStream_t st)
{
    if (a.head_dim <= 64) return a.cap > 0 ? forward_sized<T, 2, true>(a, st) : forward_sized<T, 2, false>(a, st);
    return a.cap > 0 ? forward_sized<T, 4, true>(a, st) : forward_sized<T, 4, false>(a, st);
}

template <typename T> hipError_t backward_typed(const AttnArgs &a, hipStream_t st)
{
    if (a.head_dim <= 64) return a.cap > 0 ? backward_sized<T, 2, true>(a, st) : backward_sized<T, 2, false>(a, st);
    return a.cap > 0 ? backward_sized<T, 4, true>(a, st) : backward_sized<T, 4, false>(a, st);
}

}  // namespace

hipError_t launch_attn_forward(const AttnArgs &a, int type, hipStream_t st)
{
    if (hipError_t e = doc_tiles(a, st)) return e;
    return type == 0 ? forward_typed<Bf16>(a, st) : forward_typed<Fp16>(a, st);
}

hipError_t launch_attn_backward(const AttnArgs &a, int type, hipStream_t st)
{
    if (hipError_t e = doc_tiles(a, st)) return e;
    return type == 0 ? backward_typed<Bf16>(a, st) : backward_typed<Fp16>(a, st);
}

}  // namespace dtrops
