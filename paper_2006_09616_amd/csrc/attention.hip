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
#include <type_traits>

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
    static constexpr bool narrow = false;
    static constexpr float p_gain = 1.0f, p_shift = 0.0f, lift = 0.0f, slack = 8.0f;
    static constexpr uint32_t exponent = 0x7F807F80u, least = 0x00800080u;     // of two numbers, and its lowest bits
};
// Probabilities of long rows, or beside a score far above theirs, are below
// the smallest normal number of fp16, 2^-14.  Backwards they are at most 1 and
// taken times 2^15; forwards they are at most 2^slack, for a running maximum
// that is taken `lift` below the largest score.  Score gradients have a range
// of their own (value_magnitude_kernel).
struct Fp16 {
    using raw = _Float16;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static __device__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static constexpr bool narrow = true;
    static constexpr float p_gain = 32768.0f, p_shift = 15.0f, lift = 11.0f, slack = 4.0f;
    static constexpr uint32_t exponent = 0x7C007C00u, least = 0x04000400u;
};

// eight numbers rounded to the inputs' type: an operand of the next product
template <typename T> __device__ __forceinline__ s16x8 rounded(const float *p)
{
    typename T::v8 v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (typename T::raw)p[i];
    return __builtin_bit_cast(s16x8, v);
}

// f of the numbers I .. N - 1, each a constant of its own type
template <int I, int N, typename F> __device__ __forceinline__ void static_for(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// Order for the scheduler: READS reads of LDS first, then TIMES times one
// matrix instruction, EACH reads and VALUS vector instructions.
template <int READS, int TIMES, int EACH, int VALUS> __device__ __forceinline__ void interleave()
{
    if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
    for (int i = 0; i < TIMES; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (EACH > 0) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
        if constexpr (VALUS > 0) __builtin_amdgcn_sched_group_barrier(0x002, VALUS, 0);
    }
}

template <typename T> __device__ __forceinline__ float value_of(short bits) { return (float)__builtin_bit_cast(typename T::raw, bits); }

// Infinities and NaN.  A matrix instruction multiplies them by the zero
// probability of a masked pair, which gives NaN where the definition has
// nothing.  So tiles that a mask cuts through (and only they) are searched for
// them; they are replaced by zeros, and what visible values give is added to
// the finished sums (add_nonfinite).
template <typename T> __device__ __forceinline__ uint32_t nonfinite(uint32_t two)      // top bits of those of two
{
    return ((two & T::exponent) + T::least) & 0x80008000u;
}
template <typename T> __device__ __forceinline__ bool nonfinite(const uint4 &v)
{
    return nonfinite<T>(v.x) | nonfinite<T>(v.y) | nonfinite<T>(v.z) | nonfinite<T>(v.w);
}
template <typename T> __device__ __forceinline__ uint4 cleaned(uint4 v)
{
    v.x &= ~((nonfinite<T>(v.x) >> 15) * 0xFFFFu);
    v.y &= ~((nonfinite<T>(v.y) >> 15) * 0xFFFFu);
    v.z &= ~((nonfinite<T>(v.z) >> 15) * 0xFFFFu);
    v.w &= ~((nonfinite<T>(v.w) >> 15) * 0xFFFFu);
    return v;
}
// Tiles of SIZE elements, by all 256 threads (one tile: a and b the same).
// Returns whether a and whether b had any.
struct Odd { bool a, b; };
template <typename T, int SIZE> __device__ Odd clean(short *a, short *b)
{
    constexpr int N = SIZE / 8 / 256;
    uint4 *const p = (uint4 *)a + threadIdx.x, *const q = (uint4 *)b + threadIdx.x;
    bool any_a = false, any_b = false;
#pragma unroll 2
    for (int n = 0; n < N; n++) {
        any_a |= nonfinite<T>(p[n * 256]);
        if (a != b) any_b |= nonfinite<T>(q[n * 256]);
    }
    if (!__syncthreads_or(any_a | any_b)) return {false, false};
    if (any_a)
#pragma unroll 1
        for (int n = 0; n < N; n++) p[n * 256] = cleaned<T>(p[n * 256]);
    if (any_b)
#pragma unroll 1
        for (int n = 0; n < N; n++) q[n * 256] = cleaned<T>(q[n * 256]);
    return {(bool)__syncthreads_or(any_a), (bool)__syncthreads_or(any_b)};
}

// two numbers rounded into an operand's elements i and i + 1
template <typename T> __device__ __forceinline__ void put_two(s16x8 &v, int i, const float (&x)[2])
{
    typedef typename T::raw r2 __attribute__((ext_vector_type(2)));
    typedef short s2 __attribute__((ext_vector_type(2)));
    const s2 b = __builtin_bit_cast(s2, r2{(typename T::raw)x[0], (typename T::raw)x[1]});
    v[i] = b[0];
    v[i + 1] = b[1];
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// the other half's value: lane ^ 32
__device__ __forceinline__ float other_half(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// (tanh(x) - 1) / 2 = -1 / (1 + exp(2 x)), with x2 = 2 log2(e) x: of this h
// tanh is 1 + 2 h and its derivative 1 - tanh^2 is -4 (h + h^2)
__device__ __forceinline__ float minus_half(float x2) { return __builtin_amdgcn_rcpf(-1.0f - exp2_(x2)); }

// What a cap does with the scores: none, a cap up to LARGE_CAP, a larger one.
// cap (1 + 2 h) subtracts numbers of the cap's size, so that its error is
// 1.3e-7 cap whatever the score.  Up to 128 that is below a tenth of fp16's
// unit (2^-12, as the probabilities are rounded); larger caps take the series
// of tanh where scores are below a quarter of the cap, and keep the digits of
// the score (8192 tokens in three documents, a whole pass: 1.62 ms, at a cap of
// 50 1.29).
enum { PLAIN = 0, SMALL = 1, LARGE = 2 };
constexpr float LARGE_CAP = 128.0f;

// 1 / cap that leaves a score of zero at zero however small the cap is
__device__ __forceinline__ float per_cap(float scale, float cap) { return fminf(scale / cap, -LOWEST); }

struct Capped { float score, t; };       // cap tanh(x) in units of log 2, and tanh(x)
// x tanh's series / x to x^8: 2^-26 at x = 1/4
__device__ __forceinline__ Capped large_capped(float s, float per_cap, float scale2, float cap2)
{
    const float x = s * per_cap, z = x * x;
    const float f = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 62.0f / 2835, -17.0f / 315), 2.0f / 15), -1.0f / 3), 1.0f);
    const float h = minus_half(x * (2.0f * LOG2E));
    const bool near = fabsf(x) < 0.25f;
    return {near ? s * scale2 * f : fmaf(h, 2.0f * cap2, cap2), near ? x * f : fmaf(h, 2.0f, 1.0f)};
}

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

// Moves 64 rows of a tensor (consecutive positions of a head) from memory into
// a tile in LDS without passing through registers, 256 threads.  Each
// instruction of a wavefront fills 1024 bytes of the tile in order, lane by
// lane; the swizzle is in the addresses that the lanes read.  Reads go through
// a buffer descriptor of the rows up to `end`: beyond them, and for columns
// from head_dim on, it delivers zeros.  The compiler does not see these loads:
// moved() waits for them, before the barrier that hands the tile over.  Nor
// does it know that what it places before is read by a memory instruction at
// once: one needs a wait state after a write of m0, and five after a vector
// instruction has written its scalar operands.
constexpr int STAGE_ROWS = 64;
static_assert(STAGE_ROWS == KEY_TILE, "a tile of keys is moved at once");

__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p);
}

__device__ __forceinline__ void moved() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// For the compiler: nothing that was loaded before the loop is pending within.
__device__ __forceinline__ void ready() { __builtin_amdgcn_s_waitcnt(0); }

template <int NB> struct Mover {
    using L = Tile<NB>;
    static constexpr int PER = 64 / L::CHUNKS, N = STAGE_ROWS / PER / 4;      // rows an instruction, instructions a wavefront
    uint32_t offset, bytes, step;
    __device__ Mover(int64_t stride, int head_dim)
    {
        const int lane = threadIdx.x % WAVE, row = threadIdx.x / WAVE * PER + lane / L::CHUNKS;
        const int chunk = lane % L::CHUNKS ^ L::swizzle(row);                   // the same 4 PER rows further on
        bytes = (uint32_t)stride * 2u;
        step = 4 * PER * bytes;
        offset = chunk * 8 < head_dim ? row * bytes + chunk * 16 : 0x80000000u;
    }
    __device__ void load(short *tile, const char *base, int row0, int end, int head_dim) const
    {
        const uint64_t p = (uint64_t)(base + (int64_t)row0 * bytes);
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        const u32x4 rsrc = {(uint32_t)p, (uint32_t)(p >> 32), (uint32_t)(min(end - row0, STAGE_ROWS) - 1) * bytes + head_dim * 2,
                            0x00027000u};
        const uint32_t at = lds_address(tile) + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE) * 1024;
#pragma unroll
        for (int n = 0; n < N; n++)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                         :: "s"(at + n * 4096), "v"(offset + n * step), "s"(rsrc) : "memory", "m0");
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

// The work of workgroup `id` of units x tiles: tiles of rank 0 (the longest
// under a causal mask) first, so that the short ones fill the end.  Workgroups
// go round the 8 dies; where the units divide among them, a die has units of
// its own, whose keys its cache then holds.
struct Work {
    int unit, rank;
    __device__ Work(int id, int units)
    {
        if (units % 8 == 0) {
            const int each = units / 8, i = id / 8;
            unit = id % 8 * each + i % each;
            rank = i / each;
        } else {
            unit = id % units;
            rank = id / units;
        }
    }
};

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

template <typename R> struct Four { typedef R v __attribute__((ext_vector_type(4))); };

template <typename T>
__device__ __forceinline__ void write_four(const Heads &t, int b, int head, int64_t position, int col, f32x4 v)
{
    using R = typename T::raw;
    typename Four<R>::v r;
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = (R)v[i];
    *(typename Four<R>::v *)(t.data + (b * t.batch + head * t.head + position * t.position + col) * 2) = r;
}

// adds to four columns of the output that the same lane has written
template <typename T>
__device__ __forceinline__ void add_out(const AttnArgs &a, int b, int head, int64_t query, int col, f32x4 v)
{
    using R = typename T::raw;
    auto *p = (typename Four<R>::v *)(a.out.data + (b * a.out.batch + head * a.out.head + query * a.out.position + col) * 2);
    typename Four<R>::v r = *p;
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = (R)((float)r[i] + v[i]);
    *p = r;
}

// Four columns of the output and, for the backward pass, what the rounding
// took from them: out . dout is subtracted from every score gradient of its
// row, so that its error does not average out over the keys.
template <typename T>
__device__ __forceinline__ void write_out(const AttnArgs &a, int b, int head, int query, int col, f32x4 v)
{
    using R = typename T::raw;
    write_four<T>(a.out, b, head, query, col, v);
    if (a.rest) {
        typename Four<R>::v r;
#pragma unroll
        for (int i = 0; i < 4; i++) r[i] = (R)(v[i] - (float)(R)v[i]);
        *(typename Four<R>::v *)(a.rest + (((int64_t)b * a.q_len + query) * a.k_heads * a.group + head) * a.head_dim * 2 + col * 2) = r;
    }
}

// The rows of a workgroup (ROWS from tile_row on; `mine` is the lane's, with
// 31 others in its wavefront) and the tiles of keys that any of them may see.
template <int ROWS, int THREADS> struct RowBlock {
    Unit u;
    int row, query, head, pos, doc, end;     // of the lane's row; keys from `end` on are masked for it
    int sure;                                // keys before `sure` are seen by all rows, but for documents
    int wave_end;                            // keys from here on are masked for all rows of the wavefront
    int t0, t1;                              // tiles
    int doc_lo, doc_hi;
    bool one_doc;

    __device__ RowBlock(const AttnArgs &a, int unit, int tile_row, int mine, int (&range)[4]) : u(a, unit)
    {
        const int last = a.rows - 1;
        row = mine;
        const int r = min(row, last);
        query = r / a.group;
        head = u.g * a.group + r % a.group;
        pos = u.start + query;
        const bool has_doc = !u.docs || (pos >= 0 && pos < a.k_len);
        doc = u.docs && has_doc ? u.docs[pos] : 0;
        end = has_doc ? u.end(a, pos) : 0;
        sure = u.end(a, u.start + tile_row / a.group);
        wave_end = u.end(a, u.start + min(__builtin_amdgcn_readfirstlane(mine) + 31, last) / a.group);
        t0 = 0;
        t1 = (u.end(a, u.start + min(tile_row + ROWS - 1, last) / a.group) + KEY_TILE - 1) / KEY_TILE;
        doc_lo = doc_hi = 0;
        one_doc = true;
        if (!u.docs) return;
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
        doc_lo = __builtin_amdgcn_readfirstlane(range[2]);
        doc_hi = __builtin_amdgcn_readfirstlane(range[3]);
        for (int t = threadIdx.x; t < t1; t += THREADS)
            if (near(t)) {
                atomicMin(&range[0], t);
                atomicMax(&range[1], t);
            }
        __syncthreads();
        t1 = __builtin_amdgcn_readfirstlane(range[1]) + 1;
        t0 = min(__builtin_amdgcn_readfirstlane(range[0]), t1);      // nothing near: 0, 0
        one_doc = one_doc && doc_lo == doc_hi;
    }
    // whether a tile's documents and the rows' overlap
    __device__ bool near(int t) const
    {
        const int2 d = u.doc_tiles[t];
        return d.x <= doc_hi && d.y >= doc_lo;
    }
    __device__ int next(int t) const
    {
        if (u.docs)
            while (t < t1 && !near(t)) t++;
        return t;
    }
    __device__ bool same_doc(int t) const
    {
        if (!u.docs) return true;
        const int2 d = u.doc_tiles[t];
        return one_doc && d.x == d.y;
    }
    // whether every row sees every key of the tile
    __device__ bool whole(int t) const { return (t + 1) * KEY_TILE <= sure && same_doc(t); }
    // whether some row does not see a key that is there (from u.len on there are zeros)
    __device__ bool cut(int t) const { return min((t + 1) * KEY_TILE, u.len) > sure || !same_doc(t); }
    __device__ bool sees(const AttnArgs &a, int key) const
    {
        return key < end && (!u.docs || u.docs[min(key, a.k_len - 1)] == doc);
    }
    // x = other for the lane's keys (key0 + 32 (i / 16) + 8 (i % 16 / 4) + i % 4) that its row does not see
    template <int N> __device__ void mask(const AttnArgs &a, float (&x)[N], int key0, float other) const
    {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = key0 + 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4 < end ? x[i] : other;
        if (!u.docs) return;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
#pragma unroll
            for (int n = 0; n < 4; n++)
                x[i + n] = u.docs[min(key0 + 32 * (i / 16) + 8 * (i % 16 / 4) + n, a.k_len - 1)] == doc ? x[i + n] : other;
            __builtin_amdgcn_sched_barrier(0);            // registers for four loads, not for all
        }
    }
};

// What the infinities and NaN of the values of keys j0 .. j1 - 1 add to four
// columns of a row that sees those keys: a positive probability of them is
// them.  Rarely called: for tiles that had any.
template <typename T, typename Sees>
__device__ __forceinline__ void add_nonfinite(const AttnArgs &a, const char *vb, int j0, int j1, int col, Sees sees, f32x4 &sum)
{
#pragma unroll 1
    for (int j = j0; j < j1; j++) {
        const s16x4 v = *(const s16x4 *)(vb + j * a.v.position * 2 + col * 2);
        bool any = false;
        f32x4 f;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            f[i] = value_of<T>(v[i]);
            if (fabsf(f[i]) < INFINITY) f[i] = 0.0f;
            else any = true;
        }
        if (any && sees(j)) sum += f;
    }
}

// The scores of a lane's keys (key0 + 4 (lane / 32) + 32 (i / 16) + 8 (i % 16 / 4)
// + i % 4), shaped in place: times log2(e), capped, biased.  apply_but leaves
// a gain and an offset to the exponent's fma: with a cap alone the scores are
// then minus_half (8192 tokens in three documents: 303 us, by apply 318; where
// reading the keys is the bound it only costs registers).  CAP SMALL stands for
// a cap, a bias or both.
template <int CAP> struct Shape {
    bool capped, bias;
    float scale2, per, cap2, slope2, gain, offset;
    __device__ Shape(const AttnArgs &a, int head)
    {
        capped = CAP == SMALL && a.cap > 0;
        bias = a.slopes != nullptr;
        slope2 = bias ? a.slopes[head] * LOG2E : 0.0f;
        per = CAP == PLAIN ? 0.0f : per_cap((capped ? 2.0f * LOG2E : 1.0f) * a.scale, a.cap);
        scale2 = capped ? per : a.scale * LOG2E;
        cap2 = a.cap * LOG2E;
        gain = capped && !bias ? 2.0f * cap2 : 1.0f;
        offset = capped && !bias ? cap2 : 0.0f;
    }
    template <int N> __device__ void apply(float (&x)[N], int distance0) const
    {
        if (CAP == LARGE) {
#pragma unroll
            for (int i = 0; i < N; i++) x[i] = large_capped(x[i], per, scale2, cap2).score;
        } else if (capped) {
#pragma unroll
            for (int i = 0; i < N; i++) x[i] = fmaf(minus_half(x[i] * scale2), 2.0f * cap2, cap2);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) x[i] *= scale2;
        }
        if (bias) {
            const float pf = (float)distance0;
#pragma unroll
            for (int i = 0; i < N; i++) x[i] -= slope2 * fabsf(pf - (float)(32 * (i / 16) + 8 * (i % 16 / 4) + i % 4));
        }
    }
    template <int N> __device__ void apply_but(float (&x)[N], int distance0) const
    {
        if (capped && !bias) {
#pragma unroll
            for (int i = 0; i < N; i++) x[i] = minus_half(x[i] * scale2);
        } else {
            apply(x, distance0);
        }
    }
};

// ---- forward -----------------------------------------------------------------
// One pass with a running maximum and sum a row (32 bits):
//   o = sum_j exp(s_j - m) v_j,  l = sum_j exp(s_j - m),  out = o / l,
//   log-sum-exp = m + log l.
// The probabilities are rounded to the inputs' type for the second product, as
// the matrix instruction takes them; sums are 32-bit.  A workgroup has 128
// rows, a wavefront 32, and walks over tiles of 64 keys.  The next tile is on
// its way from memory while one is worked on (two buffers, one barrier a
// tile).  Rows are packed over the heads of a group, so that shared keys are
// read once for all of them.
//   4 x 4096 tokens, 16 heads of 128, causal, bf16: 306 to 322 us, 0.87 PFLOP/s
// of the visible half; a large product reaches 1.19 to 1.35 on this card.  No
// unit is full: the matrix unit works in 42 % of the cycles, the vector unit
// issues in 47 %.  A wavefront's products and its softmax take turns, and two
// wavefronts a SIMD overlap in part.  With a cap, three transcendental
// instructions a score instead of one (8192 tokens in three documents, 16 heads
// over 4: 303 us, 0.45 PFLOP/s; 20 and 40 %, and a quarter of the card idle at
// the end).

template <typename T, int NB, bool SHAPED, int CAP>
__global__ void __launch_bounds__(256, 2) forward_kernel(AttnArgs a)
{
    using L = Tile<NB>;
    using R = typename T::raw;
    constexpr int SIZE = KEY_TILE * L::PITCH;
    __shared__ __align__(16) short tiles[4 * SIZE];     // two of keys, two of values
    __shared__ int range[4];

    const int row_tiles = (a.rows + ROW_TILE - 1) / ROW_TILE;
    const int units = a.batch * a.k_heads;
    const int split = blockIdx.x / (units * row_tiles);
    const Work work(blockIdx.x % (units * row_tiles), units);
    const int tile_row = (row_tiles - 1 - work.rank) * ROW_TILE;
    RowBlock<ROW_TILE, 256> w(a, work.unit, tile_row, tile_row + threadIdx.x / WAVE * 32 + threadIdx.x % 32, range);
    if (a.splits > 1) {                                  // this part's tiles
        const int n = max(w.t1 - w.t0, 0), per = (n + a.splits - 1) / a.splits;
        w.t0 = min(w.t0, w.t1) + per * split;
        w.t1 = min(w.t0 + per, w.t1);
    }
    const Unit &u = w.u;
    const int lane = threadIdx.x % WAVE, hi = lane / 32;

    s16x8 q[2 * NB];
    {
        const char *qp = head_base(a.q, u.b, w.head) + w.query * a.q.position * 2;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++) {
            const int d = 16 * s + 8 * hi;
            q[s] = d < a.head_dim ? *(const s16x8 *)(qp + d * 2) : s16x8{};
        }
    }
    const Shape<CAP> shape(a, w.head);

    f32x16 o[NB] = {};
    float m = LOWEST, l = 0;
    bool odd = false;                                    // whether cleaned values are to be added
    const char *kb = head_base(a.k, u.b, u.g), *vb = head_base(a.v, u.b, u.g);

    int t = w.next(w.t0);
    const Mover<NB> mk(a.k.position, a.head_dim), mv(a.v.position, a.head_dim);
    if (t < w.t1) {
        mk.load(tiles, kb, t * KEY_TILE, u.len, a.head_dim);
        mv.load(tiles + 2 * SIZE, vb, t * KEY_TILE, u.len, a.head_dim);
    }
    moved();
    ready();
    __syncthreads();
    for (int buf = 0; t < w.t1; buf ^= 1) {
        const int j0 = t * KEY_TILE, t2 = w.next(t + 1);
        if (t2 < w.t1) {
            mk.load(tiles + (buf ^ 1) * SIZE, kb, t2 * KEY_TILE, u.len, a.head_dim);
            mv.load(tiles + (2 + (buf ^ 1)) * SIZE, vb, t2 * KEY_TILE, u.len, a.head_dim);
        }
        const bool whole = w.whole(t);
        short *const vs = tiles + (2 + buf) * SIZE;
        if (w.cut(t)) odd |= clean<T, SIZE>(vs, vs).a;
        if (j0 < w.wave_end) {
            const short *ks = tiles + buf * SIZE;
            // operands are read from LDS a group of products ahead
            f32x16 s[2] = {};
            s16x8 f[2][4];
            auto keys = [&](int g) {
#pragma unroll
                for (int n = 0; n < 4; n++) f[g & 1][n] = L::row_operand(ks, 32 * (n & 1) + lane % 32, 2 * g + n / 2);
            };
            auto values = [&](int kc) {
#pragma unroll
                for (int d = 0; d < NB; d++) f[kc & 1][d] = L::column_operand(vs, 16 * kc, d);
            };
            keys(0);
#pragma unroll
            for (int g = 0; g < NB; g++) {
                if (g + 1 < NB) keys(g + 1);
#pragma unroll
                for (int n = 0; n < 4; n++) s[n & 1] = T::mfma(f[g & 1][n], q[2 * g + n / 2], s[n & 1]);
            }
            values(0);
            interleave<8, 2 * NB * 2 - 8, 1, 0>();
            interleave<0, 8, 1, 0>();
            // x: the scores times log2(e); plain ones but for a factor left to the exponent's fma
            float x[32];
            const float gain = SHAPED ? shape.gain : shape.scale2, offset = SHAPED ? shape.offset : 0.0f;
#pragma unroll
            for (int i = 0; i < 32; i++) x[i] = s[i / 16][i % 16];
            if (SHAPED) shape.apply_but(x, w.pos - j0 - 4 * hi);
            if (!whole) w.mask(a, x, j0 + 4 * hi, -INFINITY);
            float most = x[0];
#pragma unroll
            for (int i = 1; i < 32; i++) most = fmaxf(most, x[i]);
            most = fmaf(fmaxf(most, other_half(most)), gain, offset);
            // The sums are moved to a new maximum only where the old one would let
            // them grow by more than 2^slack: 32-bit sums have room, and a probability
            // is rounded relative to itself.
            if (__any(most > m + (T::lift + T::slack))) {
                const float m_new = fmaxf(m, most - T::lift), f = exp2_(m - m_new);
                m = m_new;
                l *= f;
#pragma unroll
                for (int d = 0; d < NB; d++) o[d] *= f;
            }
#pragma unroll
            for (int i = 0; i < 32; i++) {
                x[i] = exp2_(fmaf(x[i], gain, offset - m));
                l += x[i];
            }
#pragma unroll
            for (int kc = 0; kc < 4; kc++) {
                const s16x8 p = rounded<T>(x + 8 * kc);
                if (kc < 3) values(kc + 1);
#pragma unroll
                for (int d = 0; d < NB; d++) o[d] = T::mfma(f[kc & 1][d], p, o[d]);
            }
        }
        moved();
        __syncthreads();
        t = t2;
    }
    l += other_half(l);
    if (w.row >= a.rows) return;
    const bool nothing = l == 0;
    const float inv = nothing ? 0.0f : 1.0f / l;
    const int64_t part_at = ((int64_t)split * units + u.b * a.k_heads + u.g) * a.rows + w.row;
    auto write = [&](int col, f32x4 v) {
        if (a.splits > 1) *(f32x4 *)(a.part_out + part_at * a.head_dim + col) = v;
        else write_out<T>(a, u.b, w.head, w.query, col, nothing ? f32x4{} : v * inv);
    };
#pragma unroll
    for (int d = 0; d < NB; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int col = 32 * d + 8 * e + 4 * hi;
            if (col < a.head_dim) write(col, f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]});
        }
    if (hi == 0) {
        if (a.splits > 1) a.part_stat[part_at] = make_float2(m, l);
        else if (a.lse)
            a.lse[((int64_t)u.b * a.k_heads * a.group + w.head) * a.q_len + w.query] =
                nothing ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
    }
    if (!odd) return;
    for (int col = 4 * hi; col < a.head_dim; col += 8) {
        f32x4 sum = {};
        for (int t = w.next(w.t0); t < w.t1; t = w.next(t + 1))
            if (w.cut(t))
                add_nonfinite<T>(a, vb, t * KEY_TILE, min((t + 1) * KEY_TILE, u.len), col, [&](int j) { return w.sees(a, j); }, sum);
        // finite columns have been written; an infinity or NaN takes its column whole
        const bool any = !(fabsf(sum[0]) + fabsf(sum[1]) + fabsf(sum[2]) + fabsf(sum[3]) < INFINITY);
        if (!any) continue;
        if (a.splits > 1) *(f32x4 *)(a.part_out + part_at * a.head_dim + col) += sum;
        else add_out<T>(a, u.b, w.head, w.query, col, sum);
    }
}

// Few rows (at most 32 of a key head: new tokens over a cache): what bounds it
// is reading the keys and values once.  Four wavefronts have the same rows
// and take tiles of 32 keys in turn, each at its own pace: keys go from memory
// straight into the matrix operand, values through a piece of LDS that is the
// wavefront's own (no barrier), and the next tile's loads are under way before
// the softmax of this one.  At the end the four sums are joined in LDS.  Two
// workgroups of four share a compute unit (one of eight measured 47 against 39
// us on 12 units of 30011 keys: nothing runs beside its start and end).
//   One token for 32 requests of 8192 to 16384 keys, 8 key heads of 128: 289 us,
// 5.5 TB/s of keys and values (a large copy: 4.8).
constexpr int FEW_WAVES = 4, FEW_KEYS = 32;

template <typename T, int NB, bool SHAPED, int CAP>
__global__ void __launch_bounds__(256, 2) few_rows_kernel(AttnArgs a)
{
    using L = Tile<NB>;
    constexpr int SIZE = FEW_KEYS * L::PITCH, N = FEW_KEYS * L::CHUNKS / WAVE, STEP = WAVE / L::CHUNKS;
    constexpr int SUMS = FEW_WAVES * FEW_ROWS * 32 * NB;
    // values' tiles (16-bit) during the walk, sums (32-bit) afterwards
    __shared__ __align__(16) char lds[SUMS * 4 > FEW_WAVES * SIZE * 2 ? SUMS * 4 : FEW_WAVES * SIZE * 2];
    __shared__ float2 stats[FEW_WAVES][FEW_ROWS];
    __shared__ int range[4];

    const int units = a.batch * a.k_heads;
    const int id = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
    const int lane = threadIdx.x % WAVE, hi = lane / 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const RowBlock<FEW_ROWS, FEW_WAVES * WAVE> w(a, id, 0, lane % 32, range);
    const Unit &u = w.u;

    // tiles of 32 keys, a multiple of FEW_WAVES for each part
    int t0 = 2 * w.t0, t1 = min(2 * w.t1, (w.wave_end + FEW_KEYS - 1) / FEW_KEYS);
    if (a.splits > 1) {
        const int n = max(t1 - t0, 0), per = ((n + a.splits - 1) / a.splits + FEW_WAVES - 1) / FEW_WAVES * FEW_WAVES;
        t0 = min(t0, max(t1, 0)) + per * split;
        t1 = min(t0 + per, t1);
    }

    s16x8 q[2 * NB];
    {
        const char *qp = head_base(a.q, u.b, w.head) + w.query * a.q.position * 2;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++) {
            const int d = 16 * s + 8 * hi;
            q[s] = d < a.head_dim ? *(const s16x8 *)(qp + d * 2) : s16x8{};
        }
    }
    const Shape<CAP> shape(a, w.head);
    f32x16 o[NB] = {};
    float m = LOWEST, l = 0;
    bool odd = false;                                    // whether cleaned values are to be added
    const char *kb = head_base(a.k, u.b, u.g), *vb = head_base(a.v, u.b, u.g);
    short *vt = (short *)lds + wave * SIZE;
    const uint32_t koff = (uint32_t)(lane % 32 * (uint32_t)a.k.position + 8 * hi) * 2u;
    const int vrow = lane / L::CHUNKS, vchunk = lane % L::CHUNKS;
    const uint32_t voff = (uint32_t)(vrow * (uint32_t)a.v.position + vchunk * 8) * 2u;

    s16x8 kf[2 * NB];
    uint4 vr[N];
    auto load = [&](int t) {
        const int j0 = t * FEW_KEYS;
        const char *kp = kb + j0 * a.k.position * 2, *vp = vb + j0 * a.v.position * 2;
        const bool inside = j0 + FEW_KEYS <= u.len;
        const bool in = inside || j0 + lane % 32 < u.len;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++) {
            if (s * 16 + 16 <= a.head_dim ? in : in && 16 * s + 8 * hi < a.head_dim) kf[s] = *(const s16x8 *)(kp + koff + s * 32);
            else kf[s] = s16x8{};
        }
#pragma unroll
        for (int n = 0; n < N; n++) {
            if (vchunk * 8 < a.head_dim && (inside || j0 + vrow + n * STEP < u.len))
                vr[n] = *(const uint4 *)(vp + n * STEP * a.v.position * 2 + voff);
            else vr[n] = make_uint4(0, 0, 0, 0);
        }
    };
    auto next = [&](int t) {
        if (u.docs)
            while (t < t1 && !w.near(t / 2)) t += FEW_WAVES;
        return t;
    };
    int t = next(t0 + wave);
    if (t < t1) load(t);
    while (t < t1) {
        const int j0 = t * FEW_KEYS, t2 = next(t + FEW_WAVES);
        const bool masked = j0 + FEW_KEYS > w.sure || u.docs;
        if (min(j0 + FEW_KEYS, u.len) > w.sure || u.docs) {
            bool any = false;
#pragma unroll
            for (int n = 0; n < N; n++) any |= nonfinite<T>(vr[n]);
            if (__any(any)) {
                odd = true;
#pragma unroll
                for (int n = 0; n < N; n++) vr[n] = cleaned<T>(vr[n]);
            }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int n = 0; n < N; n++) *(uint4 *)(vt + L::at(vrow + n * STEP, vchunk)) = vr[n];
        f32x16 s = {};
#pragma unroll
        for (int st = 0; st < 2 * NB; st++) s = T::mfma(kf[st], q[st], s);
        if (t2 < t1) load(t2);
        float x[16];
        const float gain = SHAPED ? 1.0f : shape.scale2;
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = s[i];
        if (SHAPED) shape.apply(x, w.pos - j0 - 4 * hi);
        if (masked) w.mask(a, x, j0 + 4 * hi, -INFINITY);
        float most = x[0];
#pragma unroll
        for (int i = 1; i < 16; i++) most = fmaxf(most, x[i]);
        most = fmaxf(most, other_half(most)) * gain;
        if (__any(most > m + (T::lift + T::slack))) {    // as in the forward kernel above
            const float m_new = fmaxf(m, most - T::lift), f = exp2_(m - m_new);
            m = m_new;
            l *= f;
#pragma unroll
            for (int d = 0; d < NB; d++) o[d] *= f;
        }
#pragma unroll
        for (int i = 0; i < 16; i++) {
            x[i] = exp2_(fmaf(x[i], gain, -m));
            l += x[i];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int kc = 0; kc < 2; kc++) {
            const s16x8 p = rounded<T>(x + 8 * kc);
#pragma unroll
            for (int d = 0; d < NB; d++) o[d] = T::mfma(L::column_operand(vt, 16 * kc, d), p, o[d]);
        }
        t = t2;
    }
    l += other_half(l);

    // the wavefronts' sums: row r, columns 4 c .. of wavefront v at ((v rows + r) COLS + c), four columns each
    constexpr int COLS = 8 * NB;
    const int rows = min(a.rows, FEW_ROWS);
    __syncthreads();
    f32x4 *sums = (f32x4 *)lds;
    if (lane % 32 < rows) {
#pragma unroll
        for (int d = 0; d < NB; d++)
#pragma unroll
            for (int e = 0; e < 4; e++)
                sums[(wave * rows + lane % 32) * COLS + 8 * d + 2 * e + hi] =
                    f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
        if (hi == 0) stats[wave][lane] = make_float2(m, l);
    }
    odd = __syncthreads_or(odd);
    for (int i = threadIdx.x; i < rows * COLS; i += FEW_WAVES * WAVE) {
        const int r = i / COLS, col = i % COLS * 4;
        float most = LOWEST, total = 0;
#pragma unroll
        for (int v = 0; v < FEW_WAVES; v++) most = fmaxf(most, stats[v][r].x);
        f32x4 sum = {};
#pragma unroll
        for (int v = 0; v < FEW_WAVES; v++) {
            const float f = exp2_(stats[v][r].x - most);
            total += stats[v][r].y * f;
            sum += sums[v * rows * COLS + i] * f;
        }
        if (odd && col < a.head_dim) {
            const int pos = u.start + r / a.group, end = u.end(a, pos);
            const bool has_doc = !u.docs || (pos >= 0 && pos < a.k_len);
            const int first = u.docs ? t0 : max(t0, w.sure / FEW_KEYS);           // the tiles that were cleaned
            if (has_doc)
                add_nonfinite<T>(a, vb, first * FEW_KEYS, min(t1 * FEW_KEYS, u.len), col,
                                 [&](int j) { return j < end && (!u.docs || u.docs[j] == u.docs[pos]); }, sum);
        }
        if (a.splits > 1) {
            const int64_t at = ((int64_t)split * units + id) * a.rows + r;
            if (col < a.head_dim) *(f32x4 *)(a.part_out + at * a.head_dim + col) = sum;
            if (col == 0) a.part_stat[at] = make_float2(most, total);
        } else {
            const int query = r / a.group, head = u.g * a.group + r % a.group;
            const bool nothing = total == 0;
            if (col < a.head_dim) write_out<T>(a, u.b, head, query, col, nothing ? f32x4{} : sum * (1.0f / total));
            if (a.lse && col == 0)
                a.lse[((int64_t)u.b * a.k_heads * a.group + head) * a.q_len + query] =
                    nothing ? -INFINITY : (most + __builtin_amdgcn_logf(total)) * LN2;
        }
    }
}

// Joins the parts (at most 256) of a row: a workgroup a row, eight groups of
// 32 lanes take parts in turn, four columns a lane.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(AttnArgs a)
{
    __shared__ float factor[256];
    __shared__ float2 waves[4];
    __shared__ f32x4 sums[8][32];
    const int64_t n = (int64_t)a.batch * a.k_heads * a.rows, r = blockIdx.x;
    const int tid = threadIdx.x, g = tid / 32, c = tid % 32 * 4;
    const float2 st = tid < a.splits ? a.part_stat[tid * n + r] : make_float2(LOWEST, 0.0f);
    float m = st.x;
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    if (tid % WAVE == 0) waves[tid / WAVE].x = m;
    __syncthreads();
    m = fmaxf(fmaxf(waves[0].x, waves[1].x), fmaxf(waves[2].x, waves[3].x));
    const float f = exp2_(st.x - m);
    factor[tid] = f;
    float l = st.y * f;
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) l += __shfl_xor(l, d);
    if (tid % WAVE == 0) waves[tid / WAVE].y = l;
    __syncthreads();
    l = (waves[0].y + waves[1].y) + (waves[2].y + waves[3].y);
    f32x4 o = {};
    if (c < a.head_dim)
        for (int s = g; s < a.splits; s += 8) o += *(const f32x4 *)(a.part_out + (s * n + r) * a.head_dim + c) * factor[s];
    sums[g][tid % 32] = o;
    __syncthreads();
    if (g) return;
#pragma unroll
    for (int i = 1; i < 8; i++) o += sums[i][tid];
    const bool nothing = l == 0;
    const int64_t unit = r / a.rows;
    const int row = (int)(r % a.rows), b = (int)(unit / a.k_heads), kg = (int)(unit % a.k_heads);
    const int query = row / a.group, head = kg * a.group + row % a.group;
    if (c < a.head_dim) write_out<T>(a, b, head, query, c, nothing ? f32x4{} : o * (1.0f / l));
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
//
// fp16 holds 2^-24 to 65504: a score gradient dS = P (dP - D) of a long row,
// or of a small loss, is below that, and one of a scaled loss may be above.
// |dP| and |D| are at most columns x max |dout| x max |V|, so that a power of
// two takes the largest possible dS to 2^15: it comes off the 32-bit sums at
// the end.  Without it dQ over 6000 keys, of a dout of 1e-3, was off by 11 times
// what its own rounding takes.  Here a workgroup finds the largest finite
// number of its chunk of a unit's values; the gradients of rows that see
// something are looked at by the kernel of dQ, for that of dK and dV too.
//   4 x 4096 tokens, 16 heads of 128: 13 us (5.2 TB/s) beside 1500; 8 x 512 tokens, 12
// heads of 64: 4.5 us beside 90.
template <typename T>
__global__ void __launch_bounds__(256) value_magnitude_kernel(AttnGradArgs a)
{
    __shared__ uint32_t waves[4];
    const int unit = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const Unit u(a, unit);
    const int per = (u.len + a.chunks - 1) / a.chunks, lo = min(per * chunk, u.len), end = min(lo + per, u.len);
    const int pieces = a.head_dim / 8, step = 256 / pieces, piece = threadIdx.x % pieces;
    const char *const vb = head_base(a.v, u.b, u.g) + piece * 16;
    uint32_t most = 0;
    if ((int)threadIdx.x < step * pieces)
#pragma unroll 4
        for (int j = lo + (int)threadIdx.x / pieces; j < end; j += step) {
            const s16x8 v = *(const s16x8 *)(vb + j * a.v.position * 2);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t bits = (uint16_t)v[i] & 0x7FFFu;             // in the order of the numbers
                most = bits < (T::exponent & 0xFFFFu) ? max(most, bits) : most;
            }
        }
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    if (threadIdx.x % WAVE == 0) waves[threadIdx.x / WAVE] = most;
    __syncthreads();
    if (threadIdx.x == 0)
        a.value_magnitude[blockIdx.x] = value_of<T>((short)max(max(waves[0], waves[1]), max(waves[2], waves[3])));
}

// the largest of n numbers of at least 0; a wavefront together
__device__ __forceinline__ float largest(const float *p, int n)
{
    float most = 0;
    for (int i = threadIdx.x % WAVE; i < n; i += WAVE) most = fmaxf(most, p[i]);
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    return most;
}
__device__ __forceinline__ float value_magnitude(const AttnGradArgs &a, int unit)
{
    return largest(a.value_magnitude + (int64_t)unit * a.chunks, a.chunks);
}
// of the gradients of a row tile, a number a wavefront
__device__ __forceinline__ float *row_magnitude(const AttnGradArgs &a, int unit, int tile)
{
    return a.row_magnitude + ((int64_t)unit * ((a.rows + ROW_TILE - 1) / ROW_TILE) + tile) * 4;
}
// the power of two for score gradients
__device__ __forceinline__ int gradient_shift(int head_dim, float v, float dout)
{
    const float bound = 2.0f * head_dim * v * dout;
    return bound > 0 && bound < INFINITY ? 15 - __builtin_amdgcn_frexp_expf(bound) : 0;
}

// Rows of dQ: 128 a workgroup, as the forward pass.  P and dS are 32-bit
// numbers that are rounded to the inputs' type once, as operands of the last
// product: dQ and dK are then up to 1.5 times as far from the exact gradient as
// their own rounding makes them (0.0025 against 0.0017 of its norm in bf16).
// The other way, dS in two parts, costs every such product twice.
//   4 x 4096 tokens, 16 heads of 128, causal, bf16: 421 to 437 us for three
// products (0.96 PFLOP/s; the matrix unit works in 48 % of the cycles, the
// vector unit issues in 40 %, at a clock of 1.9 GHz under this load); 8192
// tokens in three documents, capped: 380 to 395 us (25 and 39 %).
// Two workgroups a compute unit, but for fp16's large caps at 128 columns: they
// need 8 bytes a lane more than half of the registers.
template <typename T, int NB, int CAP, bool BIAS>
__global__ void __launch_bounds__(256, CAP == LARGE && NB == 4 && T::narrow ? 1 : 2) dq_kernel(AttnGradArgs a)
{
    using L = Tile<NB>;
    constexpr int SIZE = KEY_TILE * L::PITCH;
    __shared__ __align__(16) short tiles[4 * SIZE];
    __shared__ int range[4];

    const int row_tiles = (a.rows + ROW_TILE - 1) / ROW_TILE;
    const Work work(blockIdx.x, a.batch * a.k_heads);
    const int tile_row = (row_tiles - 1 - work.rank) * ROW_TILE;
    const RowBlock<ROW_TILE, 256> w(a, work.unit, tile_row, tile_row + threadIdx.x / WAVE * 32 + threadIdx.x % 32, range);
    const Unit &u = w.u;
    const int lane = threadIdx.x % WAVE, hi = lane / 32;

    s16x8 q[2 * NB], g[2 * NB];
    float delta = 0;
    {
        const char *qp = head_base(a.q, u.b, w.head) + w.query * a.q.position * 2;
        const char *gp = head_base(a.dout, u.b, w.head) + w.query * a.dout.position * 2;
        const char *op = head_base(a.out, u.b, w.head) + w.query * a.out.position * 2;
        const char *rp = a.rest + (((int64_t)u.b * a.q_len + w.query) * a.k_heads * a.group + w.head) * a.head_dim * 2;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++) {
            const int d = 16 * s + 8 * hi;
            const bool in = d < a.head_dim;
            q[s] = in ? *(const s16x8 *)(qp + d * 2) : s16x8{};
            g[s] = in ? *(const s16x8 *)(gp + d * 2) : s16x8{};
            const s16x8 o = in ? *(const s16x8 *)(op + d * 2) : s16x8{}, r = in && a.rest ? *(const s16x8 *)(rp + d * 2) : s16x8{};
#pragma unroll
            for (int i = 0; i < 8; i++)
                delta += (value_of<T>(o[i]) + value_of<T>(r[i])) * value_of<T>(g[s][i]);
            if (nonfinite<T>(__builtin_bit_cast(uint4, q[s]))) delta = NAN;
        }
        delta += other_half(delta);
    }
    // log2-sum-exp2 (plus infinity for a row that sees nothing, so that its P
    // is 0) and D, for the kernel of dK and dV too
    const int64_t stat_at = ((int64_t)u.b * a.k_heads * a.group + w.head) * a.q_len + w.query;
    const float lse = a.lse[stat_at], lse2 = lse == -INFINITY ? INFINITY : lse * LOG2E;
    if (hi == 0 && w.row < a.rows) a.row_stat[stat_at] = make_float2(lse2, delta);
    int shift = 0;                                       // of the row's score gradients
    if constexpr (T::narrow) {
        float most = 0;
#pragma unroll
        for (int s = 0; s < 2 * NB; s++)
#pragma unroll
            for (int i = 0; i < 8; i++) most = fmaxf(most, fabsf(value_of<T>(g[s][i])));
        most = fmaxf(most, other_half(most));
        shift = gradient_shift(a.head_dim, value_magnitude(a, work.unit), most);
        most = lse2 == INFINITY || most == INFINITY ? 0.0f : most;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        if (lane == 0) row_magnitude(a, work.unit, tile_row / ROW_TILE)[threadIdx.x / WAVE] = most;
    }
    const float shifted = lse2 - (float)shift;
    const float slope2 = BIAS && a.slopes ? a.slopes[w.head] * LOG2E : 0.0f;
    const float scale2 = CAP == SMALL ? per_cap(2.0f * LOG2E * a.scale, a.cap) : a.scale * LOG2E, cap2 = a.cap * LOG2E;
    const float per = per_cap(a.scale, a.cap);
    f32x16 dq[NB] = {};
    const char *kb = head_base(a.k, u.b, u.g), *vb = head_base(a.v, u.b, u.g);

    int t = w.next(w.t0);
    const Mover<NB> mk(a.k.position, a.head_dim), mv(a.v.position, a.head_dim);
    if (t < w.t1) {
        mk.load(tiles, kb, t * KEY_TILE, u.len, a.head_dim);
        mv.load(tiles + 2 * SIZE, vb, t * KEY_TILE, u.len, a.head_dim);
    }
    moved();
    ready();
    __syncthreads();
    for (int buf = 0; t < w.t1; buf ^= 1) {
        const int j0 = t * KEY_TILE, t2 = w.next(t + 1);
        if (t2 < w.t1) {
            mk.load(tiles + (buf ^ 1) * SIZE, kb, t2 * KEY_TILE, u.len, a.head_dim);
            mv.load(tiles + (2 + (buf ^ 1)) * SIZE, vb, t2 * KEY_TILE, u.len, a.head_dim);
        }
        short *const ks = tiles + buf * SIZE, *const vs = tiles + (2 + buf) * SIZE;
        const bool whole = w.whole(t);
        // a row that sees one of them has it in its log-sum-exp or in out . dout, but for
        // infinite keys whose scores a cap or a probability of zero made finite
        if (w.cut(t) && clean<T, SIZE>(ks, vs).a) {
#pragma unroll 1
            for (int j = j0; j < min(j0 + KEY_TILE, u.len); j++) {
                bool any = false;
#pragma unroll 1
                for (int d = 0; d < a.head_dim; d += 8) any |= nonfinite<T>(*(const uint4 *)(kb + (j * a.k.position + d) * 2));
                if (any && w.sees(a, j)) delta = NAN;
            }
        }
        if (j0 < w.wave_end) {
            // The matrix instructions of both halves of the tile in order: scores
            // and dP, then dQ; operands are read from LDS four ahead (two where
            // registers are short, which measured the same).
            constexpr int M1 = 4 * NB, M = M1 + 2 * NB, AHEAD = NB == 4 ? 2 : 4;
            s16x8 ring[AHEAD];
            auto operand = [&](auto at) __attribute__((always_inline)) {
                constexpr int i = at, half = i / M, j = i % M;
                if constexpr (j < M1) return L::row_operand(j & 1 ? vs : ks, 32 * half + lane % 32, j / 2);
                else return L::column_operand(ks, 32 * half + 16 * ((j - M1) / NB), (j - M1) % NB);
            };
            auto ahead = [&](auto at) __attribute__((always_inline)) {
                if constexpr (at + AHEAD < 2 * M) ring[at % AHEAD] = operand(std::integral_constant<int, at + AHEAD>{});
                __builtin_amdgcn_sched_barrier(0);
            };
            static_for<0, AHEAD>([&](auto at) __attribute__((always_inline)) { ring[at] = operand(at); });
            static_for<0, 2>([&](auto nth) __attribute__((always_inline)) {
                constexpr int half = nth;
                f32x16 s = {}, dp = {};
                static_for<half * M, half * M + M1>([&](auto at) __attribute__((always_inline)) {
                    constexpr int j = at % M;
                    if constexpr (j & 1) dp = T::mfma(ring[at % AHEAD], g[j / 2], dp);
                    else s = T::mfma(ring[at % AHEAD], q[j / 2], s);
                    ahead(at);
                });
                float x[16];
                const float pf = (float)(w.pos - j0 - 32 * half - 4 * hi);
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    float y;
                    if (CAP == SMALL) {
                        const float h = minus_half(s[i] * scale2);
                        y = fmaf(h, 2.0f * cap2, cap2 - shifted);
                        x[i] = fmaf(dp[i], -4.0f, 4.0f * delta) * fmaf(h, h, h);
                    } else if (CAP == LARGE) {
                        const Capped c = large_capped(s[i], per, scale2, cap2);
                        y = c.score - shifted;
                        x[i] = (dp[i] - delta) * fmaf(-c.t, c.t, 1.0f);
                    } else {
                        y = fmaf(s[i], scale2, -shifted);
                        x[i] = dp[i] - delta;
                    }
                    if (BIAS) y -= slope2 * fabsf(pf - (float)(8 * (i / 4) + i % 4));
                    x[i] *= exp2_(y);
                }
                if (!whole) w.mask(a, x, j0 + 32 * half + 4 * hi, 0.0f);
                const s16x8 p[2] = {rounded<T>(x), rounded<T>(x + 8)};
                static_for<half * M + M1, half * M + M>([&](auto at) __attribute__((always_inline)) {
                    constexpr int j = at % M - M1;
                    dq[j % NB] = T::mfma(ring[at % AHEAD], p[j / NB], dq[j % NB]);
                    ahead(at);
                });
            });
        }
        moved();
        __syncthreads();
        t = t2;
    }
    if (w.row >= a.rows) return;
    const float unscale = ldexpf(a.scale, -shift);
#pragma unroll
    for (int d = 0; d < NB; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int col = 32 * d + 8 * e + 4 * hi;
            const f32x4 v = {dq[d][4 * e], dq[d][4 * e + 1], dq[d][4 * e + 2], dq[d][4 * e + 3]};
            if (col < a.head_dim) write_four<T>(a.dq, u.b, w.head, w.query, col, v * unscale);
        }
}

// A workgroup has 128 keys, a wavefront 32, and walks over steps of 64 queries
// of one head after the other of the group (two buffers in LDS, one barrier a
// step).  Where key blocks are few, the steps are cut into parts whose sums
// are added up by grad_join_kernel.  Keys and values stay in registers as
// operands, dK and dV as accumulators: from 65 columns on one workgroup a
// compute unit.
//   4 x 4096 tokens, 16 heads of 128, causal, bf16: 720 to 760 us for four
// products (0.74 PFLOP/s; one wavefront a SIMD: the matrix unit works in 33 % of
// the cycles, the vector unit issues in 27 %); 8192 tokens in three documents, 16
// heads over 4, capped: 640 us (19 and 28 %) and 33 for the join.  A cap and a
// bias are template arguments: with both tested in the loop the accumulators
// moved between register files at every step.
template <typename T, int NB, int CAP, bool BIAS>
__global__ void __launch_bounds__(256, NB == 2 ? 2 : 1) dkv_kernel(AttnGradArgs a)
{
    using L = Tile<NB>;
    constexpr int ROWS = STAGE_ROWS, SIZE = ROWS * L::PITCH;
    __shared__ __align__(16) short tiles[4 * SIZE];     // two of Q, two of dout
    __shared__ __align__(16) float lse2s[2][ROWS], deltas[2][ROWS];
    __shared__ __align__(16) int docs[2][ROWS];

    const int part = blockIdx.x % a.parts;
    const Work work(blockIdx.x / a.parts, a.batch * a.k_heads);
    const Unit u(a, work.unit);
    const int j0 = work.rank * GRAD_KEYS;
    const int lane = threadIdx.x % WAVE, hi = lane / 32;
    const int jw = j0 + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE) * 32, key = jw + lane % 32;

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
    const float scale2 = CAP == SMALL ? per_cap(2.0f * LOG2E * a.scale, a.cap) : a.scale * LOG2E, cap2 = a.cap * LOG2E;
    const float per = per_cap(a.scale, a.cap);
    // of the unit's score gradients; their probability has p_shift already
    const int shift = T::narrow ? gradient_shift(a.head_dim, value_magnitude(a, work.unit),
                                                 largest(row_magnitude(a, work.unit, 0), (a.rows + ROW_TILE - 1) / ROW_TILE * 4)) : 0;
    const float dp_gain = T::narrow ? ldexpf(CAP == SMALL ? -4.0f : 1.0f, __builtin_amdgcn_readfirstlane(shift) - (int)T::p_shift)
                                    : CAP == SMALL ? -4.0f : 1.0f;
    const float unscale = T::narrow ? ldexpf(a.scale, -shift) : a.scale;
    f32x16 dk[NB] = {}, dv[NB] = {};

    // queries that may see any of the keys: from `first` on, `tiles_q` steps a head
    const int first = a.causal && j0 >= u.prefix ? min(max(j0 - u.start, 0), a.q_len) : 0;
    const int tiles_q = j0 < u.len ? (a.q_len - first + ROWS - 1) / ROWS : 0;
    int i0 = 0, i1 = tiles_q * a.group, doc_lo = 0, doc_hi = 0;
    if (u.docs) {
        const int2 d0 = u.doc_tiles[j0 / KEY_TILE], d1 = u.doc_tiles[min(j0 / KEY_TILE + 1, a.key_tiles - 1)];
        doc_lo = min(d0.x, d1.x);
        doc_hi = max(d0.y, d1.y);
    }
    if (a.parts > 1) {
        const int per = (i1 + a.parts - 1) / a.parts;
        i0 = min(per * part, i1);
        i1 = min(i0 + per, i1);
    }
    // a step: number i, 64 queries from q0 on of one head of the group
    struct Step { int i, head, q0; };
    auto step_at = [&](int i) { return Step{i, tiles_q ? i / tiles_q : 0, tiles_q ? first + i % tiles_q * ROWS : 0}; };
    auto after = [&](Step s) {
        s.i++;
        s.q0 += ROWS;
        if (s.q0 >= a.q_len) {
            s.q0 = first;
            s.head++;
        }
        return s;
    };
    // documents of a step's queries, as the (at most two) tiles of their positions give them
    auto row_docs = [&](int q0) {
        const int p0 = max(u.start + q0, 0), p1 = min(u.start + min(q0 + ROWS, a.q_len) - 1, a.k_len - 1);
        if (p0 > p1) return make_int2(INT32_MAX, INT32_MIN);
        const int2 x = u.doc_tiles[p0 / KEY_TILE], y = u.doc_tiles[p1 / KEY_TILE];
        return make_int2(min(x.x, y.x), max(x.y, y.y));
    };
    auto same_doc = [&](int q0) {
        if (!u.docs) return true;
        const int2 d = row_docs(q0);
        return d.x == d.y && doc_lo == doc_hi && u.start + q0 >= 0 && u.start + min(q0 + ROWS, a.q_len) <= a.k_len;
    };
    // every query of the step sees every key of the workgroup
    auto whole_step = [&](int q0) { return j0 + GRAD_KEYS <= u.end(a, u.start + q0) && q0 + ROWS <= a.q_len && same_doc(q0); };
    // the first step from s on that has work, of the kind asked for: 0 not whole, 1 whole, 2 either
    auto next = [&](Step s, int kind) {
        for (; s.i < i1; s = after(s)) {
            if (u.docs) {
                const int2 d = row_docs(s.q0);
                if (d.x > doc_hi || d.y < doc_lo) continue;
            }
            if (kind == 2 || (int)whole_step(s.q0) == kind) break;
        }
        return s;
    };
    const Mover<NB> mq(a.q.position, a.head_dim), mg(a.dout.position, a.head_dim);
    float2 stat;
    int rdoc = 0;
    auto load = [&](const Step &s, int buf) {
        const int head = u.g * a.group + s.head;
        if (threadIdx.x < ROWS) {
            const int query = s.q0 + threadIdx.x, pos = u.start + query;
            stat = query < a.q_len ? a.row_stat[((int64_t)u.b * a.k_heads * a.group + head) * a.q_len + query]
                                   : make_float2(INFINITY, 0.0f);
            if (u.docs) {
                // a position without a document sees nothing
                if (pos >= 0 && pos < a.k_len) rdoc = u.docs[pos];
                else stat.x = INFINITY;
            }
        }
        mq.load(tiles + buf * SIZE, head_base(a.q, u.b, head), s.q0, a.q_len, a.head_dim);
        mg.load(tiles + (2 + buf) * SIZE, head_base(a.dout, u.b, head), s.q0, a.q_len, a.head_dim);
    };
    auto store = [&](int buf) {
        if (threadIdx.x < ROWS) {
            lse2s[buf][threadIdx.x] = stat.x - T::p_shift - (CAP == SMALL ? cap2 : 0.0f);
            deltas[buf][threadIdx.x] = stat.y * dp_gain;
            docs[buf][threadIdx.x] = rdoc;
        }
    };
    // probability and score gradient of one element: query qi of the step, of scores s and dP dp
    auto element = [&](float distance, float slope2, float s, float dp, float lse2, float delta, float &p, float &ds)
                       __attribute__((always_inline)) {
        ds = fmaf(dp, dp_gain, -delta);
        float y;
        if constexpr (CAP == SMALL) {
            const float h = minus_half(s * scale2);
            y = fmaf(h, 2.0f * cap2, -lse2);
            ds *= fmaf(h, h, h);
        } else if constexpr (CAP == LARGE) {
            const Capped c = large_capped(s, per, scale2, cap2);
            y = c.score - lse2;
            ds *= fmaf(-c.t, c.t, 1.0f);
        } else {
            y = fmaf(s, scale2, -lse2);
        }
        if (BIAS) y -= slope2 * fabsf(distance);
        p = exp2_(y);
        ds *= p;
    };

    // A step, 32 queries after the other, whatever the masks.
    auto any_step = [&](const Step &st, int buf) {
        const bool in_doc = same_doc(st.q0);
        bool odd = false;
        if (!in_doc || min(j0 + GRAD_KEYS, u.len) > u.end(a, u.start + st.q0)) {
            // of a query with one of them, log-sum-exp or out . dout has it, and so
            // has what it adds to dK; to dV out . dout takes it (below)
            const Odd found = clean<T, SIZE>(tiles + buf * SIZE, tiles + (2 + buf) * SIZE);
            odd = found.a | found.b;
        }
        const float slope2 = BIAS && a.slopes ? a.slopes[u.g * a.group + st.head] * LOG2E : 0.0f;
#pragma unroll 1
        for (int sb = 0; sb < 2; sb++) {
            const int pb = u.start + st.q0 + 32 * sb;
            if (st.q0 + 32 * sb >= a.q_len || jw >= u.end(a, pb + 31)) continue;
            short *const qh = tiles + buf * SIZE + 32 * sb * L::PITCH, *const gh = tiles + (2 + buf) * SIZE + 32 * sb * L::PITCH;
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int k = 0; k < 2 * NB; k++) {
                s = T::mfma(L::row_operand(qh, lane % 32, k), kf[k], s);
                dp = T::mfma(L::row_operand(gh, lane % 32, k), vf[k], dp);
            }
            float p[16], ds[16];
            const float d0 = (float)(key - pb - 4 * hi);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const f32x4 lse2 = *(const f32x4 *)&lse2s[buf][32 * sb + 8 * e + 4 * hi];
                const f32x4 delta = *(const f32x4 *)&deltas[buf][32 * sb + 8 * e + 4 * hi];
#pragma unroll
                for (int n = 0; n < 4; n++)
                    element(d0 - (float)(8 * e + n), slope2, s[4 * e + n], dp[4 * e + n], lse2[n], delta[n], p[4 * e + n], ds[4 * e + n]);
            }
            if (odd)
#pragma unroll
                for (int n = 0; n < 16; n++) {
                    const float delta = deltas[buf][32 * sb + 8 * (n / 4) + 4 * hi + n % 4];
                    p[n] += delta - delta;                 // NaN where it is no number
                }
            if (!in_doc || jw + 32 > u.end(a, pb)) {
                // queries of the 32 that see the key: from `from` on, and before `to`; what
                // comes after the last query, or with documents has no position in the key
                // slots, sees nothing
                int from = key >= u.len ? INT32_MAX : a.causal && key >= u.prefix ? key - pb - 4 * hi : INT32_MIN;
                int to = a.q_len - st.q0 - 32 * sb - 4 * hi;
                if (u.docs) {
                    from = max(from, -pb - 4 * hi);
                    to = min(to, a.k_len - pb - 4 * hi);
                }
#pragma unroll
                for (int n = 0; n < 16; n++) {
                    const int r = 8 * (n / 4) + n % 4;
                    const bool seen = (r >= from) & (r < to) & (docs[buf][32 * sb + 4 * hi + r] == kdoc);
                    p[n] = seen ? p[n] : 0.0f;
                    ds[n] = seen ? ds[n] : 0.0f;
                }
            }
#pragma unroll
            for (int kc = 0; kc < 2; kc++) {
                const s16x8 pr = rounded<T>(p + 8 * kc), dr = rounded<T>(ds + 8 * kc);
#pragma unroll
                for (int d = 0; d < NB; d++) {
                    dv[d] = T::mfma(L::column_operand(gh, 16 * kc, d), pr, dv[d]);
                    dk[d] = T::mfma(L::column_operand(qh, 16 * kc, d), dr, dk[d]);
                }
            }
        }
    };

    // A step whose queries all see all keys: both halves in one stretch of
    // code.  Its matrix instructions, in order: scores and dP of the halves,
    // then their sums; operands are read from LDS six instructions ahead, and
    // the elements of a half are worked out between the matrix instructions of
    // the next stage.
    auto whole = [&](const Step &st, int buf) __attribute__((always_inline)) {
        constexpr int M = 4 * NB, AHEAD = 6;              // matrix instructions of a stage
        short *const qt = tiles + buf * SIZE, *const gt = tiles + (2 + buf) * SIZE;
        const float slope2 = BIAS && a.slopes ? a.slopes[u.g * a.group + st.head] * LOG2E : 0.0f;
        const float d0 = (float)(key - u.start - st.q0 - 4 * hi);
        f32x16 s[2] = {}, dp[2] = {};
        f32x4 lse2[2], delta[2];                          // of four queries, and of the next four
        float p[2], ds[2];
        s16x8 pr[2][2], dr[2][2], ring[AHEAD];
        auto operand = [&](auto at) __attribute__((always_inline)) {
            constexpr int i = at, sb = i / M % 2, j = i % M;
            if constexpr (i < 2 * M) return L::row_operand((j & 1 ? gt : qt) + 32 * sb * L::PITCH, lane % 32, j / 2);
            else return L::column_operand((j & 1 ? qt : gt) + 32 * sb * L::PITCH, 16 * (j / (2 * NB)), j / 2 % NB);
        };
        auto row_stats = [&](int four) __attribute__((always_inline)) {
            lse2[four % 2] = *(const f32x4 *)&lse2s[buf][8 * four + 4 * hi];
            delta[four % 2] = *(const f32x4 *)&deltas[buf][8 * four + 4 * hi];
        };
        static_for<0, AHEAD>([&](auto at) __attribute__((always_inline)) { ring[at] = operand(at); });
        row_stats(0);
        static_for<0, 4 * M>([&](auto at) __attribute__((always_inline)) {
            constexpr int i = at, sb = i / M % 2, j = i % M;
            if constexpr (i < 2 * M) {
                if (j & 1) dp[sb] = T::mfma(ring[i % AHEAD], vf[j / 2], dp[sb]);
                else s[sb] = T::mfma(ring[i % AHEAD], kf[j / 2], s[sb]);
            } else {
                constexpr int kc = j / (2 * NB), d = j / 2 % NB;
                if (j & 1) dk[d] = T::mfma(ring[i % AHEAD], dr[sb][kc], dk[d]);
                else dv[d] = T::mfma(ring[i % AHEAD], pr[sb][kc], dv[d]);
            }
            if constexpr (i + AHEAD < 4 * M) ring[i % AHEAD] = operand(std::integral_constant<int, i + AHEAD>{});
            if constexpr (i >= M && i < 3 * M) {
                constexpr int h = i / M - 1;
                static_for<j * 16 / M, (j + 1) * 16 / M>([&](auto nth) __attribute__((always_inline)) {
                    constexpr int n = nth, four = 4 * h + n / 4;
                    if constexpr (n % 4 == 0 && four < 7) row_stats(four + 1);
                    element(d0 - (float)(32 * h + 8 * (n / 4) + n % 4), slope2, s[h][n], dp[h][n], lse2[four % 2][n % 4],
                            delta[four % 2][n % 4], p[n % 2], ds[n % 2]);
                    if constexpr (n % 2 == 1) {
                        put_two<T>(pr[h][n / 8], n % 8 - 1, p);
                        put_two<T>(dr[h][n / 8], n % 8 - 1, ds);
                    }
                });
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    // All steps of a kind; the next one's rows are on their way meanwhile.
    auto walk = [&](int kind, auto work) __attribute__((always_inline)) {
        Step st = next(step_at(i0), kind);
        if (st.i < i1) {
            load(st, 0);
            store(0);
        }
        moved();
        ready();
        __syncthreads();
        for (int buf = 0; st.i < i1; buf ^= 1) {
            const Step st2 = next(after(st), kind);
            if (st2.i < i1) load(st2, buf ^ 1);
            work(st, buf);
            if (st2.i < i1) store(buf ^ 1);
            moved();
            __syncthreads();
            st = st2;
        }
    };
    if constexpr (NB == 2) {
        // One loop for up to 64 columns.  Two loops, as below, spill registers where
        // there are a cap and a bias, and measured 324 us against 297 with a cap (8192
        // tokens in three documents, 16 heads over 4), 43 against 40 with a bias and
        // lengths (8 x 512 tokens, 12 heads), and without either 352 against 418 (4 x
        // 4096 tokens, 16 heads, causal).
        walk(2, any_step);
    } else {
        // in loops of their own, or the sums would move between registers in every step
        walk(0, any_step);
        walk(1, whole);
    }
    if (key >= a.k_len) return;
    const int64_t units = (int64_t)a.batch * a.k_heads;
    float *part_k = a.part_grad + (((int64_t)part * 2 * units + u.b * a.k_heads + u.g) * a.k_len + key) * a.head_dim;
    float *part_v = part_k + units * a.k_len * a.head_dim;
#pragma unroll
    for (int d = 0; d < NB; d++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int col = 32 * d + 8 * e + 4 * hi;
            f32x4 x = f32x4{dk[d][4 * e], dk[d][4 * e + 1], dk[d][4 * e + 2], dk[d][4 * e + 3]} * unscale;
            f32x4 y = f32x4{dv[d][4 * e], dv[d][4 * e + 1], dv[d][4 * e + 2], dv[d][4 * e + 3]} * (1.0f / T::p_gain);
            if (key >= u.len) x = y = f32x4{};            // whatever the queries hold
            if (col >= a.head_dim) continue;
            if (a.parts > 1) {
                *(f32x4 *)(part_k + col) = x;
                *(f32x4 *)(part_v + col) = y;
            } else {
                write_four<T>(a.dk, u.b, u.g, key, col, x);
                write_four<T>(a.dv, u.b, u.g, key, col, y);
            }
        }
}

// Adds up the parts of dK (blockIdx.y 0) and dV (1): 8 keys a workgroup, four columns a lane.
template <typename T>
__global__ void __launch_bounds__(256) grad_join_kernel(AttnGradArgs a)
{
    const int64_t n = (int64_t)a.batch * a.k_heads * a.k_len, r = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int c = threadIdx.x % 32 * 4;
    if (r >= n || c >= a.head_dim) return;
    f32x4 sum = {};
    for (int p = 0; p < a.parts; p++) sum += *(const f32x4 *)(a.part_grad + ((2 * p + blockIdx.y) * n + r) * a.head_dim + c);
    const int64_t unit = r / a.k_len;
    write_four<T>(blockIdx.y ? a.dv : a.dk, (int)(unit / a.k_heads), (int)(unit % a.k_heads), r % a.k_len, c, sum);
}

hipError_t doc_tiles(const AttnArgs &a, hipStream_t st)
{
    if (!a.docs || !a.key_tiles) return hipSuccess;
    doc_tiles_kernel<<<dim3(a.key_tiles, a.batch < 32768 ? a.batch : 32768), 64, 0, st>>>(a);
    return hipGetLastError();
}

template <typename T, int NB, bool SHAPED, int CAP> hipError_t forward_sized(const AttnArgs &a, hipStream_t st)
{
    const int64_t units = (int64_t)a.batch * a.k_heads;
    if (a.rows <= FEW_ROWS)
        few_rows_kernel<T, NB, SHAPED, CAP><<<(unsigned)(units * a.splits), FEW_WAVES * WAVE, 0, st>>>(a);
    else
        forward_kernel<T, NB, SHAPED, CAP><<<(unsigned)(units * ((a.rows + ROW_TILE - 1) / ROW_TILE) * a.splits), 256, 0, st>>>(a);
    if (a.splits > 1) {
        if (hipError_t e = hipGetLastError()) return e;
        join_kernel<T><<<(unsigned)(units * a.rows), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

template <typename T, int NB, int CAP, bool BIAS> hipError_t backward_shaped(const AttnGradArgs &a, hipStream_t st)
{
    const int64_t units = (int64_t)a.batch * a.k_heads;
    if constexpr (T::narrow) {
        value_magnitude_kernel<T><<<(unsigned)(units * a.chunks), 256, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (a.rows) {
        dq_kernel<T, NB, CAP, BIAS><<<(unsigned)(units * ((a.rows + ROW_TILE - 1) / ROW_TILE)), 256, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (a.k_len) {
        dkv_kernel<T, NB, CAP, BIAS><<<(unsigned)(units * ((a.k_len + GRAD_KEYS - 1) / GRAD_KEYS) * a.parts), 256, 0, st>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
        if (a.parts > 1) grad_join_kernel<T><<<dim3((unsigned)((units * a.k_len + 7) / 8), 2), 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

template <typename T, int NB> hipError_t backward_sized(const AttnGradArgs &a, hipStream_t st)
{
    if (a.cap > LARGE_CAP) return backward_shaped<T, NB, LARGE, true>(a, st);        // a bias or none
    if (a.cap > 0) return a.slopes ? backward_shaped<T, NB, SMALL, true>(a, st) : backward_shaped<T, NB, SMALL, false>(a, st);
    return a.slopes ? backward_shaped<T, NB, PLAIN, true>(a, st) : backward_shaped<T, NB, PLAIN, false>(a, st);
}

template <typename T, int NB> hipError_t forward_headed(const AttnArgs &a, hipStream_t st)
{
    if (a.cap > LARGE_CAP) return forward_sized<T, NB, true, LARGE>(a, st);
    return a.cap > 0 || a.slopes ? forward_sized<T, NB, true, SMALL>(a, st) : forward_sized<T, NB, false, PLAIN>(a, st);
}

template <typename T> hipError_t forward_typed(const AttnArgs &a, hipStream_t st)
{
    return a.head_dim <= 64 ? forward_headed<T, 2>(a, st) : a.head_dim <= 96 ? forward_headed<T, 3>(a, st) : forward_headed<T, 4>(a, st);
}

template <typename T> hipError_t backward_typed(const AttnGradArgs &a, hipStream_t st)
{
    return a.head_dim <= 64 ? backward_sized<T, 2>(a, st) : a.head_dim <= 96 ? backward_sized<T, 3>(a, st) : backward_sized<T, 4>(a, st);
}

}  // namespace

hipError_t launch_attn_forward(const AttnArgs &a, int type, hipStream_t st)
{
    if (hipError_t e = doc_tiles(a, st)) return e;
    return type == 0 ? forward_typed<Bf16>(a, st) : forward_typed<Fp16>(a, st);
}

hipError_t launch_attn_backward(const AttnGradArgs &a, int type, hipStream_t st)
{
    if (hipError_t e = doc_tiles(a, st)) return e;
    return type == 0 ? backward_typed<Bf16>(a, st) : backward_typed<Fp16>(a, st);
}

}  // namespace dtrops
