// rows.hip -- operators that read whole rows once: dropout with the residual
// sum, log probabilities of given tokens and their gradient.
#include "ops.h"

namespace dtrops {
namespace {

constexpr uint64_t GOLDEN = 0x9E3779B97F4A7C15ull;
constexpr int WAVE = 64;

__device__ __forceinline__ uint64_t mix64(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

struct Bf16 { using raw = __bf16; static constexpr int vec = 8; };
struct Fp16 { using raw = _Float16; static constexpr int vec = 8; };
struct Fp32 { using raw = float; static constexpr int vec = 4; };

template <typename R, int N> struct alignas(16) Pack { R e[N]; };

// A 16-byte access that, with PAST, asks the caches not to keep the line.
// The launches ask for it where one call's rows in and out are more than the
// last-level cache holds, which no reader after it could profit from; written
// lines left there would be put out during the next kernel instead.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename R, int N, bool PAST> __device__ __forceinline__ Pack<R, N> load_pack(const R *p)
{
    if (!PAST) return *(const Pack<R, N> *)p;
    return __builtin_bit_cast(Pack<R, N>, __builtin_nontemporal_load((const u32x4 *)p));
}

template <typename R, int N, bool PAST> __device__ __forceinline__ void store_pack(R *p, const Pack<R, N> &v)
{
    if (PAST)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4 *)p);
    else
        *(Pack<R, N> *)p = v;
}

constexpr int64_t LAST_CACHE = (int64_t)256 << 20;       // bytes

// ---- dropout ---------------------------------------------------------------
// out = residual + keep x / (1 - p).  The mask is a hash of the element's
// number: nothing but x, residual and out crosses the memory bus.  One 64-bit
// draw (two 64-bit products) makes the mask of two elements.  Bound by memory:
// 32768 rows of 8192 in 16 bits, 323 us with the residual (5.0 TB/s), 197 us
// without, as in the gradient (5.4 TB/s); 4096 of 768, 5 us.

template <typename T, bool PAST>
__global__ void __launch_bounds__(256) dropout_vector(DropArgs a)
{
    using R = typename T::raw;
    const int64_t r = blockIdx.y;
    for (int64_t row = r; row < a.rows; row += gridDim.y) {
        const R *x = (const R *)a.x + row * a.x_stride;
        const R *res = a.residual ? (const R *)a.residual + row * a.r_stride : nullptr;
        R *out = (R *)a.out + row * a.o_stride;
        const int64_t groups = (a.cols + 7) / 8, step = (int64_t)gridDim.x * 256;
        for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += step) {
            const int64_t c = g * 8;
            const uint64_t z0 = a.key + GOLDEN * (a.offset + (uint64_t)((row * a.cols + c) >> 1));
            uint64_t d[4];
#pragma unroll
            for (int i = 0; i < 4; i++) d[i] = mix64(z0 + GOLDEN * i);
            constexpr int N = T::vec;
            R xs[8], rs[8], os[8];
            const bool whole = c + 8 <= a.cols;
            if (whole) {
#pragma unroll
                for (int i = 0; i < 8; i += N) {
                    const auto p = load_pack<R, N, PAST>(x + c + i);
                    __builtin_memcpy(xs + i, &p, sizeof(p));
                }
                if (res)
#pragma unroll
                    for (int i = 0; i < 8; i += N) {
                        const auto p = load_pack<R, N, PAST>(res + c + i);
                        __builtin_memcpy(rs + i, &p, sizeof(p));
                    }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    xs[e] = c + e < a.cols ? x[c + e] : (R)0.0f;
                    rs[e] = res && c + e < a.cols ? res[c + e] : (R)0.0f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const uint32_t u = e & 1 ? (uint32_t)(d[e / 2] >> 32) : (uint32_t)d[e / 2];
                float v = (uint64_t)u >= a.threshold ? (float)xs[e] * a.inv : 0.0f;
                if (res) v += (float)rs[e];
                os[e] = (R)v;
            }
            if (whole) {
#pragma unroll
                for (int i = 0; i < 8; i += N) {
                    Pack<R, N> p;
                    __builtin_memcpy(&p, os + i, sizeof(p));
                    store_pack<R, N, PAST>(out + c + i, p);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (c + e < a.cols) out[c + e] = os[e];
            }
        }
    }
}

// rows whose addresses rule out 16-byte accesses: an element a lane
template <typename T>
__global__ void __launch_bounds__(256) dropout_scalar(DropArgs a)
{
    using R = typename T::raw;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const R *x = (const R *)a.x + row * a.x_stride;
        const R *res = a.residual ? (const R *)a.residual + row * a.r_stride : nullptr;
        R *out = (R *)a.out + row * a.o_stride;
        const int64_t step = (int64_t)gridDim.x * 256;
        for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < a.cols; c += step) {
            const uint64_t n = (uint64_t)(row * a.cols + c);
            const uint64_t d = mix64(a.key + GOLDEN * (a.offset + (n >> 1)));
            const uint32_t u = n & 1 ? (uint32_t)(d >> 32) : (uint32_t)d;
            float v = (uint64_t)u >= a.threshold ? (float)x[c] * a.inv : 0.0f;
            if (res) v += (float)res[c];
            out[c] = (R)v;
        }
    }
}

template <typename T> hipError_t dropout_typed(const DropArgs &a, hipStream_t st)
{
    // 32768 rows of 8192 in 16 bits: with the residual 323 us, 360 through the
    // caches; without it 197 and 211
    const bool past = a.rows * a.cols * (int64_t)sizeof(typename T::raw) * (a.residual ? 3 : 2) > LAST_CACHE;
    const int64_t items = a.vector ? (a.cols + 7) / 8 : a.cols;
    const unsigned gx = (unsigned)std::min<int64_t>((items + 255) / 256, a.rows > 1 ? 64 : 8192);
    const unsigned gy = (unsigned)std::min<int64_t>(a.rows, 32768);
    if (a.vector && past)
        dropout_vector<T, true><<<dim3(gx, gy), 256, 0, st>>>(a);
    else if (a.vector)
        dropout_vector<T, false><<<dim3(gx, gy), 256, 0, st>>>(a);
    else
        dropout_scalar<T><<<dim3(gx, gy), 256, 0, st>>>(a);
    return hipGetLastError();
}

// ---- log probabilities -------------------------------------------------------
// One pass: a running maximum m, l = sum exp(x - m) and w = sum exp(x - m)
// (x - m) give lse = m + log l and entropy = log l - w / l (w and log l
// in units of log 2, as the exponential instruction has it).  Bound by reading
// the row: 4096 rows of 32000 in 16 bits, 52 us (5.0 TB/s); with 20
// alternatives, whose vectors are read again, 8192 rows of 100003, 358-430 us
// by the inputs (3.8 to 4.6 TB/s); 4 rows of 50021 in 32 bits in 48 parts, 9 us and 4 for their join.

constexpr float LOWEST = -3.402823466e+38f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// m: maximum; l = sum exp(x - m); w = sum exp(x - m) (x - m) log2(e).  The
// maximum is subtracted before the factor log2(e): that times the type's
// lowest value would be minus infinity.
struct Stat { float m, l, w; };

__device__ __forceinline__ Stat join(Stat a, Stat b)
{
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf((a.m - m) * LOG2E, -1e4f), db = fmaxf((b.m - m) * LOG2E, -1e4f);
    const float ea = __builtin_amdgcn_exp2f(da), eb = __builtin_amdgcn_exp2f(db);
    return {m, a.l * ea + b.l * eb, (a.w + da * a.l) * ea + (b.w + db * b.l) * eb};
}

__device__ __forceinline__ Stat join_wave(Stat s)
{
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) {
        Stat o = {__shfl_xor(s.m, d), __shfl_xor(s.l, d), __shfl_xor(s.w, d)};
        s = join(s, o);
    }
    return s;
}

// Lane exchanges within the vector unit: they cost what an addition costs,
// where one through LDS would wait a hundred cycles.
template <int CONTROL> __device__ __forceinline__ float moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CONTROL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_value(float v, int lane)              // lane: uniform
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ __forceinline__ float wave_max(float v)                          // uniform
{
    v = fmaxf(v, moved<0x111>(v));                                          // row_shr:1 .. 8: rows of 16 lanes
    v = fmaxf(v, moved<0x112>(v));
    v = fmaxf(v, moved<0x114>(v));
    v = fmaxf(v, moved<0x118>(v));
    v = fmaxf(v, moved<0x142>(v));                                          // row_bcast:15, row_bcast:31
    v = fmaxf(v, moved<0x143>(v));
    return lane_value(v, WAVE - 1);
}

// A wavefront's list of alternatives, which takes elements in any number and
// order: an element is compared with the list's last, through the maximum of
// its vector.  Lane i < count holds the i-th largest value and its
// column, the lower column first among equals.
struct Top {
    float value;
    int32_t column;
    int count;                    // uniform, as all below
    float last;                   // the k-th value once the list is full
    int32_t last_column;
    float floor;                  // until then: k elements or more are at least this

    __device__ void clear()
    {
        value = 0;
        column = -1;
        count = 0;
        last = floor = -INFINITY;
        last_column = -1;
    }

    // whether an element of a later column than all in the list may enter it
    __device__ bool wants(float v, int k) const { return count < k ? v >= floor : v > last; }

    __device__ void offer(float v, int32_t c, int k)       // uniform arguments, any column
    {
        if (count == k && !(v > last || (v == last && c < last_column))) return;
        const int lane = threadIdx.x % WAVE;
        const int at = __popcll(__ballot(lane < count && (value > v || (value == v && column < c))));
        const float pv = moved<0x138>(value);                               // wave_shr:1
        const int32_t pc = __builtin_amdgcn_update_dpp(column, column, 0x138, 0xf, 0xf, false);
        value = lane > at ? pv : lane == at ? v : value;
        column = lane > at ? pc : lane == at ? c : column;
        if (count < k) count++;
        if (lane >= count) column = -1;
        if (count == k) {
            last = lane_value(value, k - 1);
            last_column = __builtin_amdgcn_readlane(column, k - 1);
        }
    }

    // The k-th largest of 64 lanes' values bounds the k-th largest of all from
    // below.  With the maxima of the first 2048 elements, 24 of them enter a
    // list of 20 where 112 would enter one that grows from nothing.
    __device__ void set_floor(float v, int k)
    {
        const int lane = threadIdx.x % WAVE;
        v = v == v ? v : -INFINITY;
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < WAVE; j++) {
            const float o = lane_value(v, j);
            rank += o > v || (o == v && j < lane);
        }
        floor = lane_value(v, __ffsll(__ballot(rank == k - 1)) - 1);
    }
};

// Candidates of one step, N a lane, all of later columns than the list's.
template <int N>
__device__ void top_step(Top &top, const float (&x)[N], bool in, int32_t column0, int k)
{
    const bool full = top.count == k;
    const float bar = full ? top.last : top.floor;
#pragma unroll
    for (int e = 0; e < N; e++) {
        const float v = x[e] == x[e] ? x[e] : -INFINITY;            // a NaN counts as the least
        for (uint64_t open = __ballot(in && (full ? v > bar : v >= bar)); open; open &= open - 1) {
            const int lane = __ffsll((unsigned long long)open) - 1;
            top.offer(lane_value(v, lane), __builtin_amdgcn_readlane(column0, lane) + e, k);
        }
    }
}

// Returns the largest of the x.
template <int N>
__device__ __forceinline__ float stat_step(Stat &s, const float (&x)[N])
{
    float most = x[0];
#pragma unroll
    for (int e = 1; e < N; e++) most = fmaxf(most, x[e]);
    if (most > s.m) {
        const float d = fmaxf((s.m - most) * LOG2E, -1e4f), f = __builtin_amdgcn_exp2f(d);
        s.w = (s.w + d * s.l) * f;
        s.l *= f;
        s.m = most;
    }
#pragma unroll
    for (int e = 0; e < N; e++) {
        const float d = (x[e] - s.m) * LOG2E;
        const float p = __builtin_amdgcn_exp2f(d);
        s.l += p;                                                  // carries a NaN
        s.w = fmaf(p, fmaxf(d, -1e4f), s.w);                       // 0 for minus infinity
    }
    return most;
}

// A row's results; lane i < top holds the i-th alternative.
__device__ void finish_row(const LogpArgs &a, int64_t row, Stat s, float value, int32_t column, float token_logit, int64_t token)
{
    const int lane = threadIdx.x % WAVE;
    const bool nothing = s.l == 0;                                  // minus infinity throughout
    const float log_l = __builtin_amdgcn_logf(s.l);
    const float lse = nothing ? -INFINITY : s.m + log_l * LN2;
    if (lane == 0) {
        a.lse[row] = lse;
        a.entropy[row] = nothing ? 0.0f : (log_l - s.w / s.l) * LN2;
        a.logp[row] = token < 0 ? 0.0f : token >= a.vocab ? NAN : nothing ? -INFINITY : token_logit - lse;
    }
    if (lane < a.top) {
        a.top_logp[row * a.top + lane] = nothing ? -INFINITY : value - lse;
        a.top_ids[row * a.top + lane] = column < 0 ? 0 : column;
    }
}

// a list entry of every lane with column >= 0
__device__ void join_list(Top &top, float v, int32_t c, int k)
{
    for (uint64_t open = __ballot(c >= 0); open; open &= open - 1) {
        const int lane = __ffsll((unsigned long long)open) - 1;
        top.offer(lane_value(v, lane), __builtin_amdgcn_readlane(c, lane), k);
    }
}

constexpr int AHEAD = 4;

// A wavefront's share of a row's part: chunks of four 16-byte vectors a lane,
// the workgroup's WAVES wavefronts in turn, so that a workgroup reads one
// stretch of memory.  Columns before the row's first 128-byte boundary go to
// the first wavefront of the first part, those after its last whole vector to
// the last of the last.
template <typename T, int WAVES> struct Segment {
    using R = typename T::raw;
    static constexpr int N = T::vec, CHUNK = AHEAD * WAVE, STEP = WAVES * CHUNK;
    const R *x;
    int head, part0, v0, v1, tail0, tails;
    bool first;

    __device__ Segment(const R *row, int vocab, int wave, int part, int parts) : x(row)
    {
        constexpr int LINE = 128 / sizeof(R);
        const int mis = (int)((uintptr_t)row % 128 / sizeof(R));
        head = min(mis ? LINE - mis : 0, vocab);
        const int vecs = (vocab - head) / N, per = parts > 1 ? (vecs + parts * 8 - 1) / (parts * 8) * 8 : vecs;
        part0 = min(per * part, vecs);
        v0 = part0 + wave * CHUNK;
        v1 = min(part0 + per, vecs);
        first = part == 0 && wave == 0;
        tail0 = head + vecs * N;
        tails = part == parts - 1 && wave == WAVES - 1 ? vocab - tail0 : 0;
    }
    __device__ Pack<R, N> vector(int v) const { return *(const Pack<R, N> *)(x + head + (int64_t)v * N); }
};

// What a lane knows of its own columns (edges aside): the largest, the chunk
// that it is in, and the largest of the other chunks.
struct LaneTop {
    float best, second;
    int chunk;
};

template <typename T, int WAVES, bool TOP>
__device__ __forceinline__ Stat segment_stat(const Segment<T, WAVES> &g, LaneTop &top)
{
    using R = typename T::raw;
    constexpr int N = T::vec;
    const int lane = threadIdx.x % WAVE;
    Stat s = {LOWEST, 0, 0};
    Pack<R, N> ahead[AHEAD];
    auto load = [&](int v) {
#pragma unroll
        for (int i = 0; i < AHEAD; i++)
            if (v + i * WAVE + lane < g.v1) ahead[i] = g.vector(v + i * WAVE + lane);
    };
    top = {-INFINITY, -INFINITY, 0};
    load(g.v0);
    for (int v = g.v0; v < g.v1; v += g.STEP) {
        float e[AHEAD][N];
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
            const bool in = v + i * WAVE + lane < g.v1;
#pragma unroll
            for (int j = 0; j < N; j++) e[i][j] = in ? (float)ahead[i].e[j] : -INFINITY;
        }
        load(v + g.STEP);
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < AHEAD; i++) most = fmaxf(most, stat_step(s, e[i]));
        if (TOP) {
            top.second = fmaxf(top.second, fminf(top.best, most));
            top.chunk = most > top.best ? v : top.chunk;
            top.best = fmaxf(top.best, most);
        }
    }
    if (g.first && lane < g.head) {
        const float e[1] = {(float)g.x[lane]};
        stat_step(s, e);
    }
    if (lane < g.tails) {
        const float e[1] = {(float)g.x[g.tail0 + lane]};
        stat_step(s, e);
    }
    return s;
}

// The alternatives of a wavefront's share, by the list.
template <typename T, int WAVES>
__device__ Top segment_top(const Segment<T, WAVES> &g, int k)
{
    constexpr int N = T::vec;
    const int lane = threadIdx.x % WAVE;
    Top top;
    top.clear();
    auto edge = [&](int c0, int n) {
        const float e[1] = {lane < n ? (float)g.x[c0 + lane] : -INFINITY};
        top_step(top, e, lane < n, c0 + lane, k);
    };
    if (g.first && g.head) edge(0, g.head);
    for (int c = g.v0; c < g.v1; c += g.STEP)
    for (int v = c; v < min(c + g.CHUNK, g.v1); v += WAVE) {
        const bool in = v + lane < g.v1;
        float e[N], most = -INFINITY;
        auto p = g.vector(in ? v + lane : v);
#pragma unroll
        for (int j = 0; j < N; j++) {
            e[j] = in ? (float)p.e[j] : -INFINITY;
            most = fmaxf(most, e[j]);
        }
        if (v == g.v0) top.set_floor(most, k);
        if (__ballot(in && top.wants(most, k))) top_step(top, e, in, g.head + (v + lane) * N, k);
    }
    if (g.tails) edge(g.tail0, g.tails);
    return top;
}

// A workgroup's alternatives among its part of a row.  The statistics' pass
// has left each lane the maximum of its own columns: a wavefront's k-th
// largest of these bounds the part's k-th largest element from below.  Of the
// lanes that reach the best of the four bounds (at most 4 k, more where maxima
// are equal), those of the k largest maxima own all elements that can count.
// The chunk of a lane's maximum is read again (all of its chunks, if the
// largest of the others reaches the bar), and of the few elements found each
// counts how many are ahead of it.  Where more are found than there is room
// for, as among many equal ones, or fewer than k numbers, the wavefronts'
// lists do it instead.
constexpr int FOUND = 512;

struct TopScratch {
    float bars[SEGS];
    struct {
        int lane, chunk;
        float best, second;
    } lanes[256];
    int kept[128];
    float2 found[FOUND];
    float2 lists[SEGS][32];
    float2 best[32];                     // the result: value, column (as bits; -1: none), largest first
    int n_lanes, n_kept, n_found;
};

template <typename T>
__device__ void part_top(TopScratch &w, const Segment<T, SEGS> &g, const LaneTop &top, int k)
{
    constexpr int N = T::vec;
    const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE;
    const float most = top.best;
    // each wavefront's k-th largest lane; the largest of these bounds the row's
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < WAVE; j++) {
        const float o = lane_value(most, j);
        rank += o > most || (o == most && j < lane);
    }
    if (rank == k - 1) w.bars[wave] = most;
    if (tid == 0) w.n_lanes = w.n_kept = w.n_found = 0;
    if (tid < 32) w.best[tid] = make_float2(0, __int_as_float(-1));
    __syncthreads();
    float bar = fmaxf(fmaxf(w.bars[0], w.bars[1]), fmaxf(w.bars[2], w.bars[3]));
    if (most >= bar) {
        const int at = atomicAdd(&w.n_lanes, 1);
        w.lanes[at] = {tid, top.chunk, most, top.second};
    }
    auto offer = [&](float v, int c) {                      // `bar` may rise between calls
        if (!(v >= bar)) return;
        const int at = atomicAdd(&w.n_found, 1);
        if (at < FOUND) w.found[at] = make_float2(v, __int_as_float(c));
    };
    if (g.first && lane < g.head) offer((float)g.x[lane], lane);
    if (lane < g.tails) offer((float)g.x[g.tail0 + lane], g.tail0 + lane);
    __syncthreads();
    const int n_lanes = w.n_lanes;
    if (n_lanes <= 4 * k) {
        // the lanes of the k largest maxima, and the k-th of those as the bar
        if (tid < n_lanes) {
            const float mine = w.lanes[tid].best;
            int ahead = 0, level = 0;
#pragma unroll 8
            for (int j = 0; j < n_lanes; j++) {
                ahead += w.lanes[j].best > mine;
                level += w.lanes[j].best == mine;
            }
            if (ahead < k) w.kept[atomicAdd(&w.n_kept, 1)] = tid;
            if (ahead < k && ahead + level >= k) w.bars[0] = mine;      // equal lanes write the same
        }
        __syncthreads();
        bar = w.bars[0];
        // their vectors: of the chunk with the largest, or of all chunks where another one reaches the bar
        const int chunks = (g.v1 - g.part0 + g.STEP - 1) / g.STEP, n_kept = w.n_kept;
        for (int i = tid / AHEAD; i < n_kept; i += 256 / AHEAD) {
            const auto &own = w.lanes[w.kept[i]];
            const int base = own.lane / WAVE * g.CHUNK + own.lane % WAVE + tid % AHEAD * WAVE;
            const bool all = own.second >= bar;
            for (int c = 0; c < (all ? chunks : 1); c++) {
                const int v = (all ? g.part0 + c * g.STEP : own.chunk - own.lane / WAVE * g.CHUNK) + base;
                if (v >= g.v1) continue;
                const auto p = g.vector(v);
#pragma unroll
                for (int e = 0; e < N; e++) offer((float)p.e[e], g.head + v * N + e);
            }
        }
    }
    __syncthreads();
    const int n = w.n_found;
    if (n_lanes <= 4 * k && n <= FOUND && n >= k) {
        for (int i = tid; i < n; i += 256) {
            const float2 mine = w.found[i];
            int ahead = 0;
#pragma unroll 8
            for (int j = 0; j < n; j++) {
                const float2 o = w.found[j];
                ahead += o.x > mine.x || (o.x == mine.x && __float_as_int(o.y) < __float_as_int(mine.y));
            }
            if (ahead < k) w.best[ahead] = mine;
        }
    } else {
        Top list = segment_top<T, SEGS>(g, k);
        if (lane < k) w.lists[wave][lane] = make_float2(list.value, __int_as_float(list.column));
        __syncthreads();
        if (wave == 0) {
            for (int i = 1; i < SEGS; i++) {
                const float2 t = lane < k ? w.lists[i][lane] : make_float2(0, __int_as_float(-1));
                join_list(list, t.x, __float_as_int(t.y), k);
            }
            if (lane < k) w.best[lane] = make_float2(list.value, __int_as_float(list.column));
        }
    }
    __syncthreads();
}

// Short rows: a wavefront each.
template <typename T, bool TOP>
__global__ void __launch_bounds__(256) logprob_short(LogpArgs a)
{
    using R = typename T::raw;
    const int64_t row = (int64_t)blockIdx.x * SEGS + threadIdx.x / WAVE;
    if (row >= a.rows) return;
    const R *x = (const R *)a.x + row * a.stride;
    const int64_t token = a.tokens[row];
    const float logit = token >= 0 && token < a.vocab ? (float)x[token] : 0.0f;
    const Segment<T, 1> g(x, (int)a.vocab, 0, 0, 1);
    LaneTop unused;
    const Stat s = join_wave(segment_stat<T, 1, false>(g, unused));
    Top top;
    top.clear();
    if (TOP) top = segment_top<T, 1>(g, a.top);
    finish_row(a, row, s, top.value, top.column, logit, token);
}

// A workgroup a row, or a part of one.
template <typename T, bool TOP>
__global__ void __launch_bounds__(256) logprob_kernel(LogpArgs a)
{
    using R = typename T::raw;
    __shared__ float part[SEGS][3];
    __shared__ TopScratch scratch;
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int row = a.splits > 1 ? (int)blockIdx.x / a.splits : (int)blockIdx.x, split = (int)blockIdx.x - row * a.splits;
    const R *x = (const R *)a.x + row * a.stride;
    const int64_t token = a.tokens[row];
    const Segment<T, SEGS> g(x, (int)a.vocab, __builtin_amdgcn_readfirstlane(wave), split, a.splits);
    LaneTop lane_top;
    Stat s = segment_stat<T, SEGS, TOP>(g, lane_top);
    const float logit = token >= 0 && token < a.vocab ? (float)x[token] : 0.0f;      // here: behind the row's loads
    s = join_wave(s);
    if (lane == 0) {
        part[wave][0] = s.m;
        part[wave][1] = s.l;
        part[wave][2] = s.w;
    }
    if (TOP) part_top<T>(scratch, g, lane_top, a.top);
    else __syncthreads();
    if (wave) return;
    s = {part[0][0], part[0][1], part[0][2]};
    for (int i = 1; i < SEGS; i++) s = join(s, {part[i][0], part[i][1], part[i][2]});
    const float2 best = TOP && lane < a.top ? scratch.best[lane] : make_float2(0, __int_as_float(-1));
    if (a.splits == 1) {
        finish_row(a, row, s, best.x, __float_as_int(best.y), logit, token);
        return;
    }
    float *o = a.part + (int64_t)blockIdx.x * 4;
    if (lane == 0) {
        o[0] = s.m;
        o[1] = s.l;
        o[2] = s.w;
        o[3] = logit;
    }
    if (TOP && lane < a.top) a.part_top[(int64_t)blockIdx.x * a.top + lane] = best;
}

// The parts of a row that several workgroups read (at most 64): the
// alternatives by counting how many of all parts' are ahead of each.
template <bool TOP>
__global__ void __launch_bounds__(256) logprob_join(LogpArgs a)
{
    __shared__ uint64_t all[64 * 32];
    __shared__ float2 best[32];
    const int tid = threadIdx.x, lane = tid % WAVE;
    const int64_t row = blockIdx.x;
    const int64_t token = a.tokens[row];
    const float logit = a.part[row * a.splits * 4 + 3];
    Stat s = {LOWEST, 0, 0};
    if (lane < a.splits) {
        const float *o = a.part + (row * a.splits + lane) * 4;
        s = {o[0], o[1], o[2]};
    }
    if (TOP) {
        const int n = a.splits * a.top;
        // an entry as one number that orders as (value, lower column first) does; none: 0.
        // Minus zero plus zero is zero.
        for (int i = tid; i < n; i += 256) {
            const float2 e = a.part_top[row * n + i];
            const uint32_t v = __float_as_uint(e.x + 0.0f), up = v & 0x80000000u ? ~v : v | 0x80000000u;
            all[i] = __float_as_int(e.y) < 0 ? 0 : (uint64_t)up << 32 | ~__float_as_uint(e.y);
        }
        if (tid < 32) best[tid] = make_float2(0, __int_as_float(-1));
        __syncthreads();
        for (int i = tid; i < n; i += 256) {
            const uint64_t mine = all[i];
            int ahead = 0;
#pragma unroll 8
            for (int j = 0; j < n; j++) ahead += all[j] > mine;
            if (mine && ahead < a.top) best[ahead] = a.part_top[row * n + i];
        }
        __syncthreads();
    }
    if (tid >= WAVE) return;
    s = join_wave(s);
    const float2 b = TOP && lane < a.top ? best[lane] : make_float2(0, __int_as_float(-1));
    finish_row(a, row, s, b.x, __float_as_int(b.y), logit, token);
}

template <typename T, bool TOP> hipError_t logprobs_typed(const LogpArgs &a, hipStream_t st)
{
    // Short rows: a wavefront each, of up to 8 vectors a lane (4096 rows of 4096
    // in 16 bits: 10 us, by workgroups 13; of 8192 no gain).  Its alternatives
    // are a serial list, so that these want shorter rows, the shorter the fewer
    // there are (8 of 1024: 4096 rows 20 us and 27, 64 rows 13 us and 9; of 512:
    // 14 and 27, 9.1 and 8.5).
    const int64_t vectors = !TOP ? 8 : a.rows > 1024 ? 2 : 1;
    if (a.vocab <= vectors * WAVE * T::vec) {
        logprob_short<T, TOP><<<(unsigned)((a.rows + SEGS - 1) / SEGS), 256, 0, st>>>(a);
        return hipGetLastError();
    }
    logprob_kernel<T, TOP><<<(unsigned)(a.rows * a.splits), 256, 0, st>>>(a);
    if (a.splits > 1) {
        if (hipError_t e = hipGetLastError()) return e;
        logprob_join<TOP><<<(unsigned)a.rows, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

// ---- gradient of the log probabilities ------------------------------------------
// dx_v = dlogp [v = token] + sum_k dtop_k [v = id_k] - p_v (G + dH (log p_v + H))
// One read and one write of the row; the few columns that get a term of their
// own are written once more, after the barrier, by the workgroup that owns them.
// Bound by memory: 4096 rows of 32000 in 16 bits, 76 us (6.9 TB/s, the row in
// part from the last-level cache).

template <typename T, bool PAST>
__global__ void __launch_bounds__(256) logprob_grad(LogpGradArgs a, int64_t per)
{
    using R = typename T::raw;
    constexpr int N = T::vec;
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
    if (row >= a.rows) return;
    const R *x = (const R *)a.x + row * a.stride;
    R *dx = (R *)a.dx + row * a.dstride;
    const float lse = a.lse[row], H = a.entropy[row];
    const int64_t token = a.tokens[row];
    const float g0 = !a.dlogp || token < 0 ? 0.0f : token >= a.vocab ? NAN : a.dlogp[row];
    const float dH = a.dentropy ? a.dentropy[row] : 0.0f;
    float G = g0;
    for (int k = 0; k < a.top; k++) G += a.dtop[row * a.top + k];
    const bool nothing = lse == -INFINITY;
    auto value = [&](float v) {
        const float d = nothing ? -INFINITY : v - lse;
        const float p = __builtin_amdgcn_exp2f(d * LOG2E);
        return -p * (G + dH * (fmaxf(d, -1e4f) + H));
    };
    const int64_t c0 = (int64_t)blockIdx.x * per, c1 = min(c0 + per, a.vocab);
    const int64_t mis = (uintptr_t)(x + c0) % 16 / sizeof(R);
    if (mis == (int64_t)((uintptr_t)(dx + c0) % 16 / sizeof(R))) {
        const int64_t head = min(mis ? N - mis : (int64_t)0, c1 - c0);
        const int64_t vecs = (c1 - c0 - head) / N, tail0 = c0 + head + vecs * N;
        if ((int64_t)threadIdx.x < head) dx[c0 + threadIdx.x] = (R)value((float)x[c0 + threadIdx.x]);
        for (int64_t v = threadIdx.x; v < vecs; v += 256) {
            const Pack<R, N> p = *(const Pack<R, N> *)(x + c0 + head + v * N);
            Pack<R, N> o;
#pragma unroll
            for (int i = 0; i < N; i++) o.e[i] = (R)value((float)p.e[i]);
            store_pack<R, N, PAST>(dx + c0 + head + v * N, o);
        }
        if (tail0 + threadIdx.x < c1) dx[tail0 + threadIdx.x] = (R)value((float)x[tail0 + threadIdx.x]);
    } else {
        for (int64_t c = c0 + threadIdx.x; c < c1; c += 256) dx[c] = (R)value((float)x[c]);
    }
    if (nothing) return;
    __syncthreads();
    if ((int)threadIdx.x <= a.top) {
        const int64_t c = threadIdx.x == 0 ? token : a.top_ids[row * a.top + threadIdx.x - 1];
        if (c >= c0 && c < c1) {
            float extra = c == token ? g0 : 0.0f;
            for (int k = 0; k < a.top; k++)
                if (a.top_ids[row * a.top + k] == c) extra += a.dtop[row * a.top + k];
            dx[c] = (R)(value((float)x[c]) + extra);
        }
    }
}

template <typename T> hipError_t logprobs_grad_typed(const LogpGradArgs &a, hipStream_t st)
{
    // 4096 rows of 32000 in 16 bits: 76 us, 80 through the caches, and the
    // forward kernel of the next step 52 us, then 75
    const bool past = a.rows * a.vocab * (int64_t)sizeof(typename T::raw) * 2 > LAST_CACHE;
    const int64_t per = 8192;                                      // columns of a workgroup
    const unsigned gx = (unsigned)((a.vocab + per - 1) / per);
    const unsigned gy = (unsigned)std::min<int64_t>(a.rows, 32768), gz = (unsigned)((a.rows + gy - 1) / gy);
    if (past)
        logprob_grad<T, true><<<dim3(gx, gy, gz), 256, 0, st>>>(a, per);
    else
        logprob_grad<T, false><<<dim3(gx, gy, gz), 256, 0, st>>>(a, per);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropArgs &a, int type, hipStream_t st)
{
    return type == 0 ? dropout_typed<Bf16>(a, st) : type == 1 ? dropout_typed<Fp16>(a, st) : dropout_typed<Fp32>(a, st);
}

hipError_t launch_logprobs(const LogpArgs &a, int type, hipStream_t st)
{
    if (a.top)
        return type == 0   ? logprobs_typed<Bf16, true>(a, st)
               : type == 1 ? logprobs_typed<Fp16, true>(a, st)
                           : logprobs_typed<Fp32, true>(a, st);
    return type == 0   ? logprobs_typed<Bf16, false>(a, st)
           : type == 1 ? logprobs_typed<Fp16, false>(a, st)
                       : logprobs_typed<Fp32, false>(a, st);
}

hipError_t launch_logprobs_grad(const LogpGradArgs &a, int type, hipStream_t st)
{
    return type == 0   ? logprobs_grad_typed<Bf16>(a, st)
           : type == 1 ? logprobs_grad_typed<Fp16>(a, st)
                       : logprobs_grad_typed<Fp32>(a, st);
}

}  // namespace dtrops
