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

// ---- dropout ---------------------------------------------------------------
// out = residual + keep x / (1 - p).  The mask is a hash of the element's
// number: nothing but x, residual and out crosses the memory bus.  One 64-bit
// draw (two 64-bit products) makes the mask of two elements.

template <typename T>
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
            R xs[8], rs[8], os[8];
            const bool whole = c + 8 <= a.cols;
            if (whole) {
                __builtin_memcpy(xs, __builtin_assume_aligned(x + c, 16), sizeof(xs));
                if (res) __builtin_memcpy(rs, __builtin_assume_aligned(res + c, 16), sizeof(rs));
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
                __builtin_memcpy(__builtin_assume_aligned(out + c, 16), os, sizeof(os));
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
    const int64_t items = a.vector ? (a.cols + 7) / 8 : a.cols;
    const unsigned gx = (unsigned)std::min<int64_t>((items + 255) / 256, a.rows > 1 ? 64 : 8192);
    const unsigned gy = (unsigned)std::min<int64_t>(a.rows, 32768);
    if (a.vector)
        dropout_vector<T><<<dim3(gx, gy), 256, 0, st>>>(a);
    else
        dropout_scalar<T><<<dim3(gx, gy), 256, 0, st>>>(a);
    return hipGetLastError();
}

// ---- log probabilities -------------------------------------------------------
// One pass: a running maximum m, l = sum exp(x - m) and w = sum exp(x - m)
// (x - m) give lse = m + log l and entropy = log l - w / l.  The alternatives
// are kept by each wavefront as a list sorted over its lanes; an element is
// compared with the list's last only, through the maximum of its vector.

constexpr float LOWEST = -3.402823466e+38f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Stat { float m, l, w; };

__device__ __forceinline__ Stat join(Stat a, Stat b)
{
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf(a.m - m, -1e4f), db = fmaxf(b.m - m, -1e4f);
    const float ea = __builtin_amdgcn_exp2f(da * LOG2E), eb = __builtin_amdgcn_exp2f(db * LOG2E);
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

// The wavefront's list: lane i < count holds the i-th largest value and its
// column.  Elements come in ascending order of columns, so among equals the
// one that came first stays in front.
struct Top {
    float value;
    int32_t column;
    int count;                    // uniform
    float last;                   // uniform: the k-th value once the list is full

    __device__ void clear()
    {
        value = 0;
        column = -1;
        count = 0;
        last = LOWEST;
    }

    __device__ bool wants(float v, int k) const { return count < k || v > last; }

    __device__ void insert(float v, int32_t c, int k)      // uniform arguments
    {
        const int lane = threadIdx.x % WAVE;
        const uint64_t ahead = __ballot(lane < count && value >= v);
        const int at = __popcll(ahead);
        const float pv = __shfl_up(value, 1);
        const int32_t pc = __shfl_up(column, 1);
        if (lane > at) {
            value = pv;
            column = pc;
        }
        if (lane == at) {
            value = v;
            column = c;
        }
        if (count < k) count++;
        if (lane >= count) column = -1;
        if (count == k) last = __shfl(value, k - 1);
    }
};

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 1; d < WAVE; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// Candidates of one step, N a lane, columns ascending over lane and element.
template <int N>
__device__ void top_step(Top &top, const float (&x)[N], uint32_t open, int32_t column0, int k)
{
    while (true) {
        float best = -INFINITY;
        int at = -1;
#pragma unroll
        for (int e = 0; e < N; e++) {
            const float v = x[e] == x[e] ? x[e] : -INFINITY;        // a NaN counts as the least
            if ((open >> e & 1) && (at < 0 || v > best)) {
                best = v;
                at = e;
            }
        }
        const bool any = at >= 0 && top.wants(best, k);
        if (!__ballot(any)) return;
        const float most = wave_max(any ? best : -INFINITY);
        const int lane = __ffsll(__ballot(any && best == most)) - 1;
        top.insert(most, __shfl(column0 + at, lane), k);
        if ((int)(threadIdx.x % WAVE) == lane) open &= ~(1u << at);
    }
}

template <int N>
__device__ __forceinline__ void stat_step(Stat &s, const float (&x)[N])
{
    float most = x[0];
#pragma unroll
    for (int e = 1; e < N; e++) most = fmaxf(most, x[e]);
    if (most > s.m) {
        const float d = fmaxf(s.m - most, -1e4f), f = __builtin_amdgcn_exp2f(d * LOG2E);
        s.w = (s.w + d * s.l) * f;
        s.l *= f;
        s.m = most;
    }
#pragma unroll
    for (int e = 0; e < N; e++) {
        const float d = x[e] - s.m;
        const float p = __builtin_amdgcn_exp2f(d * LOG2E);
        s.l += p;                                                  // carries a NaN
        s.w += p * fmaxf(d, -1e4f);                                // 0 for minus infinity
    }
}

// What a wavefront's segment or a whole row comes to: written for a join, or
// as the row's results.
__device__ void finish_row(const LogpArgs &a, int64_t row, Stat s, const Top &top, float token_logit, int64_t token)
{
    const int lane = threadIdx.x % WAVE;
    const bool nothing = s.l == 0;                                  // minus infinity throughout
    const float log_l = __builtin_amdgcn_logf(s.l) * LN2;
    const float lse = nothing ? -INFINITY : s.m + log_l;
    if (lane == 0) {
        a.lse[row] = lse;
        a.entropy[row] = nothing ? 0.0f : log_l - s.w / s.l;
        a.logp[row] = token < 0 ? 0.0f : token >= a.vocab ? NAN : nothing ? -INFINITY : token_logit - lse;
    }
    if (lane < a.top) {
        a.top_logp[row * a.top + lane] = nothing ? -INFINITY : top.value - lse;
        a.top_ids[row * a.top + lane] = top.column < 0 ? 0 : top.column;
    }
}

// a list entry of every lane with column >= 0, lists in ascending order of columns
__device__ void join_list(Top &top, float v, int32_t c, int k)
{
    bool open = c >= 0;
    while (true) {
        const bool any = open && top.wants(v, k);
        if (!__ballot(any)) return;
        const float most = wave_max(any ? v : -INFINITY);
        const int lane = __ffsll(__ballot(any && v == most)) - 1;
        top.insert(most, __shfl(c, lane), k);
        if ((int)(threadIdx.x % WAVE) == lane) open = false;
    }
}

// GROUP wavefronts read a row (one, or SEGS), each a contiguous segment.
template <typename T, int GROUP, bool TOP>
__global__ void __launch_bounds__(256) logprob_kernel(LogpArgs a)
{
    using R = typename T::raw;
    constexpr int N = T::vec;
    __shared__ float part[SEGS][3];
    __shared__ float2 lists[SEGS][32];
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const int64_t unit = GROUP == 1 ? (int64_t)blockIdx.x * SEGS + wave : blockIdx.x;
    const int64_t row = GROUP == 1 ? unit : unit / a.splits;
    if (GROUP == 1 && row >= a.rows) return;
    const int segs = GROUP == 1 ? 1 : a.splits * SEGS;
    const int seg = GROUP == 1 ? 0 : (int)(unit % a.splits) * SEGS + wave;
    const R *x = (const R *)a.x + row * a.stride;

    // head up to the first 16-byte boundary, whole vectors, tail
    const int64_t mis = (uintptr_t)x % 16 / sizeof(R);
    const int64_t head = min(mis ? N - mis : (int64_t)0, a.vocab);
    const int64_t vecs = (a.vocab - head) / N, tail0 = head + vecs * N;
    const int64_t per = (vecs + segs - 1) / segs, v0 = min(per * seg, vecs), v1 = min(v0 + per, vecs);

    Stat s = {LOWEST, 0, 0};
    Top top;
    top.clear();
    auto edge = [&](int64_t c0, int64_t n) {                        // fewer than N elements, one a lane
        float e[1] = {lane < n ? (float)x[c0 + lane] : -INFINITY};
        stat_step(s, e);
        if (TOP) top_step(top, e, lane < n ? 1u : 0u, (int32_t)c0 + lane, a.top);
    };
    if (seg == 0 && head) edge(0, head);
    for (int64_t v = v0; v < v1; v += WAVE) {
        float e[N];
        const bool in = v + lane < v1;
        Pack<R, N> p;
        if (in) p = *(const Pack<R, N> *)(x + head + (v + lane) * N);
#pragma unroll
        for (int i = 0; i < N; i++) e[i] = in ? (float)p.e[i] : -INFINITY;
        stat_step(s, e);
        if (TOP) top_step(top, e, in ? (1u << N) - 1 : 0u, (int32_t)(head + (v + lane) * N), a.top);
    }
    if (seg == segs - 1 && tail0 < a.vocab) edge(tail0, a.vocab - tail0);
    s = join_wave(s);

    const int64_t token = a.tokens[row];
    const float logit = token >= 0 && token < a.vocab ? (float)x[token] : 0.0f;
    if (GROUP == 1) {
        finish_row(a, row, s, top, logit, token);
        return;
    }
    if (a.splits > 1) {
        float *o = a.part + (row * segs + seg) * 4;
        if (lane == 0) {
            o[0] = s.m;
            o[1] = s.l;
            o[2] = s.w;
        }
        if (TOP && lane < a.top)
            a.part_top[(row * segs + seg) * a.top + lane] = make_float2(top.value, __int_as_float(top.column));
        return;
    }
    if (lane == 0) {
        part[wave][0] = s.m;
        part[wave][1] = s.l;
        part[wave][2] = s.w;
    }
    if (TOP && lane < a.top) lists[wave][lane] = make_float2(top.value, __int_as_float(top.column));
    __syncthreads();
    if (wave) return;
    s = {part[0][0], part[0][1], part[0][2]};
    for (int g = 1; g < SEGS; g++) s = join(s, {part[g][0], part[g][1], part[g][2]});
    if (TOP)
        for (int g = 1; g < SEGS; g++) {
            const float2 t = lane < a.top ? lists[g][lane] : make_float2(0, __int_as_float(-1));
            join_list(top, t.x, __float_as_int(t.y), a.top);
        }
    finish_row(a, row, s, top, logit, token);
}

// the segments of a row that several workgroups read: one wavefront a row
template <typename T, bool TOP>
__global__ void __launch_bounds__(64) logprob_join(LogpArgs a)
{
    using R = typename T::raw;
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const int segs = a.splits * SEGS;
    Stat s = {LOWEST, 0, 0};
    for (int g = lane; g < segs; g += WAVE) {
        const float *o = a.part + (row * segs + g) * 4;
        s = join(s, {o[0], o[1], o[2]});
    }
    s = join_wave(s);
    Top top;
    top.clear();
    if (TOP)
        for (int e0 = 0; e0 < segs * a.top; e0 += WAVE) {
            const int e = e0 + lane;
            const float2 t = e < segs * a.top ? a.part_top[row * segs * a.top + e] : make_float2(0, __int_as_float(-1));
            join_list(top, t.x, __float_as_int(t.y), a.top);
        }
    const int64_t token = a.tokens[row];
    const R *x = (const R *)a.x + row * a.stride;
    finish_row(a, row, s, top, token >= 0 && token < a.vocab ? (float)x[token] : 0.0f, token);
}

template <typename T, bool TOP> hipError_t logprobs_typed(const LogpArgs &a, hipStream_t st)
{
    // short rows: a wavefront each
    if (a.vocab <= (int64_t)4 * WAVE * T::vec) {
        logprob_kernel<T, 1, TOP><<<(unsigned)((a.rows + SEGS - 1) / SEGS), 256, 0, st>>>(a);
        return hipGetLastError();
    }
    logprob_kernel<T, SEGS, TOP><<<(unsigned)(a.rows * a.splits), 256, 0, st>>>(a);
    if (a.splits > 1) {
        if (hipError_t e = hipGetLastError()) return e;
        logprob_join<T, TOP><<<(unsigned)a.rows, WAVE, 0, st>>>(a);
    }
    return hipGetLastError();
}

// ---- gradient of the log probabilities ------------------------------------------
// dx_v = dlogp [v = token] + sum_k dtop_k [v = id_k] - p_v (G + dH (log p_v + H))
// One read and one write of the row; the few columns that get a term of their
// own are written once more, after the barrier, by the workgroup that owns them.

template <typename T>
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
            *(Pack<R, N> *)(dx + c0 + head + v * N) = o;
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
    const int64_t per = 8192;                                      // columns of a workgroup
    const unsigned gx = (unsigned)((a.vocab + per - 1) / per);
    const unsigned gy = (unsigned)std::min<int64_t>(a.rows, 32768), gz = (unsigned)((a.rows + gy - 1) / gy);
    logprob_grad<T><<<dim3(gx, gy, gz), 256, 0, st>>>(a, per);
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
