// Attention over packed sequences and its gradients: grouped heads, causal or not.
// See include/onebit.h for the contract of the entry points.
//
// Every product is a 32 x 32 x 16 matrix instruction whose second operand a lane holds
// whole: a query forwards and for dq, a key for dk and dv.  The scores come out with
// that query (key) in the lane's column and 16 of the 32 keys (queries) in its rows,
// which is how the next product takes them in, rounded to 16 bits, as its second
// operand: they never leave the registers.  Its first operand is the other side's tile,
// read from LDS by rows for the scores and transposed for what follows.  The summed
// index runs over a lane's 8 numbers in the order in which the scores have them: of
// 16, lanes of the lower half hold 0-3 and 8-11, those of the upper half 4-7 and 12-15.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "../../include/onebit.h"
#include "onebit_internal.h"
#include "onebit_rows.h"
#include "onebit_status.h"

namespace onebit {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
template <class T>
using vec8 = T __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kThreads = 256, kWaves = 4;
constexpr int kTile = 64;       // rows of the other side's tile in LDS
constexpr int kMostDim = 128;
constexpr int kMostParts = 1024;

__device__ __forceinline__ f32x16 mma(vec8<__bf16> a, vec8<__bf16> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(vec8<_Float16> a, vec8<_Float16> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// A lane's column in a 32 x 32 product, and the first of its rows; number i of its 16
// is row upper() * 4 + i % 4 + 8 * (i / 4).
__device__ __forceinline__ int column() { return threadIdx.x & 31; }
__device__ __forceinline__ int upper() { return threadIdx.x >> 5 & 1; }
__device__ __forceinline__ int wave_number()
{
    return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

struct Sides {
    int64_t q_ld, k_ld, v_ld, o_ld;  // elements from token to token
    const int32_t *starts;
    int tokens, sequences, heads, kv_heads, dim;
    float scale;
    int causal;
};

// The sequence of which tile `tile` of `rows` tokens is: sequence s has tiles from
// starts[s] / rows + s on, at least as many as it needs.  Each round every lane
// looks at one start.  Starts out of order or range give some range inside [0, tokens].
struct Range {
    int first, length, at;  // its first token, its length, the tile's first row in it
};

__device__ __forceinline__ Range find_sequence(const Sides &s, int tile, int rows)
{
    const int lane = threadIdx.x & 63;
    const auto start = [&](int k) { return min(max(s.starts[k], 0), s.tokens); };
    int lo = 0, n = s.sequences;  // it is one of lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 63) / 64, k = lo + lane * step;
        const bool below = lane * step < n && start(k) / rows + k <= tile;
        const int hits = __popcll(__ballot(below));
        const int skip = hits > 0 ? (hits - 1) * step : 0;
        lo += skip;
        n = min(step, n - skip);
    }
    Range r;
    r.first = __builtin_amdgcn_readfirstlane(start(lo));
    r.length = __builtin_amdgcn_readfirstlane(max(start(lo + 1) - r.first, 0));
    r.at = (tile - (r.first / rows + lo)) * rows;
    return r;
}

// 8 numbers of a row of `dim` from `at` on; zeros behind its end and without a row.
template <class T>
__device__ __forceinline__ vec8<T> load8(const T *row, int at, int dim, bool there)
{
    T t[8] = {};
    if (there) {
        if (at + 8 <= dim) {
            __builtin_memcpy(t, row + at, sizeof t);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (at + k < dim) t[k] = row[at + k];
        }
    }
    vec8<T> v;
    __builtin_memcpy(&v, t, sizeof v);
    return v;
}

// A tile of kTile rows of DP numbers in LDS, 16 bytes between rows so that 16 lanes
// with a row each reach all banks.
template <class T, int DP>
struct Tile {
    static constexpr int kPitch = DP * 2 + 16, kBytes = kTile * kPitch;
    static constexpr int kEach = kTile * (DP / 8) / kThreads;  // pieces of a thread
    vec8<T> held[kEach];
    // rows `at` and on of `rows`, into registers
    __device__ __forceinline__ void load(const T *base, int64_t ld, int at, int rows, int dim)
    {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int piece = threadIdx.x + k * kThreads, row = at + piece / (DP / 8);
            held[k] = load8(base + (int64_t)row * ld, piece % (DP / 8) * 8, dim, row < rows);
        }
    }
    __device__ __forceinline__ void store(char *lds) const
    {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int piece = threadIdx.x + k * kThreads;
            *(vec8<T> *)(lds + piece / (DP / 8) * kPitch + piece % (DP / 8) * 16) = held[k];
        }
    }
    // First operand, rows of the tile: 32 from `row` on, numbers 16 k and on.
    static __device__ __forceinline__ vec8<T> rows(const char *lds, int row, int k)
    {
        return *(const vec8<T> *)(lds + (row + column()) * kPitch + (k * 16 + upper() * 8) * 2);
    }
    // First operand, the tile's columns: 32 from 32 c on, over 16 rows from `row` on, in
    // the order of the scores (above).  A transposing read takes 4 rows x 16 columns
    // per 16 lanes.
    static __device__ __forceinline__ vec8<T> columns(const char *lds, int row, int c)
    {
        const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
        const char *at = lds + (row + 4 * (g >> 1) + (j >> 2)) * kPitch +
                         (c * 32 + (g & 1) * 16 + (j & 3) * 4) * 2;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)at);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4s *)(at + 8 * kPitch));
        return __builtin_bit_cast(vec8<T>, (v8s)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Numbers 8 half .. 8 half + 7 of a lane's scores as a second operand.
template <class T>
__device__ __forceinline__ vec8<T> narrow(const f32x16 &s, int half)
{
    vec8<T> v;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (T)s[half * 8 + k];
    return v;
}

// Both halves' values of a column.
template <class F>
__device__ __forceinline__ float both_halves(float v, F f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return f(__builtin_bit_cast(float, (uint32_t)w[0]), __builtin_bit_cast(float, (uint32_t)w[1]));
}

// Stores a lane's column of a [DP, 32] result: row `to` of a tensor, times `factor`.
template <class T, int DP>
__device__ __forceinline__ void store_column(T *to, const f32x16 (&acc)[DP / 32], float factor,
                                             int dim)
{
#pragma unroll
    for (int c = 0; c < DP / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int at = c * 32 + upper() * 4 + 8 * (i / 4);
            T t[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] = (T)(acc[c][i + k] * factor);
            if (at + 4 <= dim) {
                __builtin_memcpy(to + at, t, sizeof t);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (at + k < dim) to[at + k] = t[k];
            }
        }
}

// out = softmax(scale q k') v for QB * 32 queries of a wave, one pass over the keys
// with a running maximum m and sum l per query (both halves of a wave have a query; m
// is the same in both, l adds up at the end).
template <class T, int DP, int QB>
__global__ __launch_bounds__(kThreads) void k_attention(const T *__restrict__ q,
                                                        const T *__restrict__ k,
                                                        const T *__restrict__ v, Sides s,
                                                        T *__restrict__ out,
                                                        float *__restrict__ lse, int tiles)
{
    using Kv = Tile<T, DP>;
    constexpr int kRows = kWaves * 32 * QB;
    __shared__ __attribute__((aligned(16))) char lds[2][2][Kv::kBytes];
    const int head = blockIdx.x % s.heads, tile = tiles - 1 - blockIdx.x / s.heads;
    const Range in = find_sequence(s, tile, kRows);
    if (in.at < 0 || in.at >= in.length) return;
    const int wave = wave_number(), row0 = in.at + wave * 32 * QB;
    const int kv = head / (s.heads / s.kv_heads);
    const T *kp = k + in.first * s.k_ld + kv * s.dim, *vp = v + in.first * s.v_ld + kv * s.dim;
    vec8<T> qf[QB][DP / 16];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int row = row0 + b * 32 + column();
        const T *qp = q + (int64_t)(in.first + row) * s.q_ld + head * s.dim;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c)
            qf[b][c] = load8(qp, c * 16 + upper() * 8, s.dim, row < in.length);
    }
    const int keys = s.causal ? min(in.length, in.at + kRows) : in.length;
    const float c = s.scale * kLog2e;
    f32x16 o[QB][DP / 32] = {};
    float m[QB], l[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) m[b] = -INFINITY, l[b] = 0.f;
    Kv kt, vt;
    kt.load(kp, s.k_ld, 0, in.length, s.dim);
    vt.load(vp, s.v_ld, 0, in.length, s.dim);
    kt.store(lds[0][0]);
    vt.store(lds[0][1]);
    __syncthreads();
    for (int at = 0, turn = 0; at < keys; at += kTile, turn ^= 1) {
        const bool more = at + kTile < keys;
        if (more) {
            kt.load(kp, s.k_ld, at + kTile, in.length, s.dim);
            vt.load(vp, s.v_ld, at + kTile, in.length, s.dim);
        }
        // (with the mask, a tile that a wave does not skip leaves each of its rows a key)
        if (!(s.causal && at > row0 + 32 * QB - 1)) {
            f32x16 p[QB][2] = {};
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    const vec8<T> f = Kv::rows(lds[turn][0], h * 32, d);
#pragma unroll
                    for (int b = 0; b < QB; ++b) p[b][h] = mma(f, qf[b][d], p[b][h]);
                }
            if (at + kTile > in.length || (s.causal && at + kTile - 1 > row0)) {
#pragma unroll
                for (int b = 0; b < QB; ++b) {
                    const int row = row0 + b * 32 + column();
                    const int end = s.causal ? min(in.length, row + 1) : in.length;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (at + h * 32 + upper() * 4 + i % 4 + 8 * (i / 4) >= end)
                                p[b][h][i] = -INFINITY;
                }
            }
#pragma unroll
            for (int b = 0; b < QB; ++b) {
                const auto larger = [](float x, float y) { return fmaxf(x, y); };
                float most = p[b][0][0];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, p[b][h][i]);
                most = fmaxf(m[b], both_halves(most, larger));
                const float alpha = __builtin_amdgcn_exp2f((m[b] - most) * c), mc = most * c;
                m[b] = most;
                float sum = 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        p[b][h][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[b][h][i], c, -mc));
                        sum += p[b][h][i];
                    }
                l[b] = __builtin_fmaf(l[b], alpha, sum);
                if (__ballot(alpha != 1.f))
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[b][d][i] *= alpha;
            }
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                vec8<T> pf[QB];
#pragma unroll
                for (int b = 0; b < QB; ++b) pf[b] = narrow<T>(p[b][h / 2], h % 2);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    const vec8<T> f = Kv::columns(lds[turn][1], h * 16, d);
#pragma unroll
                    for (int b = 0; b < QB; ++b) o[b][d] = mma(f, pf[b], o[b][d]);
                }
            }
        }
        if (more) {
            kt.store(lds[turn ^ 1][0]);
            vt.store(lds[turn ^ 1][1]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int row = row0 + b * 32 + column();
        const float sum = both_halves(l[b], [](float x, float y) { return x + y; });
        if (row >= in.length) continue;
        const int64_t token = in.first + row;
        store_column<T, DP>(out + token * s.o_ld + head * s.dim, o[b], 1.f / sum, s.dim);
        if (lse && upper() == 0) lse[token * s.heads + head] = m[b] * s.scale + logf(sum);
    }
}

// ---------------------------------------------------------------------------
// Backwards, with P = exp(scale q k' - lse) formed again:
//   dv = P' dout,  dP = dout v',  dS = P (dP - D),  D = the row sums of dout out,
//   dq = scale dS k,  dk = scale dS' q.
// One kernel for D, one for dk and dv, whose workgroups own keys and go through the
// queries of all heads that share them, and one for dq, whose workgroups own queries:
// seven products instead of five, and no atomics.
// ---------------------------------------------------------------------------

// D of each token and head, by 8 lanes; with fp16 also the largest finite magnitude in
// the workgroup's dout, by which dS is scaled before it is rounded (fp16 has no room for
// gradients of 1e-6 and less).  Tokens outside the sequences are not looked at.
template <class T>
__global__ __launch_bounds__(kThreads) void k_attention_delta(const T *__restrict__ dout,
                                                              int64_t d_ld,
                                                              const T *__restrict__ out, Sides s,
                                                              float *__restrict__ delta,
                                                              float *__restrict__ parts)
{
    const auto start = [&](int k) { return (int64_t)min(max(s.starts[k], 0), s.tokens); };
    const int64_t begin = start(0) * s.heads, rows = start(s.sequences) * s.heads;
    const int lane = threadIdx.x & 7;
    float most = 0.f;
    for (int64_t r = begin + (int64_t)blockIdx.x * (kThreads / 8) + threadIdx.x / 8; r < rows;
         r += (int64_t)gridDim.x * (kThreads / 8)) {
        const int64_t token = r / s.heads;
        const int head = (int)(r - token * s.heads);
        const T *a = dout + token * d_ld + head * s.dim, *b = out + token * s.o_ld + head * s.dim;
        float sum = 0.f;
        for (int at = lane * 8; at < s.dim; at += 64) {
            const vec8<T> x = load8(a, at, s.dim, true), y = load8(b, at, s.dim, true);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                sum = __builtin_fmaf((float)x[k], (float)y[k], sum);
                if constexpr (std::is_same_v<T, _Float16>)
                    if (fabsf((float)x[k]) < INFINITY) most = fmaxf(most, fabsf((float)x[k]));
            }
        }
        sum = over_lanes<8>(sum, [](float x, float y) { return x + y; });
        if (lane == 0) delta[r] = sum;
    }
    if constexpr (std::is_same_v<T, _Float16>) {
        __shared__ float s_most[kWaves];
        most = over_lanes<64>(most, [](float x, float y) { return fmaxf(x, y); });
        if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
        __syncthreads();
        if (threadIdx.x == 0)
            parts[blockIdx.x] = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3]));
    }
}

// The power of two that brings the largest magnitude in dout (2^-24 to 2^16) to 2^-5 ..
// 2^-4, for fp16: dS then stays in range for values of v up to some thousands, and its
// step is 2^-20 of that.
template <class T>
__device__ __forceinline__ float gradient_scale(const float *__restrict__ parts, int n)
{
    if constexpr (!std::is_same_v<T, _Float16>) return 1.f;
    float most = 0.f;
    for (int k = threadIdx.x & 63; k < n; k += 64) most = fmaxf(most, parts[k]);
    most = over_lanes<64>(most, [](float x, float y) { return fmaxf(x, y); });
    const int e = (int)(__builtin_bit_cast(uint32_t, most) >> 23);
    return most > 0.f ? __builtin_bit_cast(float, (uint32_t)(249 - e) << 23) : 1.f;
}

// The sides of a backward call.
struct Grads {
    int64_t d_ld, dq_ld, dk_ld, dv_ld;
    int parts;
};

template <class T, int DP, int QB>
__global__ __launch_bounds__(kThreads) void k_attention_dq(
    const T *__restrict__ dout, const T *__restrict__ q, const T *__restrict__ k,
    const T *__restrict__ v, Sides s, Grads g, const float *__restrict__ lse,
    const float *__restrict__ delta, const float *__restrict__ parts, T *__restrict__ dq,
    int tiles)
{
    using Kv = Tile<T, DP>;
    constexpr int kRows = kWaves * 32 * QB;
    __shared__ __attribute__((aligned(16))) char lds[2][2][Kv::kBytes];
    const int head = blockIdx.x % s.heads, tile = tiles - 1 - blockIdx.x / s.heads;
    const Range in = find_sequence(s, tile, kRows);
    if (in.at < 0 || in.at >= in.length) return;
    const int wave = wave_number(), row0 = in.at + wave * 32 * QB;
    const int kv = head / (s.heads / s.kv_heads);
    const T *kp = k + in.first * s.k_ld + kv * s.dim, *vp = v + in.first * s.v_ld + kv * s.dim;
    const float grow = gradient_scale<T>(parts, g.parts);
    vec8<T> qf[QB][DP / 16], df[QB][DP / 16];
    float l2[QB], dl[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int row = row0 + b * 32 + column();
        const int64_t token = in.first + row;
        const bool there = row < in.length;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            qf[b][c] = load8(q + token * s.q_ld + head * s.dim, c * 16 + upper() * 8, s.dim, there);
            df[b][c] = load8(dout + token * g.d_ld + head * s.dim, c * 16 + upper() * 8, s.dim, there);
        }
        l2[b] = there ? lse[token * s.heads + head] * kLog2e : 0.f;
        dl[b] = there ? delta[token * s.heads + head] : 0.f;
    }
    const int keys = s.causal ? min(in.length, in.at + kRows) : in.length;
    const float c = s.scale * kLog2e;
    f32x16 acc[QB][DP / 32] = {};
    Kv kt, vt;
    kt.load(kp, s.k_ld, 0, in.length, s.dim);
    vt.load(vp, s.v_ld, 0, in.length, s.dim);
    kt.store(lds[0][0]);
    vt.store(lds[0][1]);
    __syncthreads();
    for (int at = 0, turn = 0; at < keys; at += kTile, turn ^= 1) {
        const bool more = at + kTile < keys;
        if (more) {
            kt.load(kp, s.k_ld, at + kTile, in.length, s.dim);
            vt.load(vp, s.v_ld, at + kTile, in.length, s.dim);
        }
        if (!(s.causal && at > row0 + 32 * QB - 1)) {
            const bool mask = at + kTile > in.length || (s.causal && at + kTile - 1 > row0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x16 p[QB] = {}, dp[QB] = {};
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    const vec8<T> f = Kv::rows(lds[turn][0], h * 32, d);
                    const vec8<T> w = Kv::rows(lds[turn][1], h * 32, d);
#pragma unroll
                    for (int b = 0; b < QB; ++b) {
                        p[b] = mma(f, qf[b][d], p[b]);
                        dp[b] = mma(w, df[b][d], dp[b]);
                    }
                }
#pragma unroll
                for (int b = 0; b < QB; ++b) {
                    const int row = row0 + b * 32 + column();
                    const int end = s.causal ? min(in.length, row + 1) : in.length;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(p[b][i], c, -l2[b]));
                        p[b][i] = e * ((dp[b][i] - dl[b]) * grow);
                        if (mask && at + h * 32 + upper() * 4 + i % 4 + 8 * (i / 4) >= end)
                            p[b][i] = 0.f;
                    }
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    vec8<T> pf[QB];
#pragma unroll
                    for (int b = 0; b < QB; ++b) pf[b] = narrow<T>(p[b], half);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) {
                        const vec8<T> f = Kv::columns(lds[turn][0], h * 32 + half * 16, d);
#pragma unroll
                        for (int b = 0; b < QB; ++b) acc[b][d] = mma(f, pf[b], acc[b][d]);
                    }
                }
            }
        }
        if (more) {
            kt.store(lds[turn ^ 1][0]);
            vt.store(lds[turn ^ 1][1]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int row = row0 + b * 32 + column();
        if (row < in.length)
            store_column<T, DP>(dq + (int64_t)(in.first + row) * g.dq_ld + head * s.dim, acc[b],
                                s.scale / grow, s.dim);
    }
}

template <class T, int DP, int KB>
__global__ __launch_bounds__(kThreads) void k_attention_dkv(
    const T *__restrict__ dout, const T *__restrict__ q, const T *__restrict__ k,
    const T *__restrict__ v, Sides s, Grads g, const float *__restrict__ lse,
    const float *__restrict__ delta, const float *__restrict__ parts, T *__restrict__ dk,
    T *__restrict__ dv, int tiles)
{
    using Q = Tile<T, DP>;
    constexpr int kRows = kWaves * 32 * KB;
    __shared__ __attribute__((aligned(16))) char lds[2][2][Q::kBytes];
    __shared__ float s_row[2][2][kTile];  // lse in base 2 and D of the tile's queries
    const int kv = blockIdx.x % s.kv_heads, tile = blockIdx.x / s.kv_heads;
    const Range in = find_sequence(s, tile, kRows);
    if (in.at < 0 || in.at >= in.length) return;
    const int wave = wave_number(), row0 = in.at + wave * 32 * KB;
    const int group = s.heads / s.kv_heads;
    const float grow = gradient_scale<T>(parts, g.parts);
    vec8<T> kf[KB][DP / 16], vf[KB][DP / 16];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        const int row = row0 + b * 32 + column();
        const int64_t token = in.first + row;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            kf[b][c] = load8(k + token * s.k_ld + kv * s.dim, c * 16 + upper() * 8, s.dim, row < in.length);
            vf[b][c] = load8(v + token * s.v_ld + kv * s.dim, c * 16 + upper() * 8, s.dim, row < in.length);
        }
    }
    const float c = s.scale * kLog2e;
    f32x16 dka[KB][DP / 32] = {}, dva[KB][DP / 32] = {};
    Q qt, dt;
    float row_value = 0.f;
    // the queries that see the tile's keys, a head of the group after the other
    const int from = s.causal ? in.at / kTile * kTile : 0;
    const int per_head = (in.length - from + kTile - 1) / kTile, steps = per_head * group;
    auto load = [&](int step) {
        const int head = kv * group + step / per_head, at = from + step % per_head * kTile;
        qt.load(q + in.first * s.q_ld + head * s.dim, s.q_ld, at, in.length, s.dim);
        dt.load(dout + in.first * g.d_ld + head * s.dim, g.d_ld, at, in.length, s.dim);
        if (threadIdx.x < 2 * kTile) {
            const int row = at + threadIdx.x % kTile;
            const int64_t to = (int64_t)(in.first + row) * s.heads + head;
            // (behind the end: a score of 0 less infinity has no weight)
            row_value = threadIdx.x < kTile ? (row < in.length ? lse[to] * kLog2e : INFINITY)
                                            : (row < in.length ? delta[to] : 0.f);
        }
    };
    auto store = [&](int turn) {
        qt.store(lds[turn][0]);
        dt.store(lds[turn][1]);
        if (threadIdx.x < 2 * kTile) s_row[turn][threadIdx.x / kTile][threadIdx.x % kTile] = row_value;
    };
    load(0);
    store(0);
    __syncthreads();
    for (int step = 0, turn = 0; step < steps; ++step, turn ^= 1) {
        if (step + 1 < steps) load(step + 1);
        const int at = from + step % per_head * kTile;
        if (!(s.causal && at + kTile - 1 < row0)) {
            const bool mask = s.causal && at < row0 + 32 * KB - 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x16 p[KB] = {}, dp[KB] = {};
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    const vec8<T> f = Q::rows(lds[turn][0], h * 32, d);
                    const vec8<T> w = Q::rows(lds[turn][1], h * 32, d);
#pragma unroll
                    for (int b = 0; b < KB; ++b) {
                        p[b] = mma(f, kf[b][d], p[b]);
                        dp[b] = mma(w, vf[b][d], dp[b]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = h * 32 + upper() * 4 + i % 4 + 8 * (i / 4);
                    const float l2 = s_row[turn][0][r], dl = s_row[turn][1][r];
#pragma unroll
                    for (int b = 0; b < KB; ++b) {
                        float e = __builtin_amdgcn_exp2f(__builtin_fmaf(p[b][i], c, -l2));
                        float ds = e * ((dp[b][i] - dl) * grow);
                        if (mask && at + r < row0 + b * 32 + column()) e = 0.f, ds = 0.f;
                        p[b][i] = e;
                        dp[b][i] = ds;
                    }
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    vec8<T> pf[KB], sf[KB];
#pragma unroll
                    for (int b = 0; b < KB; ++b) pf[b] = narrow<T>(p[b], half), sf[b] = narrow<T>(dp[b], half);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) {
                        const vec8<T> f = Q::columns(lds[turn][1], h * 32 + half * 16, d);
                        const vec8<T> w = Q::columns(lds[turn][0], h * 32 + half * 16, d);
#pragma unroll
                        for (int b = 0; b < KB; ++b) {
                            dva[b][d] = mma(f, pf[b], dva[b][d]);
                            dka[b][d] = mma(w, sf[b], dka[b][d]);
                        }
                    }
                }
            }
        }
        if (step + 1 < steps) store(turn ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        const int row = row0 + b * 32 + column();
        if (row >= in.length) continue;
        const int64_t token = in.first + row;
        store_column<T, DP>(dk + token * g.dk_ld + kv * s.dim, dka[b], s.scale / grow, s.dim);
        store_column<T, DP>(dv + token * g.dv_ld + kv * s.dim, dva[b], 1.f, s.dim);
    }
}

template <class F>
void with_half(int32_t dtype, F &&f)
{
    if (dtype == ONEBIT_GRAD_BF16) f((__bf16 *)nullptr);
    else f((_Float16 *)nullptr);
}

template <class F>
void with_dim(int dim, F &&f)
{
    using std::integral_constant;
    if (dim <= 32) f(integral_constant<int, 32>{});
    else if (dim <= 64) f(integral_constant<int, 64>{});
    else if (dim <= 96) f(integral_constant<int, 96>{});
    else f(integral_constant<int, 128>{});
}

int check_side(const void *p, int64_t ld, int64_t tokens, int64_t width, const char *name)
{
    return check_rows(p, ONEBIT_GRAD_BF16, ld, tokens, width, name);
}

int check_attention(int32_t dtype, int64_t tokens, int32_t heads, int32_t kv_heads, int32_t dim,
                    const int32_t *starts, int64_t sequences, float scale)
{
    if (dtype != ONEBIT_GRAD_BF16 && dtype != ONEBIT_GRAD_F16)
        return fail(ONEBIT_EINVAL, "type %d is neither ONEBIT_GRAD_BF16 nor ONEBIT_GRAD_F16", dtype);
    if (tokens < 0 || tokens > (1 << 30))
        return fail(ONEBIT_EINVAL, "tokens = %lld is not in [0, 2^30]", (long long)tokens);
    if (heads < 1 || heads > (1 << 14) || kv_heads < 1 || heads % kv_heads)
        return fail(ONEBIT_EINVAL, "%d heads on %d key heads", heads, kv_heads);
    if (dim < 1 || dim > kMostDim)
        return fail(ONEBIT_EINVAL, "dim = %d is not in [1, %d]", dim, kMostDim);
    if (sequences < 0 || sequences > (1 << 30))
        return fail(ONEBIT_EINVAL, "sequences = %lld is not in [0, 2^30]", (long long)sequences);
    if (!starts && sequences > 0) return fail(ONEBIT_EINVAL, "starts is NULL");
    if ((uintptr_t)starts % 4) return fail(ONEBIT_EALIGN, "starts is not 4-byte aligned");
    if (!(scale > 0.f) || scale > 1e30f)
        return fail(ONEBIT_EINVAL, "scale = %g is not in (0, 1e30]", (double)scale);
    return ONEBIT_OK;
}

// Tiles of `rows` tokens that cover every sequence (find_sequence), and whether a
// launch of one workgroup for each and each head is possible.
int tile_count(int64_t tokens, int64_t sequences, int heads, int rows, int *tiles)
{
    const int64_t n = tokens / rows + sequences;
    if (n * heads >= ((int64_t)1 << 32) / kThreads)
        return fail(ONEBIT_EINVAL, "%lld tokens in %lld sequences with %d heads are too many for one call",
                    (long long)tokens, (long long)sequences, heads);
    *tiles = (int)n;
    return ONEBIT_OK;
}

int delta_blocks(int64_t tokens, int heads)
{
    return (int)std::min<int64_t>((tokens * heads + kThreads / 8 - 1) / (kThreads / 8), kMostParts);
}

}  // namespace
}  // namespace onebit

using namespace onebit;

extern "C" {

int onebit_attention_forward(const void *q, int64_t q_ld, const void *k, int64_t k_ld,
                             const void *v, int64_t v_ld, int32_t dtype, int64_t tokens,
                             int32_t heads, int32_t kv_heads, int32_t dim, const int32_t *starts,
                             int64_t sequences, int32_t causal, float scale, void *out,
                             int64_t out_ld, float *lse, onebit_stream stream)
{
    TRY(check_attention(dtype, tokens, heads, kv_heads, dim, starts, sequences, scale));
    const int64_t width = (int64_t)heads * dim, kv_width = (int64_t)kv_heads * dim;
    TRY(check_side(q, q_ld, tokens, width, "q"));
    TRY(check_side(k, k_ld, tokens, kv_width, "k"));
    TRY(check_side(v, v_ld, tokens, kv_width, "v"));
    TRY(check_side(out, out_ld, tokens, width, "out"));
    if ((uintptr_t)lse % 4) return fail(ONEBIT_EALIGN, "lse is not 4-byte aligned");
    constexpr int kBlocks = 1, kRows = kWaves * 32 * kBlocks;
    int tiles;
    TRY(tile_count(tokens, sequences, heads, kRows, &tiles));
    if (tokens == 0 || sequences == 0) return ONEBIT_OK;
    const Sides s{q_ld, k_ld, v_ld, out_ld, starts, (int)tokens, (int)sequences,
                  heads, kv_heads, dim, scale, causal};
    with_half(dtype, [&](auto *t) {
        with_dim(dim, [&](auto padded) {
            using T = std::remove_pointer_t<decltype(t)>;
            k_attention<T, decltype(padded)::value, kBlocks>
                <<<tiles * heads, kThreads, 0, (hipStream_t)stream>>>(
                    (const T *)q, (const T *)k, (const T *)v, s, (T *)out, lse, tiles);
        });
    });
    return launched("attention launch");
}

int onebit_attention_grad_workspace(int64_t tokens, int32_t heads, size_t *bytes)
{
    if (!bytes) return fail(ONEBIT_EINVAL, "bytes is NULL");
    if (tokens < 0 || tokens > (1 << 30) || heads < 1 || heads > (1 << 14))
        return fail(ONEBIT_EINVAL, "%lld tokens, %d heads", (long long)tokens, heads);
    *bytes = ((size_t)kMostParts + (size_t)tokens * heads) * sizeof(float);
    return ONEBIT_OK;
}

int onebit_attention_grad(const void *dout, int64_t dout_ld, const void *q, int64_t q_ld,
                          const void *k, int64_t k_ld, const void *v, int64_t v_ld,
                          const void *out, int64_t out_ld, const float *lse, int32_t dtype,
                          int64_t tokens, int32_t heads, int32_t kv_heads, int32_t dim,
                          const int32_t *starts, int64_t sequences, int32_t causal, float scale,
                          void *dq, int64_t dq_ld, void *dk, int64_t dk_ld, void *dv,
                          int64_t dv_ld, void *workspace, onebit_stream stream)
{
    TRY(check_attention(dtype, tokens, heads, kv_heads, dim, starts, sequences, scale));
    const int64_t width = (int64_t)heads * dim, kv_width = (int64_t)kv_heads * dim;
    TRY(check_side(dout, dout_ld, tokens, width, "dout"));
    TRY(check_side(q, q_ld, tokens, width, "q"));
    TRY(check_side(k, k_ld, tokens, kv_width, "k"));
    TRY(check_side(v, v_ld, tokens, kv_width, "v"));
    TRY(check_side(out, out_ld, tokens, width, "out"));
    TRY(check_side(dq, dq_ld, tokens, width, "dq"));
    TRY(check_side(dk, dk_ld, tokens, kv_width, "dk"));
    TRY(check_side(dv, dv_ld, tokens, kv_width, "dv"));
    if (!lse && tokens > 0) return fail(ONEBIT_EINVAL, "lse is NULL");
    if ((uintptr_t)lse % 4) return fail(ONEBIT_EALIGN, "lse is not 4-byte aligned");
    if (!workspace) return fail(ONEBIT_EINVAL, "workspace is NULL");
    if ((uintptr_t)workspace % 16) return fail(ONEBIT_EALIGN, "workspace is not 16-byte aligned");
    constexpr int kBlocks = 1, kRows = kWaves * 32 * kBlocks;
    int tiles;
    TRY(tile_count(tokens, sequences, heads, kRows, &tiles));
    if (tokens == 0 || sequences == 0) return ONEBIT_OK;
    const Sides s{q_ld, k_ld, v_ld, out_ld, starts, (int)tokens, (int)sequences,
                  heads, kv_heads, dim, scale, causal};
    const Grads g{dout_ld, dq_ld, dk_ld, dv_ld, delta_blocks(tokens, heads)};
    float *parts = (float *)workspace, *delta = parts + kMostParts;
    hipStream_t st = (hipStream_t)stream;
    with_half(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        k_attention_delta<T><<<g.parts, kThreads, 0, st>>>((const T *)dout, dout_ld,
                                                           (const T *)out, s, delta, parts);
        with_dim(dim, [&](auto padded) {
            constexpr int DP = decltype(padded)::value;
            k_attention_dkv<T, DP, kBlocks><<<tiles * kv_heads, kThreads, 0, st>>>(
                (const T *)dout, (const T *)q, (const T *)k, (const T *)v, s, g, lse, delta, parts,
                (T *)dk, (T *)dv, tiles);
            k_attention_dq<T, DP, kBlocks><<<tiles * heads, kThreads, 0, st>>>(
                (const T *)dout, (const T *)q, (const T *)k, (const T *)v, s, g, lse, delta, parts,
                (T *)dq, tiles);
        });
    });
    return launched("attention gradient launch");
}

}  // extern "C"
