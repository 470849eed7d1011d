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
#include <cfloat>
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
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kThreads = 256, kWaves = 4;
constexpr int kTile = 64;       // rows of the other side's tile in LDS
constexpr int kMostDim = 128;
constexpr int kMostDeltaBlocks = 1024;

// fp16 ends at 2^-24, where a weight of one of many keys, or of one far behind another,
// soon is.  Weights are brought up by powers of two before they are rounded to it:
// forwards so that a query's largest is 2^kWeightUp or more, and below 2^(kWeightUp + 8);
// backwards P itself, which is at most 1.
template <class T>
constexpr int kWeightUp = std::is_same_v<T, _Float16> ? 7 : 0;
template <class T>
constexpr int kPUp = std::is_same_v<T, _Float16> ? 15 : 0;

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
// WHOLE: dim is a multiple of 8.
template <bool WHOLE, class T>
__device__ __forceinline__ vec8<T> load8(const T *row, int at, int dim, bool there)
{
    T t[8] = {};
    if (WHOLE) {
        if (there && at < dim) __builtin_memcpy(t, row + at, sizeof t);
    } else if (there) {
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

typedef __attribute__((address_space(3))) void lds_void;

// 16 bytes per lane, from `at` bytes behind `base` (the same in all lanes) to consecutive
// places from `lds` on; zeros from `bytes` on.  (The host compiler, which only needs the
// kernels' names, does not take the builtin at this size.)
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t bytes, char *lds, int at)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const uint64_t a = (uint64_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(((uint64_t)hi << 32) | lo), (short)0, __builtin_amdgcn_readfirstlane(bytes),
        0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)lds, 16, at, 0, 0, 0);
#endif
}

// A tile of kTile rows of DP numbers in LDS, in pieces of 16 bytes.  A row's pieces are
// permuted so that neither 16 rows' same piece nor 4 rows' 64 bytes share a bank:
// piece p of row r is at place p ^ turned(r).
template <int DP>
__device__ __forceinline__ int turned(int r)
{
    if constexpr (DP == 128) return (r & 3) << 2 | (r >> 2 & 3);
    if constexpr (DP == 64) return (r >> 1 & 1) << 2 | (r >> 2 & 3);
    return r >> 2 & 3;  // rows of 64 or 192 bytes lie in different banks by fours
}

template <class T, int DP>
struct Tile {
    static constexpr int kPitch = DP * 2, kBytes = kTile * kPitch, kPieces = DP / 8;
    // A lane's places in a fragment: rows() of 32 rows, columns() of 16.
    int row_at, low_at, high_at;
    __device__ __forceinline__ Tile()
    {
        const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
        row_at = column() * kPitch + (upper() ^ turned<DP>(column())) * 16;
        const int r = 4 * (g >> 1) + (j >> 2), p = (g & 1) * 2 + (j >> 1 & 1), in = (j & 1) * 8;
        low_at = r * kPitch + (p ^ turned<DP>(r)) * 16 + in;
        high_at = (r + 8) * kPitch + (p ^ turned<DP>(r + 8)) * 16 + in;
    }
    // ... `pieces` further on in the row (the places of rows of 192 bytes are permuted
    // by fours of pieces alone)
    static __device__ __forceinline__ int further(int at, int pieces)
    {
        if constexpr (DP == 96) return (at ^ (pieces & 3) * 16) + (pieces >> 2) * 64;
        return at ^ pieces * 16;
    }
    // First operand, rows of the tile: 32 from `row` on, numbers 16 k and on.
    __device__ __forceinline__ vec8<T> rows(const char *lds, int row, int k) const
    {
        return *(const vec8<T> *)(lds + row * kPitch + further(row_at, 2 * k));
    }
    // First operand, the tile's columns: 32 from 32 c on, over 16 rows from `row` on, in
    // the order of the scores (above).  A transposing read takes 4 rows x 16 columns
    // per 16 lanes.
    __device__ __forceinline__ vec8<T> columns(const char *lds, int row, int c) const
    {
        const char *at = lds + row * kPitch;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4s *)(at + further(low_at, 4 * c)));
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4s *)(at + further(high_at, 4 * c)));
        return __builtin_bit_cast(vec8<T>, (v8s)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Brings tiles of a side's rows to LDS, by WAVES waves of which this is the `wave`-th.
// DIRECT: rows of whole pieces on 4-byte borders, straight from memory to LDS, every wave
// 1 KB at a time; what is not there is read as zero by the buffer's bound.  Otherwise
// through registers, number by number at a row's end.  start() begins a tile's loads,
// finish() ends them (a barrier has to follow).
template <class T, int DP, int ROWS, int WAVES, bool DIRECT>
struct Loader {
    static constexpr int kEach = ROWS * (DP / 8) / (WAVES * 64);  // pieces of a thread
    int wave, at[DIRECT ? kEach : 1];
    vec8<T> held[DIRECT ? 1 : kEach];
    __device__ __forceinline__ int piece(int k) const
    {
        return (k * WAVES + wave) * 64 + (threadIdx.x & 63);
    }
    __device__ __forceinline__ Loader(int w, int64_t ld, int dim) : wave(w)
    {
        if constexpr (DIRECT) {
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const int row = piece(k) / (DP / 8);
                const int from = (piece(k) % (DP / 8) ^ turned<DP>(row)) * 8;
                at[k] = from < dim ? (row * (int)ld + from) * 2 : (int)0x80000000;
            }
        }
    }
    // rows `first` and on of the `rows` at base
    __device__ __forceinline__ void start(const T *base, int64_t ld, int dim, int first, int rows,
                                          char *lds)
    {
        if constexpr (DIRECT) {
            const int64_t bytes = ((rows - 1 - first) * ld + dim) * 2;
            const uint32_t bound = (uint32_t)(bytes < 0x7fffffff ? bytes : 0x7fffffff);
#pragma unroll
            for (int k = 0; k < kEach; ++k)
                load_to_lds(base + first * ld, bound, lds + (k * WAVES + wave) * 1024, at[k]);
        } else {
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const int row = first + piece(k) / (DP / 8);
                held[k] = load8<false>(base + (int64_t)row * ld, piece(k) % (DP / 8) * 8, dim, row < rows);
            }
        }
    }
    __device__ __forceinline__ void finish(char *lds) const
    {
        if constexpr (DIRECT) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const int row = piece(k) / (DP / 8);
                *(vec8<T> *)(lds + row * DP * 2 + (piece(k) % (DP / 8) ^ turned<DP>(row)) * 16) = held[k];
            }
        }
    }
};

// Numbers 8 half .. 8 half + 7 of a lane's scores as a second operand.
template <class T>
__device__ __forceinline__ vec8<T> narrow(const f32x16 &s, int half)
{
    typedef float pair __attribute__((ext_vector_type(2)));
    typedef T narrow_pair __attribute__((ext_vector_type(2)));
    narrow_pair v[4];  // (two at a time, an instruction each)
#pragma unroll
    for (int k = 0; k < 4; ++k)
        v[k] = __builtin_convertvector((pair{s[half * 8 + 2 * k], s[half * 8 + 2 * k + 1]}), narrow_pair);
    return __builtin_bit_cast(vec8<T>, v);
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
// WHOLE: dim is a multiple of 8.
template <bool WHOLE, class T, int DP>
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
            if (WHOLE ? at < dim : at + 4 <= dim) {
                __builtin_memcpy(to + at, t, sizeof t);
            } else if (!WHOLE) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (at + k < dim) to[at + k] = t[k];
            }
        }
}

// How a workgroup's four waves share its work: WR of them have 32 rows each (queries, or
// keys for dk and dv), and WS streams of waves take every WS-th tile of the other side,
// whose sums are joined at the end.  Each stream has STAGE rows of both of the other
// sides in LDS, NB deep.
template <int DP, int WR, int NB, int STAGE>
struct Share {
    static constexpr int kStreams = kWaves / WR, kRows = 32 * WR;
    static constexpr int kStage = STAGE;
    static constexpr int kTileBytes = kStage * DP * 2, kRowsAt = kStreams * 2 * kTileBytes;
    static constexpr int kLds = kRowsAt + kStreams * 2 * kStage * 4;  // two numbers of each row
    static_assert(kStreams * WR == kWaves, "four waves");
    static constexpr int kSums = (kWaves - WR) * 64 * (DP / 2 + 2) * 4;  // where streams are joined
    static constexpr int kFirst = kLds > kSums ? kLds : kSums;
};

// Brings what the streams' waves have of the same rows to the first stream's wave: take(i)
// gets the number of a lane of each other stream's wave where give has put it.  COUNT
// numbers per lane, in LDS (which no wave reads for anything else any more).
template <int WR, int COUNT, class Give, class Take>
__device__ __forceinline__ void join_streams(char *lds, int stream, int row_wave, Give give, Take take)
{
    constexpr int kStreams = kWaves / WR;
    float *at = (float *)lds + (threadIdx.x & 63);
    if (stream > 0) {
#pragma unroll
        for (int k = 0; k < COUNT; ++k) at[(((stream - 1) * WR + row_wave) * COUNT + k) * 64] = give(k);
    }
    __syncthreads();
    if (stream == 0)
        for (int other = 1; other < kStreams; ++other) {
            const float *from = at + ((other - 1) * WR + row_wave) * COUNT * 64;
            take([&](int k) { return from[k * 64]; });
        }
}

// out = softmax(scale q k') v for 32 queries of a wave, one pass over the keys with a
// running maximum m and sum l per query (both halves of a wave have a query; m is the
// same in both, l adds up at the end).  The matrix cores and the VALU bound it, busy 54% and
// 43% of the time and hardly ever together, although a SIMD can run products of one wave
// beside another wave's exponentials: packed prompts of up to 8,192 tokens, 16 heads on 4 of
// 128, 385 to 405 us (0.95 PFLOP/s), 64 sequences of 512 with 16 heads of 64, not causal,
// 106 us (0.65).
// Four waves with 32 rows each, four workgroups a CU with heads of 64: with 64 rows a wave
// and half the LDS reads 192 us, with tiles of 128 keys and two workgroups 129.
template <class T, int DP, int WR, int NB, bool DIRECT>
__global__ __launch_bounds__(kThreads, (WR == 1 && DP > 64 ? 1 : 2)) void k_attention(const T *__restrict__ q,
                                                           const T *__restrict__ k,
                                                           const T *__restrict__ v, Sides s,
                                                           T *__restrict__ out,
                                                           float *__restrict__ lse, int tiles)
{
    using W = Share<DP, WR, NB, kTile>;
    const Tile<T, DP> tile_at;
    // (two arrays, so that a tile's loads are not waited for before the other is read)
    __shared__ __attribute__((aligned(1024))) char lds[W::kFirst], lds2[NB > 1 ? W::kLds : 1024];
    const int head = blockIdx.x % s.heads, tile = tiles - 1 - blockIdx.x / s.heads;
    const Range in = find_sequence(s, tile, W::kRows);
    if (in.at < 0 || in.at >= in.length) return;
    const int wave = wave_number(), stream = wave / WR, row0 = in.at + wave % WR * 32;
    const int kv = head / (s.heads / s.kv_heads);
    const T *kp = k + in.first * s.k_ld + kv * s.dim, *vp = v + in.first * s.v_ld + kv * s.dim;
    const int keys = s.causal ? min(in.length, in.at + W::kRows) : in.length;
    const int own = stream * 2 * W::kTileBytes, other = own + W::kTileBytes;
    Loader<T, DP, W::kStage, WR, DIRECT> kt(wave % WR, s.k_ld, s.dim), vt(wave % WR, s.v_ld, s.dim);
    const auto start = [&](int at, char *to) {
        if (at >= keys) return;
        kt.start(kp, s.k_ld, s.dim, at, in.length, to + own);
        vt.start(vp, s.v_ld, s.dim, at, in.length, to + other);
    };
    const auto finish = [&](int at, char *to) {
        if (at >= keys) return;
        kt.finish(to + own);
        vt.finish(to + other);
    };
    start(stream * kTile, lds);
    const int row = row0 + column();
    const int64_t token = in.first + row;
    vec8<T> qf[DP / 16];
#pragma unroll
    for (int d = 0; d < DP / 16; ++d)
        qf[d] = load8<DIRECT>(q + token * s.q_ld + head * s.dim, d * 16 + upper() * 8, s.dim, row < in.length);
    const float c = s.scale * kLog2e;
    f32x16 o[DP / 32] = {};
    // (the maximum in base 2, less kWeightUp; finite from below: scores of -infinity have
    // no weight)
    float m = -FLT_MAX, l = 0.f;
    finish(stream * kTile, lds);
    __syncthreads();
    constexpr int kStep = W::kStreams * kTile;
    // A tile of keys; masked: some of them are not seen by a query of the wave.  (With
    // the mask, a tile that a wave does not skip leaves each of its rows a key.)
    const auto tile_sums = [&](int at, const char *from, bool masked) {
        f32x16 p[2] = {};
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h) p[h] = mma(tile_at.rows(from + own, h * 32, d), qf[d], p[h]);
        if (masked) {
            asm volatile("");  // (a branch, not a selection per score)
            const int end = s.causal ? min(in.length, row + 1) : in.length;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (at + h * 32 + upper() * 4 + i % 4 + 8 * (i / 4) >= end) p[h][i] = -INFINITY;
        }
        float most = p[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, p[h][i]);
        most = both_halves(most, [](float x, float y) { return fmaxf(x, y); });
        // What is summed so far is brought to the new maximum only where that is
        // 2^8 above the one in use: until then numbers grow by 2^8, and lose nothing.
        most = most * c - kWeightUp<T>;
        if (__ballot(most - m > 8.f)) {
            most = fmaxf(m, most);
            const float alpha = __builtin_amdgcn_exp2f(m - most);
            m = most;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[h][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[h][i], c, -m));
                l += p[h][i];
            }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const vec8<T> pf = narrow<T>(p[h / 2], h % 2);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
                o[d] = mma(tile_at.columns(from + other, h * 16, d), pf, o[d]);
        }
    };
    const auto step = [&](int at, const char *from, char *next) {
        if (NB > 1) start(at + kStep, next);
        if (at < keys && !(s.causal && at > row0 + 31))
            tile_sums(at, from, at + kTile > in.length || (s.causal && at + kTile - 1 > row0));
        if (NB == 1) {
            __syncthreads();
            start(at + kStep, next);
        }
        finish(at + kStep, next);
        __syncthreads();
    };
    for (int at = stream * kTile, end = keys + at; at < end; at += kStep) {
        step(at, lds, NB > 1 ? lds2 : lds);
        if (NB == 1) continue;
        if ((at += kStep) >= end) break;
        step(at, lds2, lds);
    }
    l = both_halves(l, [](float x, float y) { return x + y; });
    if constexpr (W::kStreams > 1)
        join_streams<WR, DP / 2 + 2>(lds, stream, wave % WR,
            [&](int k) { return k < DP / 2 ? o[k / 16][k % 16] : k == DP / 2 ? m : l; },
            [&](auto number) {
                const float m2 = number(DP / 2), l2 = number(DP / 2 + 1), most = fmaxf(m, m2);
                const float a = __builtin_amdgcn_exp2f(m - most);
                const float b = __builtin_amdgcn_exp2f(m2 - most);
                m = most;
                l = __builtin_fmaf(l, a, l2 * b);
#pragma unroll
                for (int k = 0; k < DP / 2; ++k)
                    o[k / 16][k % 16] = __builtin_fmaf(o[k / 16][k % 16], a, number(k) * b);
            });
    if (stream > 0 || row >= in.length) return;
    store_column<DIRECT, T, DP>(out + token * s.o_ld + head * s.dim, o, 1.f / l, s.dim);
    if (lse && upper() == 0) lse[token * s.heads + head] = m * kLn2 + logf(l);
}

// ---------------------------------------------------------------------------
// Backwards, with P = exp(scale q k' - lse) formed again:
//   dv = P' dout,  dP = dout v',  dS = P (dP - D),  D = the row sums of dout out,
//   dq = scale dS k,  dk = scale dS' q.
// One kernel for D, one for dk and dv, whose workgroups own keys and go through the
// queries of all heads that share them, and one for dq, whose workgroups own queries:
// seven products instead of five, and no atomics.  64 sequences of 512 with 16 heads of
// 64: D 23 us, dk and dv 223 (128 queries at once; 64: 235), dq 138; in fp16 23, 233 to
// 253 and 144 to 159.
// ---------------------------------------------------------------------------

// D of each token and head, by 8 lanes.  Tokens outside the sequences are not looked at.
template <class T>
__global__ __launch_bounds__(kThreads) void k_attention_delta(const T *__restrict__ dout,
                                                              int64_t d_ld,
                                                              const T *__restrict__ out, Sides s,
                                                              float *__restrict__ delta)
{
    const auto start = [&](int k) { return (int64_t)min(max(s.starts[k], 0), s.tokens); };
    const int64_t begin = start(0) * s.heads, rows = start(s.sequences) * s.heads;
    const int lane = threadIdx.x & 7;
    for (int64_t r = begin + (int64_t)blockIdx.x * (kThreads / 8) + threadIdx.x / 8; r < rows;
         r += (int64_t)gridDim.x * (kThreads / 8)) {
        const int64_t token = r / s.heads;
        const int head = (int)(r - token * s.heads);
        const T *a = dout + token * d_ld + head * s.dim, *b = out + token * s.o_ld + head * s.dim;
        float sum = 0.f;
        for (int at = lane * 8; at < s.dim; at += 64) {
            const vec8<T> x = load8<false>(a, at, s.dim, true), y = load8<false>(b, at, s.dim, true);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum = __builtin_fmaf((float)x[k], (float)y[k], sum);
        }
        sum = over_lanes<8>(sum, [](float x, float y) { return x + y; });
        if (lane == 0) delta[r] = sum;
    }
}

// dS on its way to fp16, whose numbers span 2^-24 to 2^16: a lane's column (a query's for
// dq, a key's for dk) is rounded times a power of two of its own, by which the largest that
// it has met is 2^7 or more and none above 2^15.  It is lowered, with what is summed so
// far, where a larger one comes; a column of zeros keeps the first.
constexpr float kFirstGrow = 0x1p100f;

template <class T, int N>
__device__ __forceinline__ void grow_to_range(f32x16 &ds, float &grow, f32x16 (&acc)[N])
{
    if constexpr (std::is_same_v<T, _Float16>) {
        float most = fabsf(ds[0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, fabsf(ds[i]));
        most = both_halves(most, [](float x, float y) { return fmaxf(x, y); });
        if (__ballot(most * grow > 0x1p15f)) {
            const int old = (int)(__builtin_bit_cast(uint32_t, grow) >> 23);
            const int now = min(old, 261 - (int)(__builtin_bit_cast(uint32_t, most) >> 23));
            grow = __builtin_bit_cast(float, (uint32_t)now << 23);
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] = ldexpf(acc[d][i], now - old);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] *= grow;
    }
}

// Takes the factor out of what a lane has summed, before streams of waves with other ones
// add to it.
template <class T, int N>
__device__ __forceinline__ void ungrow(float &grow, f32x16 (&acc)[N])
{
    if constexpr (std::is_same_v<T, _Float16>) {
        const float back = 1.f / grow;
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] *= back;
        grow = 1.f;
    }
}

// The sides of a backward call.
struct Grads {
    int64_t d_ld, dq_ld, dk_ld, dv_ld;
};

template <class T, int DP, int WR, int NB, bool DIRECT>
__global__ __launch_bounds__(kThreads, (WR == 1 && DP > 64 ? 1 : 2)) void k_attention_dq(
    const T *__restrict__ dout, const T *__restrict__ q, const T *__restrict__ k,
    const T *__restrict__ v, Sides s, Grads g, const float *__restrict__ lse,
    const float *__restrict__ delta, T *__restrict__ dq, int tiles)
{
    using W = Share<DP, WR, NB, kTile>;
    const Tile<T, DP> tile_at;
    // (two arrays, so that a tile's loads are not waited for before the other is read)
    __shared__ __attribute__((aligned(1024))) char lds[W::kFirst], lds2[NB > 1 ? W::kLds : 1024];
    const int head = blockIdx.x % s.heads, tile = tiles - 1 - blockIdx.x / s.heads;
    const Range in = find_sequence(s, tile, W::kRows);
    if (in.at < 0 || in.at >= in.length) return;
    const int wave = wave_number(), stream = wave / WR, row0 = in.at + wave % WR * 32;
    const int kv = head / (s.heads / s.kv_heads);
    const T *kp = k + in.first * s.k_ld + kv * s.dim, *vp = v + in.first * s.v_ld + kv * s.dim;
    const int keys = s.causal ? min(in.length, in.at + W::kRows) : in.length;
    const int own = stream * 2 * W::kTileBytes, other = own + W::kTileBytes;
    Loader<T, DP, W::kStage, WR, DIRECT> kt(wave % WR, s.k_ld, s.dim), vt(wave % WR, s.v_ld, s.dim);
    const auto start = [&](int at, char *to) {
        if (at >= keys) return;
        kt.start(kp, s.k_ld, s.dim, at, in.length, to + own);
        vt.start(vp, s.v_ld, s.dim, at, in.length, to + other);
    };
    const auto finish = [&](int at, char *to) {
        if (at >= keys) return;
        kt.finish(to + own);
        vt.finish(to + other);
    };
    start(stream * kTile, lds);
    float grow = std::is_same_v<T, _Float16> ? kFirstGrow : 1.f;
    const int row = row0 + column();
    const int64_t token = in.first + row;
    const bool there = row < in.length;
    vec8<T> qf[DP / 16], df[DP / 16];
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
        qf[d] = load8<DIRECT>(q + token * s.q_ld + head * s.dim, d * 16 + upper() * 8, s.dim, there);
        df[d] = load8<DIRECT>(dout + token * g.d_ld + head * s.dim, d * 16 + upper() * 8, s.dim, there);
    }
    const float l2 = there ? lse[token * s.heads + head] * kLog2e : 0.f;
    // (a product starts from -D instead of 0)
    const float dl = there ? -delta[token * s.heads + head] : 0.f;
    const f32x16 less_d = {dl, dl, dl, dl, dl, dl, dl, dl, dl, dl, dl, dl, dl, dl, dl, dl};
    const float c = s.scale * kLog2e;
    f32x16 acc[DP / 32] = {};
    finish(stream * kTile, lds);
    __syncthreads();
    constexpr int kStep = W::kStreams * kTile;
    // A tile of keys; masked: some of them are not seen by a query of the wave.
    const auto tile_sums = [&](int at, const char *from, bool masked) {
        const int end = s.causal ? min(in.length, row + 1) : in.length;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x16 p = {}, dp = less_d;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                p = mma(tile_at.rows(from + own, h * 32, d), qf[d], p);
                dp = mma(tile_at.rows(from + other, h * 32, d), df[d], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c, -l2)) * dp[i];
            if (masked) {
                asm volatile("");
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (at + h * 32 + upper() * 4 + i % 4 + 8 * (i / 4) >= end) p[i] = 0.f;
            }
            grow_to_range<T>(p, grow, acc);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const vec8<T> pf = narrow<T>(p, half);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
                    acc[d] = mma(tile_at.columns(from + own, h * 32 + half * 16, d), pf, acc[d]);
            }
        }
    };
    const auto step = [&](int at, const char *from, char *next) {
        if (NB > 1) start(at + kStep, next);
        if (at < keys && !(s.causal && at > row0 + 31))
            tile_sums(at, from, at + kTile > in.length || (s.causal && at + kTile - 1 > row0));
        if (NB == 1) {
            __syncthreads();
            start(at + kStep, next);
        }
        finish(at + kStep, next);
        __syncthreads();
    };
    for (int at = stream * kTile, end = keys + at; at < end; at += kStep) {
        step(at, lds, NB > 1 ? lds2 : lds);
        if (NB == 1) continue;
        if ((at += kStep) >= end) break;
        step(at, lds2, lds);
    }
    if constexpr (W::kStreams > 1) {
        ungrow<T>(grow, acc);
        join_streams<WR, DP / 2>(lds, stream, wave % WR, [&](int k) { return acc[k / 16][k % 16]; },
            [&](auto number) {
#pragma unroll
                for (int k = 0; k < DP / 2; ++k) acc[k / 16][k % 16] += number(k);
            });
    }
    if (stream == 0 && there)
        store_column<DIRECT, T, DP>(dq + token * g.dq_ld + head * s.dim, acc, s.scale / grow, s.dim);
}

template <class T, int DP, int WR, int NB, bool DIRECT>
__global__ __launch_bounds__(kThreads, (WR == 1 && DP > 64 ? 1 : 2)) void k_attention_dkv(
    const T *__restrict__ dout, const T *__restrict__ q, const T *__restrict__ k,
    const T *__restrict__ v, Sides s, Grads g, const float *__restrict__ lse,
    const float *__restrict__ delta, T *__restrict__ dk, T *__restrict__ dv, int tiles)
{
    using W = Share<DP, WR, NB, WR == 4 && DP <= 64 ? 2 * kTile : kTile>;
    const Tile<T, DP> tile_at;
    // (two arrays, so that a tile's loads are not waited for before the other is read)
    __shared__ __attribute__((aligned(1024))) char lds[W::kFirst], lds2[NB > 1 ? W::kLds : 1024];
    const int kv = blockIdx.x % s.kv_heads, tile = blockIdx.x / s.kv_heads;
    const Range in = find_sequence(s, tile, W::kRows);
    if (in.at < 0 || in.at >= in.length) return;
    const int wave = wave_number(), stream = wave / WR, row0 = in.at + wave % WR * 32;
    const int group = s.heads / s.kv_heads;
    const int own = stream * 2 * W::kTileBytes, other = own + W::kTileBytes;
    // the queries that see the workgroup's keys, a head of the group after the other
    const int begin = s.causal ? in.at / W::kStage * W::kStage : 0;
    const int per_head = (in.length - begin + W::kStage - 1) / W::kStage, steps = per_head * group;
    Loader<T, DP, W::kStage, WR, DIRECT> qt(wave % WR, s.q_ld, s.dim), dt(wave % WR, g.d_ld, s.dim);
    // lse in base 2 (less kPUp) and -D of a tile's queries lie behind the tiles
    const auto rows_of = [&](auto *buffer) {
        using F = std::conditional_t<std::is_const_v<std::remove_pointer_t<decltype(buffer)>>, const float, float>;
        return (F *)(buffer + W::kRowsAt) + stream * 2 * W::kStage;
    };
    // (waves 0 .. kStage / 64 - 1 of a stream bring 64 rows' each)
    float row_value[2];
    const auto start = [&](int step, char *to) {
        if (step >= steps) return;
        const int head = kv * group + step / per_head, at = begin + step % per_head * W::kStage;
        qt.start(q + in.first * s.q_ld + head * s.dim, s.q_ld, s.dim, at, in.length, to + own);
        dt.start(dout + in.first * g.d_ld + head * s.dim, g.d_ld, s.dim, at, in.length, to + other);
        if (wave % WR < W::kStage / 64) {
            const int row = at + wave % WR * 64 + (threadIdx.x & 63);
            const int64_t at_row = (int64_t)(in.first + row) * s.heads + head;
            // (behind the end: a score of 0 less infinity has no weight)
            row_value[0] = row < in.length ? lse[at_row] * kLog2e - kPUp<T> : INFINITY;
            row_value[1] = row < in.length ? -delta[at_row] : 0.f;
        }
    };
    const auto finish = [&](int step, char *to) {
        if (step >= steps) return;
        qt.finish(to + own);
        dt.finish(to + other);
        if (wave % WR < W::kStage / 64) {
            const int r = wave % WR * 64 + (threadIdx.x & 63);
            rows_of(to)[r] = row_value[0];
            rows_of(to)[W::kStage + r] = row_value[1];
        }
    };
    start(stream, lds);
    float grow = std::is_same_v<T, _Float16> ? kFirstGrow : 1.f;
    const int row = row0 + column();
    const int64_t token = in.first + row;
    vec8<T> kf[DP / 16], vf[DP / 16];
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) {
        kf[d] = load8<DIRECT>(k + token * s.k_ld + kv * s.dim, d * 16 + upper() * 8, s.dim, row < in.length);
        vf[d] = load8<DIRECT>(v + token * s.v_ld + kv * s.dim, d * 16 + upper() * 8, s.dim, row < in.length);
    }
    const float c = s.scale * kLog2e;
    f32x16 dka[DP / 32] = {}, dva[DP / 32] = {};
    finish(stream, lds);
    __syncthreads();
    // A tile of queries; masked: some of them are in front of a key of the wave.
    const auto tile_sums = [&](int at, const char *from, const float *of_rows, bool masked) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x16 p = {}, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                dp[i] = of_rows[W::kStage + h * 32 + upper() * 4 + i % 4 + 8 * (i / 4)];
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
                p = mma(tile_at.rows(from + own, h * 32, d), kf[d], p);
                dp = mma(tile_at.rows(from + other, h * 32, d), vf[d], dp);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = h * 32 + upper() * 4 + i % 4 + 8 * (i / 4);
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c, -of_rows[r]));
                dp[i] *= p[i];
            }
            if (masked) {
                asm volatile("");
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (at + h * 32 + upper() * 4 + i % 4 + 8 * (i / 4) < row) p[i] = 0.f, dp[i] = 0.f;
            }
            grow_to_range<T>(dp, grow, dka);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const vec8<T> pf = narrow<T>(p, half), sf = narrow<T>(dp, half);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    dva[d] = mma(tile_at.columns(from + other, h * 32 + half * 16, d), pf, dva[d]);
                    dka[d] = mma(tile_at.columns(from + own, h * 32 + half * 16, d), sf, dka[d]);
                }
            }
        }
    };
    const auto go = [&](int step, const char *from, char *next) {
        if (NB > 1) start(step + W::kStreams, next);
        const int at = begin + step % per_head * W::kStage;
        if (step < steps)
#pragma unroll 1
            for (int t = at; t < min(at + W::kStage, in.length); t += kTile)
                if (!(s.causal && t + kTile - 1 < row0))
                    tile_sums(t, from + (t - at) * DP * 2, rows_of(from) + (t - at), s.causal && t < row0 + 31);
        if (NB == 1) {
            __syncthreads();
            start(step + W::kStreams, next);
        }
        finish(step + W::kStreams, next);
        __syncthreads();
    };
    for (int step = stream, end = steps + stream; step < end; step += W::kStreams) {
        go(step, lds, NB > 1 ? lds2 : lds);
        if (NB == 1) continue;
        if ((step += W::kStreams) >= end) break;
        go(step, lds2, lds);
    }
    if constexpr (W::kStreams > 1) {
        const auto join = [&](f32x16(&acc)[DP / 32]) {
            join_streams<WR, DP / 2>(lds, stream, wave % WR, [&](int k) { return acc[k / 16][k % 16]; },
                [&](auto number) {
#pragma unroll
                    for (int k = 0; k < DP / 2; ++k) acc[k / 16][k % 16] += number(k);
                });
        };
        ungrow<T>(grow, dka);
        join(dka);
        __syncthreads();
        join(dva);
    }
    if (stream > 0 || row >= in.length) return;
    constexpr float kBack = 1.f / (1 << kPUp<T>);
    store_column<DIRECT, T, DP>(dk + token * g.dk_ld + kv * s.dim, dka, s.scale / grow * kBack, s.dim);
    store_column<DIRECT, T, DP>(dv + token * g.dv_ld + kv * s.dim, dva, kBack, s.dim);
}

template <class F>
void with_half(int32_t dtype, F &&f)
{
    if (dtype == ONEBIT_GRAD_BF16) f((__bf16 *)nullptr);
    else f((_Float16 *)nullptr);
}

// Calls f(padded dim, rows of waves, depth, direct).
template <class F>
void with_shape(int dim, bool few, bool direct, F &&f)
{
    using std::integral_constant;
    auto go = [&](auto padded, auto waves, auto depth) {
        if (direct) f(padded, waves, depth, std::true_type{});
        else f(padded, waves, depth, std::false_type{});
    };
    auto by_waves = [&](auto padded) {
        if (few) go(padded, integral_constant<int, 1>{}, integral_constant<int, 1>{});
        else go(padded, integral_constant<int, 4>{}, integral_constant<int, 2>{});
    };
    if (dim <= 32) by_waves(integral_constant<int, 32>{});
    else if (dim <= 64) by_waves(integral_constant<int, 64>{});
    else if (dim <= 96) by_waves(integral_constant<int, 96>{});
    else by_waves(integral_constant<int, 128>{});
}

// Whether a side's tiles can be read straight into LDS: pieces of 16 bytes on 4-byte
// borders, a tile's rows within the buffer's 2 GiB.
bool direct_side(const void *p, int64_t ld, int dim)
{
    return dim % 8 == 0 && (uintptr_t)p % 4 == 0 && ld % 2 == 0 && ld < (1 << 23);
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

// Tiles of `rows` tokens that cover every sequence (find_sequence): a launch has a
// workgroup for each and each head.
int check_tiles(int64_t tokens, int64_t sequences, int heads)
{
    if ((tokens / 128 + sequences) * heads >= ((int64_t)1 << 32) / kThreads)
        return fail(ONEBIT_EINVAL, "%lld tokens in %lld sequences with %d heads are too many for one call",
                    (long long)tokens, (long long)sequences, heads);
    return ONEBIT_OK;
}

int tile_count(int64_t tokens, int64_t sequences, int rows) { return (int)(tokens / rows + sequences); }

// Whether a call has so few tiles of 128 rows that its waves share the other side of 32
// rows instead.  us with whole tiles and so: attention of one prompt of 512 with 16 heads
// of 64 (80 tiles) 12.7 and 7.8, of 8,192 with 2 heads (130) 104 and 48, of 2,048 with 16
// (272) 32 and 27 causal, 33 and 40 not, of four of 1,024 (576) 27 and 39; with heads of
// 128, one of 4,096 with 4 (132) 77 and 50, of 1,000 with 32 (256) 26 and 45.  Gradients,
// whose tiles of keys go through the queries of all heads on them: 2,048 with 16 heads on
// 4 of 128 (68 tiles of keys) 629 and 177, eleven documents with 12 on 4 of 80 (228) 278
// and 160, four of 1,024 with 8 of 128 (288) 137 and 126, of 64 (576) 77 and 98.
bool few_tiles(int64_t tokens, int64_t sequences, int heads, int most)
{
    return (tokens / 128 + sequences) * heads <= most;
}
constexpr int kFewQueryTiles = 255, kFewKeyTiles = 320;

int delta_blocks(int64_t tokens, int heads)
{
    return (int)std::min<int64_t>((tokens * heads + kThreads / 8 - 1) / (kThreads / 8), kMostDeltaBlocks);
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
    TRY(check_tiles(tokens, sequences, heads));
    if (tokens == 0 || sequences == 0) return ONEBIT_OK;
    if (tokens == 1) q_ld = out_ld = width, k_ld = v_ld = kv_width;  // (not looked at above)
    const Sides s{q_ld, k_ld, v_ld, out_ld, starts, (int)tokens, (int)sequences,
                  heads, kv_heads, dim, scale, causal};
    with_half(dtype, [&](auto *t) {
        with_shape(dim, few_tiles(tokens, sequences, heads, kFewQueryTiles),
                   direct_side(k, k_ld, dim) && direct_side(v, v_ld, dim),
                   [&](auto padded, auto waves, auto depth, auto direct) {
            using T = std::remove_pointer_t<decltype(t)>;
            const int tiles = tile_count(tokens, sequences, 32 * waves);
            k_attention<T, padded(), waves(), depth(), direct()>
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
    *bytes = (size_t)tokens * heads * sizeof(float);
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
    TRY(check_tiles(tokens, sequences, heads));
    if (tokens == 0 || sequences == 0) return ONEBIT_OK;
    if (tokens == 1) {  // (not looked at above)
        dout_ld = q_ld = out_ld = dq_ld = width;
        k_ld = v_ld = dk_ld = dv_ld = kv_width;
    }
    const Sides s{q_ld, k_ld, v_ld, out_ld, starts, (int)tokens, (int)sequences,
                  heads, kv_heads, dim, scale, causal};
    const Grads g{dout_ld, dq_ld, dk_ld, dv_ld};
    float *delta = (float *)workspace;
    hipStream_t st = (hipStream_t)stream;
    with_half(dtype, [&](auto *t) {
        using T = std::remove_pointer_t<decltype(t)>;
        k_attention_delta<T><<<delta_blocks(tokens, heads), kThreads, 0, st>>>(
            (const T *)dout, dout_ld, (const T *)out, s, delta);
        with_shape(dim, few_tiles(tokens, sequences, kv_heads, kFewKeyTiles),
                   direct_side(q, q_ld, dim) && direct_side(dout, dout_ld, dim),
                   [&](auto padded, auto waves, auto depth, auto direct) {
            const int tiles = tile_count(tokens, sequences, 32 * waves);
            k_attention_dkv<T, padded(), waves(), depth(), direct()>
                <<<tiles * kv_heads, kThreads, 0, st>>>(
                    (const T *)dout, (const T *)q, (const T *)k, (const T *)v, s, g, lse, delta,
                    (T *)dk, (T *)dv, tiles);
        });
        with_shape(dim, few_tiles(tokens, sequences, heads, kFewQueryTiles),
                   direct_side(k, k_ld, dim) && direct_side(v, v_ld, dim),
                   [&](auto padded, auto waves, auto depth, auto direct) {
            const int tiles = tile_count(tokens, sequences, 32 * waves);
            k_attention_dq<T, padded(), waves(), depth(), direct()>
                <<<tiles * heads, kThreads, 0, st>>>(
                    (const T *)dout, (const T *)q, (const T *)k, (const T *)v, s, g, lse, delta,
                    (T *)dq, tiles);
        });
    });
    return launched("attention gradient launch");
}

}  // extern "C"
