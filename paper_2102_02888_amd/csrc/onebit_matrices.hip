// Orthogonalised updates of a list of matrices: Newton-Schulz products on the
// matrix cores, with the momentum before them and the parameters' update behind.
// See include/onebit.h for the formulas and the contract of the entry points.
//
// One pass over the list is two streaming launches (momentum and norm; first
// iterate) and three product launches per Newton-Schulz step:
//   gram   D = X X^T - t I            (symmetric: tiles on and below the diagonal)
//   poly   B = (b + 2 c t) D + c D D  (symmetric)
//   next   X <- (a + b t + c t^2) X + B X
// all of them over every tile of every matrix.  A product is always rows times
// rows (both operands contiguous along the summed index; D and B are symmetric),
// but for X in B X, whose fragments are read transposed from LDS.  Every operand
// lies in the workspace, padded with zeros to multiples of the tile, so that the
// product kernel has no bounds to check.
//
// Numbers.  Operands are fp16 times kScale.  PRODUCTS_F32 ("pairs"): a value is
// hi + lo, two fp16 numbers, together as fine as an fp32 one; a product adds
// hi hi + hi lo + lo hi in fp32 and leaves out lo lo, 2^-22 of it.
// PRODUCTS_F16 ("halves"): products take hi alone, and only the iterate keeps lo,
// for the term that is linear in it: rounding the iterate itself would add
// noise to every direction, which the later steps amplify in those of small
// singular values (off as a whole on gradients of rank 16 with 1e-3 of noise:
// 4e-2 without lo, 9e-4 with it).
// A matrix whose norm is far below eps starts far below 1 and may stay there.  Its
// iterate is held times gamma, a power of two that starts at no more than
// 1 / ||X||_F and falls by `fade` a step, no less than a step's growth, until it
// is 1: with Y = gamma X and E = Y Y^T - t I, the step is
//   B = (b + 2 c t / gamma^2) E + c / gamma^2 E E,   Y <- (...) Y + B Y / gamma^2.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <memory>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "../../include/onebit.h"
#include "onebit_internal.h"
#include "onebit_status.h"

namespace onebit {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// |X|, |A| and the polynomial's change stay below kRange, so that kScale times
// them stays below fp16's 65504; 2^13 leaves an iterate of 2^14 x 2^14 elements
// (2^-14 each) 2^-23 of its size as the step of its low half.
constexpr float kScale = 8192.f;
constexpr double kRange = 7.5;

constexpr int kPartGroups = 4;  // groups of waves of the tiles whose Gram sums go in parts
constexpr int kSlab = 64;    // fp16 numbers of an operand's row that are staged together
constexpr int kPrep = 64;    // rows and columns of a workgroup of the first iterate

struct Mat {
    int64_t off, ld;             // in the flat buffers
    int32_t rows, cols;          // there
    int32_t m, n;                // the smaller and the larger side
    int32_t mp, np;              // multiples of kTile
    int32_t flip;                // 1: X is the matrix transposed
    int32_t norm_first, norm_count;  // partial sums of the norm
    int32_t part_first, part_count;  // partial sums of the iterate's squares
    int32_t slot_first, slot_count;  // counters of its tiles that several workgroups form
    int32_t parts;               // of a Gram tile's summed index
    int64_t ex, em;              // elements of X and of D before this matrix's
    int64_t sums;                // where the parts' sums are
};

// A tile of a product.  (16 bytes, beside a matrix's record that its tiles share: a
// record of its own for every tile, 160 bytes, would be one load less to wait for
// but a miss for every workgroup, and costs up to 18%.)
struct MatTile {
    int32_t mat;     // < 0: none
    uint16_t i, j;
    int32_t part;    // of Mat::parts, of the summed index
    int32_t slot;    // of several parts: the counter
};

struct Item {
    int32_t mat;
    uint16_t i, j;
};

// Areas of the workspace.  Pairs: rows of X, D and B hold 32 hi numbers and then
// the same 32 lo numbers, so that 64 consecutive numbers are a slab of either
// kind.  Halves: hi alone, and x_lo holds the iterate's lo.
struct Areas {
    _Float16 *x, *x_next, *x_lo, *d, *b;
    double *norm;   // per norm chunk
    float *part;    // per tile of the iterate
    float *t;       // per matrix
    float *gamma;   // per matrix, of the first iterate
    uint32_t *counter;  // per tile in parts: parts that are done
    float *sums;        // their sums
};

struct Coefficients {
    float a, b, c;
    float fade;  // of gamma in a step: a power of two, at most 1/2
};

__device__ __forceinline__ void split(float v, _Float16 &hi, _Float16 &lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// Orders a wave's LDS accesses: what its lanes wrote is there for all of them.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Workgroup barrier behind loads straight into LDS, or behind stores that are to be
// there for other workgroups: every wave waits for its own before it arrives (a plain
// barrier waits for neither).
__device__ __forceinline__ void staged_sync()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0), the other counters at their most
    __syncthreads();
}

// Workgroup barrier that waits for no loads of the wave's own (their count is
// awaited before it, where that matters).
__device__ __forceinline__ void bare_sync()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Sum over the workgroup of 256, the same in every thread; scratch: 4 values.
template <class T>
__device__ __forceinline__ T block_sum(T v, T *scratch)
{
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    return (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
}

// ---------------------------------------------------------------------------
// Momentum, norm and the first iterate
// ---------------------------------------------------------------------------

// N consecutive elements as fp32.  Rows need no alignment: vector accesses are
// stated as copies of bytes, which become loads and stores of up to 16 bytes.
template <class T, int N>
__device__ __forceinline__ void load_vec(const T *p, float (&v)[N])
{
    T t[N];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = (float)t[k];
}

// What is orthogonalised: a tensor, or momentum and gradients of a Muon step.
// value() is N elements of it from element e of the flat buffers on; first() the
// same for the norm's pass, which sees every element once and before value().
// e_u: the element's place in the workspace.
template <class T>
struct FromTensor {
    const T *in;
    template <int N>
    __device__ __forceinline__ void value(int64_t e, int64_t, float (&v)[N]) const
    {
        load_vec(in + e, v);
    }
    template <int N>
    __device__ __forceinline__ void first(int64_t e, int64_t e_u, float (&v)[N]) const
    {
        value(e, e_u, v);
    }
};

template <class T>
struct FromMuon {
    const T *grads;
    float *m;
    float *u;  // where the norm's pass leaves the update, or NULL: it is formed again
    int64_t grad_ld;
    int n_grads;
    double n;
    float momentum;
    int nesterov;
    template <int N>
    __device__ __forceinline__ void mean(int64_t e, float (&v)[N]) const
    {
        load_vec(grads + e, v);
        if (n_grads == 1) return;
        double s[N];
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = (double)v[k];
#pragma unroll 4
        for (int i = 1; i < n_grads; ++i) {
            load_vec(grads + i * grad_ld + e, v);
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] += (double)v[k];
        }
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (float)(s[k] / n);
    }
    // the update from the new momentum
    template <int N>
    __device__ __forceinline__ void value(int64_t e, int64_t e_u, float (&v)[N]) const
    {
        if (u) return load_vec(u + e_u, v);
        float now[N];
        load_vec(m + e, now);
        if (nesterov) mean(e, v);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = nesterov ? v[k] + momentum * now[k] : now[k];
    }
    // ... which is formed and stored here
    template <int N>
    __device__ __forceinline__ void first(int64_t e, int64_t e_u, float (&v)[N]) const
    {
        float now[N];
        load_vec(m + e, now);
        mean(e, v);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            now[k] = momentum * now[k] + v[k];
            v[k] = nesterov ? v[k] + momentum * now[k] : now[k];
        }
        __builtin_memcpy(m + e, now, sizeof now);
        if (u) __builtin_memcpy(u + e_u, v, sizeof v);
    }
};

// Sum of squares (64 bits) of `size` elements of a matrix: 8 per thread at a time
// where the matrix is one run of memory, else one.  Memory bounds it: 302M fp32
// elements 204 us (5.9 TB/s), a step's momentum from bf16 gradients over the same 530 us
// (3.0 GB, 5.7 TB/s), of 8 gradients over 50M elements 274 us.
template <class S>
__global__ __launch_bounds__(256) void k_norm(const Mat *__restrict__ mats,
                                              const Item *__restrict__ items, int size, S src,
                                              double *__restrict__ norm)
{
    __shared__ double scratch[4];
    const Item it = items[blockIdx.x];
    const Mat &mt = mats[it.mat];
    const uint32_t cols = mt.cols, total = (uint32_t)mt.rows * cols;
    const int64_t off = mt.off, ld = mt.ld, at_u = mt.ex;
    const uint32_t chunk = (uint32_t)it.i << 16 | it.j;
    const uint32_t begin = chunk * size, end = min(begin + size, total);
    double sum = 0;
    if (ld == cols) {
        uint32_t e = begin + threadIdx.x * 8;
#pragma unroll 2
        for (; e + 8 <= end; e += 2048) {
            float v[8];
            src.first(off + e, at_u + e, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += (double)v[k] * (double)v[k];
        }
        for (; e < end; ++e) {  // the last thread's few, where 8 are no longer left
            float v[1];
            src.first(off + e, at_u + e, v);
            sum += (double)v[0] * (double)v[0];
        }
    } else {
        for (uint32_t e = begin + threadIdx.x; e < end; e += 256) {
            const uint32_t r = e / cols;
            float v[1];
            src.first(off + r * ld + (e - r * cols), at_u + e, v);
            sum += (double)v[0] * (double)v[0];
        }
    }
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) norm[mt.norm_first + chunk] = sum;
}

// Place of number k of an operand's row (its hi; lo follows 32 further for pairs).
template <bool PAIRS>
__device__ __forceinline__ int column(int k)
{
    return PAIRS ? (k >> 5) * 64 + (k & 31) : k;
}

// First iterate, X = u / (||u||_F + eps), padding zeroed: 64 x 64 of the matrix
// for a workgroup, 8 of a row for a thread, turned in LDS where X is the transpose.
// It is a launch of its own because the factor needs the whole norm.  Memory bounds
// it: 302M fp32 elements to hi and lo 460 to 500 us (2.4 GB, 4.8 to 5.3 TB/s).
template <bool PAIRS, class S>
__global__ __launch_bounds__(256) void k_first(const Mat *__restrict__ mats,
                                               const Item *__restrict__ items, S src, double eps,
                                               Areas w)
{
    __shared__ double scratch[4];
    __shared__ float tile[kPrep][kPrep + 1];
    const Item it = items[blockIdx.x];
    const Mat &mt = mats[it.mat];
    const int r0 = it.i * kPrep, c0 = it.j * kPrep;
    const int line = threadIdx.x >> 3, eight = (threadIdx.x & 7) * 8;
    float v[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = r0 + h * 32 + line, c = c0 + eight;
        const int64_t e = mt.off + r * mt.ld + c, e_u = mt.ex + (int64_t)r * mt.cols + c;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[h][k] = 0.f;
        if (r < mt.rows && c + 8 <= mt.cols) {
            src.value(e, e_u, v[h]);
        } else if (r < mt.rows) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < mt.cols) {
                    float one[1];
                    src.value(e + k, e_u + k, one);
                    v[h][k] = one[0];
                }
        }
    }
    double sum = 0;
    for (int k = threadIdx.x; k < mt.norm_count; k += 256) sum += w.norm[mt.norm_first + k];
    sum = block_sum(sum, scratch);
    const double size = sqrt(sum) / (sqrt(sum) + eps);
    // a NaN, zero or infinite norm, and every norm above eps: 1
    const double gamma = size > 0 && size <= 0.5 ? exp2(fmin(-ceil(log2(size)), 120.0)) : 1.0;
    if (it.i == 0 && it.j == 0) {
        if (threadIdx.x == 0) w.gamma[it.mat] = (float)gamma;
        for (int k = threadIdx.x; k < mt.slot_count; k += 256) w.counter[mt.slot_first + k] = 0;
    }
    const double factor = (double)kScale * gamma / (sqrt(sum) + eps);
    if (mt.flip) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < 8; ++k) tile[h * 32 + line][eight + k] = v[h][k];
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[h][k] = tile[eight + k][h * 32 + line];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = (mt.flip ? c0 : r0) + h * 32 + line, col = (mt.flip ? r0 : c0) + eight;
        half8 hi, lo;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            // padding stays zero beside a NaN or an infinite norm too
            const bool real = row < mt.m && col + k < mt.n;
            _Float16 a, b;
            split(real ? (float)((double)v[h][k] * factor) : 0.f, a, b);
            hi[k] = a;
            lo[k] = b;
        }
        constexpr int kind = PAIRS ? 2 : 1;
        _Float16 *to = w.x + mt.ex * kind + (int64_t)row * mt.np * kind + column<PAIRS>(col);
        *(half8 *)to = hi;
        if constexpr (PAIRS) *(half8 *)(to + 32) = lo;
        else *(half8 *)(w.x_lo + mt.ex + (int64_t)row * mt.np + col) = lo;
    }
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

constexpr int kGram = 0, kPoly = 1, kNext = 2, kLast = 3;

// Where the last product goes, 8 numbers of a row (of which `left` exist): a
// tensor, or the parameters.  Rows need no alignment: the vector accesses are
// stated as copies of bytes.
template <class T>
struct ToTensor {
    T *out;
    __device__ __forceinline__ void put(int64_t e, const float *o, int left, float) const
    {
        T t[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = (T)o[k];
        if (left >= 8) {
            __builtin_memcpy(out + e, t, sizeof t);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) out[e + k] = t[k];
        }
    }
};

struct ToMuon {
    float *x;
    float keep, lr;  // 1 - lr weight decay, lr
    __device__ __forceinline__ void put(int64_t e, const float *o, int left, float scale) const
    {
        const float by = lr * scale;
        if (left >= 8) {
            float t[8];
            __builtin_memcpy(t, x + e, sizeof t);
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = keep * t[k] - by * o[k];
            __builtin_memcpy(x + e, t, sizeof t);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left) x[e + k] = keep * x[e + k] - by * o[k];
        }
    }
};

struct NoOut {};

__device__ __forceinline__ float muon_scale(int mode, int rows, int cols)
{
    if (mode == ONEBIT_MUON_SCALE_SPECTRAL)
        return sqrtf(fmaxf(1.f, (float)rows / (float)cols));
    if (mode == ONEBIT_MUON_SCALE_RMS) return 0.2f * sqrtf((float)max(rows, cols));
    return 1.f;
}

constexpr int kRowBytes = kSlab * 2;  // 128 bytes of LDS per staged row

// Place of 16-byte chunk c of staged row r.  A fragment is chunk c of 32 rows;
// a row is 128 bytes, so that all of them would begin in the same bank: the
// row's number permutes its chunks, and any 16 consecutive rows cover all banks.
__device__ __forceinline__ int row_chunk(int r, int c)
{
    return r * kRowBytes + ((c ^ (r >> 1)) & 7) * 16;
}

// The same for an operand that is staged with the summed index along its rows
// (X in X <- B X): 32-byte chunks of row k are permuted by k mod 4 so that the four
// rows and two chunks which 32 lanes of a transposing read take lie in different
// banks, of 32 or of 64 (rows of 128 bytes have four chunks, and lie in both
// halves of 64 banks by themselves).
template <int ROW_BYTES>
__device__ __forceinline__ int deep_swizzle(int k)
{
    const int b = k & 3;
    return ROW_BYTES == 128 ? b : b << 1 | ((b >> 1) ^ (b & 1));
}

typedef __attribute__((address_space(3))) void lds_void;

// The wave's number, in a scalar register.
__device__ __forceinline__ int wave_number()
{
    return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}

// 16 bytes per lane, from `base` (the same in all lanes) + lane_at + scalar_at, to
// consecutive places from `lds` on.  The base sits in scalar registers, in a
// buffer resource of 2 GiB (its fourth word is the gfx9-family format word).  The
// host compiler, which only needs the kernels' names, does not take the builtin
// at this size.
__device__ __forceinline__ void load_to_lds(const void *base, char *lds, int lane_at, int scalar_at)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const uint64_t a = (uint64_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(((uint64_t)hi << 32) | lo), (short)0, 0x7FFFFFFF, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)lds, 16, lane_at, scalar_at, 0, 0);
#endif
}

// Stages BT rows of an operand, 8 rows of 128 bytes per instruction, straight
// into LDS: a wave's 64 lanes fill 1 KB in lane order, so the permutation is
// applied to the address that is read.  The base and a row block's offset (below
// 256 rows of 2^22 bytes) are scalars, and two lane offsets serve all.
template <int BT, int WAVES>
struct RowStager {
    static constexpr int kEach = BT / 8 / WAVES;  // instructions of a wave
    static_assert(kEach % 2 == 0, "the permutation alternates with the instruction");
    const char *base;
    int pitch, wave, lane_at[2];  // bytes, but for the wave's number
    __device__ __forceinline__ RowStager(const _Float16 *src, int64_t row_numbers, int wave_)
        : base((const char *)src), pitch((int)row_numbers * 2), wave(wave_)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            lane_at[k] = (lane >> 3) * pitch + ((lane & 7) ^ (4 * k | lane >> 4)) * 16;
    }
    __device__ __forceinline__ void operator()(int slab, char *lds) const
    {
        const char *from = base + (int64_t)slab * kRowBytes;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int block = wave * kEach + k;
            load_to_lds(from, lds + block * 1024, lane_at[k & 1], block * 8 * pitch);
        }
    }
};

// Stages a slab of an operand with the summed index along its rows: kSlab / kind
// rows of BT numbers (pairs: of BT hi and BT lo); or one of its PARTS parts.
template <bool PAIRS, int BT, int WAVES, int PARTS>
struct DeepStager {
    static constexpr int kEach = BT / 8 / WAVES / PARTS, kBytes = BT * (PAIRS ? 4 : 2);
    static constexpr int kRows = 1024 / kBytes;  // of an instruction
    // permutations of a wave's instructions
    static constexpr int kKinds = kRows >= 4 ? 1 : kEach < 4 / kRows ? kEach : 4 / kRows;
    static_assert(kEach % kKinds == 0 && (kEach % 4 == 0 || kEach == kKinds), "rows of an instruction");
    const char *base;
    int pitch, wave, lane_at[kKinds];
    __device__ __forceinline__ DeepStager(const _Float16 *src, int64_t row_numbers, int wave_)
        : base((const char *)src), pitch((int)row_numbers * 2), wave(wave_)
    {
        const int at = (threadIdx.x & 63) * 16, r = at / kBytes, p = at % kBytes / 16;
#pragma unroll
        for (int k = 0; k < kKinds; ++k)
            lane_at[k] = r * pitch +
                (((p >> 1) ^ deep_swizzle<kBytes>((wave * kEach + k) * kRows + r)) * 2 + (p & 1)) * 16;
    }
    __device__ __forceinline__ void operator()(int part, char *lds) const
    {
        constexpr int kPartRows = kSlab / (PAIRS ? 2 : 1) / PARTS;
        const char *from = base + (int64_t)part * kPartRows * pitch;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int block = wave * kEach + k;
            load_to_lds(from, lds + block * 1024, lane_at[k % kKinds], block * kRows * pitch);
        }
    }
};

// Eight numbers of the summed index for 32 columns from a deep slab: two
// transposing reads, each of 4 rows x 16 columns per 16 lanes.  at: the lane's
// place for the first (deep_place).
template <int ROW_BYTES>
__device__ __forceinline__ half8 deep_fragment(const char *at)
{
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef short v8s __attribute__((ext_vector_type(8)));
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) v4s *)at);
    const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) v4s *)(at + 4 * ROW_BYTES));
    return __builtin_bit_cast(half8, (v8s)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int ROW_BYTES>
__device__ __forceinline__ int deep_place(int byte)
{
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int r = 8 * (g >> 1) + (j >> 2), at = byte + (g & 1) * 32 + (j & 3) * 8;
    return r * ROW_BYTES + ((at >> 5) ^ deep_swizzle<ROW_BYTES>(r)) * 32 + (at & 31);
}

// One product launch: a workgroup forms a BT x BT tile, each of its waves 32 WR x
// 32 WC of it with 32 x 32 x 16 matrix instructions.  Slabs of both operands are
// staged in two buffers by turns, the next one's loads in flight under the
// present one's products.  Two buffers of their own, not halves of one: only then
// does the compiler know that reading one need not wait for loads into the other.
// With KG above 1 that many groups of waves form the same tile, each from slabs of
// its own (the k-th slab goes to group k mod KG) in buffers of its own, and their
// sums are added at the end: for lists with fewer tiles than the GPU has CUs, where
// the wait for a slab is what counts.
// A tile of 256 reads 1/128 of an operand's number per multiply-add, a tile of 64
// 1/32, which only short lists can afford.  Its 8 waves of 128 x 64 leave the matrix
// cores two waves per SIMD to draw from (4 waves of 128 x 128 read a third less from LDS
// but took 4% longer over a list of 144 matrices with halves, 11% with pairs).
// Measured on that list (96 of 1,024 x 1,024, 24 of 4,096 x 1,024, 24 of 1,024 x 4,096;
// us, and the share of the time that the matrix cores are busy):
//            gram       poly       next        last
//   pairs    963 67%    608 55%    1,683 67%   1,625 69%  (of a Muon step 1,913 56%)
//   halves   434 54%    256 44%      861 43%     816 45%
// There is no LDS bank conflict but in the last one's turned tiles.  What bounds
// pairs is the matrix cores in the slabs and memory in the epilogue, which one tile's
// products cannot hide where it has its CU to itself; for halves, with a third of the
// products, the epilogue counts for more.
template <bool PAIRS, int STEP, int BT, int WR, int WC, int KG, int THREADS, class O>
__global__ __launch_bounds__(THREADS, 2) void k_product(
    const Mat *__restrict__ mats, const MatTile *__restrict__ tiles, Areas w, Coefficients co,
    float faded, O out, int scale_mode)
{
    constexpr int kWaves = BT * BT / (1024 * WR * WC);
    static_assert(THREADS == KG * kWaves * 64, "a wave for every part of the tile");
    constexpr int kOperand = BT * kRowBytes;
    constexpr bool kDeep = STEP == kNext || STEP == kLast;
    // Tiles of 256 of B X: X in buffers of its own, for half slabs.
    constexpr bool kSplit = kDeep && BT == 256;
    constexpr int kBuffer = (kSplit ? 1 : KG * 2) * kOperand, kHalfBuffer = kSplit ? kOperand / 2 : 16;
    __shared__ __attribute__((aligned(1024))) char buffer0[kBuffer], buffer1[kBuffer];
    __shared__ __attribute__((aligned(1024))) char x00[kHalfBuffer], x01[kHalfBuffer],
        x10[kHalfBuffer], x11[kHalfBuffer];
    __shared__ float scratch[KG * kWaves];
    const MatTile it = tiles[(blockIdx.x % kXcds) * (gridDim.x / kXcds) + blockIdx.x / kXcds];
    if (it.mat < 0) return;
    const Mat mt = mats[it.mat];
    constexpr int kind = PAIRS ? 2 : 1;
    const int group = KG > 1 ? wave_number() / kWaves : 0, wave = wave_number() - group * kWaves;
    const int lane = threadIdx.x & 63;
    constexpr int kAcross = BT / (32 * WC);
    const int wr = wave / kAcross * (32 * WR), wc = wave % kAcross * (32 * WC);
    const int i0 = it.i * BT, j0 = it.j * BT;

    const int64_t ex = mt.ex * kind, em = mt.em * kind;
    const int64_t x_pitch = (int64_t)mt.np * kind, d_pitch = (int64_t)mt.mp * kind;
    const int64_t pitch = STEP == kGram ? x_pitch : d_pitch;
    const _Float16 *x = w.x + ex, *d = w.d + em, *b = w.b + em;
    const _Float16 *pa = (STEP == kGram ? x : STEP == kPoly ? d : b) + i0 * pitch;
    const _Float16 *pb = kDeep ? x + j0 * kind : (STEP == kGram ? x : d) + j0 * pitch;
    // Slabs: all of them, an even number but for tiles of 64, or this part's.
    constexpr bool kInParts = STEP == kGram && KG == kPartGroups;
    const int all_slabs = (int)(pitch / kSlab);
    const int slab0 = kInParts ? (int)((int64_t)all_slabs * it.part / mt.parts) : 0;
    const int slabs = kInParts ? (int)((int64_t)all_slabs * (it.part + 1) / mt.parts) - slab0 : all_slabs;

    f32x16 acc[WR][WC] = {};
    const RowStager<BT, kWaves> stage_a(pa, pitch, wave);
    const std::conditional_t<kDeep, DeepStager<PAIRS, BT, kWaves, kSplit ? 2 : 1>,
                             RowStager<BT, kWaves>> stage_b(pb, kDeep ? x_pitch : pitch, wave);
    auto stage = [&](int s, char *to) {
        stage_a(slab0 + s, to);
        stage_b(slab0 + s, to + kOperand);
    };
    // Fragments of 16 numbers of the summed index: of a slab's kSteps, the k-th.
    constexpr int kSteps = PAIRS ? 2 : 4, kDeepBytes = BT * 2 * kind;
    struct Fragments {
        half8 a[WR], b[WC], a_lo[PAIRS ? WR : 1], b_lo[PAIRS ? WC : 1];
    };
    // places that differ by more than a constant from one to the next
    const int row = lane & 31, up = lane >> 5;
    int place_a[4], place_b[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        place_a[c] = row_chunk(wr + row, c * 2 + up);
        if (!kDeep) place_b[c] = kOperand + row_chunk(wc + row, c * 2 + up);
        else place_b[c] = (kSplit ? 0 : kOperand) +
                          deep_place<kDeepBytes>((wc + c / kind * 32) * 2 * kind + c % kind * 64);
    }
    // b: where the second operand's slab begins, or its half with fragment k in it
    auto second = [&](const char *b, int k, int q, int lo) {
        if (kDeep)
            return deep_fragment<kDeepBytes>(b + place_b[q * kind + lo] +
                                             (kSplit ? k % (kSteps / 2) : k) * 16 * kDeepBytes);
        return *(const half8 *)(b + place_b[k + lo * 2] + q * 32 * kRowBytes);
    };
    auto load_from = [&](const char *buffer, const char *b, int k, Fragments &f) {
#pragma unroll
        for (int p = 0; p < WR; ++p) f.a[p] = *(const half8 *)(buffer + place_a[k] + p * 32 * kRowBytes);
#pragma unroll
        for (int q = 0; q < WC; ++q) f.b[q] = second(b, k, q, 0);
        if (PAIRS) {
#pragma unroll
            for (int q = 0; q < WC; ++q) f.b_lo[q] = second(b, k, q, 1);
#pragma unroll
            for (int p = 0; p < WR; ++p)
                f.a_lo[p] = *(const half8 *)(buffer + place_a[k + 2] + p * 32 * kRowBytes);
        }
    };
    auto load = [&](const char *buffer, int k, Fragments &f) { load_from(buffer, buffer, k, f); };
    auto multiply = [&](const Fragments &f) {
        auto all = [&](const half8 *fa, const half8 *fb) {
#pragma unroll
            for (int p = 0; p < WR; ++p)
#pragma unroll
                for (int q = 0; q < WC; ++q)
                    acc[p][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[p], fb[q], acc[p][q], 0, 0, 0);
        };
        all(f.a, f.b);
        if (PAIRS) {
            all(f.a, f.b_lo);
            all(f.a_lo, f.b);
        }
    };
    // The first two slabs are under way before anything else is waited for.
    char *const ours[2] = {buffer0 + group * 2 * kOperand, buffer1 + group * 2 * kOperand};
    const int own = (slabs - group + KG - 1) / KG;  // slabs of this group
    // (split: loads must start in the order in which they are waited for)
    auto in_order = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto stage_x = [&](int part, char *to) {
        in_order();
        stage_b(part, to);
        in_order();
    };
    if constexpr (kSplit) {
        stage_x(0, x00);
        stage_a(0, buffer0);
        stage_x(1, x01);
        stage_x(2, x10);
    } else {
        if (own > 0) stage(group, ours[0]);
        if (own > 1) stage(KG + group, ours[1]);
    }

    // The shift, and the step's coefficients around it.
    auto sum_over = [&](float v) {  // the workgroup's, the same in every thread
        for (int k = 32; k > 0; k /= 2) v += __shfl_xor(v, k);
        __syncthreads();
        if (lane == 0) scratch[wave_number()] = v;
        __syncthreads();
        float total = 0.f;
#pragma unroll
        for (int k = 0; k < KG * kWaves; ++k) total += scratch[k];
        return total;
    };
    const float gamma0 = w.gamma[it.mat], gamma = fmaxf(gamma0 * faded, 1.f);
    const float inv2 = 1.f / (gamma * gamma);
    float t;
    if (STEP == kGram) {
        if (faded == 1.f) {  // the first step
            t = 1.f / (float)mt.m;
        } else {
            float sum = 0.f;
            for (int k = threadIdx.x; k < mt.part_count; k += THREADS) sum += w.part[mt.part_first + k];
            t = sum_over(sum) / (float)mt.m;
            t = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, t)));
        }
        if (it.i == 0 && it.j == 0 && threadIdx.x == 0) w.t[it.mat] = t;
    } else {
        t = w.t[it.mat];
    }
    const float tx = t * inv2;  // of X, where t is of gamma X
    // to the next step's gamma; the last product's value is X itself
    const float change = STEP == kLast ? 1.f / gamma
                         : STEP == kNext ? fmaxf(gamma0 * (faded * co.fade), 1.f) / gamma : 1.f;
    const float linear = STEP == kPoly ? co.b + 2.f * co.c * tx
                                       : (co.a + (co.b + co.c * tx) * tx) * change;
    const float square = STEP == kPoly ? co.c * inv2 : inv2 * change;
    constexpr float unscale = 1.f / kScale;
    const float shift = STEP == kGram ? t * kScale : 0.f;
    const float factor = STEP == kGram ? unscale : square * unscale;

    // The old values of the linear term, 8 of a row per lane, are read a block of 32 x 64
    // ahead of their use, but where the registers are full (pairs, tiles of 256).
    constexpr bool kAhead = !(PAIRS && BT == 256);
    const int line = lane >> 3, eight = (lane & 7) * 8;  // of 8 rows, and 8 numbers of one
    constexpr int kRounds = 4 / KG, kBlocks = WR * WC / 2;
    struct Old {
        half8 hi[kRounds], lo[kRounds];
    } old[2];
    auto row_in_block = [&](int k) { return (group * kRounds + k) * 8 + line; };
    auto read_old = [&](int i1, int j1, Old &o) {
        if constexpr (STEP != kGram) {
#pragma unroll
            for (int k = 0; k < kRounds; ++k) {
                const int i = i1 + row_in_block(k), j = j1 + eight;
                const _Float16 *from = (STEP == kPoly ? d + i * d_pitch : x + i * x_pitch) + column<PAIRS>(j);
                o.hi[k] = *(const half8 *)from;
                if constexpr (PAIRS) o.lo[k] = *(const half8 *)(from + 32);
                else if constexpr (STEP != kPoly) o.lo[k] = *(const half8 *)(w.x_lo + ex + i * x_pitch + j);
            }
        }
    };
    auto block_row = [&](int n) { return i0 + wr + n / (WC / 2) * 32; };
    auto block_col = [&](int n) { return j0 + wc + n % (WC / 2) * 64; };
    if constexpr (KG > 1) read_old(block_row(0), block_col(0), old[0]);

    if constexpr (KG == 1) {
        // Each step's products run while the next step's fragments are read: two reads,
        // then one or two products, so that the reads are done well before the step is.
        constexpr int kReads = (WR + (kDeep ? 2 : 1) * WC) * kind;
        constexpr int kProducts = WR * WC * (PAIRS ? 3 : 1);
        constexpr int kGroup = kReads * 2 <= kProducts ? 2 : 1;
        constexpr int kRest = kProducts - kReads / 2 * kGroup;
        Fragments f[2];
        auto step_from = [&](const char *next, const char *b, int k, int parity) {
            load_from(next, b, k, f[parity ^ 1]);
            multiply(f[parity]);
#pragma unroll
            for (int g = 0; g < kReads / 2; ++g) {
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, kGroup, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, kRest, 0);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto step = [&](const char *next, int k, int parity) { step_from(next, next, k, parity); };
        auto inner = [&](const char *now, int parity) {  // all of a slab's steps but the last
#pragma unroll
            for (int k = 0; k < kSteps - 1; ++k) step(now, k + 1, (parity + k) & 1);
        };
        // At a slab's last step all waves have read their fragments of it: its buffer
        // takes the slab after the next, and the next one, a slab's time under way, is
        // waited for.  The loop begins there, so that nothing is under way where it
        // closes: the compiler would wait for all of it.
        constexpr int kLastParity = (kSteps - 1) & 1;
        static_assert(kLastParity == 1, "fragments change places an even number of times a slab");
        if constexpr (kSplit) {
            // X comes from memory, B from the L2 as a rule: half a slab of X is loaded again
            // as soon as it has been read, so that its loads have one and a half slab's
            // time.  Started in turn: the second half and A of a slab when the slab
            // before it begins, the first half of the slab after in its middle.  (A list of
            // 144 matrices, one slab's time for all loads and so: halves 8,248 and 8,089 us,
            // pairs 17,410 and 17,372.)
            constexpr int kHalfLoads = BT / 16 / kWaves, kLoadsA = BT / 8 / kWaves;
            static_assert(2 * kHalfLoads + kLoadsA < 16, "the counter's low bits");
            auto sync = [&](auto left) {  // all loads are there but the last `left`
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_waitcnt(0x0070 | decltype(left)::value);  // and all LDS reads
                bare_sync();
            };
            using std::integral_constant;
            constexpr integral_constant<int, 2 * kHalfLoads> at_begin{};
            constexpr integral_constant<int, 2 * kHalfLoads + kLoadsA> at_half{};
            // a slab's steps but the last, whose fragments of step 0 are there
            auto first_half = [&](const char *a, const char *x0) {
#pragma unroll
                for (int k = 1; k < kSteps / 2; ++k) step_from(a, x0, k, (k - 1) & 1);
            };
            auto second_half = [&](const char *a, const char *x1) {
#pragma unroll
                for (int k = kSteps / 2; k < kSteps; ++k) step_from(a, x1, k, (k - 1) & 1);
            };
            sync(at_begin);
            stage_a(1, buffer1);
            stage_x(3, x11);
            load_from(buffer0, x00, 0, f[0]);
            for (int s = 0; s + 2 < slabs; s += 2) {
                first_half(buffer0, x00);
                sync(at_half);
                stage_x(2 * s + 4, x00);
                second_half(buffer0, x01);
                sync(at_begin);
                stage_a(s + 2, buffer0);
                stage_x(2 * s + 5, x01);
                step_from(buffer1, x10, 0, 1);
                first_half(buffer1, x10);
                sync(at_half);
                stage_x(2 * s + 6, x10);
                second_half(buffer1, x11);
                sync(at_begin);
                stage_a(s + 3, buffer1);
                stage_x(2 * s + 7, x11);
                step_from(buffer0, x00, 0, 1);
            }
            first_half(buffer0, x00);
            sync(at_half);
            second_half(buffer0, x01);
            sync(integral_constant<int, kHalfLoads>{});
            step_from(buffer1, x10, 0, 1);
            first_half(buffer1, x10);
            staged_sync();
            second_half(buffer1, x11);
        } else {
            staged_sync();
            load(buffer0, 0, f[0]);
            inner(buffer0, 0);
            for (int s = 2; s < slabs; s += 2) {
                staged_sync();
                stage(s, buffer0);
                step(buffer1, 0, 1);
                inner(buffer1, 0);
                staged_sync();
                stage(s + 1, buffer1);
                step(buffer0, 0, 1);
                inner(buffer0, 0);
            }
            staged_sync();
            step(buffer1, 0, 1);
            inner(buffer1, 0);
        }
        multiply(f[1]);
        staged_sync();
    } else {
        const int rounds = (slabs + KG - 1) / KG;
        auto whole = [&](const char *from) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                Fragments f;
                load(from, k, f);
                multiply(f);
            }
        };
        // two slabs of the group are under way: the older one is waited for, and its
        // buffer filled again once all waves have read it
        constexpr int kLoads = 2 * BT / 8 / kWaves;  // of a wave for a slab
        auto round = [&](int s, char *from) {
            if (s < own) {
                if (s + 1 < own) __builtin_amdgcn_s_waitcnt(0x0f70 | kLoads);  // vmcnt(kLoads)
                else __builtin_amdgcn_s_waitcnt(0x0f70);
            }
            bare_sync();
            if (s < own) whole(from);
            bare_sync();
            if (s + 2 < own) stage((s + 2) * KG + group, from);
        };
        static_assert(kLoads < 16, "the counter's low bits");
        for (int s = 0; s < rounds; s += 2) {
            round(s, ours[0]);
            if (s + 1 < rounds) round(s + 1, ours[1]);
        }
        __syncthreads();
    }

    // The tile's values go through LDS, 32 x 64 of them at a time in a part of each
    // wave's own, to be read back 8 in a row: what is read and written in memory
    // is then whole lines.  A lane holds column (lane & 31) and, in register r, row
    // 8 (r / 4) + 4 (lane / 32) + r % 4 of a 32 x 32 product.
    // With several groups every wave leaves its sums there, and adds and finishes the
    // KG-th part of the rows that its group has.
    static_assert(KG == 1 || (4 % KG == 0 && WR == 1 && WC == 2), "some of 32 rows for a group");
    static_assert(kWaves * 2048 * 4 <= 2 * kOperand, "the epilogue's LDS");
    constexpr int kFit = kSplit ? kOperand / 8192 : KG * kWaves;  // waves in buffer0
    float *const mine = wave_number() < kFit ? (float *)buffer0 + wave_number() * 2048
                                             : (float *)buffer1 + (wave_number() - kFit) * 2048;
    // the first group's
    float *const sums = kSplit ? mine : (float *)buffer0 + wave * 2048;
    auto part_sync = [&] {
        if constexpr (KG > 1) __syncthreads();
        else wave_sync();
    };
    const int col = lane & 31, quad = (lane >> 5) * 4;
    auto place = [&](int r, int c) { return r * 64 + (((c >> 2) ^ r) & 15) * 4 + (c & 3); };
    auto take = [&](int r, float (&v)[8]) {
        f32x4 lo = *(const f32x4 *)(sums + place(r, eight));
        f32x4 hi = *(const f32x4 *)(sums + place(r, eight + 4));
#pragma unroll
        for (int g = 1; g < KG; ++g) {
            lo += *(const f32x4 *)(sums + g * kWaves * 2048 + place(r, eight));
            hi += *(const f32x4 *)(sums + g * kWaves * 2048 + place(r, eight + 4));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = lo[k];
            v[4 + k] = hi[k];
        }
    };
    float squares = 0.f;
    // the values of 8 numbers of the output's row i from column j on, from their sums
    auto value = [&](int i, int j, const Old &o, int k8, float (&v)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= factor;
        if constexpr (STEP == kGram) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i == j + k && i < mt.m) v[k] -= shift;
        } else {
            constexpr bool kLo = PAIRS || STEP != kPoly;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[k] += linear * (kLo ? (float)o.hi[k8][k] + (float)o.lo[k8][k] : (float)o.hi[k8][k]);
        }
    };
    auto store = [&](int i, int j, const float (&v)[8]) {
        half8 hi, lo;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            _Float16 h, l;
            split(v[k], h, l);
            hi[k] = h;
            lo[k] = l;
        }
        _Float16 *to = STEP == kNext ? w.x_next + ex + i * x_pitch
                                     : (STEP == kGram ? w.d : w.b) + em + i * d_pitch;
        *(half8 *)(to + column<PAIRS>(j)) = hi;
        if constexpr (PAIRS) *(half8 *)(to + column<PAIRS>(j) + 32) = lo;
        else if constexpr (STEP == kNext) *(half8 *)(w.x_lo + ex + i * x_pitch + j) = lo;
    };
    if constexpr (KG == 1) read_old(block_row(0), block_col(0), old[0]);
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {  // 32 rows x 64 columns
        const int p = n / (WC / 2), qq = n % (WC / 2) * 2;
        if (kAhead && n + 1 < kBlocks) read_old(block_row(n + 1), block_col(n + 1), old[(n + 1) & 1]);
        if (!kAhead && n > 0) read_old(block_row(n), block_col(n), old[n & 1]);
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                mine[place((r >> 2) * 8 + quad + (r & 3), q * 32 + col)] = acc[p][qq + q][r];
        part_sync();
        const int i1 = block_row(n), j1 = block_col(n);
        // A tile in parts: every workgroup leaves its sums, and the last one to have done
        // so (the counter, which it sets back) adds all of them in order and goes on.
        if constexpr (kInParts) {
            if (mt.parts > 1) {
                auto at = [&](int part, int k) {
                    return w.sums + mt.sums +
                           ((int64_t)(it.slot - mt.slot_first) * mt.parts + part) * (BT * BT) +
                           (wr + row_in_block(k)) * BT + wc + eight;
                };
#pragma unroll
                for (int k = 0; k < kRounds; ++k) {
                    float v[8];
                    take(row_in_block(k), v);
                    __builtin_memcpy(at(it.part, k), v, sizeof v);
                }
                // One thread's release and acquire stand for the workgroup's: every wave's
                // stores have reached the L2 before the barrier, and what they read after
                // the next one comes from behind it.  (A fence writes the whole L2 back:
                // one in every wave took 86 us where the products take 30.)
                staged_sync();
                if (threadIdx.x == 0) {
                    // The wait for the write-back is stated: behind a wait for all stores
                    // the compiler takes the release's own for done and leaves it out.
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    const uint32_t before = __hip_atomic_fetch_add(
                        w.counter + it.slot, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
                    scratch[0] = before + 1 == (uint32_t)mt.parts ? 1.f : 0.f;
                    if (before + 1 == (uint32_t)mt.parts)
                        __hip_atomic_store(w.counter + it.slot, 0u, __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_AGENT);
                }
                __syncthreads();
                if (scratch[0] == 0.f) return;
#pragma unroll
                for (int k = 0; k < kRounds; ++k) {
                    float v[8] = {};
                    for (int q = 0; q < mt.parts; ++q) {
                        float one[8];
                        __builtin_memcpy(one, at(q, k), sizeof one);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += one[e];
                    }
                    const int i = i1 + row_in_block(k), j = j1 + eight;
                    value(i, j, old[0], k, v);
                    store(i, j, v);
                }
                return;
            }
        }
#pragma unroll
        for (int k = 0; k < kRounds; ++k) {
            const int r = row_in_block(k), i = i1 + r, j = j1 + eight;
            float v[8];
            take(r, v);
            value(i, j, old[n & 1], k, v);
            if constexpr (STEP == kLast) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= unscale;
                if (!mt.flip) {
                    if (i < mt.m && j < mt.n)
                        out.put(mt.off + i * mt.ld + j, v, mt.n - j,
                                muon_scale(scale_mode, mt.rows, mt.cols));
                } else {  // back, to be read along the columns
                    *(f32x4 *)(sums + place(r, eight)) = f32x4{v[0], v[1], v[2], v[3]};
                    *(f32x4 *)(sums + place(r, eight + 4)) = f32x4{v[4], v[5], v[6], v[7]};
                }
            } else {
                if constexpr (STEP == kNext)
#pragma unroll
                    for (int e = 0; e < 8; ++e) squares += (v[e] * unscale) * (v[e] * unscale);
                store(i, j, v);
            }
        }
        part_sync();
        if constexpr (STEP == kLast) {
            if (mt.flip) {
#pragma unroll
                for (int k = 0; k < kRounds; ++k) {
                    const int c = (group * kRounds + k) * 16 + (lane >> 2), r = (lane & 3) * 8;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = sums[place(r + e, c)];
                    if (i1 + r < mt.m && j1 + c < mt.n)
                        out.put(mt.off + (j1 + c) * mt.ld + i1 + r, v, mt.m - (i1 + r),
                                muon_scale(scale_mode, mt.rows, mt.cols));
                }
                part_sync();
            }
        }
    }
    if constexpr (STEP == kNext) {
        const float sum = sum_over(squares);
        if (threadIdx.x == 0) w.part[mt.part_first + it.i * (mt.np / BT) + it.j] = sum;
    }
    if constexpr ((STEP == kGram || STEP == kPoly) && KG == 1) {
        if (it.i == it.j) return;  // a diagonal tile is its own transpose
        constexpr int kTurned = WC * WR / 2;  // of 32 columns x 64 rows
        auto turned_row = [&](int n) { return j0 + wc + n / (WR / 2) * 32; };
        auto turned_col = [&](int n) { return i0 + wr + n % (WR / 2) * 64; };
        read_old(turned_row(0), turned_col(0), old[0]);
#pragma unroll
        for (int n = 0; n < kTurned; ++n) {
            const int q = n / (WR / 2), pp = n % (WR / 2) * 2;
            if (kAhead && n + 1 < kTurned) read_old(turned_row(n + 1), turned_col(n + 1), old[(n + 1) & 1]);
            if (!kAhead && n > 0) read_old(turned_row(n), turned_col(n), old[n & 1]);
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(f32x4 *)(mine + place(col, p * 32 + g * 8 + quad)) =
                        f32x4{acc[pp + p][q][g * 4], acc[pp + p][q][g * 4 + 1],
                              acc[pp + p][q][g * 4 + 2], acc[pp + p][q][g * 4 + 3]};
            wave_sync();
#pragma unroll
            for (int k = 0; k < kRounds; ++k) {
                const int r = row_in_block(k), i = turned_row(n) + r, j = turned_col(n) + eight;
                float v[8];
                take(r, v);
                value(i, j, old[n & 1], k, v);
                store(i, j, v);
            }
            wave_sync();
        }
    }
}

}  // namespace
}  // namespace onebit

using namespace onebit;

// The tiles of one of a step's products and the kernel that forms them.
struct Product {
    int side = 0, groups = 1;  // of a tile; of waves (k_product's KG)
    int64_t blocks = 0;
    const MatTile *tiles = nullptr;
};

// What a call needs for one kind of products.
struct Side {
    int64_t ex = 0, em = 0, firsts = 0, parts = 0, slots = 0, sums = 0;
    const Mat *mats = nullptr;
    const Item *first_items = nullptr;
    Product gram, poly, next;
};

struct onebit_matrices_s {
    int device = 0;
    int32_t count = 0;
    int64_t extent = 0, norms = 0;
    int norm_size = 0;  // elements per workgroup of the norm
    bool empty = true;
    std::vector<int64_t> offset;
    char *dev = nullptr;
    const Item *norm_items = nullptr;
    Side side[2];  // by ONEBIT_PRODUCTS_*
};

namespace {

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

#define TRY(expr)                         \
    do {                                  \
        int _st = (expr);                 \
        if (_st != ONEBIT_OK) return _st; \
    } while (0)

struct WorkspaceLayout {
    size_t x0, x1, x_lo, d, b, norm, part, t, gamma, counter, sums, total;
};

WorkspaceLayout layout_of(const onebit_matrices_s *p, bool pairs)
{
    const Side &s = p->side[pairs ? ONEBIT_PRODUCTS_F32 : ONEBIT_PRODUCTS_F16];
    WorkspaceLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    const size_t half = pairs ? 4 : 2;
    l.x0 = take(half * s.ex);
    l.x1 = take(half * s.ex);
    l.x_lo = take(pairs ? 0 : 2 * s.ex);
    l.d = take(half * s.em);
    l.b = take(half * s.em);
    l.norm = take(8 * (size_t)p->norms);
    l.part = take(4 * (size_t)s.parts);
    l.t = take(4 * (size_t)p->count);
    l.gamma = take(4 * (size_t)p->count);
    l.counter = take(4 * (size_t)s.slots);
    l.sums = take(4 * (size_t)s.sums);
    l.total = at;
    return l;
}

// Workgroups go to the XCDs round-robin, and each XCD has an L2 of its own: a
// matrix's tiles go to one XCD as far as that keeps the XCDs' work even.  Tiles
// (with what one costs, the dearest first) are dealt out in runs of one matrix, each
// to the XCD with the least so far; entry x * length + k is XCD x's k-th.
struct Costed {
    MatTile tile;
    double cost;
};

std::vector<MatTile> deal(std::vector<Costed> &all)
{
    std::stable_sort(all.begin(), all.end(),
                     [](const Costed &a, const Costed &b) { return a.cost > b.cost; });
    double total = 0;
    for (const Costed &c : all) total += c.cost;
    const double most = total / (kXcds * 8) * (1 + 1e-9);  // of a run
    std::vector<MatTile> lists[kXcds];
    double load[kXcds] = {};
    for (size_t k = 0; k < all.size();) {
        const int to = (int)(std::min_element(load, load + kXcds) - load);
        double run = 0;
        const int32_t mat = all[k].tile.mat;
        do {
            lists[to].push_back(all[k].tile);
            run += all[k].cost;
            ++k;
        } while (k < all.size() && all[k].tile.mat == mat && run + all[k].cost <= most);
        load[to] += run;
    }
    size_t length = 0;
    for (const auto &l : lists) length = std::max(length, l.size());
    MatTile none{};
    none.mat = -1;
    std::vector<MatTile> out(length * kXcds, none);
    for (int x = 0; x < kXcds; ++x)
        std::copy(lists[x].begin(), lists[x].end(), out.begin() + x * length);
    return out;
}

// The kernels' shapes, and what a tile of each costs: us for a tile and for each of
// its slabs, for pairs and for halves, on a CU that has as many of them as fit;
// and for each slab of a tile that has its CU to itself.  (Fitted to lists of 1 to
// 96 matrices, 17 x 4,000 to 4,096 x 4,096.)  us of whole calls with each shape alone,
// and with those that are chosen:
//                                       64 x 4   64 x 2      128      256   chosen
//   12 of 128 x 128 to 512, pairs          101      100      149      392      101
//   11 of 17 x 4,000 to 1,001 x 257, pairs 198      277      517    1,383      177
//   1,024 x 1,024, halves                  133      141      229      433      133
//   4 of them, halves                      428      329      263      450      263
//   16 of them, pairs                    2,719    2,081    1,239    1,284    1,228
//   144 of 1,024 x 1,024 to 4,096, halves 23,602  16,987    9,022    8,089    8,089
struct Shape {
    int side, groups;
    double tile[2], slab[2], alone[2];
};
constexpr Shape kShapes[] = {
    {64, 4, {4.5, 4.5}, {0.26, 0.25}, {0.26, 0.25}},
    {64, 2, {2.5, 2.5}, {0.21, 0.21}, {0.37, 0.39}},
    {128, 1, {7.0, 5.0}, {0.64, 0.64}, {0.64, 0.64}},
    {256, 1, {10.0, 12.0}, {2.65, 2.30}, {2.65, 2.30}},
};
constexpr int kCus = 256;
constexpr int kPartSlabs = 16;    // least slabs of a part
constexpr double kPartCost = 6.0;  // us that a part's join adds

struct Sizes {
    int64_t m, n;
};

int64_t pad_to(int64_t v, int64_t side) { return (v + side - 1) / side * side; }

// Tiles of a product of one matrix (rows of tiles, and per row r their number).
int64_t tiles_of(const Sizes &z, const Shape &h, int pad, bool symmetric)
{
    const int64_t tm = pad_to(z.m, pad) / h.side, tn = pad_to(z.n, pad) / h.side;
    return !symmetric ? tm * tn : h.groups > 1 ? tm * tm : tm * (tm + 1) / 2;
}

// Slabs of a part of a Gram tile's sum: the fewest, and at least kPartSlabs, with
// which the workgroups are no more than the CUs, or than a quarter above the tiles.
int64_t part_slabs(const std::vector<Sizes> &all, const Shape &h, int pad, int kind)
{
    constexpr int64_t kWhole = (int64_t)1 << 40;
    if (h.groups != kPartGroups) return kWhole;
    int64_t tiles = 0, longest = 0;
    for (const Sizes &z : all) {
        tiles += tiles_of(z, h, pad, true);
        longest = std::max(longest, pad_to(z.n, pad) * kind / kSlab);
    }
    const int64_t most = std::max<int64_t>(kCus, tiles + tiles / 4);
    for (int64_t slabs = kPartSlabs; slabs < longest; slabs += slabs / 4) {
        int64_t parts = 0;
        for (const Sizes &z : all)
            parts += tiles_of(z, h, pad, true) * ((pad_to(z.n, pad) * kind / kSlab + slabs - 1) / slabs);
        if (parts <= most) return slabs;
    }
    return kWhole;
}

int parts_of(const Sizes &z, int pad, int kind, int64_t part)
{
    return (int)((pad_to(z.n, pad) * kind / kSlab + part - 1) / part);
}

// Estimated us of a launch: every tile goes to the CU that is free first, the dearest
// first; for long lists the mean and half of a tile.
enum Which { kIsGram, kIsPoly, kIsNext };
double launch_cost(const std::vector<Sizes> &all, const Shape &h, int pad, Which which, int kind)
{
    const int p = kind == 2 ? 0 : 1;
    const int64_t part = which == kIsGram ? part_slabs(all, h, pad, kind) : 0;
    std::vector<std::pair<double, int64_t>> work;  // cost, how many
    double total = 0, dearest = 0, longest = 0;
    for (const Sizes &z : all) {
        int64_t count = tiles_of(z, h, pad, which != kIsNext);
        double slabs = (double)(pad_to(which == kIsGram ? z.n : z.m, pad) * kind / kSlab);
        double join = 0;
        if (which == kIsGram) {
            const int parts = parts_of(z, pad, kind, part);
            count *= parts;
            slabs /= parts;
            join = parts > 1 ? kPartCost : 0;
        }
        const double cost = h.tile[p] + h.slab[p] * slabs + join;
        longest = std::max(longest, h.tile[p] + h.alone[p] * slabs + join);
        work.push_back({cost, count});
        total += cost * (double)count;
        dearest = std::max(dearest, cost);
    }
    if (total > 64.0 * kCus * dearest) return std::max(total / kCus + dearest / 2, longest);
    std::sort(work.rbegin(), work.rend());
    std::vector<double> cus(kCus, 0.0);  // a heap, the earliest on top
    auto later = [](double a, double b) { return a > b; };
    double last = longest;
    for (const auto &[cost, count] : work)
        for (int64_t k = 0; k < count; ++k) {
            std::pop_heap(cus.begin(), cus.end(), later);
            last = std::max(last, cus.back() += cost);
            std::push_heap(cus.begin(), cus.end(), later);
        }
    return last;
}

// Chooses the three products' kernels: the last one's tile sets the padding, and the
// other two take no larger one.
void choose(const std::vector<Sizes> &all, int kind, Shape (&best)[3])
{
    double least = INFINITY;
    for (const Shape &next : kShapes) {
        double cost = launch_cost(all, next, next.side, kIsNext, kind);
        Shape pick[3] = {next, next, next};
        for (int which = 0; which < 2; ++which) {
            double lowest = INFINITY;
            for (const Shape &h : kShapes) {
                if (h.side > next.side) continue;
                const double c = launch_cost(all, h, next.side, (Which)which, kind);
                if (c < lowest) {
                    lowest = c;
                    pick[which] = h;
                }
            }
            cost += lowest;
        }
        if (cost < least) {
            least = cost;
            std::copy(pick, pick + 3, best);
        }
    }
}

// Tables of one side, on the host.
struct Built {
    std::vector<Mat> mats;
    std::vector<Item> first;
    std::vector<MatTile> gram, poly, next;
};

int build_side(std::vector<Mat> mats, int kind, Side &side, Built &out)
{
    constexpr int64_t kItems = 1 << 22;
    std::vector<Sizes> sizes;
    for (const Mat &m : mats)
        if (m.m > 0) sizes.push_back(Sizes{m.m, m.n});
    if (sizes.empty()) {
        out.mats = std::move(mats);
        return ONEBIT_OK;
    }
    Shape shape[3];
    choose(sizes, kind, shape);
    const int pad = shape[kIsNext].side, p = kind == 2 ? 0 : 1;
    const int64_t part = part_slabs(sizes, shape[kIsGram], pad, kind);
    std::vector<Costed> lists[3];
    int64_t tiles = 0;
    for (size_t k = 0; k < mats.size(); ++k) {
        Mat &m = mats[k];
        if (m.m == 0) continue;
        const Sizes z{m.m, m.n};
        m.mp = (int32_t)pad_to(m.m, pad);
        m.np = (int32_t)pad_to(m.n, pad);
        m.ex = side.ex;
        m.em = side.em;
        side.ex += (int64_t)m.mp * m.np;
        side.em += (int64_t)m.mp * m.mp;
        m.part_first = (int32_t)side.parts;
        m.part_count = (int32_t)tiles_of(z, shape[kIsNext], pad, false);
        side.parts += m.part_count;
        m.slot_first = (int32_t)side.slots;
        const int parts = m.parts = parts_of(z, pad, kind, part);
        m.sums = side.sums;
        if (parts > 1) m.slot_count = (int32_t)tiles_of(z, shape[kIsGram], pad, true);
        side.slots += m.slot_count;
        side.sums += (int64_t)m.slot_count * parts * shape[kIsGram].side * shape[kIsGram].side;
        const int rp = (m.flip ? m.np : m.mp) / kPrep, cp = (m.flip ? m.mp : m.np) / kPrep;
        for (int which = 0; which < 3; ++which) tiles += tiles_of(z, shape[which], pad, which != kIsNext);
        if (tiles > kItems || (int64_t)out.first.size() + (int64_t)rp * cp > kItems)
            return fail(ONEBIT_EINVAL, "too many tiles (matrix %d)", (int)k);
        for (int i = 0; i < rp; ++i)
            for (int j = 0; j < cp; ++j) out.first.push_back(Item{(int32_t)k, (uint16_t)i, (uint16_t)j});
        int32_t slot = m.slot_first;
        for (int which = 0; which < 3; ++which) {
            const Shape &h = shape[which];
            const int tm = m.mp / h.side, tn = which == kIsNext ? m.np / h.side : tm;
            const int split = which == kIsGram ? parts : 1;
            const double slabs = (double)((which == kIsGram ? m.np : m.mp) * kind / kSlab) / split;
            for (int i = 0; i < tm; ++i)
                for (int j = 0; j < (which == kIsNext || h.groups > 1 ? tn : i + 1); ++j) {
                    MatTile t{};
                    t.mat = (int32_t)k;
                    t.i = (uint16_t)i;
                    t.j = (uint16_t)j;
                    t.slot = split > 1 ? slot++ : 0;
                    for (t.part = 0; t.part < split; ++t.part)
                        lists[which].push_back(Costed{t, h.tile[p] + h.slab[p] * slabs});
                }
        }
    }
    out.gram = deal(lists[kIsGram]);
    out.poly = deal(lists[kIsPoly]);
    out.next = deal(lists[kIsNext]);
    side.firsts = (int64_t)out.first.size();
    side.gram = Product{shape[kIsGram].side, shape[kIsGram].groups, (int64_t)out.gram.size(), nullptr};
    side.poly = Product{shape[kIsPoly].side, shape[kIsPoly].groups, (int64_t)out.poly.size(), nullptr};
    side.next = Product{shape[kIsNext].side, shape[kIsNext].groups, (int64_t)out.next.size(), nullptr};
    out.mats = std::move(mats);
    return ONEBIT_OK;
}

int check_sides(int k, int64_t r, int64_t c)
{
    constexpr int64_t kSide = 1 << 20;
    if (r < 0 || c < 0 || r > kSide || c > kSide)
        return fail(ONEBIT_EINVAL, "matrix %d is %lld x %lld: a side is at most 2^20", k,
                    (long long)r, (long long)c);
    if (r * c >= ((int64_t)1 << 31))
        return fail(ONEBIT_EINVAL, "matrix %d has 2^31 elements or more", k);
    return ONEBIT_OK;
}

int create_impl(const int64_t *rows, const int64_t *cols, const int64_t *offset,
                const int64_t *ld, int32_t count, onebit_matrices *out)
{
    std::unique_ptr<onebit_matrices_s> p(new onebit_matrices_s);
    hipError_t e = hipGetDevice(&p->device);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    std::vector<Mat> mats(count);
    std::vector<Item> norm;
    p->count = count;
    p->offset.resize(count);
    int64_t at = 0;
    // 2,048 elements are one load per thread; four where that still makes many workgroups
    double elements = 0;
    for (int32_t k = 0; k < count; ++k) elements += (double)rows[k] * (double)cols[k];
    const int size = p->norm_size = elements <= (1 << 23) ? 2048 : 8192;
    constexpr int64_t kMost = (int64_t)1 << 40, kItems = 1 << 23;
    for (int32_t k = 0; k < count; ++k) {
        const int64_t r = rows[k], c = cols[k];
        TRY(check_sides(k, r, c));
        const int64_t pitch = ld ? ld[k] : c;
        const int64_t off = offset ? offset[k] : at;
        if (pitch < c || pitch > kMost)
            return fail(ONEBIT_EINVAL, "ld[%d] = %lld, %lld columns", k, (long long)pitch,
                        (long long)c);
        if (off < 0 || off > kMost)
            return fail(ONEBIT_EINVAL, "offset[%d] = %lld", k, (long long)off);
        // (r - 1) * pitch < 2^60
        const int64_t span = r > 0 && c > 0 ? (r - 1) * pitch + c : 0;
        if (off + span > kMost)
            return fail(ONEBIT_EINVAL, "matrix %d ends above 2^40 elements", k);
        p->offset[k] = off;
        at = off + (span + 63) / 64 * 64;
        p->extent = std::max(p->extent, off + span);
        Mat &m = mats[k];
        std::memset(&m, 0, sizeof m);
        m.off = off;
        m.ld = pitch;
        m.rows = (int32_t)r;
        m.cols = (int32_t)c;
        m.flip = r > c;
        m.m = (int32_t)std::min(r, c);
        m.n = (int32_t)std::max(r, c);
        if (m.m == 0) continue;
        p->empty = false;
        m.norm_first = (int32_t)norm.size();
        m.norm_count = (int32_t)((r * c + size - 1) / size);
        if ((int64_t)norm.size() + m.norm_count > kItems)
            return fail(ONEBIT_EINVAL, "too many elements (matrix %d)", k);
        for (int32_t q = 0; q < m.norm_count; ++q)
            norm.push_back(Item{k, (uint16_t)(q >> 16), (uint16_t)q});
    }
    p->norms = (int64_t)norm.size();
    Built built[2];
    TRY(build_side(mats, 2, p->side[ONEBIT_PRODUCTS_F32], built[ONEBIT_PRODUCTS_F32]));
    TRY(build_side(mats, 1, p->side[ONEBIT_PRODUCTS_F16], built[ONEBIT_PRODUCTS_F16]));
    // one host buffer in the layout of the device allocation
    std::vector<char> host;
    auto put = [&](const auto &v) {
        const size_t here = host.size();
        host.resize(here + up256(std::max<size_t>(v.size() * sizeof(v[0]), 1)));
        if (!v.empty()) std::memcpy(host.data() + here, v.data(), v.size() * sizeof(v[0]));
        return here;
    };
    const size_t o_norm = put(norm);
    size_t o[2][5];
    for (int k = 0; k < 2; ++k) {
        o[k][0] = put(built[k].mats);
        o[k][1] = put(built[k].first);
        o[k][2] = put(built[k].gram);
        o[k][3] = put(built[k].poly);
        o[k][4] = put(built[k].next);
    }
    void *dev = nullptr;
    e = hipMalloc(&dev, host.size());
    if (e == hipErrorOutOfMemory) return fail(ONEBIT_ENOMEM, "hipMalloc of the matrix tables");
    if (e != hipSuccess) return hip_fail(e, "hipMalloc");
    e = hipMemcpy(dev, host.data(), host.size(), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        (void)hipFree(dev);
        return hip_fail(e, "copy of the matrix tables");
    }
    p->dev = (char *)dev;
    p->norm_items = (const Item *)(p->dev + o_norm);
    for (int k = 0; k < 2; ++k) {
        Side &s = p->side[k];
        s.mats = (const Mat *)(p->dev + o[k][0]);
        s.first_items = (const Item *)(p->dev + o[k][1]);
        s.gram.tiles = (const MatTile *)(p->dev + o[k][2]);
        s.poly.tiles = (const MatTile *)(p->dev + o[k][3]);
        s.next.tiles = (const MatTile *)(p->dev + o[k][4]);
    }
    *out = p.release();
    return ONEBIT_OK;
}

int kernels_impl(const int64_t *rows, const int64_t *cols, int32_t count, int kind,
                 int32_t (&side)[3], int32_t (&groups)[3], int32_t &parts)
{
    std::vector<Sizes> sizes;
    for (int32_t k = 0; k < count; ++k) {
        TRY(check_sides(k, rows[k], cols[k]));
        if (rows[k] > 0 && cols[k] > 0)
            sizes.push_back(Sizes{std::min(rows[k], cols[k]), std::max(rows[k], cols[k])});
    }
    if (sizes.empty()) return ONEBIT_OK;
    Shape shape[3];
    choose(sizes, kind, shape);
    for (int k = 0; k < 3; ++k) {
        side[k] = shape[k].side;
        groups[k] = shape[k].groups;
    }
    const int pad = shape[kIsNext].side;
    const int64_t part = part_slabs(sizes, shape[kIsGram], pad, kind);
    for (const Sizes &z : sizes) parts = std::max(parts, parts_of(z, pad, kind, part));
    return ONEBIT_OK;
}

int check_mats(const onebit_matrices_s *p)
{
    if (!p) return fail(ONEBIT_EINVAL, "matrices handle is NULL");
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != p->device)
        return fail(ONEBIT_EINVAL, "matrices were created on device %d, current device is %d",
                    p->device, dev);
    return ONEBIT_OK;
}

int type_bytes(int32_t dtype)
{
    return dtype == ONEBIT_GRAD_F32 ? 4
         : dtype == ONEBIT_GRAD_BF16 || dtype == ONEBIT_GRAD_F16 ? 2 : 0;
}

int check_buffer(const onebit_matrices_s *p, const void *ptr, int32_t dtype, const char *name)
{
    const int bytes = type_bytes(dtype);
    if (!bytes) return fail(ONEBIT_EINVAL, "%s: type %d is not one of ONEBIT_GRAD_*", name, dtype);
    if (!ptr && p->extent > 0) return fail(ONEBIT_EINVAL, "%s is NULL", name);
    if ((uintptr_t)ptr % bytes) return fail(ONEBIT_EALIGN, "%s is not %d-byte aligned", name, bytes);
    return ONEBIT_OK;
}

// Bounds of the iteration: every singular value starts in [0, 1]; a step maps s
// to s q(s^2), q(v) = a + b v + c v^2.  Refuses coefficients with which a singular
// value, its square or q's change over the interval could leave kRange (for iterates held times
// gamma: E is at most 1).  Sets fade: a step multiplies by |q| at most.
int check_coefficients(Coefficients &k, int steps)
{
    if (!std::isfinite(k.a) || !std::isfinite(k.b) || !std::isfinite(k.c))
        return fail(ONEBIT_EINVAL, "coefficients are not finite");
    const double a = k.a, b = k.b, c = k.c;
    double top = 1.0, growth = 1.0;
    for (int s = 0; s < steps; ++s) {
        const double v1 = top * top;
        auto q = [&](double v) { return a + (b + c * v) * v; };
        double lo = std::min(q(0), q(v1)), hi = std::max(q(0), q(v1));
        double peak = std::fabs(top * q(v1));
        if (c != 0) {
            const double v = -b / (2 * c);  // q's extremum
            if (v > 0 && v < v1) lo = std::min(lo, q(v)), hi = std::max(hi, q(v));
        }
        // extrema of s q(s^2): a + 3 b v + 5 c v^2 = 0
        const double disc = 9 * b * b - 20 * a * c;
        double roots[2] = {-1, -1};
        if (c != 0 && disc >= 0) {
            roots[0] = (-3 * b + std::sqrt(disc)) / (10 * c);
            roots[1] = (-3 * b - std::sqrt(disc)) / (10 * c);
        } else if (c == 0 && b != 0) {
            roots[0] = -a / (3 * b);
        }
        for (double v : roots)
            if (v > 0 && v < v1) peak = std::max(peak, std::sqrt(v) * std::fabs(q(v)));
        growth = std::max(growth, std::max(std::fabs(lo), std::fabs(hi)));
        if (v1 > kRange || std::fabs(b) + 0.75 * std::fabs(c) > kRange || hi - lo > kRange || peak > kRange)
            return fail(ONEBIT_EINVAL, "coefficients %g, %g, %g leave the range of the products "
                        "at step %d", a, b, c, s + 1);
        top = std::max(peak * 1.001, 1e-3);
    }
    k.fade = (float)std::exp2(-std::ceil(std::log2(growth * 1.001)));
    return ONEBIT_OK;
}

template <bool PAIRS, int STEP, class O>
void launch(const Mat *mats, const Product &p, const Areas &w, const Coefficients &co, float faded, const O &out,
            int scale_mode, hipStream_t st)
{
    auto run = [&](auto side, auto wr, auto wc, auto groups) {
        constexpr int BT = decltype(side)::value, WR = decltype(wr)::value, WC = decltype(wc)::value;
        constexpr int KG = decltype(groups)::value, kThreads = KG * BT * BT / (16 * WR * WC);
        k_product<PAIRS, STEP, BT, WR, WC, KG, kThreads, O><<<p.blocks, kThreads, 0, st>>>(
            mats, p.tiles, w, co, faded, out, scale_mode);
    };
    using std::integral_constant;
    if (p.side == 256)
        run(integral_constant<int, 256>{}, integral_constant<int, 4>{}, integral_constant<int, 2>{},
            integral_constant<int, 1>{});
    else if (p.side == 128)
        run(integral_constant<int, 128>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{},
            integral_constant<int, 1>{});
    else if (p.groups == 4)
        run(integral_constant<int, 64>{}, integral_constant<int, 1>{}, integral_constant<int, 2>{},
            integral_constant<int, 4>{});
    else
        run(integral_constant<int, 64>{}, integral_constant<int, 1>{}, integral_constant<int, 2>{},
            integral_constant<int, 2>{});
}

// Everything after the arguments' checks: `src` is what is orthogonalised.
template <bool PAIRS, class S, class O>
int run(const onebit_matrices_s *p, const S &src, const O &out, int scale_mode, int steps,
        const Coefficients &co, float eps, void *workspace, hipStream_t st)
{
    const Side &side = p->side[PAIRS ? ONEBIT_PRODUCTS_F32 : ONEBIT_PRODUCTS_F16];
    const WorkspaceLayout l = layout_of(p, PAIRS);
    char *ws = (char *)workspace;
    Areas w{(_Float16 *)(ws + l.x0), (_Float16 *)(ws + l.x1), (_Float16 *)(ws + l.x_lo),
            (_Float16 *)(ws + l.d), (_Float16 *)(ws + l.b),
            (double *)(ws + l.norm), (float *)(ws + l.part), (float *)(ws + l.t),
            (float *)(ws + l.gamma), (uint32_t *)(ws + l.counter), (float *)(ws + l.sums)};
    k_norm<S><<<(int)p->norms, 256, 0, st>>>(side.mats, p->norm_items, p->norm_size, src, w.norm);
    k_first<PAIRS, S><<<(int)side.firsts, 256, 0, st>>>(side.mats, side.first_items, src,
                                                        (double)eps, w);
    float faded = 1.f;
    for (int k = 0; k < steps; ++k, faded *= co.fade) {
        launch<PAIRS, kGram>(side.mats, side.gram, w, co, faded, NoOut{}, 0, st);
        launch<PAIRS, kPoly>(side.mats, side.poly, w, co, faded, NoOut{}, 0, st);
        if (k + 1 < steps) launch<PAIRS, kNext>(side.mats, side.next, w, co, faded, NoOut{}, 0, st);
        else launch<PAIRS, kLast>(side.mats, side.next, w, co, faded, out, scale_mode, st);
        std::swap(w.x, w.x_next);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ONEBIT_OK : hip_fail(e, "matrix kernel launch");
}

int check_common(const onebit_matrices_s *p, int32_t products, int32_t steps,
                 const float *coefficients, float eps, const void *workspace, Coefficients &co)
{
    if (products != ONEBIT_PRODUCTS_F32 && products != ONEBIT_PRODUCTS_F16)
        return fail(ONEBIT_EINVAL, "products %d is not one of ONEBIT_PRODUCTS_*", products);
    if (steps < 1 || steps > 64) return fail(ONEBIT_EINVAL, "steps = %d is not in 1..64", steps);
    if (!(eps > 0) || !std::isfinite(eps)) return fail(ONEBIT_EINVAL, "eps must be above 0");
    co = coefficients ? Coefficients{coefficients[0], coefficients[1], coefficients[2], 1.f}
                      : Coefficients{3.4445f, -4.7750f, 2.0315f, 1.f};
    TRY(check_coefficients(co, steps));
    if (!workspace && !p->empty) return fail(ONEBIT_EINVAL, "workspace is NULL");
    if ((uintptr_t)workspace % 256) return fail(ONEBIT_EALIGN, "workspace is not 256-byte aligned");
    return ONEBIT_OK;
}

// f is called with a null pointer of the element type.
template <class F>
int with_type(int32_t dtype, F &&f)
{
    if (dtype == ONEBIT_GRAD_F32) return f((float *)nullptr);
    if (dtype == ONEBIT_GRAD_BF16) return f((__bf16 *)nullptr);
    return f((_Float16 *)nullptr);
}

}  // namespace

extern "C" {

int onebit_matrices_create(const int64_t *rows, const int64_t *cols, const int64_t *offset,
                           const int64_t *ld, int32_t count, onebit_matrices *out)
{
    if (!out) return fail(ONEBIT_EINVAL, "out is NULL");
    *out = nullptr;
    if (!rows || !cols) return fail(ONEBIT_EINVAL, "rows or cols is NULL");
    if (count < 1) return fail(ONEBIT_EINVAL, "count < 1");
    try {
        return create_impl(rows, cols, offset, ld, count, out);
    } catch (const std::bad_alloc &) {
        return fail(ONEBIT_ENOMEM, "host memory for the matrix tables");
    }
}

int onebit_matrices_destroy(onebit_matrices mats)
{
    if (!mats) return fail(ONEBIT_EINVAL, "matrices handle is NULL");
    const hipError_t e = mats->dev ? hipFree(mats->dev) : hipSuccess;
    delete mats;
    return e == hipSuccess ? ONEBIT_OK : hip_fail(e, "hipFree");
}

int onebit_matrices_info(onebit_matrices mats, int32_t products, int64_t *extent,
                         int64_t *offset, size_t *workspace_bytes)
{
    if (!mats) return fail(ONEBIT_EINVAL, "matrices handle is NULL");
    if (products != ONEBIT_PRODUCTS_F32 && products != ONEBIT_PRODUCTS_F16)
        return fail(ONEBIT_EINVAL, "products %d is not one of ONEBIT_PRODUCTS_*", products);
    if (extent) *extent = mats->extent;
    if (offset) std::copy(mats->offset.begin(), mats->offset.end(), offset);
    if (workspace_bytes)
        *workspace_bytes = layout_of(mats, products == ONEBIT_PRODUCTS_F32).total;
    return ONEBIT_OK;
}

int onebit_matrices_kernels(const int64_t *rows, const int64_t *cols, int32_t count,
                            int32_t products, int32_t side[3], int32_t groups[3], int32_t *parts)
{
    if (!rows || !cols) return fail(ONEBIT_EINVAL, "rows or cols is NULL");
    if (count < 1) return fail(ONEBIT_EINVAL, "count < 1");
    if (products != ONEBIT_PRODUCTS_F32 && products != ONEBIT_PRODUCTS_F16)
        return fail(ONEBIT_EINVAL, "products %d is not one of ONEBIT_PRODUCTS_*", products);
    int32_t s[3] = {}, g[3] = {}, p = 0;
    try {
        TRY(kernels_impl(rows, cols, count, products == ONEBIT_PRODUCTS_F32 ? 2 : 1, s, g, p));
    } catch (const std::bad_alloc &) {
        return fail(ONEBIT_ENOMEM, "host memory for the matrix tables");
    }
    if (side) std::copy(s, s + 3, side);
    if (groups) std::copy(g, g + 3, groups);
    if (parts) *parts = p;
    return ONEBIT_OK;
}

int onebit_orthogonalize(onebit_matrices mats, const void *in, int32_t in_dtype, void *out,
                         int32_t out_dtype, int32_t products, int32_t steps,
                         const float *coefficients, float eps, void *workspace,
                         onebit_stream stream)
{
    TRY(check_mats(mats));
    TRY(check_buffer(mats, in, in_dtype, "in"));
    TRY(check_buffer(mats, out, out_dtype, "out"));
    if (in == out && in_dtype != out_dtype)
        return fail(ONEBIT_EINVAL, "in place, but in and out have different types");
    Coefficients co;
    TRY(check_common(mats, products, steps, coefficients, eps, workspace, co));
    if (mats->empty) return ONEBIT_OK;
    return with_type(in_dtype, [&](auto *i) {
        using I = std::remove_pointer_t<decltype(i)>;
        return with_type(out_dtype, [&](auto *o) {
            using O = std::remove_pointer_t<decltype(o)>;
            const FromTensor<I> src{(const I *)in};
            const ToTensor<O> dst{(O *)out};
            return products == ONEBIT_PRODUCTS_F32
                       ? run<true>(mats, src, dst, 0, steps, co, eps, workspace, (hipStream_t)stream)
                       : run<false>(mats, src, dst, 0, steps, co, eps, workspace, (hipStream_t)stream);
        });
    });
}

int onebit_muon_step(onebit_matrices mats, float *x, float *m, const void *grads,
                     int32_t grad_dtype, int64_t grad_ld, int32_t n_grads, float lr,
                     float momentum, int32_t nesterov, float weight_decay, int32_t scale,
                     int32_t products, int32_t steps, const float *coefficients, float eps,
                     void *workspace, onebit_stream stream)
{
    TRY(check_mats(mats));
    TRY(check_buffer(mats, x, ONEBIT_GRAD_F32, "x"));
    TRY(check_buffer(mats, m, ONEBIT_GRAD_F32, "m"));
    TRY(check_buffer(mats, grads, grad_dtype, "grads"));
    if (n_grads < 1) return fail(ONEBIT_EINVAL, "n_grads < 1");
    if (n_grads > 1 && grad_ld < mats->extent)
        return fail(ONEBIT_EINVAL, "grad_ld = %lld is below %lld", (long long)grad_ld,
                    (long long)mats->extent);
    if (scale < ONEBIT_MUON_SCALE_NONE || scale > ONEBIT_MUON_SCALE_RMS)
        return fail(ONEBIT_EINVAL, "scale %d is not one of ONEBIT_MUON_SCALE_*", scale);
    Coefficients co;
    TRY(check_common(mats, products, steps, coefficients, eps, workspace, co));
    if (mats->empty) return ONEBIT_OK;
    return with_type(grad_dtype, [&](auto *g) {
        using G = std::remove_pointer_t<decltype(g)>;
        // From three gradient rows on, reading them again costs more than the update's
        // own way through memory; the second iterate's place, 4 bytes an element for
        // pairs, is free until the first step's last product.
        float *u = products == ONEBIT_PRODUCTS_F32 && nesterov && n_grads >= 3
                       ? (float *)((char *)workspace + layout_of(mats, true).x1) : nullptr;
        const FromMuon<G> src{(const G *)grads, m, u, grad_ld, n_grads, (double)n_grads, momentum,
                              nesterov};
        const ToMuon dst{x, 1.f - lr * weight_decay, lr};
        return products == ONEBIT_PRODUCTS_F32
                   ? run<true>(mats, src, dst, scale, steps, co, eps, workspace, (hipStream_t)stream)
                   : run<false>(mats, src, dst, scale, steps, co, eps, workspace, (hipStream_t)stream);
    });
}

}  // extern "C"
