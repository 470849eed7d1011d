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
// rows (both operands contiguous along the summed index), for which the iterate
// is kept in both orientations, X (m x n) and XT (n x m), and D and B are
// symmetric.  Every operand lies in the workspace, padded with zeros to
// multiples of kTile, so that the product kernel has no bounds to check.
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
#include <vector>

#include "../../include/onebit.h"
#include "onebit_internal.h"
#include "onebit_status.h"

namespace onebit {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// |X|, |A| and the polynomial's change stay below kRange, so that kScale times
// them stays below fp16's 65504; 2^13 leaves an iterate of 2^14 x 2^14 elements
// (2^-14 each) 2^-23 of its size as the step of its low half.
constexpr float kScale = 8192.f;
constexpr double kRange = 7.5;

constexpr int kTile = 128;   // rows and columns of an output tile
constexpr int kSlab = 64;    // fp16 numbers of an operand's row that are staged together
constexpr int kNormChunk = 8192;  // elements of a matrix per workgroup of the norm
constexpr int kPrep = 64;    // rows and columns of a workgroup of the first iterate

struct Mat {
    int64_t off, ld;             // in the flat buffers
    int32_t rows, cols;          // there
    int32_t m, n;                // the smaller and the larger side
    int32_t mp, np;              // multiples of kTile
    int32_t flip;                // 1: X is the matrix transposed
    int32_t norm_first, norm_count;  // partial sums of the norm
    int32_t part_first, part_count;  // partial sums of the iterate's squares
    int32_t pad;
    int64_t ex, em;              // elements of X and of D before this matrix's
};

struct Item {
    int32_t mat;
    uint16_t i, j;
};

// Areas of the workspace.  Pairs: rows of X, XT, D and B hold 32 hi numbers and
// then the same 32 lo numbers, so that 64 consecutive numbers are a slab of
// either kind.  Halves: hi alone, and xt_lo holds the iterate's lo.
struct Areas {
    _Float16 *x, *xt, *xt_next, *xt_lo, *d, *b;
    double *norm;   // per norm chunk
    float *part;    // per tile of the iterate
    float *t;       // per matrix
    float *gamma;   // per matrix, of the first iterate
};

struct Coefficients {
    float a, b, c;
    float fade;  // of gamma in a step: a power of two, at most 1/2
};

// Workgroups go to the XCDs round-robin: each takes a contiguous eighth.
__device__ __forceinline__ int item_index()
{
    return (int)((blockIdx.x % kXcds) * (gridDim.x / kXcds) + blockIdx.x / kXcds);
}

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

// What is orthogonalised: a tensor, or momentum and gradients of a Muon step.
template <class T>
struct FromTensor {
    const T *in;
    __device__ __forceinline__ float value(int64_t e) const { return (float)in[e]; }
    __device__ __forceinline__ float first(int64_t e) const { return value(e); }
};

template <class T>
struct FromMuon {
    const T *grads;
    float *m;
    int64_t grad_ld;
    int n_grads;
    double n;
    float momentum;
    int nesterov;
    __device__ __forceinline__ float mean(int64_t e) const
    {
        if (n_grads == 1) return (float)grads[e];
        double s = 0;
        for (int i = 0; i < n_grads; ++i) s += (double)(float)grads[i * grad_ld + e];
        return (float)(s / n);
    }
    // the update from the new momentum
    __device__ __forceinline__ float value(int64_t e) const
    {
        return nesterov ? mean(e) + momentum * m[e] : m[e];
    }
    // ... which is formed and stored here, once for every element
    __device__ __forceinline__ float first(int64_t e) const
    {
        const float g = mean(e), now = momentum * m[e] + g;
        m[e] = now;
        return nesterov ? g + momentum * now : now;
    }
};

// Sum of squares (64 bits) of kNormChunk elements of a matrix.
template <class S>
__global__ __launch_bounds__(256) void k_norm(const Mat *__restrict__ mats,
                                              const Item *__restrict__ items, S src,
                                              double *__restrict__ norm)
{
    __shared__ double scratch[4];
    const Item it = items[blockIdx.x];
    const Mat &mt = mats[it.mat];
    const uint32_t cols = mt.cols, total = (uint32_t)mt.rows * cols;
    const int64_t off = mt.off, ld = mt.ld;
    const uint32_t chunk = (uint32_t)it.i << 16 | it.j;
    const uint32_t begin = chunk * kNormChunk, end = min(begin + kNormChunk, total);
    double sum = 0;
    for (uint32_t e = begin + threadIdx.x; e < end; e += 256) {
        const uint32_t r = e / cols;
        const float v = src.first(off + r * ld + (e - r * cols));
        sum += (double)v * (double)v;
    }
    sum = block_sum(sum, scratch);
    if (threadIdx.x == 0) norm[mt.norm_first + chunk] = sum;
}

// Writes `n` consecutive numbers (a multiple of 8, at most 32, inside one block
// of 32) of an operand's row from packed (lo << 16 | hi) words.
template <bool PAIRS, int N>
__device__ __forceinline__ void put_row(_Float16 *row, _Float16 *row_lo, int k,
                                        const uint32_t (&w)[N])
{
    uint32_t hi[N / 2], lo[N / 2];
#pragma unroll
    for (int q = 0; q < N / 2; ++q) {
        hi[q] = (w[2 * q] & 0xffffu) | w[2 * q + 1] << 16;
        lo[q] = w[2 * q] >> 16 | (w[2 * q + 1] & 0xffff0000u);
    }
    _Float16 *ph = PAIRS ? row + (k >> 5) * 64 + (k & 31) : row + k;
    _Float16 *pl = PAIRS ? ph + 32 : row_lo ? row_lo + k : nullptr;
#pragma unroll
    for (int q = 0; q < N / 2; q += 4) {
        *(v4u *)(ph + 2 * q) = v4u{hi[q], hi[q + 1], hi[q + 2], hi[q + 3]};
        if (PAIRS || pl) *(v4u *)(pl + 2 * q) = v4u{lo[q], lo[q + 1], lo[q + 2], lo[q + 3]};
    }
}

__device__ __forceinline__ uint32_t pack(float v)
{
    _Float16 hi, lo;
    split(v, hi, lo);
    return (uint32_t)__builtin_bit_cast(uint16_t, hi) |
           (uint32_t)__builtin_bit_cast(uint16_t, lo) << 16;
}

// First iterate, X = u / (||u||_F + eps) in both orientations, padding zeroed.
template <bool PAIRS, class S>
__global__ __launch_bounds__(256) void k_first(const Mat *__restrict__ mats,
                                               const Item *__restrict__ items, S src, double eps,
                                               Areas w)
{
    __shared__ double scratch[4];
    __shared__ uint32_t tile[kPrep][kPrep + 1];
    const Item it = items[blockIdx.x];
    const Mat &mt = mats[it.mat];
    double sum = 0;
    for (int k = threadIdx.x; k < mt.norm_count; k += 256) sum += w.norm[mt.norm_first + k];
    sum = block_sum(sum, scratch);
    const double size = sqrt(sum) / (sqrt(sum) + eps);
    // a NaN, zero or infinite norm, and every norm above eps: 1
    const double gamma = size > 0 && size <= 0.5 ? exp2(fmin(-ceil(log2(size)), 120.0)) : 1.0;
    if (it.i == 0 && it.j == 0 && threadIdx.x == 0) w.gamma[it.mat] = (float)gamma;
    const double factor = (double)kScale * gamma / (sqrt(sum) + eps);
    const int r0 = it.i * kPrep, c0 = it.j * kPrep;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 4
    for (int k = 0; k < kPrep / 4; ++k) {
        const int r = r0 + wave * (kPrep / 4) + k, c = c0 + lane;
        float v = 0.f;
        if (r < mt.rows && c < mt.cols)
            v = (float)((double)src.value(mt.off + r * mt.ld + c) * factor);
        tile[r - r0][lane] = pack(v);
    }
    __syncthreads();
    // along the matrix's rows: X, or XT where it is transposed; then along its columns
    const int64_t ex = mt.ex * (PAIRS ? 2 : 1);
    const int kind = PAIRS ? 2 : 1;
    const int line = threadIdx.x >> 2, part = (threadIdx.x & 3) * 16;
    uint32_t u[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) u[k] = tile[line][part + k];
    const int row_pitch = mt.flip ? mt.mp : mt.np, col_pitch = mt.flip ? mt.np : mt.mp;
    _Float16 *rows_to = (mt.flip ? w.xt : w.x) + ex;
    _Float16 *rows_lo = !PAIRS && mt.flip ? w.xt_lo + ex : nullptr;
    int64_t at = (int64_t)(r0 + line) * row_pitch;
    put_row<PAIRS>(rows_to + at * kind, rows_lo ? rows_lo + at : nullptr, c0 + part, u);
#pragma unroll
    for (int k = 0; k < 16; ++k) u[k] = tile[part + k][line];
    _Float16 *cols_to = (mt.flip ? w.x : w.xt) + ex;
    _Float16 *cols_lo = !PAIRS && !mt.flip ? w.xt_lo + ex : nullptr;
    at = (int64_t)(c0 + line) * col_pitch;
    put_row<PAIRS>(cols_to + at * kind, cols_lo ? cols_lo + at : nullptr, r0 + part, u);
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

constexpr int kGram = 0, kPoly = 1, kNext = 2, kLast = 3;

// Where the last product goes: a tensor, or the parameters.
template <class T>
struct ToTensor {
    T *out;
    __device__ __forceinline__ void put(int64_t e, float o, float) const { out[e] = (T)o; }
};

struct ToMuon {
    float *x;
    float keep, lr;  // 1 - lr weight decay, lr
    __device__ __forceinline__ void put(int64_t e, float o, float scale) const
    {
        x[e] = keep * x[e] - (lr * scale) * o;
    }
};

struct NoOut {
    __device__ __forceinline__ void put(int64_t, float, float) const {}
};

__device__ __forceinline__ float muon_scale(int mode, int rows, int cols)
{
    if (mode == ONEBIT_MUON_SCALE_SPECTRAL)
        return sqrtf(fmaxf(1.f, (float)rows / (float)cols));
    if (mode == ONEBIT_MUON_SCALE_RMS) return 0.2f * sqrtf((float)max(rows, cols));
    return 1.f;
}

constexpr int kRowBytes = kSlab * 2;            // 128 bytes of LDS per staged row
constexpr int kStage = 2 * kTile * kRowBytes;   // one slab of both operands

// Place of 16-byte chunk c of staged row r.  Eight lanes that read chunk c of
// rows r..r+7 would meet in the same banks (a row is 128 bytes); the row's number
// permutes its chunks so that any 16 consecutive rows cover all banks.
__device__ __forceinline__ int lds_chunk(int r, int c) { return r * kRowBytes + ((c ^ (r >> 1)) & 7) * 16; }

// Stages kTile rows of an operand: each wave 32 of them, 8 rows of 128 bytes per
// instruction, straight into LDS (a wave's 64 lanes fill 1 KB in lane order, so
// the permutation is applied to the address that is read).
__device__ __forceinline__ void stage_rows(const _Float16 *src, int64_t pitch, char *lds)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < kTile / 32; ++k) {
        const int r = wave * (kTile / 4) + k * 8 + (lane >> 3);
        const int c = ((lane & 7) ^ (r >> 1)) & 7;
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void *)(src + r * pitch + c * 8),
            (__attribute__((address_space(3))) void *)(lds + (wave * (kTile / 4) + k * 8) * kRowBytes),
            16, 0, 0);
    }
}

template <bool PAIRS, int STEP, class O>
__global__ __launch_bounds__(256, 2) void k_product(const Mat *__restrict__ mats,
                                                    const Item *__restrict__ items, int count,
                                                    Areas w, Coefficients co, float faded, O out,
                                                    int scale_mode)
{
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStage];
    __shared__ float scratch[4];
    const int index = item_index();
    if (index >= count) return;
    const Item it = items[index];
    const Mat mt = mats[it.mat];
    constexpr int kind = PAIRS ? 2 : 1;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wr = (wave >> 1) * 64, wc = (wave & 1) * 64;  // the wave's part of the tile
    const int i0 = it.i * kTile, j0 = it.j * kTile;

    const int64_t ex = mt.ex * kind, em = mt.em * kind;
    const int64_t pitch = (int64_t)(STEP == kGram ? mt.np : mt.mp) * kind;
    const _Float16 *pa = (STEP == kGram ? w.x + ex : STEP == kPoly ? w.d + em : w.b + em) + i0 * pitch;
    const _Float16 *pb = (STEP == kGram ? w.x + ex : STEP == kPoly ? w.d + em : w.xt + ex) + j0 * pitch;
    const int slabs = (int)(pitch / kSlab);

    f32x16 acc[2][2] = {};
    stage_rows(pa, pitch, lds);
    stage_rows(pb, pitch, lds + kTile * kRowBytes);
    __syncthreads();
    for (int s = 0; s < slabs; ++s) {
        const char *la = lds + (s & 1) * kStage, *lb = la + kTile * kRowBytes;
        if (s + 1 < slabs) {
            char *next = lds + ((s + 1) & 1) * kStage;
            stage_rows(pa + (s + 1) * kSlab, pitch, next);
            stage_rows(pb + (s + 1) * kSlab, pitch, next + kTile * kRowBytes);
        }
        const int row = lane & 31, up = lane >> 5;
        auto frag = [&](const char *base, int r, int c) {
            return *(const half8 *)(base + lds_chunk(r + row, c + up));
        };
#pragma unroll
        for (int k = 0; k < (PAIRS ? 4 : 8); k += 2) {
            half8 a[2], b[2], al[2], bl[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                a[q] = frag(la, wr + q * 32, k);
                b[q] = frag(lb, wc + q * 32, k);
                if (PAIRS) {
                    al[q] = frag(la, wr + q * 32, k + 4);
                    bl[q] = frag(lb, wc + q * 32, k + 4);
                }
            }
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    acc[p][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[p], b[q], acc[p][q], 0, 0, 0);
                    if (PAIRS) {
                        acc[p][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[p], bl[q], acc[p][q], 0, 0, 0);
                        acc[p][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(al[p], b[q], acc[p][q], 0, 0, 0);
                    }
                }
        }
        __syncthreads();
    }

    // The shift, and the step's coefficients around it.
    const float gamma0 = w.gamma[it.mat], gamma = fmaxf(gamma0 * faded, 1.f);
    const float inv2 = 1.f / (gamma * gamma);
    float t;
    if (STEP == kGram) {
        if (faded == 1.f) {  // the first step
            t = 1.f / (float)mt.m;
        } else {
            float sum = 0.f;
            for (int k = threadIdx.x; k < mt.part_count; k += 256) sum += w.part[mt.part_first + k];
            t = block_sum(sum, scratch) / (float)mt.m;
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

    // Values in place of the sums.  A lane holds column (lane & 31) and, in
    // register r, row 8 (r / 4) + 4 (lane / 32) + r % 4 of a 32 x 32 part.
    const int col = lane & 31, quad = (lane >> 5) * 4;
    const float unscale = 1.f / kScale;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int r = i0 + wr + p * 32 + g * 8 + quad, c = j0 + wc + q * 32 + col;
                half4 hi = {}, lo = {};
                if (STEP != kGram) {  // D(c, r..r+3), or XT(c, r..r+3)
                    const _Float16 *line = (STEP == kPoly ? w.d + em : w.xt + ex) + c * pitch;
                    if (PAIRS) {
                        const _Float16 *at = line + (r >> 5) * 64 + (r & 31);
                        hi = *(const half4 *)at;
                        lo = *(const half4 *)(at + 32);
                    } else {
                        hi = *(const half4 *)(line + r);
                        if (STEP != kPoly) lo = *(const half4 *)(w.xt_lo + ex + c * pitch + r);
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float v = acc[p][q][g * 4 + k] * unscale;
                    if (STEP == kGram) {
                        if (r + k == c && c < mt.m) v -= t * kScale;
                    } else {
                        const float old = (float)hi[k] + (float)lo[k];
                        v = linear * old + square * v;
                    }
                    acc[p][q][g * 4 + k] = v;
                }
            }

    if (STEP == kLast) {
        const float scale = muon_scale(scale_mode, mt.rows, mt.cols) * unscale;
        const float plain = unscale;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = i0 + wr + p * 32 + (r >> 2) * 8 + quad + (r & 3);
                    const int j = j0 + wc + q * 32 + col;
                    if (i < mt.m && j < mt.n)
                        out.put(mt.off + (mt.flip ? j * mt.ld + i : i * mt.ld + j),
                                acc[p][q][r] * plain, scale * kScale);
                }
        return;
    }

    if (STEP == kNext) {
        float sum = 0.f;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float v = acc[p][q][r] * unscale;
                    sum += v * v;
                }
        sum = block_sum(sum, scratch);
        if (threadIdx.x == 0) w.part[mt.part_first + it.i * (mt.np / kTile) + it.j] = sum;
    }

    // Both orientations, through the wave's own part of LDS, so that a row's 64
    // numbers are written by two lanes, 32 each.
    constexpr int kPitch = 68;  // words
    uint32_t *mine = (uint32_t *)(lds) + wave * (32 * kPitch);
    static_assert(4 * 32 * kPitch * 4 <= 2 * kStage, "the epilogue's LDS");
    _Float16 *rows_to = (STEP == kGram ? w.d + em : STEP == kPoly ? w.b + em : w.x + ex);
    const int64_t rows_pitch = (int64_t)(STEP == kNext ? mt.np : mt.mp) * kind;
    _Float16 *cols_to = STEP == kNext ? w.xt_next + ex : rows_to;
    const int64_t cols_pitch = (int64_t)mt.mp * kind;
    const int line = lane >> 1, part = (lane & 1) * 32;
#pragma unroll
    for (int p = 0; p < 2; ++p) {  // 32 rows x 64 columns at a time
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                mine[((r >> 2) * 8 + quad + (r & 3)) * kPitch + q * 32 + col] = pack(acc[p][q][r]);
        wave_sync();
        uint32_t u[32];
#pragma unroll
        for (int k = 0; k < 32; k += 4) *(v4u *)(u + k) = *(const v4u *)(mine + line * kPitch + part + k);
        put_row<PAIRS>(rows_to + (i0 + wr + p * 32 + line) * rows_pitch, nullptr, j0 + wc + part, u);
        wave_sync();
    }
    if (STEP != kNext && it.i == it.j) return;  // a diagonal tile is its own transpose
#pragma unroll
    for (int q = 0; q < 2; ++q) {  // 32 columns x 64 rows at a time
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(v4u *)(mine + col * kPitch + p * 32 + g * 8 + quad) =
                    v4u{pack(acc[p][q][g * 4]), pack(acc[p][q][g * 4 + 1]),
                        pack(acc[p][q][g * 4 + 2]), pack(acc[p][q][g * 4 + 3])};
        wave_sync();
        uint32_t u[32];
#pragma unroll
        for (int k = 0; k < 32; k += 4) *(v4u *)(u + k) = *(const v4u *)(mine + line * kPitch + part + k);
        const int64_t at = (int64_t)(j0 + wc + q * 32 + line) * cols_pitch;
        put_row<PAIRS>(cols_to + at, !PAIRS && STEP == kNext ? w.xt_lo + ex + at : nullptr,
                       i0 + wr + part, u);
        wave_sync();
    }
}

}  // namespace
}  // namespace onebit

using namespace onebit;

struct onebit_matrices_s {
    int device = 0;
    int32_t count = 0;
    int64_t extent = 0, ex = 0, em = 0;
    int64_t norms = 0, firsts = 0, syms = 0, nexts = 0;
    std::vector<int64_t> offset;
    char *dev = nullptr;
    const Mat *mats = nullptr;
    const Item *norm_items = nullptr, *first_items = nullptr, *sym_items = nullptr,
               *next_items = nullptr;
};

namespace {

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

#define TRY(expr)                         \
    do {                                  \
        int _st = (expr);                 \
        if (_st != ONEBIT_OK) return _st; \
    } while (0)

struct WorkspaceLayout {
    size_t x, xt0, xt1, xt_lo, d, b, norm, part, t, gamma, total;
};

WorkspaceLayout layout_of(const onebit_matrices_s *p, bool pairs)
{
    WorkspaceLayout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    const size_t half = pairs ? 4 : 2;
    l.x = take(half * p->ex);
    l.xt0 = take(half * p->ex);
    l.xt1 = take(half * p->ex);
    l.xt_lo = take(pairs ? 0 : 2 * p->ex);
    l.d = take(half * p->em);
    l.b = take(half * p->em);
    l.norm = take(8 * (size_t)p->norms);
    l.part = take(4 * (size_t)p->nexts);
    l.t = take(4 * (size_t)p->count);
    l.gamma = take(4 * (size_t)p->count);
    l.total = at;
    return l;
}

int create_impl(const int64_t *rows, const int64_t *cols, const int64_t *offset,
                const int64_t *ld, int32_t count, onebit_matrices *out)
{
    std::unique_ptr<onebit_matrices_s> p(new onebit_matrices_s);
    hipError_t e = hipGetDevice(&p->device);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    std::vector<Mat> mats(count);
    std::vector<Item> norm, first, sym, next;
    p->count = count;
    p->offset.resize(count);
    int64_t at = 0;
    constexpr int64_t kSide = 1 << 20, kMost = (int64_t)1 << 40, kItems = 1 << 23;
    for (int32_t k = 0; k < count; ++k) {
        const int64_t r = rows[k], c = cols[k];
        if (r < 0 || c < 0 || r > kSide || c > kSide)
            return fail(ONEBIT_EINVAL, "matrix %d is %lld x %lld: a side is at most 2^20", k,
                        (long long)r, (long long)c);
        if (r * c >= ((int64_t)1 << 31))
            return fail(ONEBIT_EINVAL, "matrix %d has 2^31 elements or more", k);
        const int64_t pitch = ld ? ld[k] : c;
        const int64_t off = offset ? offset[k] : at;
        if (pitch < c || pitch > kMost)
            return fail(ONEBIT_EINVAL, "ld[%d] = %lld, %lld columns", k, (long long)pitch,
                        (long long)c);
        if (off < 0 || off > kMost)
            return fail(ONEBIT_EINVAL, "offset[%d] = %lld", k, (long long)off);
        const int64_t span = r > 0 && c > 0 ? (r - 1) * pitch + c : 0;
        if (off + span > kMost || span > kMost)
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
        m.mp = (m.m + kTile - 1) / kTile * kTile;
        m.np = (m.n + kTile - 1) / kTile * kTile;
        m.ex = p->ex;
        m.em = p->em;
        p->ex += (int64_t)m.mp * m.np;
        p->em += (int64_t)m.mp * m.mp;
        const int tm = m.mp / kTile, tn = m.np / kTile;
        m.norm_first = (int32_t)norm.size();
        m.norm_count = (int32_t)((r * c + kNormChunk - 1) / kNormChunk);
        m.part_first = (int32_t)next.size();
        m.part_count = tm * tn;
        const int rp = (m.flip ? m.np : m.mp) / kPrep, cp = (m.flip ? m.mp : m.np) / kPrep;
        if ((int64_t)norm.size() + m.norm_count > kItems || (int64_t)first.size() + (int64_t)rp * cp > kItems)
            return fail(ONEBIT_EINVAL, "too many tiles (matrix %d)", k);
        for (int32_t q = 0; q < m.norm_count; ++q)
            norm.push_back(Item{k, (uint16_t)(q >> 16), (uint16_t)q});
        for (int i = 0; i < rp; ++i)
            for (int j = 0; j < cp; ++j) first.push_back(Item{k, (uint16_t)i, (uint16_t)j});
        for (int i = 0; i < tm; ++i)
            for (int j = 0; j <= i; ++j) sym.push_back(Item{k, (uint16_t)i, (uint16_t)j});
        for (int i = 0; i < tm; ++i)
            for (int j = 0; j < tn; ++j) next.push_back(Item{k, (uint16_t)i, (uint16_t)j});
    }
    p->norms = (int64_t)norm.size();
    p->firsts = (int64_t)first.size();
    p->syms = (int64_t)sym.size();
    p->nexts = (int64_t)next.size();
    // one host buffer in the layout of the device allocation
    size_t total = 0;
    auto take = [&](size_t bytes) {
        const size_t here = total;
        total += up256(bytes);
        return here;
    };
    const size_t o_mats = take(mats.size() * sizeof(Mat));
    const size_t o_norm = take(norm.size() * sizeof(Item)), o_first = take(first.size() * sizeof(Item));
    const size_t o_sym = take(sym.size() * sizeof(Item)), o_next = take(next.size() * sizeof(Item));
    std::vector<char> host(total);
    auto copy = [&](size_t to, const auto &v) {
        if (!v.empty()) std::memcpy(host.data() + to, v.data(), v.size() * sizeof(v[0]));
    };
    copy(o_mats, mats);
    copy(o_norm, norm);
    copy(o_first, first);
    copy(o_sym, sym);
    copy(o_next, next);
    void *dev = nullptr;
    e = hipMalloc(&dev, total);
    if (e == hipErrorOutOfMemory) return fail(ONEBIT_ENOMEM, "hipMalloc of the matrix tables");
    if (e != hipSuccess) return hip_fail(e, "hipMalloc");
    e = hipMemcpy(dev, host.data(), total, hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        (void)hipFree(dev);
        return hip_fail(e, "copy of the matrix tables");
    }
    p->dev = (char *)dev;
    p->mats = (const Mat *)(p->dev + o_mats);
    p->norm_items = (const Item *)(p->dev + o_norm);
    p->first_items = (const Item *)(p->dev + o_first);
    p->sym_items = (const Item *)(p->dev + o_sym);
    p->next_items = (const Item *)(p->dev + o_next);
    *out = p.release();
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

int grid8(int64_t items) { return (int)((items + kXcds - 1) / kXcds * kXcds); }

// Everything after the arguments' checks: `src` is what is orthogonalised.
template <bool PAIRS, class S, class O>
int run(const onebit_matrices_s *p, const S &src, const O &out, int scale_mode, int steps,
        const Coefficients &co, float eps, void *workspace, hipStream_t st)
{
    const WorkspaceLayout l = layout_of(p, PAIRS);
    char *ws = (char *)workspace;
    Areas w{(_Float16 *)(ws + l.x), (_Float16 *)(ws + l.xt0), (_Float16 *)(ws + l.xt1),
            (_Float16 *)(ws + l.xt_lo), (_Float16 *)(ws + l.d), (_Float16 *)(ws + l.b),
            (double *)(ws + l.norm), (float *)(ws + l.part), (float *)(ws + l.t),
            (float *)(ws + l.gamma)};
    k_norm<S><<<(int)p->norms, 256, 0, st>>>(p->mats, p->norm_items, src, w.norm);
    k_first<PAIRS, S><<<(int)p->firsts, 256, 0, st>>>(p->mats, p->first_items, src, (double)eps, w);
    const int gs = grid8(p->syms), gn = grid8(p->nexts);
    float faded = 1.f;
    for (int k = 0; k < steps; ++k, faded *= co.fade) {
        k_product<PAIRS, kGram, NoOut><<<gs, 256, 0, st>>>(p->mats, p->sym_items, (int)p->syms, w,
                                                           co, faded, NoOut{}, 0);
        k_product<PAIRS, kPoly, NoOut><<<gs, 256, 0, st>>>(p->mats, p->sym_items, (int)p->syms, w,
                                                           co, faded, NoOut{}, 0);
        if (k + 1 < steps)
            k_product<PAIRS, kNext, NoOut><<<gn, 256, 0, st>>>(
                p->mats, p->next_items, (int)p->nexts, w, co, faded, NoOut{}, 0);
        else
            k_product<PAIRS, kLast, O><<<gn, 256, 0, st>>>(
                p->mats, p->next_items, (int)p->nexts, w, co, faded, out, scale_mode);
        std::swap(w.xt, w.xt_next);
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
    if (!workspace && p->ex > 0) return fail(ONEBIT_EINVAL, "workspace is NULL");
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
    if (mats->ex == 0) return ONEBIT_OK;
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
    if (mats->ex == 0) return ONEBIT_OK;
    return with_type(grad_dtype, [&](auto *g) {
        using G = std::remove_pointer_t<decltype(g)>;
        const FromMuon<G> src{(const G *)grads, m, grad_ld, n_grads, (double)n_grads, momentum,
                              nesterov};
        const ToMuon dst{x, 1.f - lr * weight_decay, lr};
        return products == ONEBIT_PRODUCTS_F32
                   ? run<true>(mats, src, dst, scale, steps, co, eps, workspace, (hipStream_t)stream)
                   : run<false>(mats, src, dst, scale, steps, co, eps, workspace, (hipStream_t)stream);
    });
}

}  // extern "C"
