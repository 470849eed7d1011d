// Layer norm of rows, and its gradients.  Both stream: a row is read once into
// registers, where its statistics are formed, and each result is written once.
// See include/onebit.h for the contract of the entry points.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "../../include/onebit.h"
#include "onebit_internal.h"
#include "onebit_rows.h"
#include "onebit_status.h"

namespace onebit {
namespace {

// Columns that one thread holds together, and the widest row.
constexpr int kCols = 8;
constexpr int64_t kWidest = 16384;

// A row is held by L threads, C pieces of kCols columns each: piece c of thread
// `lane` is columns (c L + lane) kCols and on.  L is 8, 32 or 64 lanes of a wave,
// which holds 64 / L rows and needs no LDS, or a workgroup.
template <int L, int C, class T>
__device__ __forceinline__ void load_row(const T *p, int lane, int width, float (&v)[C][kCols])
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * L + lane) * kCols;
        load_some(p + at, v[c], width - at);
    }
}

// Weight or bias: an array of `width` numbers of any type, or none.
template <int L, int C>
__device__ __forceinline__ void load_params(const void *p, int dtype, int lane, int width,
                                            float otherwise, float (&v)[C][kCols])
{
    if (!p) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[c][k] = otherwise;
    } else if (dtype == ONEBIT_GRAD_F32) {
        load_row<L, C>((const float *)p, lane, width, v);
    } else if (dtype == ONEBIT_GRAD_BF16) {
        load_row<L, C>((const __bf16 *)p, lane, width, v);
    } else {
        load_row<L, C>((const _Float16 *)p, lane, width, v);
    }
}

// Puts `value` behind the end of the row.
template <int L, int C>
__device__ __forceinline__ void fill_tail(int lane, int width, float value, float (&v)[C][kCols])
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int left = width - (c * L + lane) * kCols;
        if (left < kCols)
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                if (k >= left) v[c][k] = value;
    }
}

// Turns a row into its differences from the mean, and gives 1 / sqrt(var + eps).
// The mean is first rounded to fp32; the differences from that are exact or nearly so
// where the mean is far above them, and their own mean is what it was off by.
template <class T, int L, int C>
__device__ __forceinline__ float centre(float (&x)[C][kCols], int lane, int width, float eps,
                                        float *lds)
{
    float sum[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kCols; ++k) sum[0] += x[c][k];
    add_lanes<L>(sum, lds);
    const float mean = sum[0] / (float)width;
    fill_tail<L, C>(lane, width, mean, x);
    float two[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
            x[c][k] -= mean;
            two[0] += x[c][k];
            two[1] = __builtin_fmaf(x[c][k], x[c][k], two[1]);
        }
    add_lanes<L>(two, lds + L / 64);
    const float shift = two[0] / (float)width;
    const float var = __builtin_fmaf(-shift, shift, two[1] / (float)width);
    float r = 1.f / sqrtf(fmaxf(var, 0.f) + eps);
    // Squares past fp32's range, which no row of fp16 numbers has: once more of the
    // differences times 2^-64.  (The sum's place is free again behind the second barrier.)
    if (!std::is_same_v<T, _Float16> && __builtin_expect(two[1] == INFINITY, 0)) {
        sum[0] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int k = 0; k < kCols; ++k) {
                const float d = x[c][k] * 0x1p-64f;
                sum[0] = __builtin_fmaf(d, d, sum[0]);
                asm volatile("" : "+v"(sum[0]));  // one at a time, for the registers
            }
        add_lanes<L>(sum, lds);
        const float s = shift * 0x1p-64f, v = __builtin_fmaf(-s, s, sum[0] / (float)width);
        r = 0x1p-64f / sqrtf(fmaxf(v, 0.f) + eps * 0x1p-128f);
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int k = 0; k < kCols; ++k) x[c][k] -= shift;
    return r;
}

template <int L>
constexpr int kThreads = L < 256 ? 256 : L;

// y = (x - mean) r w + b, a row per L threads, weight and bias in registers over all rows
// of a workgroup.  Memory bounds it: 131,072 bf16 rows of 1,024 (537 MB) take 90 us (5.9
// TB/s; a copy of 8 GiB reaches 6.8), 10,007 fp32 rows of 771 to bf16 11 us (4.2 TB/s), 16
// rows 3.8.
template <class T, class O, int L, int C>
__global__ __launch_bounds__(kThreads<L>) void k_layer_norm(const T *__restrict__ x, int64_t x_ld,
                                                      int64_t rows, int width,
                                                      const void *__restrict__ weight,
                                                      const void *__restrict__ bias, int w_dtype,
                                                      float eps, O *__restrict__ y, int64_t y_ld)
{
    constexpr int kRows = kThreads<L> / L;
    __shared__ float lds[2][L > 64 ? 3 * L / 64 : 1];
    const int lane = threadIdx.x % L;
    float w[C][kCols], b[C][kCols];
    load_params<L, C>(weight, w_dtype, lane, width, 1.f, w);
    load_params<L, C>(bias, w_dtype, lane, width, 0.f, b);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / L; row < rows;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        float v[C][kCols];
        load_row<L, C>(x + row * x_ld, lane, width, v);
        const float r = centre<T, L, C>(v, lane, width, eps, lds[turn]);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * L + lane) * kCols;
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[c][k] = __builtin_fmaf(v[c][k] * r, w[c][k], b[c][k]);
            if (at < width) store_some(y + row * y_ld + at, v[c], width - at);
        }
    }
}

// dx = r (g - mean(g) - z mean(g z)) with z = (x - mean) r and g = dy w, and the sums
// of dy z and dy over the workgroup's rows, in registers until the last one.  Sums of
// a column are added in an order that depends on the rows and the width alone.  Memory
// bounds it: 131,072 bf16 rows of 1,024 (805 MB) take 155 us (5.2 TB/s), 10,007 fp32 rows
// of 771 20, 8,192 bf16 rows of 16,384 220 (3.7).  Loading a row ahead costs a workgroup per CU in registers: 190 us.
template <class D, class T, int L, int C>
__global__ __launch_bounds__(kThreads<L>) void k_layer_norm_grad(
    const D *dy, int64_t dy_ld, const T *__restrict__ x, int64_t x_ld, int64_t rows,
    int width, const void *__restrict__ weight, int w_dtype, float eps, T *dx,
    int64_t dx_ld, float *__restrict__ partial)
{
    constexpr int kRows = kThreads<L> / L;
    __shared__ float lds[2][L > 64 ? 5 * L / 64 : 1];
    const int lane = threadIdx.x % L;
    float w[C][kCols], dw[C][kCols] = {}, db[C][kCols] = {};
    load_params<L, C>(weight, w_dtype, lane, width, 1.f, w);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / L; row < rows;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        float v[C][kCols], g[C][kCols];
        load_row<L, C>(x + row * x_ld, lane, width, v);
        load_row<L, C>(dy + row * dy_ld, lane, width, g);
        const float r = centre<T, L, C>(v, lane, width, eps, lds[turn]);
        float two[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int k = 0; k < kCols; ++k) {
                v[c][k] *= r;
                dw[c][k] = __builtin_fmaf(g[c][k], v[c][k], dw[c][k]);
                db[c][k] += g[c][k];
                g[c][k] *= w[c][k];
                two[0] += g[c][k];
                two[1] = __builtin_fmaf(g[c][k], v[c][k], two[1]);
            }
        add_lanes<L>(two, lds[turn] + 3 * L / 64);
        if (!dx) continue;
        const float mg = two[0] / (float)width, mgz = two[1] / (float)width;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * L + lane) * kCols;
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                g[c][k] = r * __builtin_fmaf(-mgz, v[c][k], g[c][k] - mg);
            if (at < width) store_some(dx + row * dx_ld + at, g[c], width - at);
        }
    }
    if (!partial) return;
    if constexpr (kRows > 1) {  // the workgroup's rows, in order
        __shared__ float sums[2][L * C * kCols];
        for (int turn = 0; turn < kRows; ++turn) {
            if ((int)threadIdx.x / L == turn)
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int k = 0; k < kCols; ++k) {
                        const int at = (c * kCols + k) * L + lane;
                        if (turn > 0) dw[c][k] += sums[0][at], db[c][k] += sums[1][at];
                        sums[0][at] = dw[c][k];
                        sums[1][at] = db[c][k];
                    }
            __syncthreads();
        }
        if ((int)threadIdx.x / L != kRows - 1) return;
    }
    float *to = partial + (int64_t)blockIdx.x * 2 * width;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * L + lane) * kCols;
        if (at >= width) break;
        store_some(to + at, dw[c], width - at);
        store_some(to + width + at, db[c], width - at);
    }
}

// Adds the workgroups' sums: 16 columns a workgroup, whose 64 groups of threads take
// every 64th sum, up to kJoinAhead of them loaded before the first is added (1,024 sums
// of 2,048 columns: 6 us; 16 groups of 16 threads, one load behind the other, 29).
constexpr int kJoinCols = 16, kJoinParts = 64, kJoinAhead = 8;

template <class G>
__device__ __forceinline__ void put_sum(void *to, int k, float s, int accumulate)
{
    G *q = (G *)to + k;
    *q = (G)(accumulate ? (float)*q + s : s);
}

__global__ __launch_bounds__(kJoinCols *kJoinParts) void k_layer_norm_join(
    const float *__restrict__ partial, int parts, int width, void *__restrict__ dweight,
    void *__restrict__ dbias, int dtype, int accumulate)
{
    __shared__ float sums[kJoinParts][kJoinCols];
    const int col = threadIdx.x % kJoinCols, part = threadIdx.x / kJoinCols;
    const int at = blockIdx.x * kJoinCols + col;
    float s = 0.f;
    if (at < 2 * width)
        for (int first = part; first < parts; first += kJoinParts * kJoinAhead) {
            float v[kJoinAhead];
#pragma unroll
            for (int k = 0; k < kJoinAhead; ++k) {
                const int p = first + k * kJoinParts;
                v[k] = p < parts ? partial[(int64_t)p * 2 * width + at] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < kJoinAhead; ++k) s += v[k];
        }
    sums[part][col] = s;
    __syncthreads();
    if (part > 0 || at >= 2 * width) return;
#pragma unroll
    for (int p = 1; p < kJoinParts; ++p) s += sums[p][col];
    void *to = at < width ? dweight : dbias;
    const int k = at < width ? at : at - width;
    if (!to) return;
    if (dtype == ONEBIT_GRAD_F32) put_sum<float>(to, k, s, accumulate);
    else if (dtype == ONEBIT_GRAD_BF16) put_sum<__bf16>(to, k, s, accumulate);
    else put_sum<_Float16>(to, k, s, accumulate);
}

// Calls f(L, C) for rows of this width.
template <class F>
void with_shape(int64_t width, F &&f)
{
    auto go = [&](auto l, auto c) { f(l, c); };
    using std::integral_constant;
    if (width <= 64) go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (width <= 256) go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (width <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (width <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (width <= 2048) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (width <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (width <= 8192) go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    else go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

// Workgroups of 256 threads that a launch has at most: as many as the GPU's 256 CUs
// hold at once, each of which goes on to further rows with its weights (and, backwards,
// its sums) in registers.
constexpr int kMostBlocks = 2048, kMostParts = 1024;

int blocks_for(int64_t rows, int lanes, int most)
{
    const int threads = lanes < 256 ? 256 : lanes;
    const int64_t at_once = threads / lanes;
    return (int)std::min<int64_t>((rows + at_once - 1) / at_once, most / (threads / 256));
}

int check_norm(int64_t rows, int64_t width)
{
    TRY(check_size(rows, "rows"));
    if (width < 0 || width > kWidest)
        return fail(ONEBIT_EINVAL, "width = %lld is not in [0, %lld]", (long long)width,
                    (long long)kWidest);
    return ONEBIT_OK;
}

int check_params(const void *p, int32_t dtype, const char *name)
{
    const int bytes = elem_bytes(dtype);
    if (!bytes) return fail(ONEBIT_EINVAL, "%s: type %d is not one of ONEBIT_GRAD_*", name, dtype);
    if ((uintptr_t)p % bytes) return fail(ONEBIT_EALIGN, "%s is not %d-byte aligned", name, bytes);
    return ONEBIT_OK;
}

int check_eps(float eps)
{
    if (!(eps >= 0.f) || eps > 3e38f) return fail(ONEBIT_EINVAL, "eps = %g", (double)eps);
    return ONEBIT_OK;
}

}  // namespace
}  // namespace onebit

using namespace onebit;

extern "C" {

int onebit_layer_norm_forward(const void *x, int32_t x_dtype, int64_t x_ld, int64_t rows,
                              int64_t width, const void *weight, const void *bias,
                              int32_t w_dtype, float eps, void *y, int32_t y_dtype, int64_t y_ld,
                              onebit_stream stream)
{
    TRY(check_norm(rows, width));
    TRY(check_rows(x, x_dtype, x_ld, rows, width, "x"));
    TRY(check_rows(y, y_dtype, y_ld, rows, width, "y"));
    TRY(check_params(weight, w_dtype, "weight"));
    TRY(check_params(bias, w_dtype, "bias"));
    TRY(check_eps(eps));
    if (rows == 0 || width == 0) return ONEBIT_OK;
    with_type(x_dtype, [&](auto *t) {
        with_type(y_dtype, [&](auto *o) {
            with_shape(width, [&](auto lanes, auto pieces) {
                using T = std::remove_pointer_t<decltype(t)>;
                using O = std::remove_pointer_t<decltype(o)>;
                constexpr int L = decltype(lanes)::value, C = decltype(pieces)::value;
                k_layer_norm<T, O, L, C><<<blocks_for(rows, L, kMostBlocks), kThreads<L>, 0,
                                     (hipStream_t)stream>>>((const T *)x, x_ld, rows, (int)width,
                                                            weight, bias, w_dtype, eps, (O *)y,
                                                            y_ld);
            });
        });
    });
    return launched("layer norm launch");
}

int onebit_layer_norm_grad_workspace(int64_t rows, int64_t width, size_t *bytes)
{
    if (!bytes) return fail(ONEBIT_EINVAL, "bytes is NULL");
    TRY(check_norm(rows, width));
    *bytes = (size_t)std::min<int64_t>(rows, kMostParts) * 2 * (size_t)width * sizeof(float);
    return ONEBIT_OK;
}

int onebit_layer_norm_grad(const void *dy, int32_t dy_dtype, int64_t dy_ld, const void *x,
                           int32_t x_dtype, int64_t x_ld, int64_t rows, int64_t width,
                           const void *weight, int32_t w_dtype, float eps, void *dx,
                           int64_t dx_ld, void *dweight, void *dbias, int32_t dw_dtype,
                           int32_t accumulate, void *workspace, onebit_stream stream)
{
    TRY(check_norm(rows, width));
    TRY(check_rows(dy, dy_dtype, dy_ld, rows, width, "dy"));
    TRY(check_rows(x, x_dtype, x_ld, rows, width, "x"));
    if (dx) TRY(check_rows(dx, x_dtype, dx_ld, rows, width, "dx"));
    TRY(check_params(weight, w_dtype, "weight"));
    TRY(check_params(dweight, dw_dtype, "dweight"));
    TRY(check_params(dbias, dw_dtype, "dbias"));
    TRY(check_eps(eps));
    const bool sums = dweight || dbias;
    if (sums && !workspace) return fail(ONEBIT_EINVAL, "workspace is NULL");
    if ((uintptr_t)workspace % 16) return fail(ONEBIT_EALIGN, "workspace is not 16-byte aligned");
    if (width == 0 || (!dx && !sums) || (rows == 0 && (accumulate || !sums))) return ONEBIT_OK;
    hipStream_t st = (hipStream_t)stream;
    float *partial = sums ? (float *)workspace : nullptr;
    int parts = 0;
    if (rows > 0)
        with_type(dy_dtype, [&](auto *d) {
            with_type(x_dtype, [&](auto *t) {
                with_shape(width, [&](auto lanes, auto pieces) {
                    using D = std::remove_pointer_t<decltype(d)>;
                    using T = std::remove_pointer_t<decltype(t)>;
                    constexpr int L = decltype(lanes)::value, C = decltype(pieces)::value;
                    parts = blocks_for(rows, L, kMostParts);
                    k_layer_norm_grad<D, T, L, C><<<parts, kThreads<L>, 0, st>>>(
                        (const D *)dy, dy_ld, (const T *)x, x_ld, rows, (int)width, weight,
                        w_dtype, eps, (T *)dx, dx_ld, partial);
                });
            });
        });
    TRY(launched("layer norm gradient launch"));
    if (!sums) return ONEBIT_OK;
    k_layer_norm_join<<<(int)((2 * width + kJoinCols - 1) / kJoinCols), kJoinCols * kJoinParts, 0, st>>>(
        partial, parts, (int)width, dweight, dbias, dw_dtype, accumulate);
    return launched("layer norm join launch");
}

}  // extern "C"
