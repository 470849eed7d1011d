// What the operators over rows of numbers share: loads and stores of a row's
// pieces, sums over lanes, and the checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/onebit.h"
#include "onebit_status.h"

namespace onebit {

// N consecutive elements of type T as fp32.  Rows need no alignment (an odd
// width leaves every second row of a 16-bit table on an odd element), so the
// vector access is stated as a copy of bytes, which the compiler turns into one
// load or store of up to 16 bytes (gfx950 takes them at any address).
template <class T, int N>
__device__ __forceinline__ void load_vec(const T *p, float (&v)[N])
{
    T t[N];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = (float)t[k];
}

template <class T, int N>
__device__ __forceinline__ void store_vec(T *p, const float (&v)[N])
{
    T t[N];
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = (T)v[k];
    __builtin_memcpy(p, t, sizeof t);
}

// ... past the caches: what a call writes once and does not read again leaves the
// rows that it reads in them (131,072 rows of 1,024 bf16 numbers from an fp32 table:
// 118 us with plain stores, 76 so).
template <class T, int N>
__device__ __forceinline__ void stream_vec(T *p, const float (&v)[N])
{
    constexpr int kBytes = sizeof(T) * N;
    if constexpr (kBytes < 4) {
        store_vec(p, v);
    } else {
        constexpr int kWords = kBytes % 16 == 0 ? 4 : kBytes % 8 == 0 ? 2 : 1, kPieces = kBytes / (4 * kWords);
        typedef uint32_t words __attribute__((ext_vector_type(kWords), aligned(sizeof(T))));
        T t[N];
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] = (T)v[k];
        words w[kPieces];
        __builtin_memcpy(w, t, kBytes);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) __builtin_nontemporal_store(w[k], (words *)p + k);
    }
}

// The first `left` of N elements (a row's end); the others are 0 or not stored.
template <class T, int N>
__device__ __forceinline__ void load_some(const T *p, float (&v)[N], int left)
{
    if (left >= N) return load_vec(p, v);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = k < left ? (float)p[k] : 0.f;
}

template <class T, int N>
__device__ __forceinline__ void store_some(T *p, const float (&v)[N], int left)
{
    if (left >= N) return stream_vec(p, v);
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < left) p[k] = (T)v[k];
}

__device__ __forceinline__ int64_t load_id(const void *ids, int ids_bytes, int64_t t)
{
    return ids_bytes == 8 ? ((const int64_t *)ids)[t] : (int64_t)((const int32_t *)ids)[t];
}

// The other half's value of each 32, 16, 8, 4, 2 or 1 lanes is brought beside a lane's
// own without LDS: rotations and mirrors within 16 lanes, swaps of halves above.
template <int CTRL>
__device__ __forceinline__ float lanes(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL,
                                                                 0xf, 0xf, true));
}

// f over the values of each L lanes (8, 16, 32 or 64); every lane gets the same result,
// from the same tree.
template <int L, class F>
__device__ __forceinline__ float over_lanes(float v, F f)
{
    v = f(v, lanes<0xB1>(v));   // lane ^ 1
    v = f(v, lanes<0x4E>(v));   // lane ^ 2
    v = f(v, lanes<0x141>(v));  // the mirror of 8: the other 4
    if constexpr (L >= 16) v = f(v, lanes<0x140>(v));  // the mirror of 16: the other 8
    if constexpr (L >= 32) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v);
        const auto w = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = f(__builtin_bit_cast(float, (uint32_t)w[0]), __builtin_bit_cast(float, (uint32_t)w[1]));
    }
    if constexpr (L >= 64) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v);
        const auto w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        v = f(__builtin_bit_cast(float, (uint32_t)w[0]), __builtin_bit_cast(float, (uint32_t)w[1]));
    }
    return v;
}

// Sums over L lanes of N values; with L above 64, over the workgroup of L threads
// (all call it), through `at`, N * L / 64 floats that no other call uses until a
// barrier behind this one.
template <int L, int N>
__device__ __forceinline__ void add_lanes(float (&v)[N], float *at)
{
    const auto add = [](float a, float b) { return a + b; };
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = over_lanes<(L < 64 ? L : 64)>(v[k], add);
    if constexpr (L > 64) {
        constexpr int kWaves = L / 64;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) at[k * kWaves + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += at[k * kWaves + w];
            v[k] = s;
        }
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int64_t kSizeLimit = (int64_t)1 << 31;

inline size_t round_up(size_t a, size_t m) { return (a + m - 1) / m * m; }

inline int check_size(int64_t v, const char *name)
{
    if (v < 0 || v >= kSizeLimit)
        return fail(ONEBIT_EINVAL, "%s = %lld is not in [0, 2^31)", name, (long long)v);
    return ONEBIT_OK;
}

inline int elem_bytes(int32_t dtype)
{
    return dtype == ONEBIT_GRAD_F32 ? 4
         : dtype == ONEBIT_GRAD_BF16 || dtype == ONEBIT_GRAD_F16 ? 2 : 0;
}

inline int check_rows(const void *p, int32_t dtype, int64_t ld, int64_t rows, int64_t width,
                      const char *name)
{
    const int bytes = elem_bytes(dtype);
    if (!bytes) return fail(ONEBIT_EINVAL, "%s: type %d is not one of ONEBIT_GRAD_*", name, dtype);
    if (rows > 1 && (ld < width || ld > ((int64_t)1 << 40)))
        return fail(ONEBIT_EINVAL, "%s: leading dimension %lld, width %lld", name, (long long)ld,
                    (long long)width);
    if (!p && rows > 0 && width > 0) return fail(ONEBIT_EINVAL, "%s is NULL", name);
    if ((uintptr_t)p % bytes) return fail(ONEBIT_EALIGN, "%s is not %d-byte aligned", name, bytes);
    return ONEBIT_OK;
}

inline int check_ids(const void *ids, int32_t ids_bytes, int64_t tokens)
{
    if (ids_bytes != 4 && ids_bytes != 8)
        return fail(ONEBIT_EINVAL, "ids_bytes = %d is neither 4 nor 8", ids_bytes);
    if (!ids && tokens > 0) return fail(ONEBIT_EINVAL, "ids is NULL");
    if ((uintptr_t)ids % ids_bytes)
        return fail(ONEBIT_EALIGN, "ids is not %d-byte aligned", ids_bytes);
    return ONEBIT_OK;
}

#define TRY(expr)                         \
    do {                                  \
        int _st = (expr);                 \
        if (_st != ONEBIT_OK) return _st; \
    } while (0)

// Calls f with a null pointer of the element type's C++ type.
template <class F>
void with_type(int32_t dtype, F &&f)
{
    if (dtype == ONEBIT_GRAD_F32) f((float *)nullptr);
    else if (dtype == ONEBIT_GRAD_BF16) f((__bf16 *)nullptr);
    else f((_Float16 *)nullptr);
}

inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ONEBIT_OK : hip_fail(e, what);
}

}  // namespace onebit
