// Token embedding: lookup with scaling, and the table's gradient by sorted
// tokens.  Both stream: the lookup reads a row and writes a row per token; the
// gradient reads every token's row once and writes every row of the table once.
// See include/onebit.h for the contract of the entry points.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "../../include/onebit.h"
#include "onebit_internal.h"
#include "onebit_status.h"

namespace onebit {
namespace {

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

// Columns that one thread holds of a row.
constexpr int kCols = 8;

// Item `base + threadIdx.x` of items that are rows of `per_row`: its row, and its
// place in the row.  base is the same in every lane, so that the 64-bit
// division is done once per wave and a lane's own is in 32 bits.
__device__ __forceinline__ int64_t row_of(int64_t base, int per_row, int &in_row)
{
    const int64_t first = base / per_row;
    const uint32_t at = (uint32_t)(base - first * per_row) + threadIdx.x;
    const uint32_t row = at / (uint32_t)per_row;
    in_row = (int)(at - row * per_row);
    return first + row;
}

// out[t] = scale * table[ids[t]]: one thread per kCols columns of a place, so that a
// row of any width is read and written in pieces of 16 or 32 bytes and a call of a
// few hundred places still fills the GPU's CUs.  Memory bounds it: 131,072 places
// of 1,024 columns, fp32 table of 30,522 rows to bf16, move at least 394 MB and take
// 76 us (5.2 TB/s; a copy of 8 GiB reaches 6.8); 10,007 places of 771, bf16 to fp32,
// 46 MB and 8.8 us; 512 places of 1,024 take 2.8 us, the call around them 7.
template <class T, class O>
__global__ __launch_bounds__(256) void k_embedding(const T *__restrict__ table, int64_t table_ld,
                                                   int64_t vocab, int width, int per_row,
                                                   const void *__restrict__ ids, int ids_bytes,
                                                   int64_t tokens, float scale,
                                                   O *__restrict__ out, int64_t out_ld)
{
    for (int64_t base = (int64_t)blockIdx.x * 256; base < tokens * per_row;
         base += (int64_t)gridDim.x * 256) {
        int c;
        const int64_t t = row_of(base, per_row, c);
        if (t >= tokens) return;
        c *= kCols;
        const int64_t id = load_id(ids, ids_bytes, t);
        float v[kCols] = {};
        if (id >= 0 && id < vocab) {
            load_some(table + id * table_ld + c, v, width - c);
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[k] *= scale;
        }
        store_some(out + t * out_ld + c, v, width - c);
    }
}

// ---------------------------------------------------------------------------
// Sorting the places by id: a stable radix sort, least significant digit first.
// A key is the id, or `vocab` for a place that adds nothing (these come last).
// Sorted places make the gradient a sum of runs: every row of dout is read once,
// every row of the table's gradient written once, and the order of a row's sum is
// that of its places (atomics would give another order in every call, and read
// and write each row of the gradient as often as its token occurs).
// ---------------------------------------------------------------------------

constexpr int kDigits = 256;
// Places that one workgroup sorts, in LDS (whose size sets the limit): one launch for
// the sort and one for the sums, where the longer way takes two for every 8 bits of
// the id, one for the sums and one for the rows that cross pieces.  us this way and
// that (vocabulary 30,522, Zipf-distributed ids): 128 places of 1,024 bf16 columns
// 24.3 / 42.8, 1,024 of them 26.1 / 46.9, 4,096 45.4 / 53.5, 4,096 of 256 29.1 / 36.6,
// 4,096 of 771 in fp32 on top of a gradient 34.5 / 34.5.  The sums are one workgroup's
// for each row and group of columns, so that a single id throughout costs more this
// way: 128 places 31 / 43, 1,024 90 / 52, 4,096 303 / 75.
constexpr int kSmallTokens = 4096;
constexpr int kSmallThreads = 1024;
constexpr int kSmallRows = 1 << 18;  // rows that the sorting workgroup has bits for
// Workgroups of a pass over more (each reads the counts of all).  A pass waits for
// memory and does little else: 131,072 places take 5 us to count and 9 to move.
constexpr int kSortBlocks = 128;
constexpr int kFillBlocks = 512;

struct Key {
    int64_t vocab, padding;
    __device__ __forceinline__ uint32_t of(int64_t id) const
    {
        return id >= 0 && id < vocab && id != padding ? (uint32_t)id : (uint32_t)vocab;
    }
};

// Zeros rows [begin, end) of the gradient, by workgroup `part` of `parts`: those
// without a place, once the list is sorted; all of them beside the sort of a short
// list, which keeps few CUs busy and no memory.
struct Fill {
    void *grad;
    int64_t ld;
    int64_t begin, end;  // rows
    int width, elem;     // elem: bytes of an element
};

// Zeros `len` bytes, an even number from an even address on, by `threads` threads.
__device__ __forceinline__ void fill_bytes(char *at, int64_t len, int thread, int threads)
{
    char *stop = at + len;
    char *first = (char *)(((uintptr_t)at + 15) & ~(uintptr_t)15);
    char *last = (char *)((uintptr_t)stop & ~(uintptr_t)15);
    if (first > last) first = last = stop;  // a short run that crosses no 16 bytes
    for (char *q = at + thread * 2; q < first && q < stop; q += threads * 2) *(uint16_t *)q = 0;
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    for (char *q = first + thread * 16; q < last; q += threads * 16)
        __builtin_nontemporal_store(words{0, 0, 0, 0}, (words *)q);
    for (char *q = last + thread * 2; q < stop; q += threads * 2) *(uint16_t *)q = 0;
}

__device__ __forceinline__ void fill_range(const Fill &f, int part, int parts, int64_t &r0,
                                           int64_t &r1)
{
    r0 = f.begin + (f.end - f.begin) * part / parts;
    r1 = f.begin + (f.end - f.begin) * (part + 1) / parts;
}

__device__ void fill_rows(const Fill &f, int part, int parts)
{
    int64_t r0, r1;
    fill_range(f, part, parts, r0, r1);
    const int64_t bytes = (int64_t)f.width * f.elem, pitch = f.ld * f.elem;
    char *base = (char *)f.grad + r0 * pitch;
    if (r0 < r1 && f.ld == f.width)
        fill_bytes(base, bytes * (r1 - r0), threadIdx.x, blockDim.x);  // one run
    else
        for (int64_t r = r0; r < r1; ++r, base += pitch)
            fill_bytes(base, bytes, threadIdx.x, blockDim.x);
}

// The rows that have no bit, a wave for each.
__device__ void fill_unmarked(const Fill &f, const uint32_t *__restrict__ present, int part,
                              int parts)
{
    int64_t r0, r1;
    fill_range(f, part, parts, r0, r1);
    for (int64_t r = r0 + (threadIdx.x >> 6); r < r1; r += blockDim.x >> 6)
        if (!(present[r >> 5] >> (r & 31) & 1))
            fill_bytes((char *)f.grad + r * f.ld * f.elem, (int64_t)f.width * f.elem,
                       threadIdx.x & 63, 64);
}

// The rows without a place: a thread looks its row up in the sorted keys, and a
// wave zeros a row.
__device__ void fill_absent(const Fill &f, const uint32_t *__restrict__ keys, int64_t tokens,
                            int part, int parts)
{
    __shared__ bool absent[256];
    int64_t r0, r1;
    fill_range(f, part, parts, r0, r1);
    for (int64_t r = r0; r < r1; r += 256) {
        const uint32_t row = (uint32_t)(r + threadIdx.x);
        int64_t lo = 0, hi = tokens;  // the first key that is not below the row's
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (keys[mid] < row) lo = mid + 1;
            else hi = mid;
        }
        __syncthreads();
        absent[threadIdx.x] = r + threadIdx.x < r1 && (lo == tokens || keys[lo] != row);
        __syncthreads();
        for (int k = threadIdx.x >> 6; k < 256; k += 4)
            if (absent[k])
                fill_bytes((char *)f.grad + (r + k) * f.ld * f.elem, (int64_t)f.width * f.elem,
                           threadIdx.x & 63, 64);
    }
}

// Orders a wave's LDS accesses: every lane has read (written) what comes before.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Lanes of the wave that hold the same digit as this one (bits: its width), of
// those that are `on`.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool on)
{
    uint64_t same = __ballot(on);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? set : ~set;
    }
    return same;
}

// Exclusive sums of v over the workgroup's first 256 threads (all call it).
__device__ __forceinline__ uint32_t scan256(uint32_t v, uint32_t *wave_sums)
{
    const int tid = threadIdx.x, lane = tid & 63;
    uint32_t x = v;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (tid < kDigits && lane == 63) wave_sums[tid >> 6] = x;
    __syncthreads();
    if (tid < kDigits)
        for (int w = 0; w < (tid >> 6); ++w) x += wave_sums[w];
    __syncthreads();
    return x - v;
}

// Up to kSmallTokens places: workgroup 0 sorts them whole, the others zero rows of
// the gradient.  Every wave owns consecutive keys, so that ranks within a wave and
// waves in order keep the sort stable.  It also leaves where every row's places
// begin (begins[k] for the k-th row that has any, behind them the number of places;
// *rows is their number) and a bit for every row that has any.
__global__ __launch_bounds__(kSmallThreads) void k_sort_small(const void *__restrict__ ids,
                                                              int ids_bytes, int tokens, Key key,
                                                              int bits, uint32_t *keys,
                                                              uint32_t *order,
                                                              uint32_t *begins, uint32_t *rows,
                                                              uint32_t *present, int words,
                                                              Fill fill)
{
    if (blockIdx.x > 0) return fill_rows(fill, blockIdx.x - 1, gridDim.x - 1);
    constexpr int kWaves = kSmallThreads / 64;
    __shared__ uint32_t s_key[2][kSmallTokens], s_at[2][kSmallTokens];
    __shared__ uint32_t s_count[kWaves][kDigits];
    __shared__ uint32_t s_sums[4];
    __shared__ uint32_t s_present[kSmallRows / 32], s_heads[kWaves], s_valid;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    for (int k = tid; k < words; k += kSmallThreads) s_present[k] = 0;
    if (tid == 0) s_valid = 0;
    const int per_wave = (tokens + kWaves * 64 - 1) / (kWaves * 64) * 64;
    const int begin = min(wave * per_wave, tokens), end = min(begin + per_wave, tokens);
    for (int t = tid; t < tokens; t += kSmallThreads) {
        s_key[0][t] = key.of(load_id(ids, ids_bytes, t));
        s_at[0][t] = t;
    }
    int from = 0;
    for (int shift = 0; shift < bits; shift += 8, from ^= 1) {
        const int width = min(8, bits - shift);
        for (int d = tid; d < kWaves * kDigits; d += kSmallThreads) (&s_count[0][0])[d] = 0;
        __syncthreads();
        for (int t = begin + lane; t < end; t += 64)
            atomicAdd(&s_count[wave][(s_key[from][t] >> shift) & 255], 1u);
        __syncthreads();
        uint32_t total = 0;
        if (tid < kDigits)
            for (int w = 0; w < kWaves; ++w) total += s_count[w][tid];
        uint32_t at = scan256(total, s_sums);
        if (tid < kDigits)
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t n = s_count[w][tid];
                s_count[w][tid] = at;
                at += n;
            }
        __syncthreads();
        for (int t0 = begin; t0 < end; t0 += 64) {
            const int t = t0 + lane;
            const bool on = t < end;
            const uint32_t k = on ? s_key[from][t] : 0;
            const uint32_t digit = (k >> shift) & 255;
            const uint64_t same = same_digit(digit, width, on);
            const int rank = __popcll(same & ((1ull << lane) - 1));
            uint32_t pos = 0;
            if (on) {
                pos = s_count[wave][digit] + rank;
                s_key[from ^ 1][pos] = k;
                s_at[from ^ 1][pos] = s_at[from][t];
            }
            wave_sync();  // every lane has read its digit's place
            if (on && rank == 0) s_count[wave][digit] += (uint32_t)__popcll(same);
            wave_sync();
        }
        __syncthreads();
    }
    // heads: places where another row begins
    auto head = [&](int t) {
        const uint32_t k = s_key[from][t];
        return k < key.vocab && (t == 0 || s_key[from][t - 1] != k);
    };
    uint32_t heads = 0, valid = 0;
    for (int t0 = begin; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        const bool on = t < end;
        heads += __popcll(__ballot(on && head(t)));
        valid += __popcll(__ballot(on && s_key[from][t] < key.vocab));
    }
    if (lane == 0) {
        s_heads[wave] = heads;
        atomicAdd(&s_valid, valid);
    }
    __syncthreads();
    uint32_t at = 0;
    for (int w = 0; w < wave; ++w) at += s_heads[w];
    for (int t0 = begin; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        const bool on = t < end && head(t);
        const uint64_t all = __ballot(on);
        if (on) {
            begins[at + __popcll(all & ((1ull << lane) - 1))] = t;
            const uint32_t k = s_key[from][t];
            if (words > 0) atomicOr(&s_present[k >> 5], 1u << (k & 31));
        }
        at += __popcll(all);
    }
    if (wave == kWaves - 1 && lane == 0) {
        begins[at] = s_valid;
        *rows = at;
    }
    for (int t = tid; t < tokens; t += kSmallThreads) {
        keys[t] = s_key[from][t];
        order[t] = s_at[from][t];
    }
    __syncthreads();
    for (int k = tid; k < words; k += kSmallThreads) present[k] = s_present[k];
}

// One digit's counts per workgroup.  FIRST: keys come from the ids.
template <bool FIRST>
__device__ __forceinline__ uint32_t key_at(const void *src, int ids_bytes, const Key &key,
                                           int64_t t)
{
    return FIRST ? key.of(load_id(src, ids_bytes, t)) : ((const uint32_t *)src)[t];
}

template <bool FIRST>
__global__ __launch_bounds__(256) void k_sort_count(const void *__restrict__ src, int ids_bytes,
                                                    int64_t tokens, int64_t per_block, int blocks,
                                                    Key key, int shift, uint32_t *counts)
{
    __shared__ uint32_t s_count[kDigits];
    s_count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * per_block, end = min(begin + per_block, tokens);
    for (int64_t t = begin + threadIdx.x; t < end; t += 256)
        atomicAdd(&s_count[(key_at<FIRST>(src, ids_bytes, key, t) >> shift) & 255], 1u);
    __syncthreads();
    counts[blockIdx.x * kDigits + threadIdx.x] = s_count[threadIdx.x];
}

// Moves a workgroup's keys to their places, from the counts of all workgroups.
template <bool FIRST>
__global__ __launch_bounds__(256) void k_sort_move(const void *__restrict__ src,
                                                   const uint32_t *__restrict__ src_at,
                                                   int ids_bytes, int64_t tokens,
                                                   int64_t per_block, int blocks, Key key,
                                                   int shift, int width,
                                                   const uint32_t *__restrict__ counts,
                                                   uint32_t *__restrict__ keys,
                                                   uint32_t *__restrict__ order)
{
    __shared__ uint32_t s_count[4][kDigits];
    __shared__ uint32_t s_sums[4];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    uint32_t before = 0, total = 0;
#pragma unroll 32
    for (int b = 0; b < blocks; ++b) {
        const uint32_t n = counts[b * kDigits + tid];
        total += n;
        if (b < (int)blockIdx.x) before += n;
    }
    for (int w = 0; w < 4; ++w) s_count[w][tid] = 0;
    const uint32_t base = scan256(total, s_sums) + before;
    const int64_t per_wave = per_block / 4;  // a multiple of 64
    const int64_t block_end = min((blockIdx.x + 1) * per_block, tokens);
    const int64_t begin = min(blockIdx.x * per_block + wave * per_wave, block_end);
    const int64_t end = min(begin + per_wave, block_end);
#pragma unroll 4
    for (int64_t t = begin + lane; t < end; t += 64)
        atomicAdd(&s_count[wave][(key_at<FIRST>(src, ids_bytes, key, t) >> shift) & 255], 1u);
    __syncthreads();
    uint32_t at = base;
    for (int w = 0; w < 4; ++w) {
        const uint32_t n = s_count[w][tid];
        s_count[w][tid] = at;
        at += n;
    }
    __syncthreads();
    constexpr int kBatch = 4;  // rounds of 64 whose keys are loaded together
    for (int64_t t0 = begin; t0 < end; t0 += 64 * kBatch) {
        uint32_t k[kBatch], from[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t t = min(t0 + u * 64 + lane, end - 1);
            k[u] = key_at<FIRST>(src, ids_bytes, key, t);
            from[u] = FIRST ? (uint32_t)t : src_at[t];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const bool on = t0 + u * 64 + lane < end;
            const uint32_t digit = (k[u] >> shift) & 255;
            const uint64_t same = same_digit(digit, width, on);
            const int rank = __popcll(same & ((1ull << lane) - 1));
            if (on) {
                const uint32_t pos = s_count[wave][digit] + rank;
                keys[pos] = k[u];
                order[pos] = from[u];
            }
            wave_sync();
            if (on && rank == 0) s_count[wave][digit] += (uint32_t)__popcll(same);
            wave_sync();
        }
    }
}

// ---------------------------------------------------------------------------
// Sums over the sorted places
// ---------------------------------------------------------------------------

// The sorted list is cut into pieces of `piece` places, whatever rows they
// belong to, so that a frequent token costs what its places do.  A thread adds
// V columns of a piece's places in order.  A row that lies inside a piece is
// finished there; a row that crosses a piece's end leaves one partial sum per
// piece it touches (slot 0: it began in an earlier piece, slot 1: it begins
// here), which k_grad_join adds.
struct Sums {
    const uint32_t *keys, *order;
    int64_t tokens, vocab;
    int width, per_row, piece;  // per_row: threads that share a row
    int64_t pieces;
    float scale;
    int accumulate;
    int64_t dout_ld, grad_ld;
    float *partial;  // [pieces][2][per_row * V]
};

// Columns of a row's thread number n: V from n V on, or, so that every load is a
// whole one, the row's last V.  skip: those that the thread before has too.
template <int V>
struct Columns {
    int first, skip;
    __device__ __forceinline__ Columns(int n, int width)
        : first(V == 1 ? n : min(n * V, width - V)), skip(n * V - first) {}
};

template <int V, class G>
__device__ __forceinline__ void finish_row(const Sums &s, G *__restrict__ grad, uint32_t row,
                                           const Columns<V> &c, const float (&acc)[V])
{
    G *p = grad + (int64_t)row * s.grad_ld + c.first;
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = s.scale * acc[k];
    if (c.skip == 0) {
        if (s.accumulate) {
            float old[V];
            load_vec(p, old);
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] += old[k];
        }
        stream_vec(p, v);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k >= c.skip) p[k] = (G)(s.accumulate ? v[k] + (float)p[k] : v[k]);
    }
}

template <int V>
__device__ __forceinline__ float *partial_at(const Sums &s, int64_t piece, int slot, int n)
{
    return s.partial + ((piece * 2 + slot) * s.per_row + n) * V;
}

constexpr int kAhead = 4;  // rows whose loads are in flight together
constexpr int kJoin = 8;   // threads that share a crossing row's partial sums

template <class T, int V>
struct Raw {  // elements as they lie in memory
    T v[V];
    // every row is read once, so that it need not stay in the caches
    __device__ __forceinline__ void load(const T *p)
    {
        constexpr int kBytes = sizeof(T) * V;
        if constexpr (kBytes < 4) {
            __builtin_memcpy(v, p, kBytes);
        } else {
            static_assert(kBytes == 4 || kBytes == 16, "one load");
            typedef uint32_t words __attribute__((ext_vector_type(kBytes / 4), aligned(sizeof(T))));
            const words w = __builtin_nontemporal_load((const words *)p);
            __builtin_memcpy(v, &w, kBytes);
        }
    }
};

// A thread's work is a chain: the list's entries, the rows they name, their sums.
// (Memory bounds it where the list is long: 131,072 bf16 places of 1,024 columns,
// fp32 gradient of 30,522 rows, move 394 MB in 80 to 93 us, 4.2 to 4.9 TB/s, a third of
// the rows zeroed in between; 33,333 fp32 places of 771 columns added to 5,003 rows, 134
// MB in 31 us.)
// Each part runs a batch ahead of the next: while a batch is added, the next one's
// rows and the entries of the one after are under way.  The loads stand outside of
// every branch (an entry that adds nothing reads row 0 instead): where their
// number is not known the compiler waits for all of them.
template <class D, class G, int V>
__global__ __launch_bounds__(256) void k_grad_sum(Sums s, const D *__restrict__ dout,
                                                  G *__restrict__ grad, int blocks, Fill fill)
{
    if ((int)blockIdx.x >= blocks)
        return fill_absent(fill, s.keys, s.tokens, blockIdx.x - blocks, gridDim.x - blocks);
    int n;
    const int64_t piece = row_of((int64_t)blockIdx.x * 256, s.per_row, n);
    if (piece >= s.pieces) return;
    const Columns<V> c(n, s.width);
    const int64_t begin = piece * s.piece, end = min(begin + s.piece, s.tokens);
    const uint32_t none = (uint32_t)s.vocab;
    const D *from = dout + c.first;
    struct Batch {
        uint32_t key[kAhead], at[kAhead];
    };
    // (the list's areas reach four batches past the last piece)
    auto entries = [&](int64_t at, Batch &b) {
        __builtin_memcpy(b.key, __builtin_assume_aligned(s.keys + at, 16), sizeof b.key);
        __builtin_memcpy(b.at, __builtin_assume_aligned(s.order + at, 16), sizeof b.at);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool on = at + u < end && b.key[u] < none;
            b.key[u] = on ? b.key[u] : none;
            b.at[u] = on ? b.at[u] : 0;
        }
    };
    auto rows = [&](const Batch &b, Raw<D, V> (&r)[kAhead]) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            r[u].load(from + (int64_t)b.at[u] * s.dout_ld);
    };
    Batch entry[2];
    Raw<D, V> r[2][kAhead];
    entries(begin, entry[0]);
    entries(begin + kAhead, entry[1]);
    const uint32_t previous = begin > 0 ? s.keys[begin - 1] : none;
    const uint32_t following = end < s.tokens ? s.keys[end] : none;
    rows(entry[0], r[0]);
    uint32_t row = entry[0].key[0];
    if (row == none) return;  // places that add nothing, as all that follow
    bool before = previous == row;
    float acc[V] = {};
    // (two batches by turns, with no copies from one to the other: a copy would wait)
    auto batch = [&](int64_t at, Batch &now, const Raw<D, V> (&mine)[kAhead], const Batch &next,
                     Raw<D, V> (&theirs)[kAhead]) {
        Batch after;
        entries(at + 2 * kAhead, after);
        rows(next, theirs);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (now.key[u] != row) {  // the row ends here
                if (now.key[u] == none) break;
                if (before)
                    store_vec(partial_at<V>(s, piece, 0, n), acc);
                else
                    finish_row<V>(s, grad, row, c, acc);
                row = now.key[u];
                before = false;
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += (float)mine[u].v[i];
        }
        now = after;
    };
    for (int64_t at = begin; at < end; at += 2 * kAhead) {
        batch(at, entry[0], r[0], entry[1], r[1]);
        batch(at + kAhead, entry[1], r[1], entry[0], r[0]);
    }
    if (before)
        store_vec(partial_at<V>(s, piece, 0, n), acc);
    else if (following == row)
        store_vec(partial_at<V>(s, piece, 1, n), acc);
    else
        finish_row<V>(s, grad, row, c, acc);
}

// Rows that cross pieces, by the piece they begin in: of the pieces that follow,
// each of kJoin threads adds every kJoin-th, and their sums are added in order.  The
// chain of the most frequent row's pieces bounds it (131,072 places: 12 us).
template <class G, int V>
__global__ __launch_bounds__(256) void k_grad_join(Sums s, G *__restrict__ grad)
{
    __shared__ float part[kJoin][256 / kJoin][V + 1];
    const int groups = (s.per_row + 256 / kJoin - 1) / (256 / kJoin);  // of columns
    const int64_t piece = blockIdx.x / groups;
    const int64_t begin = piece * s.piece, end = begin + s.piece;
    if (end >= s.tokens) return;
    const uint32_t row = s.keys[end];
    if (row >= s.vocab || s.keys[end - 1] != row) return;
    if (begin > 0 && s.keys[begin] == row && s.keys[begin - 1] == row) return;  // it began earlier
    const int lane = threadIdx.x % (256 / kJoin), turn = threadIdx.x / (256 / kJoin);
    const int n = (int)(blockIdx.x % groups) * (256 / kJoin) + lane;
    const bool mine = n < s.per_row;
    float acc[V] = {};
    if (turn == 0 && mine) load_vec(partial_at<V>(s, piece, 1, n), acc);
    constexpr int kBatch = 4;
    for (int64_t q = piece + 1 + turn; q < s.pieces; q += kBatch * kJoin) {
        float v[kBatch][V];
        bool on[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t p = min(q + u * kJoin, s.pieces - 1);
            on[u] = q + u * kJoin < s.pieces && s.keys[p * s.piece] == row;
            if (mine) load_vec(partial_at<V>(s, p, 0, n), v[u]);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (on[u])
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += v[u][i];
        if (!on[kBatch - 1]) break;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) part[turn][lane][i] = acc[i];
    __syncthreads();
    if (turn > 0 || !mine) return;
#pragma unroll
    for (int t = 1; t < kJoin; ++t)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += part[t][lane][i];
    finish_row<V>(s, grad, row, Columns<V>(n, s.width), acc);
}

// Sums of a short list: a workgroup takes one row's places, or up to `across`
// threads' columns of them, with kSmallThreads / across threads per column that add
// every so manieth place; their sums are added in order.  The workgroups behind the
// rows' zero the rows without a place, which bounds it: for 512 places of 1,024
// columns and 30,522 fp32 rows the sort takes 12 us and this 14, each with half of the
// 125 MB to be zeroed.
template <class D, class G, int V>
__global__ __launch_bounds__(kSmallThreads) void k_grad_rows(Sums s, const D *__restrict__ dout,
                                                             G *__restrict__ grad, int across,
                                                             int groups,
                                                             const uint32_t *__restrict__ begins,
                                                             const uint32_t *__restrict__ rows,
                                                             const uint32_t *__restrict__ present,
                                                             Fill fill)
{
    __shared__ float part[kSmallThreads * V];
    const int blocks = (int)s.tokens * groups;
    if ((int)blockIdx.x >= blocks)
        return fill_unmarked(fill, present, blockIdx.x - blocks, gridDim.x - blocks);
    const int index = blockIdx.x / groups;
    if (index >= (int)*rows) return;
    const int begin = begins[index], end = begins[index + 1];
    const int turns = kSmallThreads / across, turn = threadIdx.x / across;
    const int n = blockIdx.x % groups * across + threadIdx.x % across;
    const bool mine = n < s.per_row && turn < turns;
    const Columns<V> c(min(n, s.per_row - 1), s.width);
    const D *from = dout + c.first;
    float acc[V] = {};
    if (mine)
        for (int at = begin + turn; at < end; at += turns * kAhead) {
            Raw<D, V> r[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)  // (past the end: the last place again)
                r[u].load(from + (int64_t)s.order[min(at + u * turns, end - 1)] * s.dout_ld);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (at + u * turns < end)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[i] += (float)r[u].v[i];
        }
    const int used = min(turns, end - begin);
    if (used > 1) {
        if (turn > 0 && turn < used)
#pragma unroll
            for (int i = 0; i < V; ++i) part[threadIdx.x * V + i] = acc[i];
        __syncthreads();
    }
    if (turn > 0 || !mine) return;
    for (int t = 1; t < used; ++t)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += part[(t * across + threadIdx.x) * V + i];
    finish_row<V>(s, grad, s.keys[begin], c, acc);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------

constexpr int64_t kSizeLimit = (int64_t)1 << 31;

struct GradLayout {
    int piece, columns;  // columns: of a thread
    int64_t pieces, per_row;
    size_t keys[2], order[2], counts, partial, begins, rows, present;  // byte offsets
};

size_t round_up(size_t a, size_t m) { return (a + m - 1) / m * m; }

// Columns of a thread: 16 bytes of dout, or one where a row is shorter than that.
// Places per piece: as many as still leave 2^18 threads, from 8 to 128, which bounds
// the partial sums and the join's chains.  us of the call, pieces of 8 / 16 / 32 / 64 /
// 128: 131,072 bf16 places of 1,024 columns 179 / 147 / 128 / 126 / 123 (64 here), of a
// single id 894 / 496 / 296 / 192 / 153; 33,333 fp32 ones of 771, added, 76 / 72 / 79 /
// 95 / 140 (16; 193 threads a row); 20,000 bf16 ones of 1,024 81 / 76 / 75 / 76 / 98
// (8).
constexpr int kLeastPiece = 8, kMostPiece = 128;
constexpr int64_t kPieceThreads = 1 << 18;

GradLayout grad_layout(int64_t tokens, int64_t width, int elem)
{
    GradLayout l{};
    l.columns = width >= 16 / elem ? 16 / elem : 1;
    l.per_row = (width + l.columns - 1) / l.columns;
    l.piece = kLeastPiece;
    while (l.piece < kMostPiece && tokens / (2 * l.piece) * l.per_row >= kPieceThreads) l.piece *= 2;
    l.pieces = (tokens + l.piece - 1) / l.piece;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    for (int k = 0; k < 2; ++k) {
        l.keys[k] = take((round_up(tokens, kMostPiece) + 4 * kAhead) * 4);
        l.order[k] = take((round_up(tokens, kMostPiece) + 4 * kAhead) * 4);
    }
    l.begins = take(((size_t)std::min<int64_t>(tokens, kSmallTokens) + 1) * 4);
    l.rows = take(4);
    l.present = take(kSmallRows / 8);
    l.counts = take((size_t)kSortBlocks * kDigits * 4);
    l.partial = at;
    return l;
}

// Bytes that serve every call of up to so many tokens and columns.  The areas before
// the partial sums grow with the tokens, but there are fewer partial sums where a
// longer piece begins: a call has pieces * 2 * (its columns, padded to its threads').
// With the longest piece that is at most the first number below; with a shorter one
// tokens / (2 piece) * per_row stayed below kPieceThreads, so that pieces * per_row is
// below 2 kPieceThreads + 2 per_row, and pieces are at least kLeastPiece places.
size_t grad_workspace(int64_t tokens, int64_t width, int elem)
{
    const GradLayout l = grad_layout(tokens, width, elem);
    const size_t padded = (size_t)(l.per_row * l.columns);
    auto pieces = [&](int piece) { return round_up(tokens, piece) / piece; };
    const size_t longest = pieces(kMostPiece) * padded;
    const size_t shorter = std::min(pieces(kLeastPiece) * padded,
                                    2 * (size_t)kPieceThreads * (16 / elem) + 2 * padded);
    return l.partial + round_up(std::max(longest, shorter) * 2 * 4, 256);
}

int check_size(int64_t v, const char *name)
{
    if (v < 0 || v >= kSizeLimit)
        return fail(ONEBIT_EINVAL, "%s = %lld is not in [0, 2^31)", name, (long long)v);
    return ONEBIT_OK;
}

int elem_bytes(int32_t dtype)
{
    return dtype == ONEBIT_GRAD_F32 ? 4
         : dtype == ONEBIT_GRAD_BF16 || dtype == ONEBIT_GRAD_F16 ? 2 : 0;
}

int check_rows(const void *p, int32_t dtype, int64_t ld, int64_t rows, int64_t width,
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

int check_ids(const void *ids, int32_t ids_bytes, int64_t tokens)
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

int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ONEBIT_OK : hip_fail(e, what);
}

}  // namespace
}  // namespace onebit

using namespace onebit;

extern "C" {

int onebit_embedding_forward(const void *table, int32_t table_dtype, int64_t table_ld,
                             int64_t vocab, int64_t width, const void *ids, int32_t ids_bytes,
                             int64_t tokens, float scale, void *out, int32_t out_dtype,
                             int64_t out_ld, onebit_stream stream)
{
    TRY(check_size(vocab, "vocab"));
    TRY(check_size(width, "width"));
    TRY(check_size(tokens, "tokens"));
    TRY(check_rows(table, table_dtype, table_ld, vocab, width, "table"));
    TRY(check_rows(out, out_dtype, out_ld, tokens, width, "out"));
    TRY(check_ids(ids, ids_bytes, tokens));
    if (tokens == 0 || width == 0) return ONEBIT_OK;
    const int per_row = (int)((width + kCols - 1) / kCols);
    const int64_t items = tokens * per_row;
    const int blocks = (int)std::min<int64_t>((items + 255) / 256, 1 << 22);
    with_type(table_dtype, [&](auto *t) {
        with_type(out_dtype, [&](auto *o) {
            using T = std::remove_pointer_t<decltype(t)>;
            using O = std::remove_pointer_t<decltype(o)>;
            k_embedding<T, O><<<blocks, 256, 0, (hipStream_t)stream>>>(
                (const T *)table, table_ld, vocab, (int)width, per_row, ids, ids_bytes, tokens,
                scale, (O *)out, out_ld);
        });
    });
    return launched("embedding kernel launch");
}

int onebit_embedding_grad_workspace(int64_t tokens, int64_t vocab, int64_t width, size_t *bytes)
{
    if (!bytes) return fail(ONEBIT_EINVAL, "bytes is NULL");
    TRY(check_size(tokens, "tokens"));
    TRY(check_size(vocab, "vocab"));
    TRY(check_size(width, "width"));
    *bytes = std::max(grad_workspace(tokens, width, 2), grad_workspace(tokens, width, 4));
    return ONEBIT_OK;
}

int onebit_embedding_grad(const void *dout, int32_t dout_dtype, int64_t dout_ld, const void *ids,
                          int32_t ids_bytes, int64_t tokens, int64_t vocab, int64_t width,
                          int64_t padding_id, float scale, void *grad, int32_t grad_dtype,
                          int64_t grad_ld, int32_t accumulate, void *workspace,
                          onebit_stream stream)
{
    TRY(check_size(vocab, "vocab"));
    TRY(check_size(width, "width"));
    TRY(check_size(tokens, "tokens"));
    TRY(check_rows(dout, dout_dtype, dout_ld, tokens, width, "dout"));
    TRY(check_rows(grad, grad_dtype, grad_ld, vocab, width, "grad"));
    TRY(check_ids(ids, ids_bytes, tokens));
    if (!workspace) return fail(ONEBIT_EINVAL, "workspace is NULL");
    if ((uintptr_t)workspace % 16) return fail(ONEBIT_EALIGN, "workspace is not 16-byte aligned");
    if (vocab == 0 || width == 0 || (tokens == 0 && accumulate)) return ONEBIT_OK;
    hipStream_t st = (hipStream_t)stream;
    const GradLayout l = grad_layout(tokens, width, elem_bytes(dout_dtype));
    // Launches stay below 2^32 threads: where a short list's sums would not, because its
    // rows are very wide, it goes the longer way, whose workgroups take many places.
    const int across = (int)std::min<int64_t>(l.per_row, 128);
    const int64_t groups = (l.per_row + across - 1) / across;
    const bool small = tokens <= kSmallTokens &&
                       tokens * groups + 4 * kFillBlocks < ((int64_t)1 << 32) / kSmallThreads;
    const int64_t blocks = (l.pieces * l.per_row + 255) / 256;
    const int64_t joins = (l.per_row + 256 / kJoin - 1) / (256 / kJoin);  // workgroups of a piece
    if (!small && (blocks > (1 << 23) || l.pieces * joins > (1 << 23)))
        return fail(ONEBIT_EINVAL, "%lld places of %lld columns are too many for one call",
                    (long long)tokens, (long long)width);
    char *ws = (char *)workspace;
    const Key key{vocab, padding_id < 0 ? -1 : padding_id};
    const int bits = 32 - __builtin_clz((uint32_t)vocab);  // keys are 0..vocab
    Fill fill{grad, vocab > 1 ? grad_ld : width, 0, accumulate ? 0 : vocab, (int)width,
              elem_bytes(grad_dtype)};
    const int fills = accumulate ? 0 : (int)std::min<int64_t>(kFillBlocks, vocab);
    int now = 0;
    // Half of the rows are zeroed beside the sort of a short list, all of them where
    // there are too many for its bits; the others beside the sums.
    const int words = small && vocab <= kSmallRows ? (int)((vocab + 31) / 32) : 0;
    Fill rest = fill;
    if (small) {
        rest.begin = tokens == 0 || words == 0 ? fill.end : fill.end / 2;
        fill.end = rest.begin;
        k_sort_small<<<1 + fills, kSmallThreads, 0, st>>>(
            ids, ids_bytes, (int)tokens, key, bits, (uint32_t *)(ws + l.keys[0]),
            (uint32_t *)(ws + l.order[0]), (uint32_t *)(ws + l.begins), (uint32_t *)(ws + l.rows),
            (uint32_t *)(ws + l.present), words, fill);
    } else {
        const int sorters = (int)std::min<int64_t>(kSortBlocks, (tokens + 1023) / 1024);
        const int64_t per_block = ((tokens + sorters - 1) / sorters + 255) / 256 * 256;
        uint32_t *counts = (uint32_t *)(ws + l.counts);
        const int passes = (bits + 7) / 8;
        const void *src = ids;
        const uint32_t *src_at = nullptr;
        for (int p = 0; p < passes; ++p) {
            const int shift = 8 * p, width_bits = std::min(8, bits - shift);
            uint32_t *keys = (uint32_t *)(ws + l.keys[p & 1]);
            uint32_t *order = (uint32_t *)(ws + l.order[p & 1]);
            if (p == 0) {
                k_sort_count<true><<<sorters, 256, 0, st>>>(
                    src, ids_bytes, tokens, per_block, sorters, key, shift, counts);
                k_sort_move<true><<<sorters, 256, 0, st>>>(
                    src, src_at, ids_bytes, tokens, per_block, sorters, key, shift, width_bits,
                    counts, keys, order);
            } else {
                k_sort_count<false><<<sorters, 256, 0, st>>>(
                    src, ids_bytes, tokens, per_block, sorters, key, shift, counts);
                k_sort_move<false><<<sorters, 256, 0, st>>>(
                    src, src_at, ids_bytes, tokens, per_block, sorters, key, shift, width_bits,
                    counts, keys, order);
            }
            src = keys;
            src_at = order;
            now = p & 1;
        }
    }
    TRY(launched("embedding gradient sort launch"));
    if (tokens == 0) return ONEBIT_OK;
    Sums s{(const uint32_t *)(ws + l.keys[now]), (const uint32_t *)(ws + l.order[now]), tokens,
           vocab, (int)width, (int)l.per_row, l.piece, l.pieces, scale, accumulate, dout_ld,
           grad_ld, (float *)(ws + l.partial)};
    const int absent = accumulate ? 0 : (int)std::min<int64_t>(4 * kFillBlocks, (rest.end - rest.begin + 31) / 32);
    auto sums = [&](auto columns, auto *d, auto *g) {
        using D = std::remove_pointer_t<decltype(d)>;
        using G = std::remove_pointer_t<decltype(g)>;
        constexpr int V = decltype(columns)::value;
        if (small) {
            k_grad_rows<D, G, V><<<(int)(tokens * groups) + absent, kSmallThreads, 0, st>>>(
                s, (const D *)dout, (G *)grad, across, (int)groups, (const uint32_t *)(ws + l.begins),
                (const uint32_t *)(ws + l.rows), (const uint32_t *)(ws + l.present), rest);
            return;
        }
        k_grad_sum<D, G, V><<<blocks + absent, 256, 0, st>>>(s, (const D *)dout, (G *)grad,
                                                             (int)blocks, rest);
        if (l.pieces > 1) k_grad_join<G, V><<<l.pieces * joins, 256, 0, st>>>(s, (G *)grad);
    };
    with_type(grad_dtype, [&](auto *g) {
        with_type(dout_dtype, [&](auto *d) {
            constexpr int kWide = 16 / sizeof(*d);
            if (l.columns == 1) sums(std::integral_constant<int, 1>{}, d, g);
            else sums(std::integral_constant<int, kWide>{}, d, g);
        });
    });
    return launched("embedding gradient launch");
}

}  // extern "C"
