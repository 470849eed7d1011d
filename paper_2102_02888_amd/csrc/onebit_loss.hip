// What a language model's logits are turned into: log-probabilities of given tokens
// with the rows' entropies and top alternatives, the divergence from a teacher's top
// logits, and the logits' gradient of either.  Every call is one launch in which a
// workgroup reads a row once, into registers where it fits, and forms everything that
// is wanted of it.  See include/onebit.h for the contract of the entry points.
//
// Numbers.  With M the row's largest logit, d = x - M, e = 2^(d scale log2(e)) and
// S the sum of e, all fp32:  log p = d scale - ln S,  p = e / S,
// entropy = ln S - scale (sum of e d) / S.  M starts at the lowest finite number, so
// that a row whose logits are all that number is uniform, and one whose logits are all
// -infinity has S = 0: it has no distribution.
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

constexpr int kCols = 8;         // logits that a thread holds together
constexpr int kMostTop = 64;     // alternatives of a row
constexpr int kMostTeacher = 256;
constexpr int64_t kMostVocab = 1 << 30;
constexpr int kCandidates = 512;
constexpr float kLowest = -FLT_MAX;
constexpr float kLog2e = 1.44269504088896340736f;

// kCols logits as the words that they are; -infinity behind the end.
template <class T>
struct Piece {
    static constexpr int kWords = kCols * sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T *row, int at, int vocab)
    {
        if (at + kCols <= vocab) {
            __builtin_memcpy(w, row + at, sizeof w);
        } else {
            T t[kCols];
#pragma unroll
            for (int k = 0; k < kCols; ++k) t[k] = at + k < vocab ? row[at + k] : (T)-INFINITY;
            __builtin_memcpy(w, t, sizeof w);
        }
    }
    __device__ __forceinline__ void widen(float (&x)[kCols]) const
    {
        T t[kCols];
        __builtin_memcpy(t, w, sizeof t);
#pragma unroll
        for (int k = 0; k < kCols; ++k) x[k] = (float)t[k];
    }
};

// A row of logits over the TH threads of a workgroup, in registers: piece c of a
// thread is kCols logits from (c TH + thread) kCols on; -infinity behind the end.
template <class T, int TH, int C>
struct Held {
    static constexpr bool kHeld = true;
    Piece<T> piece[C];
    __device__ __forceinline__ Held(const T *row, int vocab)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) piece[c].load(row, (c * TH + (int)threadIdx.x) * kCols, vocab);
    }
    // f(kCols logits as fp32, the first one's column).  Every pass converts them anew:
    // the compiler is kept from holding what another pass made of them, which would
    // take two to four times the registers.
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int k = 0; k < Piece<T>::kWords; ++k) asm volatile("" : "+v"(piece[c].w[k]));
            float x[kCols];
            piece[c].widen(x);
            f(x, (c * TH + (int)threadIdx.x) * kCols);
            __builtin_amdgcn_sched_barrier(0);  // one piece at a time, for the same reason
        }
    }
};

// ... one that does not fit: read again by every pass over it.
template <class T, int TH>
struct Held<T, TH, 0> {
    static constexpr bool kHeld = false;
    const T *row;
    int vocab;
    __device__ __forceinline__ Held(const T *r, int n) : row(r), vocab(n) {}
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
        for (int at = (int)threadIdx.x * kCols; at < vocab; at += TH * kCols) {
            Piece<T> piece;
            piece.load(row, at, vocab);
            float x[kCols];
            piece.widen(x);
            f(x, at);
        }
    }
};

// Waves that a SIMD has to hold: two of the largest workgroups on a CU, so that one
// computes while the other's loads and stores run (8,192 rows of 30,522 bf16 logits, the
// distillation's gradient: 316 us with one, 214 with two).
template <int TH>
constexpr int kWavesFor = TH == 1024 ? 8 : 4;

// LDS of a workgroup of TH threads.
template <int TH>
struct Shared {
    float most[TH / 64], sums[2 * TH / 64];
    float taken[2];  // logit of the given token, teacher's total
};

template <int TH>
__device__ __forceinline__ float most_of(float m, Shared<TH> &s)
{
    m = over_lanes<64>(m, [](float a, float b) { return fmaxf(a, b); });
    if constexpr (TH > 64) {
        if ((threadIdx.x & 63) == 0) s.most[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TH / 64; ++w) m = fmaxf(m, s.most[w]);
    }
    return m;
}

// The row's largest logit, and of all of it the sum of e and, with ENT, of e d.
// mine: the largest of this thread's.  before: called before the barrier behind which
// the sums are known.
template <int TH, bool ENT, class Row, class Before>
__device__ __forceinline__ void statistics(Row &row, float c, Shared<TH> &s, float &most,
                                           float &mine, bool &mine_nan, float &sum, float &moment,
                                           Before before)
{
    mine = kLowest;
    float two[ENT ? 2 : 1] = {};
    const auto add = [&](const float(&x)[kCols], float m) {
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
            const float d = x[k] - m;
            const float e = __builtin_amdgcn_exp2f(d * c);
            two[0] += e;
            // (0 times -infinity is not wanted)
            if constexpr (ENT) two[1] = __builtin_fmaf(e, fmaxf(d, kLowest), two[1]);
        }
    };
    // brings the sums from this thread's maximum to another
    const auto rebase = [&](float m) {
        const float d = mine - m, f = __builtin_amdgcn_exp2f(d * c);
        if constexpr (ENT) two[1] = f == 0.f ? 0.f : f * __builtin_fmaf(two[0], d, two[1]);
        two[0] *= f;
    };
    if constexpr (Row::kHeld) {
        row.each([&](float(&x)[kCols], int) {
#pragma unroll
            for (int k = 0; k < kCols; ++k) mine = fmaxf(mine, x[k]);
        });
        most = most_of<TH>(mine, s);
        row.each([&](float(&x)[kCols], int) { add(x, most); });
    } else {  // in one pass over the memory, each thread with a maximum of its own
        row.each([&](float(&x)[kCols], int) {
            float m = mine;
#pragma unroll
            for (int k = 0; k < kCols; ++k) m = fmaxf(m, x[k]);
            if (m > mine) {
                rebase(m);
                mine = m;
            }
            add(x, m);
        });
        most = most_of<TH>(mine, s);
        rebase(most);
    }
    mine_nan = two[0] != two[0];
    before();
    add_lanes<TH>(two, s.sums);
    sum = two[0];
    moment = ENT ? two[ENT ? 1 : 0] : 0.f;
}

// ---------------------------------------------------------------------------
// Top alternatives.  A key orders by the logit, then the lowest column first; NaN is
// above all numbers.  The largest logits of 128 (64) groups of threads are known; the
// k-th largest of those bounds the row's k-th largest from below, and little more than
// k logits reach it unless many are equal or fewer than k groups hold a finite one.  Those
// are gathered and ranked; too many of them are taken one by one, each by a pass over the
// row (4,096 rows of 30,522 bf16 logits, 20 alternatives: 80 us, of equal logits or all but
// three masked 1,490; of 1,000, whose groups are fewer than 64 alternatives, 274, of 1,100
// 35).
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t order_of(float x)
{
    if (x != x) return 0xffffffffu;
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);  // -0 as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint64_t key_of(float x, int column)
{
    return (uint64_t)order_of(x) << 32 | ~(uint32_t)column;
}

template <int TH>
struct SharedTop {
    static constexpr int kGroups = TH >= 128 ? 128 : TH;
    float group[kGroups];
    float bound;
    int count;
    uint64_t best[TH / 64];
    uint64_t key[kCandidates + 8];
};

// What top_of() needs before the barrier that it begins behind.
template <int TH>
__device__ __forceinline__ void prepare_top(float mine, SharedTop<TH> &s)
{
    constexpr int kPer = TH / SharedTop<TH>::kGroups;
    const int tid = threadIdx.x;
    float m = mine;
    const auto larger = [](float a, float b) { return fmaxf(a, b); };
    if constexpr (kPer == 8) m = over_lanes<8>(m, larger);
    if constexpr (kPer == 4) m = larger(m, lanes<0xB1>(m)), m = larger(m, lanes<0x4E>(m));
    if constexpr (kPer == 2) m = larger(m, lanes<0xB1>(m));
    if (tid % kPer == 0) s.group[tid / kPer] = m;
    if (tid == 0) s.count = 0;
    for (int i = tid; i < kCandidates + 8; i += TH) s.key[i] = 0;  // below every key
}

// put(rank, column, logit) for the k largest of the row, by one thread each.
template <int TH, class T, class Row, class Put>
__device__ __forceinline__ void top_of(Row &row, const T *logits, int vocab, int k, float mine,
                                       bool mine_nan, SharedTop<TH> &s, Put put)
{
    constexpr int kGroups = SharedTop<TH>::kGroups;
    const int tid = threadIdx.x;
    {
        // Every wave looks at some of the groups' values: the one that fewer than k are
        // above, and k or more are not below, is the k-th.
        constexpr int kEach = kGroups / (TH / 64);
        const int lane = tid & 63, first = __builtin_amdgcn_readfirstlane(tid >> 6) * kEach;
        const float a = s.group[lane], b = kGroups > 64 ? s.group[kGroups - 64 + lane] : -INFINITY;
        const float mine_of = s.group[first + lane % kEach];
#pragma unroll 8
        for (int i = 0; i < kEach; ++i) {
            const float x = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, mine_of), i));
            const int above = __popcll(__ballot(a > x)) + __popcll(__ballot(b > x));
            const int reach = __popcll(__ballot(a >= x)) + __popcll(__ballot(b >= x));
            // fewer than k groups with a logit above the lowest number (the largest of the
            // others starts there): all logits
            if (above < k && reach >= k && lane == 0) s.bound = x > kLowest ? x : -INFINITY;
        }
    }
    __syncthreads();
    const float bound = s.bound;
    if (!(mine < bound) || mine_nan)
        row.each([&](float(&x)[kCols], int at) {
            bool any = false;
#pragma unroll
            for (int i = 0; i < kCols; ++i) any |= !(x[i] < bound);
            if (!any) return;
#pragma unroll
            for (int i = 0; i < kCols; ++i)
                if (!(x[i] < bound) && at + i < vocab) {
                    const int to = atomicAdd(&s.count, 1);
                    if (to < kCandidates) s.key[to] = key_of(x[i], at + i);
                }
        });
    __syncthreads();
    const int count = s.count;
    const auto give = [&](int rank, uint64_t key) {
        const uint32_t o = (uint32_t)(key >> 32);
        const uint32_t u = o & 0x80000000u ? o & 0x7fffffffu : ~o;
        put(rank, (int)~(uint32_t)key, __builtin_bit_cast(float, u));
    };
    if (count <= kCandidates) {
        for (int i = tid; i < count; i += TH) {
            const uint64_t key = s.key[i];
            int rank = 0;
            for (int j = 0; j < count; j += 8)  // (zeros behind the last)
#pragma unroll
                for (int k = 0; k < 8; ++k) rank += s.key[j + k] > key;
            if (rank < k) give(rank, key);
        }
    } else {  // many equal logits: one after another, each by a pass over the row in memory
        Held<T, TH, 0> again(logits, vocab);
        uint64_t most = ~0ull;  // (itself a key: NaN in the first column)
        for (int r = 0; r < k; ++r) {
            uint64_t best = 0;
            again.each([&](float(&x)[kCols], int at) {
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const uint64_t key = key_of(x[i], at + i);
                    if (at + i < vocab && key <= most && key > best) best = key;
                }
            });
            for (int d = 1; d < 64; d *= 2) {
                const uint64_t other = __shfl_xor(best, d);
                best = other > best ? other : best;
            }
            if constexpr (TH > 64) {
                if ((tid & 63) == 0) s.best[tid >> 6] = best;
                __syncthreads();
                for (int w = 0; w < TH / 64; ++w) best = s.best[w] > best ? s.best[w] : best;
                __syncthreads();
            }
            if (tid == 0) give(r, best);
            most = best - 1;
        }
    }
    for (int r = min(vocab, k) + tid; r < k; r += TH) put(r, -1, -INFINITY);
}

struct Logits {
    int64_t ld, first;  // first: the launch's first row
    int vocab;
    float scale;
};

// What a call gives of each row; pointers may be null.
struct Values {
    float *logprob, *entropy;
    void *top_ids;
    float *top_logprob;
    int top, top_bytes;
};

// 4,096 rows of 30,522 bf16 logits (a floor of 37 us): the log-probabilities 45 us, with
// entropies 54, with 20 alternatives too 86, bounded by the VALU, which is busy 89% of the
// time.
template <class T, int TH, int C, bool ENT, bool TOP>
__global__ __launch_bounds__(TH, (kWavesFor<TH>)) void k_logprobs(const T *__restrict__ logits, Logits in,
                                                 const void *__restrict__ ids, int ids_bytes,
                                                 Values out)
{
    __shared__ Shared<TH> s;
    const int64_t r = in.first + blockIdx.x;
    const T *at = logits + r * in.ld;
    Held<T, TH, C> row(at, in.vocab);
    float taken = 0.f;
    bool on = false;
    if (threadIdx.x == 0 && ids) {
        const int64_t id = load_id(ids, ids_bytes, r);
        on = id >= 0 && id < in.vocab;
        if (on) taken = (float)at[id];
    }
    float most, mine, sum, moment;
    bool mine_nan;
    __shared__ SharedTop<TOP ? TH : 64> top;
    statistics<TH, ENT>(row, in.scale * kLog2e, s, most, mine, mine_nan, sum, moment, [&] {
        if constexpr (TOP) prepare_top(mine, top);
    });
    if constexpr (TOP && TH == 64) __syncthreads();
    const float ln = logf(sum);  // -infinity without a distribution
    const auto logprob = [&](float x) {
        return sum == 0.f ? -INFINITY : (x - most) * in.scale - ln;
    };
    if (threadIdx.x == 0) {
        if (out.logprob) out.logprob[r] = on ? logprob(taken) : 0.f;
        if (ENT) out.entropy[r] = sum == 0.f ? 0.f : ln - in.scale * (moment / sum);
    }
    if constexpr (TOP) {
        top_of<TH>(row, at, in.vocab, out.top, mine, mine_nan, top,
                   [&](int rank, int column, float x) {
            const int64_t to = r * out.top + rank;
            if (out.top_ids) {
                if (out.top_bytes == 8) ((int64_t *)out.top_ids)[to] = column;
                else ((int32_t *)out.top_ids)[to] = column;
            }
            if (out.top_logprob) out.top_logprob[to] = column < 0 ? -INFINITY : logprob(x);
        });
    }
}

// dx_v = scale (g ([v = t] - p_v) - h p_v (log p_v + entropy)); a row without a token
// or without a distribution gets zeros.  8,192 rows of 30,522 bf16 logits (1 GB) take 175
// us (5.7 TB/s), with the entropy's gradient 208.
template <class T, int TH, int C, bool ENT>
__global__ __launch_bounds__(TH, (kWavesFor<TH>)) void k_logprobs_grad(const T *logits, Logits in,
                                                      const void *__restrict__ ids, int ids_bytes,
                                                      const float *__restrict__ grad_logprob,
                                                      const float *__restrict__ grad_entropy,
                                                      T *dlogits, int64_t d_ld, Values out)
{
    __shared__ Shared<TH> s;
    const int64_t r = in.first + blockIdx.x;
    const T *at = logits + r * in.ld;
    T *to = dlogits + r * d_ld;
    const int64_t id = load_id(ids, ids_bytes, r);
    const bool on = id >= 0 && id < in.vocab;
    if (!on && !(ENT && out.entropy)) {
        for (int v = (int)threadIdx.x * kCols; v < in.vocab; v += TH * kCols) {
            const float zero[kCols] = {};
            store_some(to + v, zero, in.vocab - v);
        }
        if (threadIdx.x == 0 && out.logprob) out.logprob[r] = 0.f;
        return;
    }
    Held<T, TH, C> row(at, in.vocab);
    // (its value is waited for before the barriers behind which the row may be
    // written in place)
    if (threadIdx.x == 0) s.taken[0] = on ? (float)at[id] : 0.f;
    const float g = grad_logprob ? grad_logprob[r] : 0.f;
    float most, mine, sum, moment;
    bool mine_nan;
    const float c = in.scale * kLog2e;
    statistics<TH, ENT>(row, c, s, most, mine, mine_nan, sum, moment, [] {});
    const float ln = logf(sum);
    const float entropy = ENT ? ln - in.scale * (moment / sum) : 0.f;
    if (threadIdx.x == 0) {
        if (out.logprob)
            out.logprob[r] = !on ? 0.f : sum == 0.f ? -INFINITY
                                       : (s.taken[0] - most) * in.scale - ln;
        if (ENT && out.entropy) out.entropy[r] = sum == 0.f ? 0.f : entropy;
    }
    const bool zero = !on || sum == 0.f;
    const float a = zero ? 0.f : -g * in.scale / sum, one = zero ? 0.f : g * in.scale;
    const float b = ENT && grad_entropy && !zero ? -grad_entropy[r] * in.scale / sum : 0.f;
    const float nothing = (a - a) + (b - b);  // where p is 0: NaN in a row that is NaN
    row.each([&](float(&x)[kCols], int v) {
        if (v >= in.vocab) return;
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
            const float d = x[k] - most;
            const float e = __builtin_amdgcn_exp2f(d * c);
            if constexpr (ENT) {
                const float more = __builtin_fmaf(b, d * in.scale - ln + entropy, a);
                x[k] = zero || e == 0.f ? nothing : e * more;
            } else {
                x[k] = zero ? 0.f : a * e;
            }
        }
        if ((uint64_t)(id - v) < kCols) {
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                if (v + k == id) x[k] += one;
        }
        store_some(to + v, x, in.vocab - v);
    });
}

// ---------------------------------------------------------------------------
// Distillation
// ---------------------------------------------------------------------------

struct Teacher {
    const void *ids, *logits;
    int64_t ld;
    int top, ids_bytes, dtype;
};

__device__ __forceinline__ float load_teacher(const Teacher &t, int64_t at)
{
    return t.dtype == ONEBIT_GRAD_F32 ? ((const float *)t.logits)[at]
         : t.dtype == ONEBIT_GRAD_BF16 ? (float)((const __bf16 *)t.logits)[at]
                                       : (float)((const _Float16 *)t.logits)[at];
}

// loss = sum of q_k (log q_k - log p of its token), q = softmax(scale teacher's logits)
// over the alternatives whose token is one of the vocabulary;
// dx_v = g scale ((sum of q) p_v - sum of q_k over id_k = v).  A thread brings an
// alternative to LDS and, once the row is written, sets the column that it names; the
// first wave makes the teacher's softmax and the loss of them.  8,192 rows of 30,522 bf16
// logits with 64 alternatives and the gradient take 215 us, 39 more than without a teacher;
// the loss alone 113.
template <class T, int TH, int C, bool GRAD>
__global__ __launch_bounds__(TH, (kWavesFor<TH>)) void k_distill(const T *logits, Logits in, Teacher t,
                                                const float *__restrict__ grad_loss, T *dlogits,
                                                int64_t d_ld, float *__restrict__ loss)
{
    __shared__ Shared<TH> s;
    // an alternative's token (-1: none), teacher's and student's logit, and q
    __shared__ __attribute__((aligned(16))) int32_t s_id[kMostTeacher];
    __shared__ float s_z[kMostTeacher], s_x[kMostTeacher];
    __shared__ __attribute__((aligned(16))) float s_q[kMostTeacher];
    const int tid = threadIdx.x, top = (t.top + 3) & ~3;
    const int64_t r = in.first + blockIdx.x;
    const T *at = logits + r * in.ld;
#pragma unroll 1
    for (int j = tid; j < top; j += TH) {
        int id = -1;
        float z = -INFINITY;
        if (j < t.top) {
            const int64_t v = load_id(t.ids, t.ids_bytes, r * t.top + j);
            if (v >= 0 && v < in.vocab) id = (int)v, z = load_teacher(t, r * t.ld + j);
        }
        s_id[j] = id, s_z[j] = z, s_q[j] = 0.f;
    }
    Held<T, TH, C> row(at, in.vocab);
    float most, mine, sum, moment;
    bool mine_nan;
    const float c = in.scale * kLog2e;
    statistics<TH, false>(row, c, s, most, mine, mine_nan, sum, moment, [&] {
        // (the logits that are looked up are waited for here, before the barrier behind
        // which the row may be written in place)
#pragma unroll 1
        for (int j = tid; j < t.top; j += TH) s_x[j] = s_id[j] >= 0 ? (float)at[s_id[j]] : 0.f;
        if (tid >= 64) return;
        float m = kLowest, all[1] = {0.f};
#pragma unroll 1
        for (int j = tid; j < t.top; j += 64) m = fmaxf(m, s_z[j]);
        m = over_lanes<64>(m, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll 1
        for (int j = tid; j < t.top; j += 64) all[0] += __builtin_amdgcn_exp2f((s_z[j] - m) * c);
        add_lanes<64>(all, nullptr);
        if (tid == 0) s.taken[0] = m, s.taken[1] = all[0];
    });
    if constexpr (TH == 64) __syncthreads();
    const float teacher_most = s.taken[0], teacher_sum = s.taken[1];
    if (tid < 64) {
        const float ln = logf(sum), teacher_ln = logf(teacher_sum);
        const float inverse = teacher_sum == 0.f ? 0.f : 1.f / teacher_sum;
        float part[1] = {0.f};
#pragma unroll 1
        for (int j = tid; j < t.top; j += 64) {
            const float q = __builtin_amdgcn_exp2f((s_z[j] - teacher_most) * c) * inverse;
            const float logq = (s_z[j] - teacher_most) * in.scale - teacher_ln;
            const float logp = sum == 0.f ? -INFINITY : (s_x[j] - most) * in.scale - ln;
            if (s_id[j] >= 0 && q != 0.f) part[0] += q * (logq - logp);
            s_q[j] = q;
        }
        add_lanes<64>(part, nullptr);
        if (tid == 0 && loss) loss[r] = part[0];
    }
    if constexpr (GRAD) {
        T *to = dlogits + r * d_ld;
        const float g = grad_loss[r] * in.scale;
        const bool zero = sum == 0.f || teacher_sum == 0.f;
        const float a = zero ? 0.f : g * (teacher_sum / teacher_sum) / sum;  // (NaN stays)
        row.each([&](float(&v)[kCols], int col) {
            if (col >= in.vocab) return;
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                v[k] = zero ? 0.f : a * __builtin_amdgcn_exp2f((v[k] - most) * c);
            store_some(to + col, v, in.vocab - col);
        });
        // Two stores to one place: the first has arrived before the second is sent.
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (!zero)
#pragma unroll 1
            for (int j = tid; j < t.top; j += TH) {
                const int id = s_id[j];
                if (id < 0) continue;
                float all = 0.f;  // a token that is named twice: each thread writes the same
                for (int k = 0; k < top; k += 4) {
                    const int4 others = *(const int4 *)(s_id + k);
                    const float4 theirs = *(const float4 *)(s_q + k);
                    all += others.x == id ? theirs.x : 0.f;
                    all += others.y == id ? theirs.y : 0.f;
                    all += others.z == id ? theirs.z : 0.f;
                    all += others.w == id ? theirs.w : 0.f;
                }
                to[id] = (T)(a * __builtin_amdgcn_exp2f((s_x[j] - most) * c) - g * all);
            }
    }
}

// Calls f(threads, pieces) for rows of this many logits.  A row in registers is read
// once; a longer one twice, the second time from the caches for the most part.  us with
// 1,024 threads, from registers and from memory (a floor of 74 for reading, 147 with the
// gradient): 8,192 rows of 30,522 bf16 logits 109 and 128, gradient 186 and 295,
// distillation 215 and 319; 4,096 rows of 30,522 fp32 ones 80 and 80, 236 and 233, 341
// and 247 (half the row's registers are left, and two workgroups no longer fit a CU; LDS,
// of which 5 of 160 KB are used, could hold part of such a row, and does not).
// 8,192 rows of 9,000 bf16 ones 76 with 1,024 threads.
template <class T, class F>
void with_shape(int64_t vocab, F &&f)
{
    using std::integral_constant;
    if (vocab <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (vocab <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (vocab <= 8192) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (vocab <= 16384) f(integral_constant<int, 512>{}, integral_constant<int, 4>{});
    else if constexpr (sizeof(T) == 4) f(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
    else if (vocab <= 32768) f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    else f(integral_constant<int, 1024>{}, integral_constant<int, 0>{});
}

template <class F>
void with_flag(bool flag, F &&f)
{
    if (flag) f(std::true_type{});
    else f(std::false_type{});
}

// Launches of a workgroup for every row stay below 2^32 threads.
template <class F>
void with_rows(int64_t rows, F &&f)
{
    constexpr int64_t kMost = 1 << 21;
    for (int64_t first = 0; first < rows; first += kMost)
        f(first, (int)std::min(rows - first, kMost));
}

int check_logits(const void *logits, int32_t dtype, int64_t ld, int64_t rows, int64_t vocab,
                 float scale)
{
    TRY(check_size(rows, "rows"));
    if (vocab < 0 || vocab > kMostVocab)
        return fail(ONEBIT_EINVAL, "vocab = %lld is not in [0, 2^30]", (long long)vocab);
    TRY(check_rows(logits, dtype, ld, rows, vocab, "logits"));
    if (!(scale > 0.f) || scale > 1e30f)
        return fail(ONEBIT_EINVAL, "scale = %g is not in (0, 1e30]", (double)scale);
    return ONEBIT_OK;
}

int check_floats(const void *p, const char *name)
{
    if ((uintptr_t)p % 4) return fail(ONEBIT_EALIGN, "%s is not 4-byte aligned", name);
    return ONEBIT_OK;
}

int check_teacher(const Teacher &t, int64_t rows)
{
    if (t.top < 1 || t.top > kMostTeacher)
        return fail(ONEBIT_EINVAL, "top = %d is not in [1, %d]", t.top, kMostTeacher);
    TRY(check_rows(t.logits, t.dtype, t.ld, rows, t.top, "teacher's logits"));
    return check_ids(t.ids, t.ids_bytes, rows);
}

}  // namespace
}  // namespace onebit

using namespace onebit;

extern "C" {

int onebit_logprobs_forward(const void *logits, int32_t dtype, int64_t ld, int64_t rows,
                            int64_t vocab, const void *ids, int32_t ids_bytes, float scale,
                            float *logprobs, float *entropy, int32_t top, void *top_ids,
                            float *top_logprobs, onebit_stream stream)
{
    TRY(check_logits(logits, dtype, ld, rows, vocab, scale));
    TRY(check_floats(logprobs, "logprobs"));
    TRY(check_floats(entropy, "entropy"));
    TRY(check_floats(top_logprobs, "top_logprobs"));
    if (top < 0 || top > kMostTop)
        return fail(ONEBIT_EINVAL, "top = %d is not in [0, %d]", top, kMostTop);
    if (ids_bytes != 4 && ids_bytes != 8)
        return fail(ONEBIT_EINVAL, "ids_bytes = %d is neither 4 nor 8", ids_bytes);
    if (logprobs) TRY(check_ids(ids, ids_bytes, rows));
    if ((uintptr_t)top_ids % ids_bytes)
        return fail(ONEBIT_EALIGN, "top_ids is not %d-byte aligned", ids_bytes);
    if (rows == 0 || !(logprobs || entropy || top)) return ONEBIT_OK;
    const Values out{logprobs, entropy, top_ids, top_logprobs, top, ids_bytes};
    with_type(dtype, [&](auto *t) {
        with_shape<std::remove_pointer_t<decltype(t)>>(vocab, [&](auto threads, auto pieces) {
            with_flag(entropy, [&](auto ent) {
                with_flag(top > 0, [&](auto tops) {
                    using T = std::remove_pointer_t<decltype(t)>;
                    constexpr int TH = decltype(threads)::value, C = decltype(pieces)::value;
                    with_rows(rows, [&](int64_t first, int blocks) {
                        k_logprobs<T, TH, C, decltype(ent)::value, decltype(tops)::value>
                            <<<blocks, TH, 0, (hipStream_t)stream>>>(
                                (const T *)logits, Logits{ld, first, (int)vocab, scale},
                                logprobs ? ids : nullptr, ids_bytes, out);
                    });
                });
            });
        });
    });
    return launched("log-probabilities launch");
}

int onebit_logprobs_grad(const void *logits, int32_t dtype, int64_t ld, int64_t rows,
                         int64_t vocab, const void *ids, int32_t ids_bytes, float scale,
                         const float *grad_logprobs, const float *grad_entropy, void *dlogits,
                         int64_t d_ld, float *logprobs, float *entropy, onebit_stream stream)
{
    TRY(check_logits(logits, dtype, ld, rows, vocab, scale));
    TRY(check_rows(dlogits, dtype, d_ld, rows, vocab, "dlogits"));
    TRY(check_ids(ids, ids_bytes, rows));
    TRY(check_floats(grad_logprobs, "grad_logprobs"));
    TRY(check_floats(grad_entropy, "grad_entropy"));
    TRY(check_floats(logprobs, "logprobs"));
    TRY(check_floats(entropy, "entropy"));
    if (rows == 0) return ONEBIT_OK;
    const Values out{logprobs, entropy, nullptr, nullptr, 0, 4};
    with_type(dtype, [&](auto *t) {
        with_shape<std::remove_pointer_t<decltype(t)>>(vocab, [&](auto threads, auto pieces) {
            with_flag(grad_entropy || entropy, [&](auto ent) {
                using T = std::remove_pointer_t<decltype(t)>;
                constexpr int TH = decltype(threads)::value, C = decltype(pieces)::value;
                with_rows(rows, [&](int64_t first, int blocks) {
                    k_logprobs_grad<T, TH, C, decltype(ent)::value>
                        <<<blocks, TH, 0, (hipStream_t)stream>>>(
                            (const T *)logits, Logits{ld, first, (int)vocab, scale}, ids,
                            ids_bytes, grad_logprobs, grad_entropy, (T *)dlogits, d_ld, out);
                });
            });
        });
    });
    return launched("log-probabilities gradient launch");
}

int onebit_distill_forward(const void *logits, int32_t dtype, int64_t ld, int64_t rows,
                           int64_t vocab, const void *teacher_ids, int32_t ids_bytes,
                           const void *teacher_logits, int32_t teacher_dtype, int64_t teacher_ld,
                           int32_t top, float scale, float *loss, onebit_stream stream)
{
    TRY(check_logits(logits, dtype, ld, rows, vocab, scale));
    const Teacher teacher{teacher_ids, teacher_logits, teacher_ld, top,
                          ids_bytes, teacher_dtype};
    TRY(check_teacher(teacher, rows));
    TRY(check_floats(loss, "loss"));
    if (!loss && rows > 0) return fail(ONEBIT_EINVAL, "loss is NULL");
    if (rows == 0) return ONEBIT_OK;
    with_type(dtype, [&](auto *t) {
        with_shape<std::remove_pointer_t<decltype(t)>>(vocab, [&](auto threads, auto pieces) {
            using T = std::remove_pointer_t<decltype(t)>;
            constexpr int TH = decltype(threads)::value, C = decltype(pieces)::value;
            with_rows(rows, [&](int64_t first, int blocks) {
                k_distill<T, TH, C, false><<<blocks, TH, 0, (hipStream_t)stream>>>(
                    (const T *)logits, Logits{ld, first, (int)vocab, scale}, teacher, nullptr,
                    (T *)nullptr, 0, loss);
            });
        });
    });
    return launched("distillation launch");
}

int onebit_distill_grad(const void *logits, int32_t dtype, int64_t ld, int64_t rows,
                        int64_t vocab, const void *teacher_ids, int32_t ids_bytes,
                        const void *teacher_logits, int32_t teacher_dtype, int64_t teacher_ld,
                        int32_t top, float scale, const float *grad_loss, void *dlogits,
                        int64_t d_ld, float *loss, onebit_stream stream)
{
    TRY(check_logits(logits, dtype, ld, rows, vocab, scale));
    const Teacher teacher{teacher_ids, teacher_logits, teacher_ld, top,
                          ids_bytes, teacher_dtype};
    TRY(check_teacher(teacher, rows));
    TRY(check_rows(dlogits, dtype, d_ld, rows, vocab, "dlogits"));
    TRY(check_floats(grad_loss, "grad_loss"));
    TRY(check_floats(loss, "loss"));
    if (!grad_loss && rows > 0) return fail(ONEBIT_EINVAL, "grad_loss is NULL");
    if (rows == 0) return ONEBIT_OK;
    with_type(dtype, [&](auto *t) {
        with_shape<std::remove_pointer_t<decltype(t)>>(vocab, [&](auto threads, auto pieces) {
            using T = std::remove_pointer_t<decltype(t)>;
            constexpr int TH = decltype(threads)::value, C = decltype(pieces)::value;
            with_rows(rows, [&](int64_t first, int blocks) {
                k_distill<T, TH, C, true><<<blocks, TH, 0, (hipStream_t)stream>>>(
                    (const T *)logits, Logits{ld, first, (int)vocab, scale}, teacher, grad_loss,
                    (T *)dlogits, d_ld, loss);
            });
        });
    });
    return launched("distillation gradient launch");
}

}  // extern "C"
