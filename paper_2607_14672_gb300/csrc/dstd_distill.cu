// Learning from a teacher: the largest logits of each row (the teacher's record) and
// the distillation loss from such a record, with its gradient.
//
// The logit of an output y is factor y; where that is -infinity (a silent output,
// whose spike time is +infinity, or a masked class) it is factor silent, a constant.
#include "dstd_rows.cuh"
#include "dstd_tc_ptx.cuh"

#include <algorithm>
#include <cfloat>

namespace dstd {
namespace {

using tc::cluster_arrive;
using tc::cluster_ctarank;
using tc::cluster_sync;
using tc::cluster_wait;
using tc::mapa_rank;
using tc::smem_u32;

// exp2 as the special-function unit gives it (off by 2^-22 or so)
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.44269504f;

// two fp32 at a time
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ float2 of_pair(uint64_t p) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// both 16-bit values of a word as fp32, and two fp32 rounded to a word
template <class T>
__device__ __forceinline__ uint64_t word_pair(uint32_t w);
template <>
__device__ __forceinline__ uint64_t word_pair<__nv_bfloat16>(uint32_t w) {
    return pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ uint64_t word_pair<__half>(uint32_t w) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    return pair_of(f.x, f.y);
}
template <class T>
__device__ __forceinline__ uint32_t pair_word(uint64_t p);
template <>
__device__ __forceinline__ uint32_t pair_word<__nv_bfloat16>(uint64_t p) {
    const float2 f = of_pair(p);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <>
__device__ __forceinline__ uint32_t pair_word<__half>(uint64_t p) {
    const float2 f = of_pair(p);
    const __half2 h = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&h);
}

struct Logit {
    float factor, none;
    __device__ __forceinline__ explicit Logit(const LogitArgs &a) : factor(a.factor), none(a.factor * a.silent) {}
    __device__ __forceinline__ float of(float y, bool &silent) const {
        const float z = factor * y;
        silent = z == -INFINITY;
        return silent ? none : z;
    }
    __device__ __forceinline__ float of(float y) const {
        bool silent;
        return of(y, silent);
    }
};

// A block's share of a row, in 16-byte pieces from the row's first aligned address: packs
// [first, last) at column head + k P. Up to P - 1 columns before and after all packs are
// taken singly, by the first and the last share; columns [low, high) are the share's.
template <class T>
struct RowView {
    static constexpr int P = Pack<T>::P;
    const T *row;
    int cols, head, packs, first, last, low, high;
    __device__ __forceinline__ RowView(const LogitArgs &a, long long r, int part = 0, int parts = 1) {
        row = static_cast<const T *>(a.y) + r * a.ld;
        cols = a.cols;
        head = min(cols, (int)((0 - reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (P - 1)));
        packs = (cols - head) / P;
        first = (int)((long long)packs * part / parts);
        last = (int)((long long)packs * (part + 1) / parts);
        low = part == 0 ? 0 : head + first * P;
        high = part == parts - 1 ? cols : head + last * P;
    }
    // column of a thread's single element (t below 2 P), -1: none
    __device__ __forceinline__ int single(int t) const {
        const int c = t < P ? t : head + packs * P + t - P;
        return (t < P ? t < head : t < 2 * P) && c >= low && c < high ? c : -1;
    }
    __device__ __forceinline__ uint4 pack(int k) const {
        return __ldg(reinterpret_cast<const uint4 *>(row + head + (long long)k * P));
    }
};

// A thread's packs of a block's share, read in every pass (from L2 after the first), BATCH at a time.
template <class T, int THREADS, int BATCH>
struct OwnPacks {
    float one;
    int at;  // column of `one`, or -1
    __device__ __forceinline__ OwnPacks(const RowView<T> &v, bool mine) {
        at = mine ? v.single(threadIdx.x) : -1;
        one = at >= 0 ? to_f32<T>(v.row[at]) : 0.f;
    }
    // f(packs, the first one's number); those from v.last on are not set
    template <class F>
    __device__ __forceinline__ void batches(const RowView<T> &v, F f) const {
        for (int k = v.first + (int)threadIdx.x; k < v.last; k += BATCH * THREADS) {
            uint4 w[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i == 0 || k + i * THREADS < v.last) w[i] = v.pack(k + i * THREADS);
            f(w, k);
        }
    }
    // f(pack, its number) for every pack of this thread
    template <class F>
    __device__ __forceinline__ void each(const RowView<T> &v, F f) const {
        batches(v, [&](const uint4 (&w)[BATCH], int k) {
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i == 0 || k + i * THREADS < v.last) f(w[i], k + i * THREADS);
        });
    }
};

// ---------------------------------------------------------------------------
// The K largest logits of a row, descending, equal ones by ascending column. The
// logits are ordered as 32-bit keys (-0 as 0, NaN above all). Each thread takes
// the largest of its columns; the K-th largest of those is a bound that none of
// the row's K largest is below, and few are above it: with 512 threads and K = 64
// about 68. Those are gathered and put in order by counting, for each, the larger ones. Of rows
// with many more logits at the bound (equal ones) those above it are gathered, and the first
// columns of the equal ones. Few long rows
// are shared by the blocks of a cluster, which then count each other's. A row is not held: the few packs with logits at the
// bound come from L2 once more (held in shared memory, three rows to an SM: 71 us). What bounds it is the latency of
// those steps, with six rows to an SM: 4096 rows of 32768 bf16, K = 64, in 58 us, 4.7 TB/s (62 when the threads at the
// bound read their own packs again).
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(float z) {
    if (z != z) return 0xfffffffeu;
    const uint32_t u = __float_as_uint(z + 0.f);  // -0 + 0 = 0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of_key(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// the larger of two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
template <class T>
struct Two;  // two 16-bit values in a word
template <>
struct Two<__half> { using type = __half2; };
template <>
struct Two<__nv_bfloat16> { using type = __nv_bfloat162; };

constexpr int kTopGroups = 4;  // of a thread's packs; those of one with a logit at the bound are read again
template <int BATCH>
constexpr int kTopThreads = BATCH == 2 ? 2048 : 1536;  // threads on an SM
constexpr int kFew = 512;  // as many at most are put in order by counting, the square of them; kTopMax * 3 / 2 + 64 fit

__device__ __forceinline__ uint64_t ld_cluster64(uint32_t addr) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}

// Largest logits of packs. PAIRS (16-bit outputs, none of whose logits is a stand-in): the order of the logits is that
// of the outputs, or of the negated ones (flip), and two are compared at once. Without WITH_NAN a NaN is passed
// over, unless there is nothing else.
template <class T, bool PAIRS, bool WITH_NAN>
struct PackMax {
    Logit logit;
    uint32_t flip;
    __device__ __forceinline__ explicit PackMax(const Logit &l) : logit(l), flip(l.factor < 0.f ? 0x80008000u : 0u) {}
    static __device__ __forceinline__ uint32_t two(uint32_t a, uint32_t b) {
        using V = typename Two<T>::type;
        const V x = *reinterpret_cast<const V *>(&a), y = *reinterpret_cast<const V *>(&b);
        const V m = WITH_NAN ? __hmax2_nan(x, y) : __hmax2(x, y);
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    __device__ __forceinline__ uint32_t words(const uint4 &w) const {
        if (flip) return two(two(w.x ^ flip, w.y ^ flip), two(w.z ^ flip, w.w ^ flip));
        return two(two(w.x, w.y), two(w.z, w.w));
    }
    // of both halves of a word from words()
    __device__ __forceinline__ float of_words(uint32_t u) const { return unit() * output(u); }
    static __device__ __forceinline__ float output(uint32_t u) {
        using V = typename Two<T>::type;
        const V m = *reinterpret_cast<const V *>(&u);
        return to_f32<T>(WITH_NAN ? __hmax_nan(m.x, m.y) : __hmax(m.x, m.y));
    }
    // The largest as it is before the factor (PAIRS: outputs, negated for a negative factor; else logits), of a pack and
    // of one output; unit() times that is the logit.
    __device__ __forceinline__ float unit() const { return PAIRS ? fabsf(logit.factor) : 1.f; }
    __device__ __forceinline__ float level(const uint4 &w) const {
        if constexpr (PAIRS) return output(words(w));
        else return (*this)(w);
    }
    __device__ __forceinline__ float level(float y) const {
        if constexpr (PAIRS) return flip ? -y : y;
        else return logit.of(y);
    }
    __device__ __forceinline__ float operator()(const uint4 &w) const {
        if constexpr (PAIRS) {
            return of_words(words(w));
        } else {
            float m = logit.of(Pack<T>::one(w, 0));
#pragma unroll
            for (int i = 1; i < Pack<T>::P; ++i) {
                const float z = logit.of(Pack<T>::one(w, i));
                m = WITH_NAN ? max_nan(m, z) : fmaxf(m, z);
            }
            return m;
        }
    }
    // the largest of packs k0, k0 + STEP and so on, COUNT of them or fewer, all loads first; there is one at least
    template <int COUNT, int STEP, class View>
    __device__ __forceinline__ float of_packs(const View &v, int k0) const {
        uint4 w[COUNT];
#pragma unroll
        for (int i = 0; i < COUNT; ++i) w[i] = v.pack(k0 + i * STEP < v.last ? k0 + i * STEP : k0);
        if constexpr (PAIRS) {
            uint32_t m = words(w[0]);
#pragma unroll
            for (int i = 1; i < COUNT; ++i) m = two(m, words(w[i]));
            return of_words(m);
        } else {
            float m = (*this)(w[0]);
#pragma unroll
            for (int i = 1; i < COUNT; ++i) m = WITH_NAN ? max_nan(m, (*this)(w[i])) : fmaxf(m, (*this)(w[i]));
            return m;
        }
    }
};

template <class T, int THREADS, int BATCH, bool PAIRS>  // BATCH: packs that a thread loads at once
__global__ void __launch_bounds__(THREADS, kTopThreads<BATCH> / THREADS)
    k_top_logits(const LogitArgs a, const int parts, const int K, float *top, int32_t *index) {
    constexpr int P = Pack<T>::P;
    __shared__ uint64_t s_cand[kFew], s_best[kTopMax];
    __shared__ unsigned s_n, s_groups, s_hits, s_hist[256], s_digit[2], s_warp[THREADS / 32];
    __shared__ int s_group[kFew], s_hit[kFew];
    __shared__ uint4 s_pack[kFew];
    extern __shared__ uint64_t s_all[];
    const int t = threadIdx.x, part = parts > 1 ? (int)cluster_ctarank() : 0;
    const long long r = blockIdx.x / parts;
    const RowView<T> v(a, r, part, parts);
    const Logit logit(a);
    const PackMax<T, PAIRS, true> pack_max(logit);
    if (t == 0) s_n = s_groups = s_hits = 0;
    const int single = v.single(t);
    const float one = single >= 0 ? logit.of(to_f32<T>(v.row[single])) : 0.f;
    // every column of the share once, in any order
    const auto each = [&](auto f) {
        if (single >= 0) f(single, key_of(one));
        for (int k = v.first + t; k < v.last; k += THREADS) {
            const uint4 w = v.pack(k);
#pragma unroll
            for (int i = 0; i < P; ++i) f(v.head + k * P + i, key_of(logit.of(Pack<T>::one(w, i))));
        }
    };
    const int want = min(K, v.high - v.low);
    // the largest of each group of this thread's packs
    float largest[kTopGroups];
    uint32_t mine = 0, bound = 0;  // 0: below every logit's key
    constexpr int step = BATCH * THREADS;
    const int group = step * max(1, (v.last - v.first + kTopGroups * step - 1) / (kTopGroups * step));
#pragma unroll
    for (int q = 0; q < kTopGroups; ++q) {
        const int from = v.first + t + q * group, to = min(v.last, from - t + group);
        largest[q] = -INFINITY;
        for (int k0 = from; k0 < to; k0 += step)
            largest[q] = max_nan(largest[q], pack_max.template of_packs<BATCH, THREADS>(v, k0));
    }
    if (single >= 0 || v.first + t < v.last) {
        float m = single >= 0 ? one : -INFINITY;
#pragma unroll
        for (int q = 0; q < kTopGroups; ++q) m = max_nan(m, largest[q]);
        mine = key_of(m);
    }
    // the upper half of the key will do: a bound lower by 2^-7 at most lets few more pass
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t trial = bound | (1u << bit);
        if (__syncthreads_count(mine >= trial) >= want) bound = trial;
    }
    // groups with a logit at the bound; then their packs once more, from L2, a thread to each; then the columns of those
    // with such a logit, a thread to each
    const auto gather = [&](int c, float z) {
        const uint32_t k = key_of(z);
        if (k < bound) return;
        const unsigned at = atomicAdd(&s_n, 1u);
        if (at < kFew) s_cand[at] = (uint64_t)k << 32 | (uint32_t)~c;
    };
    if (single >= 0) gather(single, one);
    const float least = bound ? logit_of_key(bound) : -INFINITY;
    if (mine >= bound) {
#pragma unroll
        for (int q = 0; q < kTopGroups; ++q) {
            const int from = v.first + t + q * group;
            if (from >= v.last || largest[q] < least) continue;
            const unsigned at = atomicAdd(&s_groups, 1u);
            if (at < kFew) s_group[at] = from;
        }
    }
    __syncthreads();
    if (s_groups > kFew) {
        if (t == 0) s_hits = kFew + 1u;
    } else {
        const unsigned each_group = group / THREADS, all = s_groups * each_group;
        for (unsigned i = t; i < all; i += THREADS) {
            const unsigned q = i / each_group;
            const int k = s_group[q] + (int)(i - q * each_group) * THREADS;
            if (k >= v.last) continue;
            const uint4 w = v.pack(k);
            if (pack_max(w) < least) continue;
            const unsigned at = atomicAdd(&s_hits, 1u);
            if (at < kFew) {
                s_hit[at] = k;
                s_pack[at] = w;
            }
        }
    }
    __syncthreads();
    if (s_hits > kFew) {
        if (t == 0) s_n = kFew + 1u;
    } else {
        for (unsigned i = t; i < s_hits * P; i += THREADS)
            gather(v.head + s_hit[i / P] * P + (int)(i % P),
                   logit.of(to_f32<T>(reinterpret_cast<const T *>(s_pack + i / P)[i % P])));
    }
    __syncthreads();
    unsigned n = s_n;
    if (n > (unsigned)(K + K / 2 + 64)) {
        // many equal logits at the bound. Those above the exact K-th largest of the threads' largest are few, as a rule:
        uint32_t last = bound;
        for (int bit = 15; bit >= 0; --bit) {
            const uint32_t trial = last | (1u << bit);
            if (__syncthreads_count(mine >= trial) >= want) last = trial;
        }
        const auto above = [&](uint32_t least) {
            if (t == 0) s_n = 0;
            __syncthreads();
            if (mine > least)
                each([&](int c, uint32_t k) {
                    if (k <= least) return;
                    const unsigned at = atomicAdd(&s_n, 1u);
                    if (at < kFew) s_cand[at] = (uint64_t)k << 32 | (uint32_t)~c;
                });
            __syncthreads();
            return s_n;
        };
        n = above(last);
        if (n > kFew) {
            // the K-th largest digit by digit
            uint32_t mask = 0;
            unsigned need = want;
            last = 0;
            for (int shift = 24; shift >= 0; shift -= 8) {
                for (int i = t; i < 256; i += THREADS) s_hist[i] = 0;
                __syncthreads();
                each([&](int, uint32_t k) {
                    if ((k & mask) == last) atomicAdd(&s_hist[(k >> shift) & 255u], 1u);
                });
                __syncthreads();
                if (t == 0) {
                    unsigned over = 0;
                    int d = 255;
                    while (d > 0 && over + s_hist[d] < need) over += s_hist[d--];
                    s_digit[0] = (unsigned)d;
                    s_digit[1] = over;
                }
                __syncthreads();
                last |= s_digit[0] << shift;
                mask |= 255u << shift;
                need -= s_digit[1];
                __syncthreads();
            }
            n = above(last);
        }
        // then the first columns of those equal to it
        const unsigned need = n < (unsigned)want ? want - n : 0;
        unsigned found = 0;
        for (int c0 = v.low; c0 < v.high && found < need; c0 += THREADS) {
            const bool here = c0 + t < v.high && key_of(logit.of(to_f32<T>(v.row[c0 + t]))) == last;
            const unsigned ballot = __ballot_sync(0xffffffffu, here);
            if ((t & 31) == 0) s_warp[t >> 5] = __popc(ballot);
            __syncthreads();
            unsigned before = found, all = found;
            for (int w = 0; w < THREADS / 32; ++w) {
                if (w < (t >> 5)) before += s_warp[w];
                all += s_warp[w];
            }
            before += __popc(ballot & ((1u << (t & 31)) - 1u));
            if (here && before < need) s_cand[n + before] = (uint64_t)last << 32 | (uint32_t)~(uint32_t)(c0 + t);
            found = all;
            __syncthreads();
        }
        n += need;
        __syncthreads();
    }
    const auto put = [&](uint64_t e, int rank) {
        if (rank >= K) return;
        top[r * K + rank] = logit_of_key((uint32_t)(e >> 32));
        index[r * K + rank] = (int32_t)~(uint32_t)e;
    };
    for (unsigned i = t; i < n; i += THREADS) {
        const uint64_t me = s_cand[i];
        int rank = 0;
#pragma unroll 8
        for (unsigned j = 0; j < n; ++j) rank += s_cand[j] > me;
        if (parts == 1) put(me, rank);
        else if (rank < K) s_best[rank] = me;
    }
    if (parts > 1) {
        if (t >= want && t < K) s_best[t] = 0;  // below every entry
        __syncwarp();
        cluster_sync();
        // all shares' entries, in the blocks' order
        for (int i = t; i < parts * K; i += THREADS)
            s_all[i] = ld_cluster64(mapa_rank(smem_u32(s_best + i % K), (uint32_t)(i / K)));
        __syncwarp();
        cluster_sync();
        if (t < want) {
            const uint64_t me = s_best[t];
            int rank = t;
            for (int q = 0; q < parts && rank < K; ++q) {
                if (q == part) continue;
                int lo = 0, hi = K;  // entries above me
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (s_all[q * K + mid] > me) lo = mid + 1;
                    else hi = mid;
                }
                rank += lo;
            }
            put(me, rank);
        }
    }
}

// Rows of up to 32 E classes: a warp to a row; a logit's place is the number of logits before it (larger, or equal
// in an earlier column).
template <class T, int E>
__global__ void __launch_bounds__(256) k_top_small(const LogitArgs a, const int K, float *top, int32_t *index) {
    __shared__ uint32_t s_key[8][32 * E];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long r = (long long)blockIdx.x * 8 + warp;
    if (r >= a.rows) return;
    const Logit logit(a);
    const T *row = static_cast<const T *>(a.y) + r * a.ld;
    uint32_t key[E];
    int rank[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = lane + 32 * e;
        key[e] = c < a.cols ? key_of(logit.of(to_f32<T>(row[c]))) : 0u;
        s_key[warp][c] = key[e];
        rank[e] = 0;
    }
    __syncwarp();
#pragma unroll 4
    for (int j = 0; j < a.cols; ++j) {
        const uint32_t other = s_key[warp][j];
#pragma unroll
        for (int e = 0; e < E; ++e) rank[e] += other >= key[e] + (j < lane + 32 * e ? 0u : 1u);
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (lane + 32 * e < a.cols && rank[e] < K) {
            top[r * K + rank[e]] = logit_of_key(key[e]);
            index[r * K + rank[e]] = lane + 32 * e;
        }
}

// Rows of up to 32 E columns and K <= 128: a warp to a row, whose keys stay in registers. The least of the lanes' largest
// (in two groups of a lane's columns for K > 32, in four for K > 64) is a bound with K logits or more at or above it; halving the
// interval from there to the row's largest narrows them to a list that is put in order by counting. Where equal logits
// keep the list long, their first columns are taken. Instructions bound it: 10000 rows of 1000 fp32, K = 10, 18 us, 2.2
// TB/s (in blocks 46).
constexpr int kTopWarp = 128;
template <class T, int E>
__global__ void __launch_bounds__(256) k_top_packs(const LogitArgs a, const int K, float *top, int32_t *index) {
    constexpr int P = Pack<T>::P, N = E / P;
    constexpr uint32_t ALL = 0xffffffffu;
    __shared__ unsigned long long s_list[8][kTopWarp + 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long r = (long long)blockIdx.x * 8 + warp;
    if (r >= a.rows) return;
    const Logit logit(a);
    const RowView<T> v(a, r);
    uint32_t key[E + 1];  // 0: none
    uint4 raw[N];
#pragma unroll
    for (int j = 0; j < N; ++j) raw[j] = lane + 32 * j < v.packs ? v.pack(lane + 32 * j) : make_uint4(0, 0, 0, 0);
    const int at = v.single(lane);
    const float one = at >= 0 ? to_f32<T>(v.row[at]) : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
        key[e] = lane + 32 * (e / P) < v.packs ? key_of(logit.of(Pack<T>::one(raw[e / P], e % P))) : 0u;
    key[E] = at >= 0 ? key_of(logit.of(one)) : 0u;

    uint32_t most_of[4] = {key[E], 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < E; ++e) most_of[e % 4] = max(most_of[e % 4], key[e]);
    const uint32_t even = max(most_of[0], most_of[2]), odd = max(most_of[1], most_of[3]);
    const uint32_t least = K <= 32 ? max(even, odd)
                                   : K <= 64 ? min(even, odd) : min(min(most_of[0], most_of[1]), min(most_of[2], most_of[3]));
    const auto count = [&](uint32_t bound) {
        unsigned c = 0;
#pragma unroll
        for (int e = 0; e <= E; ++e) c += key[e] >= bound;
        return c;
    };
    const unsigned wanted = (unsigned)K, most = (wanted + 39) & ~31u;
    uint32_t low = max(1u, __reduce_min_sync(ALL, least));
    uint32_t high = __reduce_max_sync(ALL, max(even, odd)) + 1;  // fewer than K from here on
    unsigned n = __reduce_add_sync(ALL, count(low));
    while (n > most && high - low > 1) {
        const uint32_t middle = low + (high - low) / 2;
        const unsigned c = __reduce_add_sync(ALL, count(middle));
        if (c >= wanted) low = middle, n = c;
        else high = middle;
    }
    if (n > most) {
        // equal ones: as many as are wanted, by columns (single ones before the packs, packs, single ones behind)
        unsigned left = wanted - __reduce_add_sync(ALL, count(high));
        const auto keep = [&](unsigned equal) {  // how many of a lane's equal ones, and of all lanes'
            unsigned before = equal;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const unsigned other = __shfl_up_sync(ALL, before, d);
                if (lane >= d) before += other;
            }
            const unsigned all = __shfl_sync(ALL, before, 31);
            before -= equal;
            const unsigned kept = before < left ? left - before : 0u;
            left -= min(left, all);
            return kept;
        };
        if (keep(key[E] == low && at < v.head) == 0 && key[E] == low && at < v.head) key[E] = 0u;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            unsigned equal = 0;
#pragma unroll
            for (int i = 0; i < P; ++i) equal += key[j * P + i] == low;
            unsigned kept = keep(equal);
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (key[j * P + i] == low) {
                    if (kept) --kept;
                    else key[j * P + i] = 0u;
                }
        }
        if (keep(key[E] == low && at >= v.head) == 0 && key[E] == low && at >= v.head) key[E] = 0u;
        n = wanted;
    }
    const unsigned own = count(low);
    unsigned place = own;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const unsigned other = __shfl_up_sync(ALL, place, d);
        if (lane >= d) place += other;
    }
    place -= own;
    const auto list = [&](uint32_t k, int column) {
        if (k >= low) s_list[warp][place++] = (unsigned long long)k << 32 | (uint32_t)~column;
    };
#pragma unroll
    for (int e = 0; e < E; ++e) list(key[e], v.head + (lane + 32 * (e / P)) * P + e % P);
    list(key[E], at);
    __syncwarp();
    for (unsigned i = lane; i < n; i += 32) {
        const unsigned long long mine = s_list[warp][i];
        unsigned rank = 0;
#pragma unroll 8
        for (unsigned j = 0; j < n; ++j) rank += s_list[warp][j] > mine;
        if (rank < wanted) {
            top[r * K + rank] = logit_of_key((uint32_t)(mine >> 32));
            index[r * K + rank] = (int32_t)~(uint32_t)mine;
        }
    }
}

// blocks that share a row: where the rows alone do not fill the GPU, up to 8 of at least `least` packs
int shares(int rows, int packs, int least) {
    int parts = 1;
    while (parts < 8 && rows * 2ll * parts <= 304 && packs >= 2 * parts * least) parts *= 2;
    return parts;
}

template <auto KERNEL, int THREADS, int SHARED, class... A>  // SHARED: bytes of dynamic shared memory
cudaError_t launch_shared(int rows, int parts, cudaStream_t st, const A &...args) {
    if ((long long)rows * parts > 0x7fffffff) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)parts;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    cfg.gridDim = dim3((unsigned)(rows * parts));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SHARED;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, KERNEL, args...);
}

template <class T, bool PAIRS>
cudaError_t top_rows(const LogitArgs &a, int K, float *top, int32_t *index, cudaStream_t st) {
    const int packs = (int)(((long long)a.cols * sizeof(T) + 15) / 16), parts = shares(a.rows, packs, 512);
    constexpr int all = 8 * kTopMax * 8;
    // 256 threads have enough largest ones to bound 128 logits closely (32768 fp32: 95 us with 512 threads, 99 with them);
    // short rows want more blocks on an SM (16384 rows of 1500 bf16: 71 us, with the long ones' form 87)
    if (parts == 1 && K <= 128 && packs <= 1280)
        return launch_shared<k_top_logits<T, 256, 2, PAIRS>, 256, 0>(a.rows, parts, st, a, parts, K, top, index);
    if (parts == 1 && K <= 128 && packs <= 4096)
        return launch_shared<k_top_logits<T, 256, 4, PAIRS>, 256, 0>(a.rows, parts, st, a, parts, K, top, index);
    return launch_shared<k_top_logits<T, 512, 4, PAIRS>, 512, all>(a.rows, parts, st, a, parts, K, top, index);
}

template <class T>
cudaError_t top_logits(const LogitArgs &a, int K, float *top, int32_t *index, cudaStream_t st) {
    const unsigned blocks = ((unsigned)a.rows + 7) / 8;
    if (a.cols <= 32) {
        k_top_small<T, 1><<<blocks, 256, 0, st>>>(a, K, top, index);
        return cudaGetLastError();
    }
    const int packs = (int)(((long long)a.cols * sizeof(T) + 15) / 16);
    // few rows of more than 256 columns, or with more than 64 logits to find, are faster in blocks (300 fp32, K = 20: 608 rows 4.3 us both ways, 152 rows 4.2
    // and 3.3, 912 rows 4.7 and 6.8, 10000 rows 12 and 42; 200 bf16, K = 100: 152 rows 7.4 and 4.9, 1216 rows 7.5 and 14)
    const int warp_columns = a.rows > 5 * 152 ? 32 * 32 : K <= 64 ? 32 * 8 : 0;
    if (K <= kTopWarp && packs * Pack<T>::P <= warp_columns) {
        if (packs * Pack<T>::P <= 32 * 8) k_top_packs<T, 8><<<blocks, 256, 0, st>>>(a, K, top, index);
        else if (packs * Pack<T>::P <= 32 * 16) k_top_packs<T, 16><<<blocks, 256, 0, st>>>(a, K, top, index);
        else k_top_packs<T, 32><<<blocks, 256, 0, st>>>(a, K, top, index);
        return cudaGetLastError();
    }
    if (a.cols <= 128) {
        k_top_small<T, 4><<<blocks, 256, 0, st>>>(a, K, top, index);
        return cudaGetLastError();
    }
    if constexpr (sizeof(T) == 2)
        if (a.factor * a.silent == -INFINITY) return top_rows<T, true>(a, K, top, index, st);
    return top_rows<T, false>(a, K, top, index, st);
}

// ---------------------------------------------------------------------------
// Distillation. With p = softmax(teacher_factor top) over a row's used entries
// and q = softmax of its logits:
//     L_r = sum_k p_k (log p_k - log q_{i_k}),
//     dL_r / dy_c = factor (q_c - sum_{k: i_k = c} p_k)   (0 where silent).
// First the largest logit and the sum of exp(z - largest), by warps, then over
// the block (or the cluster that shares the row), then exp(z - m) times a
// constant. A row that a warp has stays in its registers in between; a block's is
// read a second time, from L2 while the rows under way fit there (4096 rows of
// 32768 bf16: 292 MB read from HBM for 268; 1000 rows of 100000 fp32: 752 for
// 400). The few columns that the teacher names are written once more, from
// fp32, so that every gradient is rounded once; entries of the same column are
// added up in their order.
// ---------------------------------------------------------------------------
struct Teacher {
    int at;       // column of this thread's entry, -1: none
    float log_p, p, z, old;
    bool silent;
};

// A row's entries, EACH to a lane of a warp: lane l has entries l, 32 + l, ...; at: the column, -1 where it is not used.
template <int EACH>
struct Record {
    int at[EACH];
    float z[EACH];
    __device__ __forceinline__ Record(const DistillArgs &a, long long r, int lane) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int k = e * 32 + lane;
            at[e] = k < a.K ? a.index[r * a.K + k] : -1;
            z[e] = k < a.K ? a.teacher_factor * a.top[r * a.K + k] : -INFINITY;
            if (at[e] >= a.y.cols || z[e] == -INFINITY) at[e] = -1;
        }
    }
    __device__ __forceinline__ bool any() const {
        bool some = false;
#pragma unroll
        for (int e = 0; e < EACH; ++e) some = some || at[e] >= 0;
        return __any_sync(0xffffffffu, some);
    }
    // the softmax's largest logit and the log of its sum
    __device__ __forceinline__ void softmax(float &m, float &log_sum) const {
        m = -INFINITY;
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (at[e] >= 0) m = fmaxf(m, z[e]);
#pragma unroll
        for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (at[e] >= 0) sum += expf(z[e] - m);
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        log_sum = logf(sum);
    }
    // entry e of this lane, given its output y and what its gradient holds
    __device__ __forceinline__ Teacher entry(int e, float m, float log_sum, const Logit &logit, float y,
                                             float old) const {
        Teacher t;
        t.at = at[e];
        t.z = logit.of(y, t.silent);
        t.old = old;
        t.log_p = z[e] - m - log_sum;
        t.p = t.at >= 0 ? expf(t.log_p) : 0.f;
        return t;
    }
};
// What entry k's column gets: its p and those of later entries of the same column; false where an
// earlier entry has it.
__device__ __forceinline__ bool column_mass(const int *at, const float *p, int k, int K, float &mass) {
    const int own = at[k];
    bool first = true;
    mass = 0.f;
#pragma unroll 8
    for (int j = 0; j < K; ++j) {
        const bool same = at[j] == own;
        first = first && !(same && j < k);
        mass += same && j >= k ? p[j] : 0.f;
    }
    return first;
}
// this entry's share of the row's loss, given the log of the softmax's denominator
__device__ __forceinline__ float teacher_loss(const Teacher &t, float m, float log_sum) {
    return t.at >= 0 && t.p != 0.f ? t.p * (t.log_p - (t.z - m - log_sum)) : 0.f;
}

// largest and sum of (m, s) pairs of all lanes; `unit` times m is a logit
__device__ __forceinline__ void join_lanes(float &m, float &s, float unit) {
    const float own = m;
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    // an infinite m has nothing to rescale: such a sum is 0 or already NaN
    s = own == m ? s : s * expf((own - m) * unit);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
}

// Counts a row (or a block's rows) whose losses this thread has written; true for the last one.
__device__ __forceinline__ bool last_counted(const DistillArgs &a, unsigned all) {
    __threadfence();
    return atomicAdd(reinterpret_cast<unsigned *>(a.loss + 1), 1u) == all - 1;
}

// the last block adds the rows' losses up, in a fixed order
__device__ __forceinline__ void add_losses(const DistillArgs &a) {
    __shared__ float s_total[32];
    __threadfence();
    // each thread's sum with what its additions lost (64-bit additions took most of a readout's time)
    float sum = 0.f, lost = 0.f;
    const float even = 1.f / (float)a.y.rows;
    for (long long i0 = threadIdx.x; i0 < a.y.rows; i0 += 8 * blockDim.x) {
        float w[8], loss[8];
        // the last row again behind it, with no weight: eight loads under way at once
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const long long i = i0 + e * blockDim.x, at = min(i, (long long)a.y.rows - 1);
            loss[e] = __ldcg(a.row_loss + at);
            w[e] = i < a.y.rows ? even : 0.f;
        }
        if (a.row_weight) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const long long i = i0 + e * blockDim.x;
                const float given = a.row_weight[min(i, (long long)a.y.rows - 1)];
                w[e] = i < a.y.rows ? given : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = w[e] != 0.f ? __fmul_rn(w[e], loss[e]) : 0.f, all = __fadd_rn(sum, x);
            const float part = __fsub_rn(all, sum);
            lost = __fadd_rn(lost, __fadd_rn(__fsub_rn(sum, __fsub_rn(all, part)), __fsub_rn(x, part)));
            sum = all;
        }
    }
    // an infinite sum has lost nothing that could be told
    if (isfinite(sum)) sum += lost;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) s_total[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x < 32) {
        sum = threadIdx.x < blockDim.x / 32 ? s_total[threadIdx.x] : 0.f;
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (threadIdx.x == 0) {
            a.loss[0] = a.weight * sum;
            *reinterpret_cast<unsigned *>(a.loss + 1) = 0u;
        }
    }
}

// Whether one of a warp's K columns (negative: none) is named twice. Entries of one place in the table meet in rounds;
// each leaves one of them there for the others to look at, so that every round ends some of them (single steps of
// compare-and-swap took 5 us of 13, as lanes went their own ways).
template <int EACH, int SLOTS>
__device__ __forceinline__ bool named_twice(const int *at, int *slot, int K, int lane) {
    int column[EACH];  // -1: none, or through
    bool open = false, again = false;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        column[e] = 32 * e + lane < K ? at[32 * e + lane] : -1;
        open = open || column[e] >= 0;
    }
    while (__any_sync(0xffffffffu, open)) {
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (32 * e < K && column[e] >= 0) slot[column[e] & (SLOTS - 1)] = 32 * e + lane;
        __syncwarp();
        open = false;
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (32 * e < K && column[e] >= 0) {
                const int there = slot[column[e] & (SLOTS - 1)];
                const bool own = there == 32 * e + lane, met = !own && at[there] == column[e];
                again = again || met;
                if (own || met) column[e] = -1;
                else open = true;
            }
        __syncwarp();
    }
    return __any_sync(0xffffffffu, again);
}

// exp(z - m) of outputs, m the largest logit, given as PackMax's level (nothing but -infinity: every exp is 0 with any
// finite m, and NaN stays NaN). FAST: 16-bit outputs without a stand-in for silent ones, whose exp is 0 by itself:
// with m = factor y*, exp(z - m) = 2^((y - y*) factor log2(e)), on the special-function unit, two at a time. The difference
// comes first, so that the roundings are of the size of z - m, not of z (y - y* is exact for near ones): the argument
// is off by 2^-22 |z - m|, and where the difference of finite outputs is infinite the exp is 0 anyway (least_factor).
constexpr float least_factor = 0x1p-120f, most_factor = 1e30f;
template <class T, bool FAST>
struct ExpOf {
    static constexpr int P = Pack<T>::P;
    Logit logit;
    float minus, scale;  // what is added to a logit (FAST: to an output) before the factor
    __device__ __forceinline__ ExpOf(const Logit &l, float level)
        : logit(l), minus(fmaxf(level, -FLT_MAX) * (FAST && l.factor < 0.f ? 1.f : -1.f)), scale(l.factor * kLog2e) {}
    __device__ __forceinline__ float one(float y) const {
        if constexpr (FAST) return exp2_fast((y + minus) * scale);
        else return expf(logit.of(y) + minus);
    }
    __device__ __forceinline__ uint64_t two(uint32_t w) const {
        const float2 x = of_pair(mul_pair(add_pair(word_pair<T>(w), pair_of(minus, minus)), pair_of(scale, scale)));
        return pair_of(exp2_fast(x.x), exp2_fast(x.y));
    }
    __device__ __forceinline__ float sum(const uint4 &w) const {
        if constexpr (FAST) {
            const float2 f = of_pair(add_pair(add_pair(two(w.x), two(w.y)), add_pair(two(w.z), two(w.w))));
            return f.x + f.y;
        } else {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < P; ++i) s += one(Pack<T>::one(w, i));
            return s;
        }
    }
    // over exp(z - m), 0 where silent
    __device__ __forceinline__ float grad(float y, float over) const {
        bool silent;
        const float z = logit.of(y, silent);
        return silent ? 0.f : (FAST ? one(y) : expf(z + minus)) * over;
    }
    __device__ __forceinline__ void grads(const uint4 &w, float over, T (&out)[P]) const {
        // a silent one's exp is 0, and so is its product, unless `over` is infinite or NaN
        if constexpr (FAST) {
            if (isfinite(over)) {
                const uint64_t c = pair_of(over, over);
                *reinterpret_cast<uint4 *>(out) =
                    make_uint4(pair_word<T>(mul_pair(two(w.x), c)), pair_word<T>(mul_pair(two(w.y), c)),
                               pair_word<T>(mul_pair(two(w.z), c)), pair_word<T>(mul_pair(two(w.w), c)));
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i) out[i] = round_out<T>(grad(Pack<T>::one(w, i), over));
    }
};

// What a warp that has a row to itself knows of the teacher: EACH entries a lane.
template <int EACH>
struct WarpShared {
    static constexpr int SLOTS = 128 * EACH;
    int at[32 * EACH], slot[SLOTS];
    float p[32 * EACH];
};
template <int EACH>
struct WarpTeacher {
    Teacher entry[EACH];
    bool any, twice;
    template <class T>
    __device__ __forceinline__ void read(const DistillArgs &a, const Logit &logit, const T *row, const T *g, long long r,
                                         int lane, WarpShared<EACH> &s) {
        const Record<EACH> record(a, r, lane);
        any = record.any();
        float y[EACH], old[EACH], m, log_sum;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            y[e] = record.at[e] >= 0 ? to_f32<T>(row[record.at[e]]) : 0.f;
            old[e] = record.at[e] >= 0 && a.accumulate && g ? to_f32<T>(g[record.at[e]]) : 0.f;
        }
        record.softmax(m, log_sum);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            entry[e] = record.entry(e, m, log_sum, logit, y[e], old[e]);
            s.at[32 * e + lane] = entry[e].at;
            s.p[32 * e + lane] = entry[e].p;
        }
        __syncwarp();
        twice = named_twice<EACH, WarpShared<EACH>::SLOTS>(s.at, s.slot, a.K, lane);
    }
    // the row's loss, in every lane
    __device__ __forceinline__ float loss(float m, float sum, bool done) const {
        const float log_sum = logf(sum);
        float l = 0.f;
        if (done) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) l += teacher_loss(entry[e], m, log_sum);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
        return l;
    }
    // the named columns' gradients, once all others have been written
    template <class T>
    __device__ __forceinline__ void write(const DistillArgs &a, T *g, float m, float sum, float coef, int lane,
                                          const WarpShared<EACH> &s) const {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const Teacher &t = entry[e];
            float mass = t.p;
            if (t.at >= 0 && !t.silent && (!twice || column_mass(s.at, s.p, 32 * e + lane, a.K, mass)))
                g[t.at] = round_out<T>(t.old + (expf(t.z - m) / sum - mass) * coef);
        }
    }
};

__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
// From the level of a row's largest to its logit. An infinite one has no softmax: its sum is NaN, also where the output
// is finite and only factor y is infinite.
__device__ __forceinline__ float largest_logit(float level, float unit, float &sum) {
    const float m = level * unit;
    if (m == INFINITY) sum = __uint_as_float(0x7fffffffu);
    return m;
}
// a row without logits has no softmax: it is left out (a NaN counts as a logit)
__device__ __forceinline__ bool has_logits(float m, float sum) { return !(m == -INFINITY && !(sum != sum)); }

// a block's rows counted, and the losses added up by the last one
__device__ __forceinline__ void finish_block(const DistillArgs &a) {
    __shared__ int s_last;
    if (!a.ticket) return;
    __syncthreads();
    if (threadIdx.x == 0) s_last = last_counted(a, gridDim.x);
    __syncthreads();
    if (s_last) add_losses(a);
}

// Rows of up to 32 E classes: a warp to a row, E columns a lane.
template <class T, int E>
__global__ void __launch_bounds__(256) k_distill_small(const DistillArgs a) {
    __shared__ WarpShared<2> s_warp[8];
    let_next_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long r = (long long)blockIdx.x * 8 + warp;
    if (r < a.y.rows) {
        const Logit logit(a.y);
        const T *row = static_cast<const T *>(a.y.y) + r * a.y.ld;
        T *g = a.g ? static_cast<T *>(a.g) + r * a.ld_g : nullptr;
        const float rw = a.row_weight ? a.row_weight[r] : 1.f / (float)a.y.rows;
        float z[E];
        bool silent[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = lane + 32 * i;
            silent[i] = true;
            z[i] = c < a.y.cols ? logit.of(to_f32<T>(row[c]), silent[i]) : -INFINITY;
        }
        WarpTeacher<2> teacher{};
        teacher.read<T>(a, logit, row, g, r, lane, s_warp[warp]);
        float m = -INFINITY, s = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) m = fmaxf(m, z[i]);
        m = lanes_max(m);
#pragma unroll
        for (int i = 0; i < E; ++i) s += z[i] == -INFINITY ? 0.f : expf(z[i] - m);
        s = lanes_sum(s);
        const bool done = teacher.any && rw != 0.f && has_logits(m, s);
        const float loss = teacher.loss(m, s, done);
        if (lane == 0) a.row_loss[r] = loss;
        if (g && (done || !a.accumulate)) {
            const float coef = a.weight * rw * logit.factor, over = coef / s;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int c = lane + 32 * i;
                if (c >= a.y.cols) continue;
                const float d = silent[i] || !done ? 0.f : expf(z[i] - m) * over;
                g[c] = round_out<T>(a.accumulate ? to_f32<T>(g[c]) + d : d);
            }
            __syncwarp();
            if (done) teacher.write<T>(a, g, m, s, coef, lane, s_warp[warp]);
        }
    }
    finish_block(a);
}

// Rows of up to 32 N packs: a warp to a row, N packs of 16 bytes a lane, in registers (13319 rows of 698 16-bit
// classes, 64 entries: 22 us, 1.7 TB/s; when in blocks 133 and with single columns 71, both before the losses had a
// launch of their own). Instructions bound it: exponentials, the teacher's entries, and sums across lanes.
template <class T, int N, int EACH, bool FAST>
__global__ void __launch_bounds__(256) k_distill_packs(const DistillArgs a) {
    constexpr int P = Pack<T>::P;
    __shared__ WarpShared<EACH> s_warp[8];
    let_next_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long r = (long long)blockIdx.x * 8 + warp;
    if (r < a.y.rows) {
        const Logit logit(a.y);
        const RowView<T> v(a.y, r);
        T *g = a.g ? static_cast<T *>(a.g) + r * a.ld_g : nullptr;
        const float rw = a.row_weight ? a.row_weight[r] : 1.f / (float)a.y.rows;
        uint4 raw[N];
#pragma unroll
        for (int j = 0; j < N; ++j) raw[j] = lane + 32 * j < v.packs ? v.pack(lane + 32 * j) : make_uint4(0, 0, 0, 0);
        const int at = v.single(lane);
        const float one = at >= 0 ? to_f32<T>(v.row[at]) : 0.f;
        const auto each = [&](auto f) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (lane + 32 * j < v.packs) f(raw[j], lane + 32 * j);
        };
        WarpTeacher<EACH> teacher{};
        teacher.template read<T>(a, logit, v.row, g, r, lane, s_warp[warp]);
        const PackMax<T, FAST, false> pack_max(logit);
        float level = at >= 0 ? pack_max.level(one) : -INFINITY, s = 0.f;
        each([&](const uint4 &w, int) { level = fmaxf(level, pack_max.level(w)); });
        level = lanes_max(level);
        const ExpOf<T, FAST> e(logit, level);
        each([&](const uint4 &w, int) { s += e.sum(w); });
        if (at >= 0) s += e.one(one);
        s = lanes_sum(s);
        const float m = largest_logit(level, pack_max.unit(), s);
        const bool done = teacher.any && rw != 0.f && has_logits(m, s);
        const float loss = teacher.loss(m, s, done);
        if (lane == 0) a.row_loss[r] = loss;
        if (g && (done || !a.accumulate)) {
            const float coef = a.weight * rw * logit.factor, over = done ? coef / s : 0.f;
            if (at >= 0) {
                const float d = done ? e.grad(one, over) : 0.f;
                g[at] = round_out<T>(a.accumulate ? to_f32<T>(g[at]) + d : d);
            }
            T *dst = g + v.head;
            const bool wide = (reinterpret_cast<uintptr_t>(dst) & 15) == 0;
            each([&](const uint4 &w, int k) {
                T *to = dst + k * P;
                alignas(16) T out[P];
                if (a.accumulate) {
#pragma unroll
                    for (int i = 0; i < P; ++i) out[i] = round_out<T>(to_f32<T>(to[i]) + e.grad(Pack<T>::one(w, i), over));
                } else if (done) {
                    e.grads(w, over, out);
                } else {
#pragma unroll
                    for (int i = 0; i < P; ++i) out[i] = round_out<T>(0.f);
                }
                if (wide) {
                    *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(out);
                } else {
#pragma unroll
                    for (int i = 0; i < P; ++i) to[i] = out[i];
                }
            });
            __syncwarp();
            if (done) teacher.template write<T>(a, g, m, s, coef, lane, s_warp[warp]);
        }
    }
    finish_block(a);
}

template <int BATCH>
constexpr int kRowThreads = BATCH == 2 ? 2048 : 1280;  // threads on an SM

// Longer rows, or longer records: the last warp of a block has the teacher's entries, the others the row, with the sum
// of exp(z - m) brought up to each new largest logit m as it comes. HBM bounds it, with the latency of a row's steps
// between barriers, five rows of 32768 to an SM: 4096 of them in bf16 in 98 us, 5.5 TB/s (held in shared memory, three
// rows to an SM: 121; in registers, two: 157). Without CLUSTER a block has a row to itself and knows it: fewer registers
// to keep (16384 rows of 3000 bf16: 77 us, with the form for clusters 89).
template <class T, int THREADS, int BATCH, bool FAST, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, kRowThreads<BATCH> / THREADS)
    k_distill(const DistillArgs a, const int shared_by) {
    constexpr int P = Pack<T>::P, ROW = THREADS - 32, WARPS = ROW / 32, SLOTS = 2 * kTopMax;
    __shared__ float2 s_stat[WARPS], s_share[8];
    __shared__ float s_p[kTopMax], s_log[kTopMax], s_z[kTopMax], s_old[kTopMax];
    __shared__ int s_any, s_twice, s_last, s_at[kTopMax], s_slot[SLOTS];
    const int parts = CLUSTER ? shared_by : 1;
    let_next_launch();
    if (parts > 1) cluster_arrive();  // waited for before the first store to another block
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, part = parts > 1 ? (int)cluster_ctarank() : 0;
    const long long r = blockIdx.x / parts;
    const bool teaches = warp == WARPS;
    const RowView<T> v(a.y, r, part, parts);
    const Logit logit(a.y);
    T *g = a.g ? static_cast<T *>(a.g) + r * a.ld_g : nullptr;
    const float rw = a.row_weight ? a.row_weight[r] : 1.f / (float)a.y.rows;
    const OwnPacks<T, ROW, BATCH> h(v, !teaches);
    const PackMax<T, FAST, false> pack_max(logit);
    float level = -INFINITY, s = 0.f;
    if (teaches) {
        // the teacher's softmax, and which of its columns are named twice, beside the others' work on the row
        float tm = -INFINITY;
        bool some = false;
        for (int k = lane; k < a.K; k += 32) {
            int at = a.index[r * a.K + k];
            const float z = a.teacher_factor * a.top[r * a.K + k];
            if (at >= a.y.cols || z == -INFINITY) at = -1;
            s_at[k] = at;
            s_log[k] = z;
            if (at < 0) continue;
            some = true;
            tm = fmaxf(tm, z);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) tm = fmaxf(tm, __shfl_xor_sync(0xffffffffu, tm, d));
        __syncwarp();
        float sum = 0.f;
        for (int k = lane; k < a.K; k += 32) {
            const int at = s_at[k];
            if (at < 0) continue;
            bool silent;
            const float z = logit.of(to_f32<T>(v.row[at]), silent);
            s_z[k] = z;
            s_old[k] = a.accumulate && g ? to_f32<T>(g[at]) : 0.f;
            if (silent) s_at[k] = at | (1 << 30);  // its column gets no gradient
            sum += expf(s_log[k] - tm);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const float log_sum = logf(sum);
        for (int k = lane; k < a.K; k += 32) {
            const float log_p = s_log[k] - tm - log_sum;
            s_log[k] = log_p;
            s_p[k] = s_at[k] >= 0 ? expf(log_p) : 0.f;
        }
        some = __any_sync(0xffffffffu, some);
        __syncwarp();
        const bool again = named_twice<kTopMax / 32, SLOTS>(s_at, s_slot, a.K, lane);
        if (lane == 0) {
            s_any = some;
            s_twice = again;
        }
    } else {
        // largest and sum, over the warp's columns
        const auto raise = [&](float to) {
            if (to > level) {
                s *= expf((level - to) * pack_max.unit());
                level = to;
            }
        };
        h.batches(v, [&](const uint4 (&w)[BATCH], int k) {
            float most = pack_max.level(w[0]);
#pragma unroll
            for (int i = 1; i < BATCH; ++i)
                if (k + i * ROW < v.last) most = fmaxf(most, pack_max.level(w[i]));
            raise(most);
            const ExpOf<T, FAST> e(logit, level);
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i == 0 || k + i * ROW < v.last) s += e.sum(w[i]);
        });
        if (h.at >= 0) {
            raise(pack_max.level(h.one));
            s += ExpOf<T, FAST>(logit, level).one(h.one);
        }
        join_lanes(level, s, pack_max.unit());
        if (lane == 0) s_stat[warp] = make_float2(level, s);
    }
    __syncthreads();
    const bool any = s_any != 0;
    {
        const float2 w = lane < WARPS ? s_stat[lane] : make_float2(-INFINITY, 0.f);
        level = w.x;
        s = w.y;
        join_lanes(level, s, pack_max.unit());
    }
    if (parts > 1) {
        __syncwarp();
        cluster_wait();  // every block of the cluster has started (behind the row's first pass: nothing is left to wait for)
        if (t < parts) {
            const uint32_t to = mapa_rank(smem_u32(s_share + part), (uint32_t)t);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(level), "f"(s) : "memory");
        }
        __syncwarp();
        cluster_sync();
        const float2 w = lane < parts ? s_share[lane] : make_float2(-INFINITY, 0.f);
        level = w.x;
        s = w.y;
        join_lanes(level, s, pack_max.unit());
    }
    const float m = largest_logit(level, pack_max.unit(), s);
    const bool done = any && rw != 0.f && has_logits(m, s);
    const float coef = a.weight * rw * logit.factor, over = done ? coef / s : 0.f;
    const ExpOf<T, FAST> e(logit, level);
    // each pack of the share to g: made(pack, its place) gives the P gradients
    const auto write = [&](auto made) {
        T *dst = g + v.head;
        if ((reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
            h.each(v, [&](const uint4 &w, int k) {
                T *to = dst + (long long)k * P;
                alignas(16) T out[P];
                made(w, to, out);
                *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(out);
            });
        } else {
            h.each(v, [&](const uint4 &w, int k) {
                T *to = dst + (long long)k * P;
                alignas(16) T out[P];
                made(w, to, out);
#pragma unroll
                for (int i = 0; i < P; ++i) to[i] = out[i];
            });
        }
    };
    if (teaches) {
        // (it has no columns)
    } else if (g && done) {
        if (h.at >= 0) g[h.at] = round_out<T>(e.grad(h.one, over) + (a.accumulate ? to_f32<T>(g[h.at]) : 0.f));
        if (a.accumulate)
            write([&](const uint4 &w, const T *was, T (&out)[P]) {
#pragma unroll
                for (int i = 0; i < P; ++i) out[i] = round_out<T>(to_f32<T>(was[i]) + e.grad(Pack<T>::one(w, i), over));
            });
        else
            write([&](const uint4 &w, const T *, T (&out)[P]) { e.grads(w, over, out); });
    } else if (g && !a.accumulate) {
        if (h.at >= 0) g[h.at] = round_out<T>(0.f);
        write([&](const uint4 &, const T *, T (&out)[P]) {
#pragma unroll
            for (int i = 0; i < P; ++i) out[i] = round_out<T>(0.f);
        });
    }
    if (teaches && part == 0) {
        float loss = 0.f;
        const float log_sum = logf(s);
        if (done)
            for (int k = lane; k < a.K; k += 32)
                if (s_p[k] != 0.f) loss += s_p[k] * (s_log[k] - (s_z[k] - m - log_sum));
#pragma unroll
        for (int d = 16; d; d >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, d);
        // counted here, where this warp has written nothing else that the fence would wait for
        if (lane == 0) {
            a.row_loss[r] = loss;
            if (a.ticket) s_last = last_counted(a, (unsigned)a.y.rows);
        }
    }
    __syncthreads();
    if (teaches && g && done)
        for (int k = lane; k < a.K; k += 32) {
            const int at = s_at[k];
            float mass = s_p[k];
            if (at < 0 || (at >> 30) || at < v.low || at >= v.high) continue;
            if (!s_twice || column_mass(s_at, s_p, k, a.K, mass))
                g[at] = round_out<T>(s_old[k] + (expf(s_z[k] - m) / s - mass) * coef);
        }
    if (a.ticket && part == 0 && s_last) add_losses(a);
}

// the losses of many rows, where a block should not wait for its stores to be counted
__global__ void __launch_bounds__(512) k_distill_sum(const DistillArgs a) {
    wait_launch_before();
    add_losses(a);
}

template <class T, bool FAST>
cudaError_t distill_rows(const DistillArgs &a, cudaStream_t st) {
    const int packs = (int)(((long long)a.y.cols * sizeof(T) + 15) / 16), parts = shares(a.y.rows, packs, 512);
    const int blocks = a.y.rows * parts, each = packs / parts;
    // short rows have less to load than to wait for, and want more blocks on an SM (4000 rows of 5000 fp32: 40 us; by a
    // form that could share rows 42, with six of its blocks to an SM 44, with five 52); long ones are read with more loads
    // under way (4096 of 32768 bf16: 98, with the short ones' form 129)
    if (each <= 1280 && blocks > 5 * 152)  // (rows are not shared there)
        return launch_shared<k_distill<T, 256, 2, FAST, false>, 256, 0>(a.y.rows, 1, st, a, 1);
    // few blocks have more threads each
    if (each <= 4096 && (blocks >= 152 || each <= 512)) {
        if (parts == 1) return launch_shared<k_distill<T, 256, 4, FAST, false>, 256, 0>(a.y.rows, 1, st, a, 1);
        return launch_shared<k_distill<T, 256, 4, FAST, true>, 256, 0>(a.y.rows, parts, st, a, parts);
    }
    return launch_shared<k_distill<T, 512, 4, FAST, true>, 512, 0>(a.y.rows, parts, st, a, parts);
}

// blocks that count their rows: as many as two to an SM. More have the losses added up by a launch of their own, since
// a block that counts waits for its stores (13319 rows of 698 fp16: 38 us counted, 32 with the launch).
constexpr int kCounting = 304;
// up to here, rows with records of more than 64 entries are as fast in blocks or faster (1000 fp32, K = 128: 304 rows 9.5
// us by warps and 8.5 in blocks, 1216 rows 9.7 and 11.3, 16384 rows 64 and 103)
constexpr int kFewRows = 608;

template <class T, bool FAST>
cudaError_t distill_by_size(DistillArgs &a, cudaStream_t st) {
    const int packs = (int)(((long long)a.y.cols * sizeof(T) + 15) / 16);
    const unsigned blocks = ((unsigned)a.y.rows + 7) / 8;
    a.ticket = blocks <= kCounting;
    if (a.y.cols <= 64 && a.K <= 64) {
        k_distill_small<T, 2><<<blocks, 256, 0, st>>>(a);
    } else if (a.K <= 64 && packs <= 32 * 2) {
        k_distill_packs<T, 2, 2, FAST><<<blocks, 256, 0, st>>>(a);
    } else if (a.K <= 64 && packs <= 32 * 8) {
        k_distill_packs<T, 8, 2, FAST><<<blocks, 256, 0, st>>>(a);
    } else if (a.K <= 128 && packs <= 32 * 8 && a.y.rows > kFewRows) {
        k_distill_packs<T, 8, 4, FAST><<<blocks, 256, 0, st>>>(a);
    } else {
        a.ticket = a.y.rows <= kCounting;
        return distill_rows<T, FAST>(a, st);
    }
    return cudaGetLastError();
}

template <class T>
cudaError_t distill(DistillArgs a, int &launches, cudaStream_t st) {
    const bool fast = sizeof(T) == 2 && a.y.factor * a.y.silent == -INFINITY && fabsf(a.y.factor) < most_factor &&
                      fabsf(a.y.factor) >= least_factor;
    const cudaError_t e = fast ? distill_by_size<T, sizeof(T) == 2>(a, st) : distill_by_size<T, false>(a, st);
    launches = a.ticket ? 1 : 2;
    return e != cudaSuccess || a.ticket ? e : launch_dependent(k_distill_sum, 1, 512, st, a);
}

}  // namespace

cudaError_t launch_top_logits(const LogitArgs &a, int K, float *top, int32_t *index, cudaStream_t st) {
    if (a.type == DSTD_TYPE_F32) return top_logits<float>(a, K, top, index, st);
    if (a.type == DSTD_TYPE_BF16) return top_logits<__nv_bfloat16>(a, K, top, index, st);
    return top_logits<__half>(a, K, top, index, st);
}

cudaError_t launch_distill(const DistillArgs &a, int &launches, cudaStream_t st) {
    if (a.y.type == DSTD_TYPE_F32) return distill<float>(a, launches, st);
    if (a.y.type == DSTD_TYPE_BF16) return distill<__nv_bfloat16>(a, launches, st);
    return distill<__half>(a, launches, st);
}

}  // namespace dstd
