// Learning from a teacher: the largest logits of each row (the teacher's record) and
// the distillation loss from such a record, with its gradient.
//
// The logit of an output y is factor y; where that is -infinity (a silent output,
// whose spike time is +infinity, or a masked class) it is factor silent, a constant.
#include "dstd_rows.cuh"
#include "dstd_tc_ptx.cuh"

#include <algorithm>

namespace dstd {
namespace {

template <class T>
__device__ __forceinline__ float logit_of(float y, float factor, float none, bool &silent) {
    const float z = factor * y;
    silent = z == -INFINITY;
    return silent ? none : z;
}

// A row in 16-byte pieces from its first aligned address: packs cover
// [head, head + packs P), up to P - 1 columns before and after them are taken singly.
template <class T>
struct RowView {
    const T *row;
    int cols, head, packs;
    __device__ __forceinline__ RowView(const LogitArgs &a, long long r) {
        constexpr int P = Pack<T>::P;
        row = static_cast<const T *>(a.y) + r * a.ld;
        cols = a.cols;
        head = min(cols, (int)((0 - reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (P - 1)));
        packs = (cols - head) / P;
    }
    // column of a thread's single element (t below 2 P), -1: none
    __device__ __forceinline__ int single(int t) const {
        constexpr int P = Pack<T>::P;
        if (t < P) return t < head ? t : -1;
        const int c = head + packs * P + t - P;
        return t < 2 * P && c < cols ? c : -1;
    }
    __device__ __forceinline__ uint4 pack(int k) const {
        return __ldg(reinterpret_cast<const uint4 *>(row + head + (long long)k * Pack<T>::P));
    }
};

// ---------------------------------------------------------------------------
// The K largest logits of a row, descending, equal ones by ascending column. The
// logits are ordered as 32-bit keys (-0 as 0, NaN above all). Each thread takes
// the largest of its columns; the K-th largest of those is a bound that no
// smaller logit of the row can be among the K largest below, and few are above
// it: with 1024 threads about K. Those are gathered and put in order by counting,
// for each, the larger ones. Rows with more than CAP logits at the bound (many equal
// ones) go digit by digit.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(float z) {
    if (z != z) return 0xffffffffu;
    const uint32_t u = __float_as_uint(z + 0.f);  // -0 + 0 = 0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of_key(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

constexpr int kCap = 2048;

template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS) k_top_logits(const LogitArgs a, const int K, float *top, int32_t *index) {
    constexpr int P = Pack<T>::P;
    __shared__ uint64_t s_cand[kCap];
    __shared__ unsigned s_n, s_hist[256], s_digit[2], s_warp[THREADS / 32];
    const int t = threadIdx.x;
    const long long r = blockIdx.x;
    const RowView<T> v(a, r);
    const float none = a.factor * a.silent;
    const auto key = [&](float y) {
        bool silent;
        return key_of(logit_of<T>(y, a.factor, none, silent));
    };
    // every column once, in any order
    const auto each = [&](auto f) {
        const int c = v.single(t);
        if (c >= 0) f(c, key(to_f32<T>(v.row[c])));
        for (int k = t; k < v.packs; k += THREADS) {
            const uint4 w = v.pack(k);
#pragma unroll
            for (int i = 0; i < P; ++i) f(v.head + k * P + i, key(Pack<T>::one(w, i)));
        }
    };
    if (t == 0) s_n = 0;
    uint32_t mine = 0, bound = 0;
    each([&](int, uint32_t k) { mine = max(mine, k); });
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = bound | (1u << bit);
        if (__syncthreads_count(mine >= trial) >= K) bound = trial;
    }
    __syncthreads();
    each([&](int c, uint32_t k) {
        if (k >= bound) {
            const unsigned at = atomicAdd(&s_n, 1u);
            if (at < kCap) s_cand[at] = (uint64_t)k << 32 | (uint32_t)~c;
        }
    });
    __syncthreads();
    unsigned n = s_n;
    if (n > kCap) {
        uint32_t prefix = 0, mask = 0;
        unsigned need = K;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = t; i < 256; i += THREADS) s_hist[i] = 0;
            __syncthreads();
            each([&](int, uint32_t k) {
                if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> shift) & 255u], 1u);
            });
            __syncthreads();
            if (t == 0) {
                unsigned above = 0;
                int d = 255;
                while (d > 0 && above + s_hist[d] < need) above += s_hist[d--];
                s_digit[0] = (unsigned)d;
                s_digit[1] = above;
            }
            __syncthreads();
            prefix |= s_digit[0] << shift;
            mask |= 255u << shift;
            need -= s_digit[1];
            __syncthreads();
        }
        if (t == 0) s_n = 0;
        __syncthreads();
        each([&](int c, uint32_t k) {
            if (k > prefix) s_cand[atomicAdd(&s_n, 1u)] = (uint64_t)k << 32 | (uint32_t)~c;
        });
        // the first `need` columns of those equal to the K-th
        unsigned found = 0;
        for (long long c0 = 0; c0 < v.cols && found < need; c0 += THREADS) {
            const bool here = c0 + t < v.cols && key(to_f32<T>(v.row[c0 + t])) == prefix;
            const unsigned ballot = __ballot_sync(0xffffffffu, here);
            if ((t & 31) == 0) s_warp[t >> 5] = __popc(ballot);
            __syncthreads();
            unsigned before = found, all = found;
            for (int w = 0; w < THREADS / 32; ++w) {
                if (w < (t >> 5)) before += s_warp[w];
                all += s_warp[w];
            }
            before += __popc(ballot & ((1u << (t & 31)) - 1u));
            if (here && before < need) s_cand[K - need + before] = (uint64_t)prefix << 32 | (uint32_t)~(uint32_t)(c0 + t);
            found = all;
            __syncthreads();
        }
        n = K;
        __syncthreads();
    }
    for (unsigned i = t; i < n; i += THREADS) {
        const uint64_t me = s_cand[i];
        int rank = 0;
        for (unsigned j = 0; j < n; ++j) rank += s_cand[j] > me;
        if (rank < K) {
            top[r * K + rank] = logit_of_key((uint32_t)(me >> 32));
            index[r * K + rank] = (int32_t)~(uint32_t)me;
        }
    }
}

template <class T>
cudaError_t top_logits(const LogitArgs &a, int K, float *top, int32_t *index, cudaStream_t st) {
    if (a.cols <= 8192) k_top_logits<T, 256><<<(unsigned)a.rows, 256, 0, st>>>(a, K, top, index);
    else k_top_logits<T, 1024><<<(unsigned)a.rows, 1024, 0, st>>>(a, K, top, index);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// Distillation. With p = softmax(teacher_factor top) over a row's used entries
// and q = softmax of its logits:
//     L_r = sum_k p_k (log p_k - log q_{i_k}),
//     dL_r / dy_c = factor (q_c - sum_{k: i_k = c} p_k)   (0 where silent).
// The first pass takes the largest logit m and sum_c exp(z_c - m), rescaling when
// m grows; the second writes exp(z - m) times a constant. The few columns that
// the teacher names are written once more, from fp32, so that every gradient is
// rounded once; entries of the same column are added up in their order.
// ---------------------------------------------------------------------------
template <class T>
__device__ __forceinline__ float exp_of(float x) {
    if constexpr (sizeof(T) == 4) return expf(x);
    else return __expf(x);  // off by 2^-21 or so near 0, far below a 16-bit rounding
}

template <int THREADS>
__device__ __forceinline__ void group_sync() {
    if constexpr (THREADS == 32) __syncwarp();
    else __syncthreads();
}
template <int THREADS>
__device__ __forceinline__ float group_sum(float v, float *s_part) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if constexpr (THREADS > 32) {
        const int t = threadIdx.x;
        __syncthreads();
        if ((t & 31) == 0) s_part[t >> 5] = v;
        __syncthreads();
        v = s_part[0];
        for (int i = 1; i < THREADS / 32; ++i) v += s_part[i];
    }
    return v;
}
template <int THREADS>
__device__ __forceinline__ float group_max(float v, float *s_part) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    if constexpr (THREADS > 32) {
        const int t = threadIdx.x;
        __syncthreads();
        if ((t & 31) == 0) s_part[t >> 5] = v;
        __syncthreads();
        v = s_part[0];
        for (int i = 1; i < THREADS / 32; ++i) v = fmaxf(v, s_part[i]);
    }
    return v;
}

// THREADS to a row: a warp, 8 rows to a block, or a whole block. VEC: y's and g's
// rows have their aligned 16 bytes at the same columns.
template <class T, int THREADS, bool VEC>
__global__ void __launch_bounds__(THREADS == 32 ? 256 : THREADS) k_distill(const DistillArgs a) {
    constexpr int P = Pack<T>::P, ROWS = THREADS == 32 ? 8 : 1;
    __shared__ float s_p[ROWS][kTopMax];
    __shared__ int s_at[ROWS][kTopMax];
    __shared__ float s_part[32];
    __shared__ double s_total[32];
    __shared__ unsigned s_last;
    const int t = threadIdx.x % THREADS, sub = threadIdx.x / THREADS;
    const long long r = (long long)blockIdx.x * ROWS + sub;
    const LogitArgs &y = a.y;
    const float none = y.factor * y.silent;
    if (r < y.rows) {
        const RowView<T> v(y, r);
        const float rw = a.row_weight ? a.row_weight[r] : 1.f / (float)y.rows;
        float *p = s_p[sub];
        int *at = s_at[sub];
        // the teacher's softmax
        float m = -INFINITY;
        for (int k = t; k < a.K; k += THREADS) {
            const int i = a.index[r * a.K + k];
            const float z = a.teacher_factor * a.top[r * a.K + k];
            const bool used = i >= 0 && i < y.cols && z != -INFINITY;
            at[k] = used ? i : -1;
            p[k] = z;
            if (used) m = fmaxf(m, z);
        }
        m = group_max<THREADS>(m, s_part);
        float s = 0.f;
        for (int k = t; k < a.K; k += THREADS)
            if (at[k] >= 0) s += expf(p[k] - m);
        s = group_sum<THREADS>(s, s_part);
        const bool any = group_max<THREADS>([&] {
            float u = 0.f;
            for (int k = t; k < a.K; k += THREADS) u = at[k] >= 0 ? 1.f : u;
            return u;
        }(), s_part) > 0.f;
        const bool taught = any && rw != 0.f;
        const float t_max = m, t_log = logf(s);
        // the row's largest logit and its sum
        float z_max = -INFINITY, z_sum = 0.f;
        const auto take = [&](float yv) {
            bool silent;
            const float z = logit_of<T>(yv, y.factor, none, silent);
            if (z > z_max) {
                z_sum *= expf(z_max - z);
                z_max = z;
            }
            z_sum += z == -INFINITY ? 0.f : exp_of<T>(z - z_max);
        };
        if (taught) {
            for (int c = t; c < 2 * P; c += THREADS) {
                const int i = v.single(c);
                if (i >= 0) take(to_f32<T>(v.row[i]));
            }
            for (int k = t; k < v.packs; k += THREADS) {
                const uint4 w = v.pack(k);
#pragma unroll
                for (int i = 0; i < P; ++i) take(Pack<T>::one(w, i));
            }
        }
        const float row_max = group_max<THREADS>(z_max, s_part);
        z_sum = group_sum<THREADS>(z_max == row_max ? z_sum : z_sum * expf(z_max - row_max), s_part);
        // a row without logits has no softmax: it is left out (a NaN counts as a logit)
        const bool empty = row_max == -INFINITY && !(z_sum != z_sum);
        const float z_log = logf(z_sum);
        const bool done = taught && !empty;
        float part = 0.f;
        if (done)
            for (int k = t; k < a.K; k += THREADS) {
                if (at[k] < 0) continue;
                bool silent;
                const float z = logit_of<T>(to_f32<T>(v.row[at[k]]), y.factor, none, silent);
                const float log_p = p[k] - t_max - t_log, pk = expf(log_p);
                if (pk != 0.f) part += pk * (log_p - (z - row_max - z_log));
                p[k] = pk;
            }
        const float loss = group_sum<THREADS>(part, s_part);
        if (t == 0) a.row_loss[r] = loss;
        if (a.g && (done || !a.accumulate)) {
            T *g = static_cast<T *>(a.g) + r * a.ld_g;
            const float coef = a.weight * rw * y.factor, scale = done ? coef / z_sum : 0.f;
            const auto grad = [&](float yv, float old) {
                bool silent;
                const float z = logit_of<T>(yv, y.factor, none, silent);
                return old + (silent || !done ? 0.f : exp_of<T>(z - row_max) * scale);
            };
            // what the named columns hold before they are written
            constexpr int EACH = kTopMax / THREADS > 0 ? kTopMax / THREADS : 1;
            float old[EACH];
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int k = e * THREADS + t;
                old[e] = k < a.K && at[k] >= 0 && a.accumulate ? to_f32<T>(g[at[k]]) : 0.f;
            }
            group_sync<THREADS>();
            if constexpr (VEC) {
                for (int c = t; c < 2 * P; c += THREADS) {
                    const int i = v.single(c);
                    if (i >= 0) g[i] = round_out<T>(grad(to_f32<T>(v.row[i]), a.accumulate ? to_f32<T>(g[i]) : 0.f));
                }
                for (int k = t; k < v.packs; k += THREADS) {
                    const uint4 w = v.pack(k);
                    uint4 *dst = reinterpret_cast<uint4 *>(g + v.head + (long long)k * P);
                    uint4 was = make_uint4(0, 0, 0, 0);
                    if (a.accumulate) was = *dst;
                    alignas(16) T out[P];
#pragma unroll
                    for (int i = 0; i < P; ++i) out[i] = round_out<T>(grad(Pack<T>::one(w, i), Pack<T>::one(was, i)));
                    *dst = *reinterpret_cast<const uint4 *>(out);
                }
            } else {
                for (long long c = t; c < v.cols; c += THREADS)
                    g[c] = round_out<T>(grad(to_f32<T>(v.row[c]), a.accumulate ? to_f32<T>(g[c]) : 0.f));
            }
            group_sync<THREADS>();
            if (done) {
#pragma unroll
                for (int e = 0; e < EACH; ++e) {
                    const int k = e * THREADS + t;
                    if (k >= a.K || at[k] < 0) continue;
                    const int c = at[k];
                    bool first = true;
                    for (int j = 0; j < k; ++j) first = first && at[j] != c;
                    if (!first) continue;
                    float mass = p[k];
                    for (int j = k + 1; j < a.K; ++j)
                        if (at[j] == c) mass += p[j];
                    bool silent;
                    const float z = logit_of<T>(to_f32<T>(v.row[c]), y.factor, none, silent);
                    if (!silent) g[c] = round_out<T>(old[e] + (expf(z - row_max) / z_sum - mass) * coef);
                }
            }
        }
    }
    // the last block adds the rows' losses up, in a fixed order
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(reinterpret_cast<unsigned *>(a.loss + 1), 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    double sum = 0.0;
    for (long long i = threadIdx.x; i < y.rows; i += blockDim.x) {
        const float w = a.row_weight ? a.row_weight[i] : 1.f / (float)y.rows;
        if (w != 0.f) sum += (double)w * __ldcg(a.row_loss + i);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) s_total[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = s_total[0];
        for (unsigned i = 1; i < blockDim.x / 32; ++i) sum += s_total[i];
        a.loss[0] = (float)(a.weight * sum);
        *reinterpret_cast<unsigned *>(a.loss + 1) = 0u;
    }
}

template <class T>
cudaError_t distill(const DistillArgs &a, cudaStream_t st) {
    constexpr int P = Pack<T>::P;
    const auto phase = [](const void *p) { return (long long)(reinterpret_cast<uintptr_t>(p) / sizeof(T)); };
    const bool vec = !a.g || (((phase(a.y.y) - phase(a.g)) | (a.y.ld - a.ld_g)) & (P - 1)) == 0;
    const unsigned rows = (unsigned)a.y.rows;
    if (a.y.cols <= 1024 && a.K <= 64) {
        if (vec) k_distill<T, 32, true><<<(rows + 7) / 8, 256, 0, st>>>(a);
        else k_distill<T, 32, false><<<(rows + 7) / 8, 256, 0, st>>>(a);
    } else if (a.y.cols <= 8192) {
        if (vec) k_distill<T, 256, true><<<rows, 256, 0, st>>>(a);
        else k_distill<T, 256, false><<<rows, 256, 0, st>>>(a);
    } else {
        if (vec) k_distill<T, 1024, true><<<rows, 1024, 0, st>>>(a);
        else k_distill<T, 1024, false><<<rows, 1024, 0, st>>>(a);
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_top_logits(const LogitArgs &a, int K, float *top, int32_t *index, cudaStream_t st) {
    if (a.type == DSTD_TYPE_F32) return top_logits<float>(a, K, top, index, st);
    if (a.type == DSTD_TYPE_BF16) return top_logits<__nv_bfloat16>(a, K, top, index, st);
    return top_logits<__half>(a, K, top, index, st);
}

cudaError_t launch_distill(const DistillArgs &a, cudaStream_t st) {
    if (a.y.type == DSTD_TYPE_F32) return distill<float>(a, st);
    if (a.y.type == DSTD_TYPE_BF16) return distill<__nv_bfloat16>(a, st);
    return distill<__half>(a, st);
}

}  // namespace dstd
