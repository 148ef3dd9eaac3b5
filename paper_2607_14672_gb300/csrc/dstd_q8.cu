// 8-bit rows and their products: the row quantiser and
// y_tn = sx_t sw_n sum_k x_tk w_nk with the sum exact in whole numbers.
#include "dstd_rows.cuh"
#include "dstd_tc_ptx.cuh"

#include <algorithm>

namespace dstd {

// ---------------------------------------------------------------------------
// Row quantiser. With a = max_k |x_k|:
//     scale = a / 127,  q_k = rint(x_k (127 (1 / a))),  value_k = q_k scale,
// each operation rounded to fp32 (three roundings move x 127 / a by less than
// 127 * 3 * 2^-24 code steps; above a = 2^126, where 1 / a is subnormal, by less
// than twice that). 1 / a overflows for a below 2^-128; rows of
// very small a are multiplied by 2^64 first (exact), which gives the same codes.
// A row of zeros has scale 0; a row that holds an infinity or a NaN has scale
// NaN and codes 0, so that whatever is computed from it is NaN. The largest |x|
// is taken on the bit patterns: without the sign they order like the values,
// with infinities and NaN on top.
// ---------------------------------------------------------------------------
struct RowCode {
    float pre, inv, scale;  // q = rint((x pre) inv), value = q scale
};
__device__ __forceinline__ RowCode row_code(unsigned top_bits) {
    RowCode c{1.f, 0.f, 0.f};
    if (top_bits >= 0x7f800000u) {
        c.pre = 0.f;
        c.scale = __uint_as_float(0x7fffffffu);
    } else if (top_bits != 0) {
        const float a = __uint_as_float(top_bits);
        c.scale = __fdiv_rn(a, 127.f);
        if (a < 1e-30f) c.pre = 18446744073709551616.f;
        c.inv = __frcp_rn(a * c.pre) * 127.f;
    }
    return c;
}
// an infinity times pre = 0 is NaN, whose conversion to an integer is 0
__device__ __forceinline__ int code_of(float x, const RowCode &c) { return __float2int_rn((x * c.pre) * c.inv); }

struct QuantArgs {
    int rows, cols;
    long long ld_x, ld_q, ld_v;
    int8_t *q;
    float *scale, *values;
};

// One pass: THREADS threads (a warp, or a whole block) hold their row in
// registers, find the largest |x|, and write. PACKED: 16 bytes of x at a time,
// from the first aligned one of the row; up to P - 1 elements at each end are
// taken singly. That needs the row's codes (and values) aligned at the same
// element, as they are when x and q are both contiguous. Otherwise one element
// at a time (loads and stores of neighbouring threads are still neighbours).
// A thread has up to 4 or 8 of these loads under way, and a block's threads are
// few enough for several rows to be on an SM (4153 rows of 4480 16-bit elements:
// 13 us; with 512 threads a row and one load each 21 us). HBM bounds it: 16384 x
// 16384 fp32 with values in 345 us, 7.0 TB/s.
template <class T, bool PACKED, int L, int THREADS, int BLOCK = THREADS == 32 ? 256 : THREADS>
__global__ void __launch_bounds__(BLOCK, THREADS == 32 ? 1 : (BLOCK == 1024 ? 2 : (L == 8 ? 1024 : 1536) / BLOCK)) k_quantize_rows(const T *__restrict__ x, const QuantArgs a) {
    constexpr int P = PACKED ? Pack<T>::P : 1;
    __shared__ unsigned s_top[32];
    let_next_launch();
    const int t = threadIdx.x % THREADS;
    const long long r = (long long)blockIdx.x * (BLOCK / THREADS) + threadIdx.x / THREADS;
    if (r >= a.rows) return;  // a whole warp, or never
    const T *row = x + r * a.ld_x;
    int8_t *q = a.q + r * a.ld_q;
    float *val = a.values ? a.values + r * a.ld_v : nullptr;
    // packs cover [head, head + packs P); `edge` are this thread's elements before and after them
    const int head = PACKED ? min(a.cols, (int)((0 - reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (P - 1))) : 0;
    const int packs = (a.cols - head) / P, done = head + packs * P;
    const int edge[2] = {t < head ? t : -1, PACKED && done + t < a.cols ? done + t : -1};
    uint4 raw[PACKED ? L : 1];
    float one[PACKED ? 2 : L];
    auto value = [&](int j, int i) { return PACKED ? Pack<T>::one(raw[PACKED ? j : 0], i) : one[PACKED ? 0 : j]; };
#pragma unroll
    for (int j = 0; j < L; ++j) {
        const int k = j * THREADS + t;
        if constexpr (PACKED) {
            raw[j] = k < packs ? *reinterpret_cast<const uint4 *>(row + head + k * P) : make_uint4(0, 0, 0, 0);
        } else {
            one[j] = k < a.cols ? to_f32<T>(row[k]) : 0.f;
        }
    }
    unsigned top = 0;
    if constexpr (PACKED) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            one[e] = edge[e] >= 0 ? to_f32<T>(row[edge[e]]) : 0.f;
            top = max(top, __float_as_uint(one[e]) & 0x7fffffffu);
        }
    }
#pragma unroll
    for (int j = 0; j < L; ++j)
#pragma unroll
        for (int i = 0; i < P; ++i) top = max(top, __float_as_uint(value(j, i)) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (THREADS > 32) {
        if ((t & 31) == 0) s_top[t >> 5] = top;
        __syncthreads();
        top = s_top[(t & 31) % (THREADS / 32)];
        top = __reduce_max_sync(0xffffffffu, top);
    }
    const RowCode c = row_code(top);
    if (t == 0) a.scale[r] = c.scale;
    auto put = [&](int k, float v) {
        const int n = code_of(v, c);
        q[k] = (int8_t)n;
        if (val) val[k] = n * c.scale;
    };
    if constexpr (PACKED) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (edge[e] >= 0) put(edge[e], one[e]);
    }
#pragma unroll
    for (int j = 0; j < L; ++j) {
        const int k = j * THREADS + t;
        if constexpr (PACKED) {
            if (k >= packs) break;
            int n[P];
#pragma unroll
            for (int i = 0; i < P; ++i) n[i] = code_of(value(j, i), c);
            uint32_t w[P / 4];
#pragma unroll
            for (int i = 0; i < P / 4; ++i)
                w[i] = (uint32_t)(n[4 * i] & 255) | (uint32_t)(n[4 * i + 1] & 255) << 8 |
                       (uint32_t)(n[4 * i + 2] & 255) << 16 | (uint32_t)n[4 * i + 3] << 24;
            if constexpr (P == 4) *reinterpret_cast<uint32_t *>(q + head + k * P) = w[0];
            else *reinterpret_cast<uint2 *>(q + head + k * P) = make_uint2(w[0], w[1]);
            if (val) {
#pragma unroll
                for (int i = 0; i < P; i += 4)
                    *reinterpret_cast<float4 *>(val + head + k * P + i) =
                        make_float4(n[i] * c.scale, n[i + 1] * c.scale, n[i + 2] * c.scale, n[i + 3] * c.scale);
            }
        } else {
            if (k >= a.cols) break;
            put(k, one[j]);
        }
    }
}

// rows too long for the registers: read twice (the second time mostly from L2).
// Columns are counted without a sign: a row may have up to 2^31 - 1 of them, and
// the count passes that by a step before the loop ends. One element a load, so
// neither the loads nor HBM are used fully: 1024 rows of 40000 fp32 with values in
// 97 us (3.8 TB/s), 8192 rows of 32768 bf16 in 245 us (3.3 TB/s).
template <class T>
__global__ void __launch_bounds__(256) k_quantize_long(const T *__restrict__ x, const QuantArgs a) {
    __shared__ unsigned s_top[8];
    const long long r = blockIdx.x;
    const unsigned cols = (unsigned)a.cols;
    const T *row = x + r * a.ld_x;
    unsigned top = 0;
#pragma unroll 8
    for (unsigned k = threadIdx.x; k < cols; k += 256)
        top = max(top, __float_as_uint(to_f32<T>(row[k])) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, s_top[i]);
    const RowCode c = row_code(top);
    if (threadIdx.x == 0) a.scale[r] = c.scale;
#pragma unroll 4
    for (unsigned k = threadIdx.x; k < cols; k += 256) {
        const int v = code_of(to_f32<T>(row[k]), c);
        a.q[r * a.ld_q + k] = (int8_t)v;
        if (a.values) a.values[r * a.ld_v + k] = (float)v * c.scale;
    }
}

template <class T>
void quantize(const T *x, const QuantArgs &a, cudaStream_t st) {
    constexpr int P = Pack<T>::P;
    // element of the first aligned 16 bytes, codes and values, in every row the same for all three
    const auto phase = [](const void *p, size_t bytes) { return (long long)(reinterpret_cast<uintptr_t>(p) / bytes); };
    const bool packed = ((phase(x, sizeof(T)) - phase(a.q, 1)) & (P - 1)) == 0 && ((a.ld_x - a.ld_q) & (P - 1)) == 0 &&
                        (!a.values || (((phase(x, sizeof(T)) - phase(a.values, 4)) & 3) == 0 &&
                                       ((a.ld_x - a.ld_v) & 3) == 0));
    const int cols = a.cols;
    if (cols > 16384) {
        k_quantize_long<T><<<(unsigned)a.rows, 256, 0, st>>>(x, a);
    } else if (!packed) {
        if (cols <= 256) k_quantize_rows<T, false, 8, 32><<<((unsigned)a.rows + 7) / 8, 256, 0, st>>>(x, a);
        else if (cols <= 1024) k_quantize_rows<T, false, 32, 32><<<((unsigned)a.rows + 7) / 8, 256, 0, st>>>(x, a);
        else if (cols <= 4096) k_quantize_rows<T, false, 16, 256><<<(unsigned)a.rows, 256, 0, st>>>(x, a);
        else if (cols <= 8192) k_quantize_rows<T, false, 16, 512><<<(unsigned)a.rows, 512, 0, st>>>(x, a);
        else k_quantize_rows<T, false, 16, 1024><<<(unsigned)a.rows, 1024, 0, st>>>(x, a);
    } else {
        const int bytes = cols * (int)sizeof(T);
        if (bytes <= 1024) k_quantize_rows<T, true, 2, 32><<<((unsigned)a.rows + 7) / 8, 256, 0, st>>>(x, a);
        else if (bytes <= 4096) k_quantize_rows<T, true, 8, 32><<<((unsigned)a.rows + 7) / 8, 256, 0, st>>>(x, a);
        else if (bytes <= 8192) k_quantize_rows<T, true, 4, 128><<<(unsigned)a.rows, 128, 0, st>>>(x, a);
        else if (bytes <= 16384) k_quantize_rows<T, true, 4, 256><<<(unsigned)a.rows, 256, 0, st>>>(x, a);
        else if (bytes <= 32768) k_quantize_rows<T, true, 8, 256><<<(unsigned)a.rows, 256, 0, st>>>(x, a);
        else k_quantize_rows<T, true, 8, 512><<<(unsigned)a.rows, 512, 0, st>>>(x, a);
    }
}

cudaError_t launch_quantize_rows(const void *x, dstd_type type, int rows, int cols, long long ld_x, int8_t *q,
                                 long long ld_q, float *scale, float *values, long long ld_v, cudaStream_t st) {
    if (rows == 0) return cudaSuccess;
    const QuantArgs a{rows, cols, ld_x, ld_q, ld_v, q, scale, values};
    if (type == DSTD_TYPE_F32) quantize((const float *)x, a, st);
    else if (type == DSTD_TYPE_BF16) quantize((const __nv_bfloat16 *)x, a, st);
    else quantize((const __half *)x, a, st);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// Grid weights of a layer's inputs straight to tokens: t [B, N] -> codes of row
// (b, m), zero for M <= m < Mp, and the rows' scales; the same codes as from
// writing the grid weights out and quantising their rows. An input touches two
// grid points, so the fp32 rows (M times the inputs) never exist: a block first
// takes the largest weight of every grid point over all inputs of its sample
// (in shared memory; the bits of positive floats order like the floats; a plain
// look first keeps all but the early ones from the atomics), then writes the
// codes of its 4 THREADS inputs, four to a word.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void raise_top(unsigned *top, float w) {
    const unsigned bits = __float_as_uint(w) & 0x7fffffffu;
    if (bits > *(volatile unsigned *)top) atomicMax(top, bits);
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_bin_codes(const float *__restrict__ t, int N, const LifConst c, int8_t *q,
                                                   long long ld_q, float *scale) {
    __shared__ unsigned s_top[128];
    const int b = blockIdx.y;
    const float *row = t + (long long)b * N;
    for (int m = threadIdx.x; m < c.Mp; m += THREADS) s_top[m] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < N; j += 4 * THREADS) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = j + i * THREADS < N ? __ldg(row + j + i * THREADS) : INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!isfinite(x[i])) continue;
            const BinW w = bin_weights(c, x[i], false);
            if (w.k >= 0 && w.k < c.M) raise_top(&s_top[w.k], w.wR);
            if (w.k >= -1 && w.k + 1 < c.M) raise_top(&s_top[w.k + 1], w.wL);
        }
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int m = threadIdx.x; m < c.Mp; m += THREADS) scale[(long long)b * c.Mp + m] = row_code(s_top[m]).scale;
    const int j0 = (blockIdx.x * THREADS + threadIdx.x) * 4;
    if (j0 >= ld_q) return;
    int k[4], first[4], second[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k[i] = -100;
        first[i] = second[i] = 0;
        const float x = j0 + i < N ? row[j0 + i] : INFINITY;
        if (!isfinite(x)) continue;
        const BinW w = bin_weights(c, x, false);
        k[i] = w.k;
        if (w.k >= 0 && w.k < c.M) first[i] = code_of(w.wR, row_code(s_top[w.k])) & 255;
        if (w.k >= -1 && w.k + 1 < c.M) second[i] = code_of(w.wL, row_code(s_top[w.k + 1])) & 255;
    }
    int8_t *out = q + (long long)b * c.Mp * ld_q + j0;
    for (int m = 0; m < c.Mp; ++m, out += ld_q) {
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) word |= (uint32_t)(m == k[i] ? first[i] : (m == k[i] + 1 ? second[i] : 0)) << (8 * i);
        *reinterpret_cast<uint32_t *>(out) = word;
    }
}

cudaError_t launch_bin_codes(const float *t, int B, int N, const LifConst &c, int8_t *q, long long ld_q, float *scale,
                             cudaStream_t st) {
    // every block passes over all inputs of its sample: long rows take blocks of more threads
    if (ld_q <= 1024) k_bin_codes<256><<<dim3(1, (unsigned)B), 256, 0, st>>>(t, N, c, q, ld_q, scale);
    else k_bin_codes<1024><<<dim3((unsigned)((ld_q + 4095) / 4096), (unsigned)B), 1024, 0, st>>>(t, N, c, q, ld_q, scale);
    return cudaGetLastError();
}

// row sums of the weights' values: rowsum_n = scale_n sum_k q_nk (one warp per
// row, whose start is at any address: words of four codes from the first aligned one)
__global__ void __launch_bounds__(256) k_q8_rowsum(const int8_t *__restrict__ w, long long ld, int N, int K,
                                                   const float *__restrict__ scale, float *rowsum) {
    const int n = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (n >= N) return;
    const int8_t *row = w + (long long)n * ld;
    const int head = min(K, (int)(-reinterpret_cast<uintptr_t>(row) & 3)), words = (K - head) / 4;
    int sum = 0;
    const int *p = reinterpret_cast<const int *>(row + head);
#pragma unroll 8
    for (int i = lane; i < words; i += 32) sum = __dp4a(__ldg(p + i), 0x01010101, sum);
    const int done = head + 4 * words;
    if (lane < head) sum += row[lane];
    if (done + lane < K) sum += row[done + lane];
    sum = __reduce_add_sync(0xffffffffu, sum);
    if (lane == 0) rowsum[n] = scale[n] * (float)sum;
}

cudaError_t launch_q8_rowsum(const int8_t *w, long long ld, int N, int K, const float *scale, float *rowsum,
                             cudaStream_t st) {
    k_q8_rowsum<<<(N + 7) / 8, 256, 0, st>>>(w, ld, N, K, scale, rowsum);
    return cudaGetLastError();
}

// 16 codes from any address. Aligned ones take one load; others the two aligned
// 16-byte words that hold them, shifted together (the first may begin up to 15
// bytes before the codes: in the same word as a code, so in the same allocation).
template <bool ALIGNED>
__device__ __forceinline__ uint4 load_codes(const int8_t *p) {
    if constexpr (ALIGNED) {
        return __ldg(reinterpret_cast<const uint4 *>(p));
    } else {
        const int r = (int)(reinterpret_cast<uintptr_t>(p) & 15), shift = 8 * (r & 3);
        const uint4 *word = reinterpret_cast<const uint4 *>(p - r);
        const uint4 u = __ldg(word), n = __ldg(word + 1);
        const bool two = r & 8, one = r & 4;
        const uint32_t w0 = two ? u.z : u.x, w1 = two ? u.w : u.y, w2 = two ? n.x : u.z, w3 = two ? n.y : u.w,
                       w4 = two ? n.z : n.x, w5 = two ? n.w : n.y;
        const uint32_t x0 = one ? w1 : w0, x1 = one ? w2 : w1, x2 = one ? w3 : w2, x3 = one ? w4 : w3,
                       x4 = one ? w5 : w4;
        return make_uint4(__funnelshift_r(x0, x1, shift), __funnelshift_r(x1, x2, shift),
                          __funnelshift_r(x2, x3, shift), __funnelshift_r(x3, x4, shift));
    }
}
// the same near a row's end: zeros beyond `left` (which may be negative); words
// that would pass the matrix's end are read by bytes
template <bool ALIGNED>
__device__ __noinline__ uint4 load_codes(const int8_t *p, int left, const int8_t *end) {
    uint32_t v[4] = {0, 0, 0, 0};
    if (left > 0) {
        if (p + (ALIGNED ? 16 : 32) <= end) {
            const uint4 u = load_codes<ALIGNED>(p);
            v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int keep = left - 4 * i;
                v[i] = keep <= 0 ? 0u : (keep < 4 ? v[i] & ((1u << (8 * keep)) - 1u) : v[i]);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < 16 && i < left; ++i) {
                const uint32_t byte = (uint32_t)(unsigned char)p[i] << (8 * (i & 3));
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] |= (i >> 2) == j ? byte : 0u;
            }
        }
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}
// the end of a matrix of codes
__host__ __device__ __forceinline__ const int8_t *matrix_end(const int8_t *p, int rows, int cols, long long ld) {
    return p + (long long)(rows - 1) * ld + cols;
}

__device__ __forceinline__ void store_out(const Q8Out &o, long long t, long long n, float y) {
    const long long at = t * o.ld_t + n * o.ld_n;
    if (o.type == DSTD_TYPE_F32) ((float *)o.p)[at] = y;
    else if (o.type == DSTD_TYPE_BF16) ((__nv_bfloat16 *)o.p)[at] = __float2bfloat16_rn(y);
    else ((__half *)o.p)[at] = __float2half_rn(y);
}

// four codes (one word) to two fp16 pairs: 1024 + (code + 128) as fp16 bits
// (0x6400 | byte), minus 1152
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = __half2half2(__ushort_as_half(0x6480));
    uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hsub2(*reinterpret_cast<__half2 *>(&a), off), y = __hsub2(*reinterpret_cast<__half2 *>(&b), off);
    lo = *reinterpret_cast<const uint32_t *>(&x);
    hi = *reinterpret_cast<const uint32_t *>(&y);
}

// ---------------------------------------------------------------------------
// Product for few tokens or small sizes: one launch, the weights from memory
// straight into registers. 8-bit dot instructions run at a fraction of their
// usual rate on this part (dp4a: about 70 products a cycle and SM, which made 8
// tokens take twice as long as reading the weights), so the codes become fp16
// here too and go through mma.sync (16 channels x 8 tokens x 16 codes, fp32
// sums, exact up to 1024 codes as on the big path): at these sizes the
// products are few and the point is to spend nothing between memory and the
// tensor core. Any order of K will do as long as both operands have the same, so a
// lane takes 16 consecutive codes of its rows, one load each, as its share of
// four instructions.
// A block has 16 channels and 8 NT tokens; its warps (1 to 8) share K in blocks
// of 128 codes (whole 128-byte lines): as many as fit the GPU in one round of
// blocks, so that there are loads enough under way and no second, half-empty round.
// Memory bounds it: 8 tokens x 16384 x 16384 in 47 us, 5.7 TB/s of weights (two
// blocks' loads under way per warp took registers from other warps: 57 us). Small
// layers are bound by the launch: 16 tokens x 784 x 800 in about 2.5 us.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int i) {
    return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w));
}

// warps on an SM, as the registers allow
template <int NT>
constexpr int few_resident() { return NT == 1 ? 32 : (NT == 2 ? 24 : 16); }

template <int NT, bool ALIGNED>
__global__ void __launch_bounds__(256, few_resident<NT>() / 8) k_q8_few(const Q8Args a, const int tiles_t) {
    __shared__ int s_sum[8][4 * NT][32];
    const int part = threadIdx.x >> 5, wpk = blockDim.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int t0 = (int)(blockIdx.x % tiles_t) * (8 * NT);
    const long long n0 = (long long)(blockIdx.x / tiles_t) * 16;
    wait_launch_before();
    // rows and tokens beyond the end repeat the last (their results are not stored)
    const int8_t *row0 = a.w + min(n0 + g, (long long)a.N - 1) * a.ld_w + 16 * q;
    const int8_t *row1 = a.w + min(n0 + g + 8, (long long)a.N - 1) * a.ld_w + 16 * q;
    const int8_t *tok[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) tok[j] = a.x + (long long)min(t0 + 8 * j + g, a.T - 1) * a.ld_x + 16 * q;
    const int8_t *w_end = matrix_end(a.w, a.N, a.K, a.ld_w), *x_end = matrix_end(a.x, a.T, a.K, a.ld_x);
    float c[NT][4] = {};
    int sum[NT][4] = {};
    // blocks whose loads need no care, for any row
    const int blocks = (a.K + 127) / 128, whole = ALIGNED ? a.K / 128 : (a.K < 16 ? 0 : (a.K - 16) / 128);
    int run = 0;
    for (int b = part; b < blocks; b += wpk) {
        uint4 w0[2], w1[2], x[2][NT];
        if (b < whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = b * 128 + h * 64;
                w0[h] = load_codes<ALIGNED>(row0 + k);
                w1[h] = load_codes<ALIGNED>(row1 + k);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < NT; ++j) x[h][j] = load_codes<ALIGNED>(tok[j] + b * 128 + h * 64);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = b * 128 + h * 64, left = a.K - k - 16 * q;
                w0[h] = load_codes<ALIGNED>(row0 + k, left, w_end);
                w1[h] = load_codes<ALIGNED>(row1 + k, left, w_end);
#pragma unroll
                for (int j = 0; j < NT; ++j) x[h][j] = load_codes<ALIGNED>(tok[j] + k, left, x_end);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t a0, a1, a2, a3;
                codes_to_half(word_of(w0[h], i), a0, a2);
                codes_to_half(word_of(w1[h], i), a1, a3);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    uint32_t b0, b1;
                    codes_to_half(word_of(x[h][j], i), b0, b1);
                    mma_16x8x16(c[j], a0, a1, a2, a3, b0, b1);
                }
            }
        if (++run == 8) {  // 1024 codes
            run = 0;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sum[j][i] += __float2int_rn(c[j][i]);
                    c[j][i] = 0.f;
                }
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[j][i] += __float2int_rn(c[j][i]);
    if (wpk > 1) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) s_sum[part][4 * j + i][lane] = sum[j][i];
        __syncthreads();
        if (part != 0) return;
        for (int v = 1; v < wpk; ++v)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[j][i] += s_sum[v][4 * j + i][lane];
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + 8 * j + 2 * q + (i & 1);
            const long long n = n0 + g + (i >> 1) * 8;
            if (t >= a.T || n >= a.N) continue;
            const float first = a.swapped ? a.w_scale[n] : a.x_scale[t], second = a.swapped ? a.x_scale[t] : a.w_scale[n];
            store_out(a.out, t, n, ((float)sum[j][i] * first) * second);
        }
}

struct FewPlan {
    int tiles_t, wpk, blocks;  // blocks of 128 along K
    long long grid;
    int rounds;
};
template <int NT>
FewPlan few_plan(int T, int N, int K) {
    FewPlan p{(T + 8 * NT - 1) / (8 * NT), 1, (K + 127) / 128, 0, 0};
    constexpr int warps = 152 * few_resident<NT>();
    p.grid = ((long long)N + 15) / 16 * p.tiles_t;
    while (p.wpk < 8 && p.grid * p.wpk * 2 <= warps && p.blocks > p.wpk) p.wpk *= 2;
    p.rounds = (int)std::min<long long>((p.grid * p.wpk + warps - 1) / warps, 1 << 20);
    return p;
}

template <int NT>
cudaError_t launch_few(const Q8Args &a, bool aligned, cudaStream_t st) {
    const FewPlan p = few_plan<NT>(a.T, a.N, a.K);
    if (p.grid > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_dependent(aligned ? k_q8_few<NT, true> : k_q8_few<NT, false>, (unsigned)p.grid, 32 * p.wpk, st, a,
                            p.tiles_t);
}

// ---------------------------------------------------------------------------
// Product on tensor cores. sm_103a has no fast 8-bit integer rate, but a code
// is exact in fp16 and so is a product of two in fp32, so the 16-bit tensor
// cores give the whole-number sum as long as it stays within 2^24, which 1024
// products of at most 2^14 do. Computed transposed, D[n, t]: the weights are
// the M operand. They stay 8 bits wide until they are in the SM (TMA tiles of
// 128 rows x 128 codes): with both operands in 16 bits the widest tile would take
// in 83 bytes a cycle and SM, where 16-bit tiles were measured to get about 57
// from L2. Eight warps turn them into fp16 pairs in TMEM, from where the tensor
// core reads them, two groups of four taking blocks in turn (one group's chain of
// load, convert, store and signal was longer than the block's MMAs). The tokens,
// which every tile row shares, are turned into fp16 once per call and read
// through TMA.
// A pair of SMs works on 256 channels x NT tokens: each holds 128 channels and
// half of the tokens' operand. Two accumulators of NT columns alternate every
// 1024 codes of K; eight epilogue warps take the full one into 32-bit integers
// in registers while the other fills.
// Whole rounds of tiles go one to a pair. The tiles left over (all of them, when
// there are few) are cut along K into equal shares for all pairs, where that
// is shorter than one more round: a pair adds its integer sums into the
// workspace with atomics, and the last one of a part (a ticket counts them)
// stores the result. Whole-number sums do not depend on the order.
// The tensor pipe bounds large products: 4096 x 16384 x 16384 in 1.09 ms, 2.0
// PFLOP/s, with the preparation 1.17 (cuBLAS bf16 burst: 1.91 PFLOP/s); 4096^3 in
// 97 us as a call with cold caches (the pipe is active 82% of the time at 4096 x
// 4096 x 8192; the rest are the pipeline's ends and the last round). Small ones are bound by the pipeline's ends, about 8 us from launch to
// the last store.
// ---------------------------------------------------------------------------
__device__ unsigned int g_status_q8 = 0;

cudaError_t q8_status_read(unsigned int *out, int clear) {
    cudaError_t e = cudaMemcpyFromSymbol(out, g_status_q8, sizeof(unsigned int));
    if (e != cudaSuccess || !clear) return e;
    unsigned int z = 0;
    return cudaMemcpyToSymbol(g_status_q8, &z, sizeof(z));
}

namespace {
using namespace tc;

constexpr int KB = 128;          // codes of K per stage
constexpr int FOLD = 1024 / KB;  // stages per accumulator
constexpr int W_BYTES = 128 * KB;
constexpr int CONV_WARPS = 8, EPI_WARPS = 8, TC_THREADS = 32 * (CONV_WARPS + EPI_WARPS + 4);
// registers a thread of each role, where the kernel splits them (whole warpgroups)
constexpr int REGS_CONV = 72, REGS_EPI = 136, REGS_REST = 48;
constexpr int REGS_SUM = 32 * (CONV_WARPS * REGS_CONV + EPI_WARPS * REGS_EPI + 4 * REGS_REST);

template <int NT>
struct Q8Cfg {
    static constexpr int X_BYTES = NT / 2 * 128;  // 64 fp16 of K for this SM's half of the tokens
    static constexpr int STAGE = W_BYTES + 2 * X_BYTES;
    static constexpr int STAGES = 200 * 1024 / STAGE > 8 ? 8 : 200 * 1024 / STAGE;
    static constexpr int SMEM = STAGES * STAGE + 1024 + 512;
    static constexpr int A_STAGES = (512 - 2 * NT) / 64 > 4 ? 4 : (512 - 2 * NT) / 64;  // of 128 codes, 64 columns each
    static constexpr int A_COL = 2 * NT;
    static constexpr int COLS = NT / 2;                   // columns of one epilogue warp
    // the epilogue's sums do not fit an even share of the registers: the other warps give some of theirs
    // (REGS_SUM = 59392, of the 640 x 96 = 61440 that the block is launched with; checked before the launch)
    static constexpr bool SPLIT_REGS = NT > 64;
    static constexpr int CH = COLS == 32 ? 32 : 16;  // columns per TMEM read
};

struct Q8Plan {
    int nt, tiles_n, tiles_t, blocks;  // blocks of 128 along K
    int whole;                         // tiles computed in one piece
    int share;                         // blocks of one pair's share of the others (0: none are left)
    double cycles;                     // estimate
};

struct Q8Tc {
    int T, N, K;
    bool w_copied, swapped;
    Q8Plan p;
    const float *x_scale, *w_scale;
    Q8Out out;
    int *partial;      // [tile][16 warps][COLS][32] of the tiles that are cut, zeroed before the launch
    unsigned *ticket;  // [tile][16 warps], too
};

// What a pair works on, in order: tile and blocks [b0, b1) of K, cut into `parts` shares among pairs.
struct Work {
    int tile, b0, b1, parts;
    int i, step, g, end;
    __device__ __forceinline__ Work(const Q8Plan &p, int cid, int ncl) : i(cid), step(ncl) {
        const long long rest = (long long)(p.tiles_n * p.tiles_t - p.whole) * p.blocks;
        const long long lo = (long long)cid * p.share, hi = lo + p.share;
        g = (int)(lo < rest ? lo : rest);
        end = (int)(hi < rest ? hi : rest);
    }
    __device__ __forceinline__ bool next(const Q8Plan &p) {
        if (i < p.whole) {
            tile = i;
            b0 = 0;
            b1 = p.blocks;
            parts = 1;
            i += step;
            return true;
        }
        if (g >= end) return false;
        const int r = g / p.blocks;
        tile = p.whole + r;
        b0 = g - r * p.blocks;
        b1 = min(p.blocks, b0 + end - g);
        parts = (r * p.blocks + p.blocks - 1) / p.share - r * p.blocks / p.share + 1;
        g += b1 - b0;
        return true;
    }
};

// tiles are taken in groups of 8 token tiles, so that the pairs at work at one
// time share both operands in L2
__device__ __forceinline__ void tile_of(int i, int tiles_n, int tiles_t, int &tn, int &tt) {
    const int per_group = 8 * tiles_n;
    const int group = i / per_group, r = i - group * per_group;
    const int left = tiles_t - group * 8, wide = left < 8 ? left : 8;
    tn = r / wide;
    tt = group * 8 + r - tn * wide;
}

template <int CH>
__device__ __forceinline__ void tmem_ld(uint32_t addr, float (&v)[CH]) {
    if constexpr (CH == 32) tmem_ld32(addr, v);
    else tmem_ld16(addr, v);
}

__device__ __forceinline__ void q8_timeout() { atomicOr(&g_status_q8, STATUS_TIMEOUT); }

// column c of this lane's channel: the token's scale is held by lane c % 32, and
// multiplied first (the lane's own, where the lanes hold tokens)
template <int COLS>
__device__ __forceinline__ float scaled(const int (&sum)[COLS], const float (&xs)[(COLS + 31) / 32], float ws,
                                        bool swapped, int c) {
    const float x = __shfl_sync(0xffffffffu, xs[c / 32], c % 32);
    return ((float)sum[c] * (swapped ? ws : x)) * (swapped ? x : ws);
}
// a warp's lanes hold neighbouring channels: each column is one row segment
template <class O, int COLS>
__device__ __forceinline__ void store_columns(O *dst, long long ld, const int (&sum)[COLS],
                                              const float (&xs)[(COLS + 31) / 32], float ws, bool swapped, int left) {
#pragma unroll
    for (int c = 0; c < COLS; ++c, dst += ld) {
        const float y = scaled<COLS>(sum, xs, ws, swapped, c);
        if (c < left) *dst = round_out<O>(y);
    }
}
// the columns lie next to each other: 16 bytes at a time where the row allows it
template <class O, int COLS>
__device__ __forceinline__ void store_row(O *dst, const int (&sum)[COLS], const float (&xs)[(COLS + 31) / 32],
                                          float ws, bool swapped, int left) {
    constexpr int P = 16 / sizeof(O);
    const bool vec = (reinterpret_cast<uintptr_t>(dst) & 15) == 0;
#pragma unroll
    for (int c = 0; c < COLS; c += P) {
        alignas(16) O y[P];
#pragma unroll
        for (int u = 0; u < P; ++u) y[u] = round_out<O>(scaled<COLS>(sum, xs, ws, swapped, c + u));
        if (vec && c + P <= left) {
            *reinterpret_cast<uint4 *>(dst + c) = *reinterpret_cast<const uint4 *>(y);
        } else {
#pragma unroll
            for (int u = 0; u < P; ++u)
                if (c + u < left) dst[c + u] = y[u];
        }
    }
}
template <class O, int COLS>
__device__ __forceinline__ void store_tile(const Q8Out &o, long long at, const int (&sum)[COLS],
                                           const float (&xs)[(COLS + 31) / 32], float ws, bool swapped, int left) {
    if (o.ld_t == 1) store_row<O, COLS>((O *)o.p + at, sum, xs, ws, swapped, left);
    else store_columns<O, COLS>((O *)o.p + at, o.ld_t, sum, xs, ws, swapped, left);
}

template <int NT>
__global__ void __launch_bounds__(TC_THREADS, 1)
    k_q8_tc(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const Q8Tc a) {
    using C = Q8Cfg<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t *w_full = reinterpret_cast<uint64_t *>(smem + C::STAGES * C::STAGE);  // own weights have landed
    // (leader) both halves of the tokens have, and both SMs' fp16 weights are in TMEM
    uint64_t *ready = w_full + C::STAGES;
    uint64_t *empty = ready + C::STAGES;          // the pair's MMAs have read the stage
    uint64_t *acc_full = empty + C::STAGES;       // [2]
    uint64_t *acc_empty = acc_full + 2;           // [2] (leader)
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(acc_empty + 2);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank();
    Work wk(a.p, (int)cluster_id_x(), (int)cluster_count_x());

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&w_full[s], 1);
            mbar_init(&ready[s], 1 + 2 * CONV_WARPS / 2);  // one group of each SM takes a block
            mbar_init(&empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&acc_full[s], 1);
            mbar_init(&acc_empty[s], 2 * EPI_WARPS);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == CONV_WARPS + EPI_WARPS + 1) tmem_alloc_pair(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both SMs' barriers exist before any remote signal
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if constexpr (C::SPLIT_REGS) {
        if (warp >= CONV_WARPS + EPI_WARPS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_REST));
    }
    if (warp == CONV_WARPS + EPI_WARPS || warp == CONV_WARPS + EPI_WARPS + 2) {
        // TMA producers, of this SM's weights and of its half of the tokens. The weights, unless they were copied into
        // place, do not wait for the launch before.
        const bool tokens = warp == CONV_WARPS + EPI_WARPS + 2;
        if (tokens || a.w_copied) wait_launch_before();
        const uint32_t ready0 = mapa_rank(smem_u32(&ready[0]), 0);
        uint32_t it = 0;
        bool ok = true;
        while (ok && wk.next(a.p)) {
            int tn, tt;
            tile_of(wk.tile, a.p.tiles_n, a.p.tiles_t, tn, tt);
            const int n0 = tn * 256 + rank * 128, t0 = tt * NT + rank * (NT / 2);
            for (int b = wk.b0; b < wk.b1; ++b, ++it) {
                const int s = it % C::STAGES;
                ok = mbar_wait_cycles(&empty[s], ((it / C::STAGES) & 1u) ^ 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t st = smem_u32(smem + s * C::STAGE);
                if (elect_one()) {
                    if (!tokens) {
                        mbar_expect_tx(&w_full[s], (uint32_t)W_BYTES);
                        tma_load_2d(st, &map_w, &w_full[s], b * KB, n0);
                    } else {
                        const bool two = b * KB + 64 < a.K;  // a second half of the stage to read
                        if (rank == 0) mbar_expect_tx(&ready[s], (uint32_t)((two ? 4 : 2) * C::X_BYTES));
                        const uint32_t rb = ready0 + (uint32_t)(s * sizeof(uint64_t));
                        tma_load_2d_pair(st + W_BYTES, &map_x, rb, b * KB, t0);
                        if (two) tma_load_2d_pair(st + W_BYTES + C::X_BYTES, &map_x, rb, b * KB + 64, t0);
                    }
                }
                __syncwarp();
            }
        }
        // every stage released: no copy is in flight and no commit targets this SM's stages afterwards
        for (int i = 0; i < C::STAGES && ok; ++i, ++it)
            ok = mbar_wait_cycles(&empty[it % C::STAGES], ((it / C::STAGES) & 1u) ^ 1u);
        if (!ok) q8_timeout();
        __syncwarp();
    } else if (warp == CONV_WARPS + EPI_WARPS + 1) {
        if (rank == 0) {
            // MMA issuer of the pair
            constexpr uint32_t idesc = idesc_16bit(256, NT, true);
            uint32_t it = 0, j = 0;
            bool ok = true;
            while (ok && wk.next(a.p)) {
                int in_chunk = 0;
                for (int b = wk.b0; b < wk.b1; ++b, ++it) {
                    const int s = it % C::STAGES, as = it % C::A_STAGES;
                    ok = (in_chunk > 0 || mbar_wait_cycles(&acc_empty[j & 1u], ((j >> 1) & 1u) ^ 1u)) &&
                         mbar_wait_cycles(&ready[s], (it / C::STAGES) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t acc = tmem + (j & 1u) * NT, at = tmem + C::A_COL + as * 64;
                    const uint64_t xd = sdesc_sw128(smem_u32(smem + s * C::STAGE + W_BYTES));
                    const bool two = b * KB + 64 < a.K, last = in_chunk + 1 == FOLD || b + 1 == wk.b1;
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            mma_pair_ts(acc, at + kk * 8, xd + kk * 2, idesc, (in_chunk > 0 || kk > 0) ? 1u : 0u);
                        if (two) {
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                mma_pair_ts(acc, at + 32 + kk * 8, xd + C::X_BYTES / 16 + kk * 2, idesc, 1u);
                        }
                        mma_commit_pair(&empty[s]);
                        if (last) mma_commit_pair(&acc_full[j & 1u]);
                    }
                    __syncwarp();
                    in_chunk = last ? 0 : in_chunk + 1;
                    j += last ? 1 : 0;
                }
            }
            if (!ok) q8_timeout();
        }
        __syncwarp();
    } else if (warp < CONV_WARPS) {
        // weights to fp16: a thread takes one row; two groups of four warps take the blocks in turn
        if constexpr (C::SPLIT_REGS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_CONV));
        const int group = warp >> 2, row = (warp & 3) * 32 + lane, swz = row & 7;
        const uint32_t ready0 = mapa_rank(smem_u32(&ready[0]), 0);
        const uint32_t tbase = tmem + ((uint32_t)((warp & 3) * 32) << 16) + C::A_COL;
        uint32_t it = 0;
        bool ok = true;
        while (ok && wk.next(a.p)) {
            for (int b = wk.b0; b < wk.b1; ++b, ++it) {
                if ((it & 1u) != (uint32_t)group) continue;
                const int s = it % C::STAGES, as = it % C::A_STAGES;
                ok = mbar_wait_cycles(&w_full[s], (it / C::STAGES) & 1u);
                // the block that used these columns has been multiplied
                if (ok && it >= C::A_STAGES) {
                    const uint32_t old = it - C::A_STAGES;
                    ok = mbar_wait_cycles(&empty[old % C::STAGES], (old / C::STAGES) & 1u);
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint8_t *src = smem + s * C::STAGE + row * 128;
                const int halves = b * KB + 64 < a.K ? 2 : 1;
                for (int h = 0; h < halves; ++h) {
                    uint32_t r[32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(src + (((h * 4 + c) ^ swz) << 4));
                        codes_to_half(v.x, r[8 * c], r[8 * c + 1]);
                        codes_to_half(v.y, r[8 * c + 2], r[8 * c + 3]);
                        codes_to_half(v.z, r[8 * c + 4], r[8 * c + 5]);
                        codes_to_half(v.w, r[8 * c + 6], r[8 * c + 7]);
                    }
                    tmem_st32(tbase + as * 64 + h * 32, r);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_pair(ready0 + (uint32_t)(s * sizeof(uint64_t)));
            }
        }
        if (!ok) q8_timeout();
    } else if (warp < CONV_WARPS + EPI_WARPS) {
        // epilogue: rows of quarter (warp & 3), half of the columns
        if constexpr (C::SPLIT_REGS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_EPI));
        const int ew = warp - CONV_WARPS, quarter = warp & 3, group = ew >> 2;
        const uint32_t tbase = tmem + ((uint32_t)(quarter * 32) << 16) + group * C::COLS;
        const uint32_t acc_empty0 = mapa_rank(smem_u32(&acc_empty[0]), 0);
        uint32_t j = 0;
        wait_launch_before();  // sums and tickets have been set to zero
        while (wk.next(a.p)) {
            int tn, tt;
            tile_of(wk.tile, a.p.tiles_n, a.p.tiles_t, tn, tt);
            const int n = tn * 256 + rank * 128 + quarter * 32 + lane, t0 = tt * NT + group * C::COLS;
            // the scales, on their way while the tile is computed: token t0 + c is held by lane c % 32
            const float ws = n < a.N ? a.w_scale[n] : 0.f;
            float xs[(C::COLS + 31) / 32];
#pragma unroll
            for (int c = 0; c < (C::COLS + 31) / 32; ++c)
                xs[c] = t0 + 32 * c + lane < a.T ? a.x_scale[t0 + 32 * c + lane] : 0.f;
            int sum[C::COLS];
#pragma unroll
            for (int c = 0; c < C::COLS; ++c) sum[c] = 0;
            bool ok = true;
            for (int b = wk.b0; b < wk.b1; b += FOLD, ++j) {
                if (!mbar_wait_cycles(&acc_full[j & 1u], (j >> 1) & 1u)) {
                    q8_timeout();
                    ok = false;
                    break;
                }
                __syncwarp();
                tc_fence_after();
#pragma unroll
                for (int c0 = 0; c0 < C::COLS; c0 += C::CH) {
                    float v[C::CH];
                    tmem_ld<C::CH>(tbase + (j & 1u) * NT + c0, v);
#pragma unroll
                    for (int c = 0; c < C::CH; ++c) sum[c0 + c] += __float2int_rn(v[c]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_pair(acc_empty0 + (uint32_t)((j & 1u) * sizeof(uint64_t)));
            }
            if (!ok) break;
            if (wk.parts > 1) {
                const int cut = (wk.tile - a.p.whole) * 16 + rank * EPI_WARPS + ew;
                int *all = a.partial + (long long)cut * C::COLS * 32 + lane;
#pragma unroll
                for (int c = 0; c < C::COLS; ++c) atomicAdd(all + c * 32, sum[c]);
                __threadfence();
                __syncwarp();
                unsigned drawn = 0;
                if (lane == 0) drawn = atomicAdd(&a.ticket[cut], 1u);
                drawn = __shfl_sync(0xffffffffu, drawn, 0);
                if (drawn != (unsigned)(wk.parts - 1)) continue;
                __threadfence();
#pragma unroll
                for (int c = 0; c < C::COLS; ++c) sum[c] = __ldcg(all + c * 32);
            }
            const int left = n < a.N ? a.T - t0 : 0;  // this lane's columns that exist
            const long long at = (long long)t0 * a.out.ld_t + (long long)n * a.out.ld_n;
            if (a.out.type == DSTD_TYPE_F32) store_tile<float, C::COLS>(a.out, at, sum, xs, ws, a.swapped, left);
            else if (a.out.type == DSTD_TYPE_BF16)
                store_tile<__nv_bfloat16, C::COLS>(a.out, at, sum, xs, ws, a.swapped, left);
            else store_tile<__half, C::COLS>(a.out, at, sum, xs, ws, a.swapped, left);
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both SMs are done with TMEM, every remote arrive has landed
    if (warp == CONV_WARPS + EPI_WARPS + 1) tmem_dealloc_pair(tmem, 512);
}

// What the tensor-core launch needs first, 16 codes a thread: the tokens as fp16
// rows [T, ld], the weights copied to rows [N, ld_wc] where theirs are not
// aligned (wc not null), and zeros for the sums and tickets of the tiles that are cut.
struct PrepArgs {
    const int8_t *x, *w;
    long long ld_x, ld_w;
    int T, N, K;
    bool x_aligned;
    __half *xh;
    int ld;
    int8_t *wc;
    int ld_wc;
    uint4 *zero;
    long long x_threads, w_threads, zeros;
};

__device__ __forceinline__ long long quotient(long long i, int d) {
    return i < (1ll << 31) ? (long long)((unsigned)i / (unsigned)d) : i / d;
}

__global__ void __launch_bounds__(256) k_q8_prep(const PrepArgs a) {
    wait_launch_before();
    let_next_launch();
    long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i < a.x_threads) {
        const int chunks = (a.ld + 15) / 16;
        const long long t = quotient(i, chunks);
        const int k = (int)(i - t * chunks) * 16;
        const int8_t *p = a.x + t * a.ld_x + k;
        const int8_t *end = matrix_end(a.x, a.T, a.K, a.ld_x);
        const uint4 v = k + 32 <= a.K ? (a.x_aligned ? load_codes<true>(p) : load_codes<false>(p))
                        : a.x_aligned ? load_codes<true>(p, a.K - k, end)
                                      : load_codes<false>(p, a.K - k, end);
        uint4 lo, hi;
        codes_to_half(v.x, lo.x, lo.y);
        codes_to_half(v.y, lo.z, lo.w);
        codes_to_half(v.z, hi.x, hi.y);
        codes_to_half(v.w, hi.z, hi.w);
        __half *y = a.xh + t * a.ld + k;
        *reinterpret_cast<uint4 *>(y) = lo;
        if (k + 8 < a.ld) *reinterpret_cast<uint4 *>(y + 8) = hi;
        return;
    }
    i -= a.x_threads;
    if (i < a.w_threads) {
        const int chunks = a.ld_wc / 16;
        const long long n = quotient(i, chunks);
        const int k = (int)(i - n * chunks) * 16;
        const int8_t *p = a.w + n * a.ld_w + k;
        *reinterpret_cast<uint4 *>(a.wc + n * a.ld_wc + k) =
            k + 32 <= a.K ? load_codes<false>(p) : load_codes<false>(p, a.K - k, matrix_end(a.w, a.N, a.K, a.ld_w));
        return;
    }
    i -= a.w_threads;
    if (i < a.zeros) a.zero[i] = make_uint4(0, 0, 0, 0);
}

constexpr int kPairs = 76;  // SM pairs of the GPU, for planning

// fewer tokens than this never go to the big form
constexpr int kTcMinTokens = 9;

// Time of one block of 128 codes in a pair's pipeline, in cycles, measured with
// 4096 tokens, 16384 inputs and channels (the MMAs alone: 4 nt). The conversion
// and the issue of the MMAs hold it at about 700 up to 128 tokens a tile; 160
// reach the tensor pipe's rate (that product's call in 1.17 ms); with 192 only two
// blocks fit beside the accumulators in TMEM (1.19 ms).
struct TileCost {
    int nt, block;
};
constexpr TileCost kTiles[] = {{32, 680}, {64, 680}, {96, 770}, {128, 800}, {160, 830}, {192, 1010}};

// `pairs`: SM pairs at work at a time. Whole rounds of tiles, then the rest
// either as one more round or in shares along K; the tile width by the sum.
Q8Plan q8_plan(int T, int N, int K, int pairs) {
    Q8Plan best{};
    double best_cost = 0;
    for (const TileCost &tc : kTiles) {
        Q8Plan p{};
        p.nt = tc.nt;
        p.tiles_n = (N + 255) / 256;
        p.tiles_t = (T + tc.nt - 1) / tc.nt;
        p.blocks = (K + KB - 1) / KB;
        const int tiles = p.tiles_n * p.tiles_t, rest = tiles % pairs;
        p.whole = tiles;
        const double tile = (double)p.blocks * tc.block;
        double cost = (tiles / pairs) * tile + 12.0 * tc.nt;
        if (rest > 0) {
            // a share of at least two blocks; adding up and the wait for the last part cost about 6000 + 30 nt
            // cycles
            const long long blocks = (long long)rest * p.blocks;
            const int share = (int)std::max((blocks + pairs - 1) / pairs, 2ll);
            const double cut = (double)share * tc.block + 6000 + 30.0 * tc.nt;
            if (cut < tile) {
                p.whole = tiles - rest;
                p.share = share;
            }
            cost += std::min(cut, tile);
        }
        if (best.nt == 0 || cost < best_cost) {
            best_cost = cost;
            best = p;
            best.cycles = cost;
        }
    }
    return best;
}

// Scratch of the tensor-core form: the fp16 tokens, a copy of the weights
// (used where their rows are not aligned), then tickets and sums of the tiles
// that are cut (fewer than kPairs, of at most 192 tokens, whatever the plan).
struct Q8Scratch {
    __half *x;
    int8_t *w;
    unsigned *ticket;
    int *partial;
    int ld, ld_w;
    long long zeros;  // 16-byte words from ticket on
    size_t bytes;
};
Q8Scratch q8_scratch(void *base, int T, int N, int K, bool copy, long long cut, int nt) {
    Q8Scratch s{};
    char *b = static_cast<char *>(base);
    s.ld = (K + 7) / 8 * 8;
    s.ld_w = (K + 15) / 16 * 16;
    const size_t x = ((size_t)T * s.ld * 2 + 255) / 256 * 256, w = copy ? ((size_t)N * s.ld_w + 255) / 256 * 256 : 0;
    s.x = (__half *)b;
    s.w = (int8_t *)(b + x);
    s.ticket = (unsigned *)(b + x + w);
    s.partial = (int *)(b + x + w + cut * 64);
    s.zeros = (cut * 64 + cut * 1024 * nt) / 16;
    s.bytes = x + w + (size_t)cut * (64 + 1024 * nt);
    return s;
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                             const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                             CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// rows of 128-byte boxes, swizzled; beyond the matrix zeros are read
bool row_map(CUtensorMap *m, CUtensorMapDataType type, int bytes, const void *p, int rows, int cols, long long ld,
             int box_rows) {
    EncodeFn enc = reinterpret_cast<EncodeFn>(tensor_map_encoder());
    if (!enc) return false;
    const cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t stride[1] = {(cuuint64_t)ld * bytes};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / bytes), (cuuint32_t)box_rows};
    const cuuint32_t one[2] = {1, 1};
    return enc(m, type, 2, const_cast<void *>(p), dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool rows_aligned(const int8_t *p, long long ld) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)ld) & 15) == 0; }
bool w_rows_aligned(const Q8Args &a) { return rows_aligned(a.w, a.ld_w); }

template <int NT>
cudaLaunchConfig_t tc_config(cudaLaunchAttribute (&attr)[2]) {
    cudaLaunchConfig_t cfg = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cfg.blockDim = dim3(TC_THREADS);
    cfg.dynamicSmemBytes = Q8Cfg<NT>::SMEM;
    return cfg;
}

// Kernel attributes of a tile width: the grant of shared memory belongs to the
// device that is current. False on an error.
template <int NT>
bool tc_setup() {
    using C = Q8Cfg<NT>;
    static PerDevice done;
    return done.get([](int) {
        if (cudaFuncSetAttribute(k_q8_tc<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) != cudaSuccess)
            return 0;
        if (!C::SPLIT_REGS) return 1;
        // a split of more registers than the block has would wait forever
        cudaFuncAttributes at;
        if (cudaFuncGetAttributes(&at, k_q8_tc<NT>) != cudaSuccess) return 0;
        return at.numRegs * TC_THREADS >= REGS_SUM && at.numRegs >= REGS_CONV && at.numRegs <= REGS_EPI ? 1 : 0;
    }) != 0;
}

// SM pairs that can be at work at once (0: an error); every tile width takes a whole SM
int resident_pairs() {
    static PerDevice resident;
    return resident.get([](int) {
        cudaLaunchAttribute attr[2];
        cudaLaunchConfig_t cfg = tc_config<192>(attr);
        cfg.gridDim = dim3(2 * kPairs);
        cfg.numAttrs = 1;
        int n = 0;
        if (!tc_setup<192>() || cudaOccupancyMaxActiveClusters(&n, k_q8_tc<192>, &cfg) != cudaSuccess)
            return 0;
        return std::min(n, kPairs);
    });
}

template <int NT>
cudaError_t launch_tc(const Q8Args &q, const Q8Plan &p, const Q8Scratch &s, int pairs, cudaStream_t st) {
    if (!tc_setup<NT>()) return cudaErrorInvalidConfiguration;
    CUtensorMap map_w, map_x;
    const bool copied = !w_rows_aligned(q);
    if (!row_map(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, copied ? s.w : q.w, q.N, q.K, copied ? s.ld_w : q.ld_w, 128) ||
        !row_map(&map_x, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, s.x, q.T, q.K, s.ld, NT / 2))
        return cudaErrorInvalidValue;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = tc_config<NT>(attr);
    cfg.stream = st;
    cfg.gridDim = dim3(2 * (unsigned)(p.share ? pairs : std::min(p.whole, pairs)));
    const Q8Tc a{q.T, q.N, q.K, copied, q.swapped, p, q.x_scale, q.w_scale, q.out, s.partial, s.ticket};
    return cudaLaunchKernelEx(&cfg, k_q8_tc<NT>, map_w, map_x, a);
}

// Estimates in microseconds, without what any launch costs, fitted to times with
// cold caches. mma.sync: rounds of resident blocks, each warp passing `steps`
// blocks of 128 codes of K, or the weights' reading time. The big form: its plan,
// 4 us for the pipeline's ends and 2 for its second launch, the preparation's
// traffic (the tokens to 16 bits, a copy of weights whose rows are not aligned)
// and, where a lane's row goes out piece by piece, the stores. Measured with the
// other form beside it (us, with 6.5 of launch and events): 32 x 784 x 800 10.8
// and 12.9, 16 x 4096 x 4096 12.9 and 18.0, 64 x 4096 x 4096 23.1 and 19.1,
// 32 x 16384 x 16384 103 and 56, 256 x 3000 x 1000 (not aligned) 31 and 17.
double few_time(const Q8Args &a) {
    const int nt = a.T <= 8 ? 1 : (a.T <= 16 ? 2 : 4);
    const FewPlan f = nt == 1 ? few_plan<1>(a.T, a.N, a.K) : (nt == 2 ? few_plan<2>(a.T, a.N, a.K) : few_plan<4>(a.T, a.N, a.K));
    const bool aligned = rows_aligned(a.x, a.ld_x) && rows_aligned(a.w, a.ld_w);
    const double steps = (double)((f.blocks + f.wpk - 1) / f.wpk) * f.rounds;
    const double each = (nt == 1 ? 1.0 : (nt == 2 ? 1.1 : 1.5)) * (aligned ? 1.0 : 1.5);
    return 3.5 + std::max(steps * each, (double)a.N * a.K / 6.2e6) + (aligned ? 0.0 : 4.0);
}
double tc_time(const Q8Args &a, const Q8Plan &p) {
    const double prep = (3.0 * a.T + (w_rows_aligned(a) ? 0.0 : 2.0 * a.N)) * a.K / 6.0e6;
    const bool pieces = a.out.ld_t == 1, wide = pieces && a.out.ld_n % 8 == 0;
    const double stores = pieces ? (double)a.T * a.N / (152.0 * (wide ? 4 : 1)) : 0.0;
    return 6.0 + prep + (p.cycles + stores) / 1900.0;
}
// the same product with the sides exchanged
Q8Args exchanged(const Q8Args &a) {
    return Q8Args{a.w, a.x, a.ld_w, a.ld_x, a.w_scale, a.x_scale, a.N, a.T, a.K,
                  Q8Out{a.out.p, a.out.type, a.out.ld_n, a.out.ld_t}, !a.swapped};
}

cudaError_t run_few(const Q8Args &a, cudaStream_t st) {
    const bool aligned = rows_aligned(a.x, a.ld_x) && rows_aligned(a.w, a.ld_w);
    if (a.T <= 8) return launch_few<1>(a, aligned, st);
    if (a.T <= 16) return launch_few<2>(a, aligned, st);
    return launch_few<4>(a, aligned, st);
}

cudaError_t run_tc(const Q8Args &a, const Q8Plan &p, int pairs, void *workspace, cudaStream_t st) {
    const Q8Scratch s = q8_scratch(workspace, a.T, a.N, a.K, !w_rows_aligned(a),
                                   (long long)p.tiles_n * p.tiles_t - p.whole, p.nt);
    PrepArgs pa{a.x, a.w, a.ld_x, a.ld_w, a.T, a.N, a.K, rows_aligned(a.x, a.ld_x), s.x, s.ld, s.w, s.ld_w,
                (uint4 *)s.ticket, (long long)a.T * ((s.ld + 15) / 16),
                w_rows_aligned(a) ? 0 : (long long)a.N * (s.ld_w / 16), s.zeros};
    const long long blocks = (pa.x_threads + pa.w_threads + pa.zeros + 255) / 256;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    cudaError_t e = launch_dependent(k_q8_prep, (unsigned)blocks, 256, st, pa);
    if (e != cudaSuccess) return e;
    switch (p.nt) {
        case 32: return launch_tc<32>(a, p, s, pairs, st);
        case 64: return launch_tc<64>(a, p, s, pairs, st);
        case 96: return launch_tc<96>(a, p, s, pairs, st);
        case 128: return launch_tc<128>(a, p, s, pairs, st);
        case 160: return launch_tc<160>(a, p, s, pairs, st);
        default: return launch_tc<192>(a, p, s, pairs, st);
    }
}

}  // namespace

// The big form counts whole tiles of up to 256 rows of either side.
bool q8_sizes_ok(int T, int N) {
    constexpr int most = 0x7fffffff - 255;
    return T < kTcMinTokens || (T <= most && N <= most);
}

// Then no copy is made, whichever side is which.
bool q8_rows_aligned(const Q8Args &a) { return rows_aligned(a.x, a.ld_x) && rows_aligned(a.w, a.ld_w); }

// The sides are exchanged only where there are more tokens than channels.
size_t q8_workspace_bytes(int T, int N, int K, bool aligned) {
    if (T < kTcMinTokens || N < 1 || K < 1) return 256;
    const long long cut = std::min<long long>((long long)((N + 255) / 256) * ((T + 31) / 32), kPairs);
    const long long cut_exchanged = std::min<long long>((long long)((T + 255) / 256) * ((N + 31) / 32), kPairs);
    const size_t bytes = q8_scratch(nullptr, T, N, K, !aligned, cut, 192).bytes;
    return T > N ? std::max(bytes, q8_scratch(nullptr, N, T, K, !aligned, cut_exchanged, 192).bytes) : bytes;
}

// The big form computes 256 rows of one side by up to 192 of the other at a
// time, and reads the first in 8 bits; mma.sync streams one side past up to 32
// rows of the other. So which side is which is chosen with the form: with more
// tokens than channels they are exchanged where that is estimated to be faster
// (7561 tokens, 4181 inputs, 21 channels: 25 us instead of 42).
cudaError_t launch_q8_product(const Q8Args &a, void *workspace, int &launches, cudaStream_t st) {
    launches = 0;
    if (a.T == 0 || a.N == 0) return cudaSuccess;
    const int pairs = resident_pairs();
    if (pairs < 1) return cudaErrorInvalidConfiguration;
    const Q8Args b = exchanged(a);
    const bool may_exchange = a.T > a.N, may_tc = a.T >= kTcMinTokens && a.K >= 16;
    double best = few_time(a);
    int form = 0;  // 1: exchanged, 2: big
    Q8Plan plan{};
    if (may_exchange && few_time(b) < best) {
        best = few_time(b);
        form = 1;
    }
    for (int i = 0; may_tc && i < (may_exchange ? 2 : 1); ++i) {
        const Q8Args &c = i ? b : a;
        const Q8Plan p = q8_plan(c.T, c.N, c.K, pairs);
        if (tc_time(c, p) < best) {
            best = tc_time(c, p);
            form = 2 + i;
            plan = p;
        }
    }
    const Q8Args &c = form & 1 ? b : a;
    launches = form & 2 ? 2 : 1;
    return form & 2 ? run_tc(c, plan, pairs, workspace, st) : run_few(c, st);
}

}  // namespace dstd
