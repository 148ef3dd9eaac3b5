// 8-bit rows and their products: the row quantiser and
// y_tn = sx_t sw_n sum_k x_tk w_nk with the sum exact in whole numbers.
#include "dstd_internal.cuh"

#include <limits.h>

namespace dstd {

// ---------------------------------------------------------------------------
// Row quantiser. With a = max_k |x_k|:
//     scale = a / 127,  q_k = rint(x_k (127 (1 / a))),  value_k = q_k scale,
// each operation rounded to fp32 (three roundings move x 127 / a by less than
// 127 * 3 * 2^-24 code steps). 1 / a overflows for a below 2^-128; rows of
// very small a are multiplied by 2^64 first (exact), which gives the same codes. A row of zeros has scale 0; a row
// that holds an infinity or a NaN has scale NaN and codes 0, so that whatever
// is computed from it is NaN. The largest |x| is taken on the bit patterns:
// without the sign they order like the values, with infinities and NaN on top.
// ---------------------------------------------------------------------------
template <class T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }

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

template <class T>
__global__ void __launch_bounds__(256) k_quantize_rows(const T *__restrict__ x, int cols, long long ld_x, int8_t *q,
                                                       long long ld_q, float *scale, float *values,
                                                       long long ld_v) {
    __shared__ unsigned s_top[8];
    const long long r = blockIdx.x;
    const T *row = x + r * ld_x;
    unsigned top = 0;
    for (int k = threadIdx.x; k < cols; k += 256)
        top = max(top, __float_as_uint(to_f32<T>(row[k])) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, s_top[i]);
    const RowCode c = row_code(top);
    if (threadIdx.x == 0) scale[r] = c.scale;
    for (int k = threadIdx.x; k < cols; k += 256) {
        const int v = code_of(to_f32<T>(row[k]), c);
        q[r * ld_q + k] = (int8_t)v;
        if (values) values[r * ld_v + k] = (float)v * c.scale;
    }
}

cudaError_t launch_quantize_rows(const void *x, dstd_type type, int rows, int cols, long long ld_x, int8_t *q,
                                 long long ld_q, float *scale, float *values, long long ld_v, cudaStream_t st) {
    if (rows == 0) return cudaSuccess;
    if (type == DSTD_TYPE_F32)
        k_quantize_rows<float><<<rows, 256, 0, st>>>((const float *)x, cols, ld_x, q, ld_q, scale, values, ld_v);
    else if (type == DSTD_TYPE_BF16)
        k_quantize_rows<__nv_bfloat16>
            <<<rows, 256, 0, st>>>((const __nv_bfloat16 *)x, cols, ld_x, q, ld_q, scale, values, ld_v);
    else
        k_quantize_rows<__half><<<rows, 256, 0, st>>>((const __half *)x, cols, ld_x, q, ld_q, scale, values, ld_v);
    return cudaGetLastError();
}

// row sums of the weights' values: rowsum_n = scale_n sum_k q_nk (one warp per row)
__global__ void __launch_bounds__(256) k_q8_rowsum(const int8_t *__restrict__ w, long long ld, int N, int K,
                                                   const float *__restrict__ scale, float *rowsum) {
    const int n = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (n >= N) return;
    int sum = 0;
    for (int k = threadIdx.x & 31; k < K; k += 32) sum += w[(long long)n * ld + k];
    sum = __reduce_add_sync(0xffffffffu, sum);
    if ((threadIdx.x & 31) == 0) rowsum[n] = scale[n] * (float)sum;
}

cudaError_t launch_q8_rowsum(const int8_t *w, long long ld, int N, int K, const float *scale, float *rowsum,
                             cudaStream_t st) {
    k_q8_rowsum<<<(N + 7) / 8, 256, 0, st>>>(w, ld, N, K, scale, rowsum);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// Product, dot form: a warp holds R channels x TT tokens of 32-bit sums; its
// lanes split K in chunks of 16 codes (four dp4a each per pair).
// ---------------------------------------------------------------------------
__device__ __forceinline__ int4 load16(const int8_t *p, int left, bool aligned) {
    if (aligned && left >= 16) return *reinterpret_cast<const int4 *>(p);
    int v[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < left) v[i >> 2] |= (int)(unsigned char)p[i] << (8 * (i & 3));
    return make_int4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void store_out(const Q8Out &o, long long t, long long n, float y) {
    const long long at = t * o.ld_t + n * o.ld_n;
    if (o.type == DSTD_TYPE_F32) ((float *)o.p)[at] = y;
    else if (o.type == DSTD_TYPE_BF16) ((__nv_bfloat16 *)o.p)[at] = __float2bfloat16_rn(y);
    else ((__half *)o.p)[at] = __float2half_rn(y);
}

template <int TT, int R>
__global__ void __launch_bounds__(256) k_q8_dot(Q8Args a, bool aligned) {
    const int lane = threadIdx.x & 31;
    const long long n0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * R;
    const int t0 = blockIdx.y * TT;
    if (n0 >= a.N) return;
    int acc[R][TT] = {};
    for (int k = lane * 16; k < a.K; k += 512) {
        int4 w[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            w[r] = n0 + r < a.N ? load16(a.w + (n0 + r) * a.ld_w + k, a.K - k, aligned) : make_int4(0, 0, 0, 0);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            if (t0 + t >= a.T) break;
            const int4 x = load16(a.x + (long long)(t0 + t) * a.ld_x + k, a.K - k, aligned);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                acc[r][t] = __dp4a(x.x, w[r].x, acc[r][t]);
                acc[r][t] = __dp4a(x.y, w[r].y, acc[r][t]);
                acc[r][t] = __dp4a(x.z, w[r].z, acc[r][t]);
                acc[r][t] = __dp4a(x.w, w[r].w, acc[r][t]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int sum = __reduce_add_sync(0xffffffffu, acc[r][t]);
            if (lane == 0 && t0 + t < a.T && n0 + r < a.N)
                store_out(a.out, t0 + t, n0 + r, ((float)sum * a.x_scale[t0 + t]) * a.w_scale[n0 + r]);
        }
}

size_t q8_workspace_bytes(int T, int N, int K) {
    (void)T, (void)N, (void)K;
    return 256;
}

cudaError_t launch_q8_product(const Q8Args &a, void *workspace, cudaStream_t st) {
    (void)workspace;
    if (a.T == 0 || a.N == 0) return cudaSuccess;
    constexpr int TT = 8, R = 2;
    const bool aligned = ((reinterpret_cast<uintptr_t>(a.w) | reinterpret_cast<uintptr_t>(a.x) | (uintptr_t)a.ld_w |
                           (uintptr_t)a.ld_x) & 15) == 0;
    const int tt_max = 65535 * TT;  // tokens of one launch
    for (int t = 0; t < a.T; t += tt_max) {
        Q8Args b = a;
        b.T = a.T - t < tt_max ? a.T - t : tt_max;
        b.x += (long long)t * a.ld_x;
        b.x_scale += t;
        b.out.p = (char *)a.out.p + (long long)t * a.out.ld_t * (a.out.type == DSTD_TYPE_F32 ? 4 : 2);
        k_q8_dot<TT, R><<<dim3((a.N + 8 * R - 1) / (8 * R), (b.T + TT - 1) / TT), 256, 0, st>>>(b, aligned);
    }
    return cudaGetLastError();
}

}  // namespace dstd
