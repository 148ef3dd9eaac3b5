// 4-bit rows with a power of two for each block of 32 columns, and their
// products y_tn = sum_k x_tk w_nk.
//
// A row of codes is 16 bytes for each block (the even column in a byte's low
// half), zero beyond the last column. The exponents are bytes, in tiles of 128
// rows by 4 blocks of 512 bytes: the order in which the tensor cores take them.
#include "dstd_rows.cuh"
#include "dstd_tc_ptx.cuh"

#include <cuda_fp4.h>

#include <algorithm>

namespace dstd {

size_t mx4_scale_bytes(long long rows, int cols) {
    return (size_t)((rows + 127) / 128) * ((mx4_blocks(cols) + 3) / 4) * 512;
}

// ---------------------------------------------------------------------------
// A block's exponent is the least e >= -127 with max |x| <= 6 2^e, so that no
// code is beyond the largest, 6: with max |x| = 1.m 2^E that is E - 2, or E - 1 for 1.m > 1.5.
// x 2^-e is exact (or below the least code by far), so the codes are the nearest
// ones, ties to the even code, whatever the order of the work. A block that holds
// an infinity or a NaN has exponent byte 255, which stands for NaN, and codes 0.
// ---------------------------------------------------------------------------
struct BlockCode {
    uint32_t byte;  // e + 127
    float pre;      // 2^-e; 0 where the block is not finite
};
__device__ __forceinline__ BlockCode block_code(uint32_t top_bits) {
    if (top_bits >= 0x7f800000u) return BlockCode{255u, 0.f};
    const int byte = max(0, (int)(top_bits >> 23) - 2 + ((top_bits & 0x7fffffu) > 0x400000u ? 1 : 0));
    return BlockCode{(uint32_t)byte, __uint_as_float((uint32_t)(254 - byte) << 23)};
}
// 2^(byte - 127), NaN for 255
__device__ __forceinline__ float block_scale(uint32_t byte) {
    return byte == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(byte == 0u ? 0x400000u : byte << 23);
}
__device__ __forceinline__ uint32_t code_pair(float lo, float hi) {
    return (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(lo, hi), __NV_E2M1, cudaRoundNearest);
}
__device__ __forceinline__ float2 pair_values(uint32_t byte) {
    const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)byte, __NV_E2M1);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
// place of the exponent byte of row r, block b; ktiles tiles of 4 blocks to a row
__device__ __forceinline__ long long scale_at(long long r, int b, int ktiles) {
    return ((r >> 7) * ktiles + (b >> 2)) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (b & 3);
}

struct Quant4Args {
    int rows, cols, blocks;
    long long ld_x, ld_q, ld_v, items;
    uint8_t *q, *scale;
    float *values;
};

// A lane holds P = 16 / sizeof(T) columns of a block, 32 / P lanes make a block and a
// warp takes U runs of 32 P columns of one row, all loads first.
template <class T, bool PACKED, int U>
__global__ void __launch_bounds__(256) k_quantize_mx4(const T *__restrict__ x, const Quant4Args a) {
    constexpr int P = Pack<T>::P, LANES = 32 / P, RUN = 32 * P;
    let_next_launch();
    const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (item >= a.items) return;
    const int lane = threadIdx.x & 31;
    const int runs = (a.cols + U * RUN - 1) / (U * RUN);
    const long long r = item < (1ll << 31) ? (long long)((unsigned)item / (unsigned)runs) : item / runs;
    const long long c0 = (item - r * runs) * (U * RUN) + lane * P;
    const T *row = x + r * a.ld_x;
    float v[U][P];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long c = c0 + u * RUN;
        if (PACKED && c + P <= a.cols) {
            const uint4 w = __ldg(reinterpret_cast<const uint4 *>(row + c));
#pragma unroll
            for (int i = 0; i < P; ++i) v[u][i] = Pack<T>::one(w, i);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) v[u][i] = c + i < a.cols ? to_f32<T>(row[c + i]) : 0.f;
        }
    }
    const int ktiles = (a.blocks + 3) / 4;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long c = c0 + u * RUN;
        const int b = (int)(c >> 5);  // this lane's block
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < P; ++i) top = max(top, __float_as_uint(v[u][i]) & 0x7fffffffu);
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        const BlockCode k = block_code(top);
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < P; i += 2) word |= code_pair(v[u][i] * k.pre, v[u][i + 1] * k.pre) << (4 * i);
        if (k.byte == 255u) word = 0;
        // the exponents of a tile's four blocks are one word
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            bytes |= __shfl_sync(0xffffffffu, k.byte, (lane & ~(4 * LANES - 1)) + i * LANES) << (8 * i);
        if (b < a.blocks) {
            uint8_t *q = a.q + r * a.ld_q + (c >> 1);
            if constexpr (P == 4) *reinterpret_cast<uint16_t *>(q) = (uint16_t)word;
            else *reinterpret_cast<uint32_t *>(q) = word;
            if (a.values) {
                const float s = block_scale(k.byte);
                float *val = a.values + r * a.ld_v + c;
                float y[P];
#pragma unroll
                for (int i = 0; i < P; i += 2) {
                    const float2 f = pair_values((word >> (4 * i)) & 255u);
                    y[i] = f.x * s;
                    y[i + 1] = f.y * s;
                }
                if (PACKED && c + P <= a.cols) {
#pragma unroll
                    for (int i = 0; i < P; i += 4)
                        *reinterpret_cast<float4 *>(val + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < P; ++i)
                        if (c + i < a.cols) val[i] = y[i];
                }
            }
            if ((lane & (4 * LANES - 1)) == 0) *reinterpret_cast<uint32_t *>(a.scale + scale_at(r, b, ktiles)) = bytes;
        }
    }
}

template <class T>
cudaError_t quantize_mx4(const T *x, Quant4Args a, cudaStream_t st) {
    constexpr int U = 2;
    const auto at16 = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool packed = at16(x) && (a.ld_x * (long long)sizeof(T)) % 16 == 0 &&
                        (!a.values || (at16(a.values) && a.ld_v % 4 == 0));
    const int runs = (int)(((long long)a.cols + U * 32 * Pack<T>::P - 1) / (U * 32 * Pack<T>::P));
    a.items = (long long)a.rows * runs;
    if ((a.items + 7) / 8 > 0x7fffffff) return cudaErrorInvalidValue;
    const unsigned grid = (unsigned)((a.items + 7) / 8);
    if (packed) k_quantize_mx4<T, true, U><<<grid, 256, 0, st>>>(x, a);
    else k_quantize_mx4<T, false, U><<<grid, 256, 0, st>>>(x, a);
    return cudaGetLastError();
}

cudaError_t launch_quantize_mx4(const void *x, dstd_type type, int rows, int cols, long long ld_x, uint8_t *q,
                                long long ld_q, uint8_t *scale, float *values, long long ld_v, cudaStream_t st) {
    if (rows == 0 || cols == 0) return cudaSuccess;
    const Quant4Args a{rows, cols, mx4_blocks(cols), ld_x, ld_q, ld_v, 0, q, scale, values};
    if (type == DSTD_TYPE_F32) return quantize_mx4((const float *)x, a, st);
    if (type == DSTD_TYPE_BF16) return quantize_mx4((const __nv_bfloat16 *)x, a, st);
    return quantize_mx4((const __half *)x, a, st);
}

// ---------------------------------------------------------------------------
// Grid weights of a layer's inputs straight to tokens: t [B, N] -> codes and
// exponents of row (b, m), the same as from writing the grid weights out and
// quantising their rows; zero for M <= m < Mp. A warp takes a block of 32 inputs: an
// input touches two grid points, whose largest weights and codes are gathered in
// shared memory; then each lane writes the 16 bytes of its grid points. The 4
// warps of a block have 4 neighbouring blocks, whose exponents are one word.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(128) k_bin_mx4(const float *__restrict__ t, int N, const LifConst c, uint8_t *q,
                                                 long long ld_q, uint8_t *scale) {
    __shared__ uint4 s_code[4][128];
    __shared__ uint32_t s_top[4][128];
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.y, blocks = mx4_blocks(N), block = blockIdx.x * 4 + w, j = block * 32 + lane;
    for (int m = lane; m < c.Mp; m += 32) {
        s_code[w][m] = make_uint4(0, 0, 0, 0);
        s_top[w][m] = 0;
    }
    __syncwarp();
    const float x = j < N ? __ldg(t + (long long)b * N + j) : INFINITY;
    int k = -100;
    BinW bw{};
    if (isfinite(x)) {
        bw = bin_weights(c, x, false);
        k = bw.k;
        if (k >= 0 && k < c.M) atomicMax(&s_top[w][k], __float_as_uint(bw.wR) & 0x7fffffffu);
        if (k >= -1 && k + 1 < c.M) atomicMax(&s_top[w][k + 1], __float_as_uint(bw.wL) & 0x7fffffffu);
    }
    __syncwarp();
    uint32_t *code = reinterpret_cast<uint32_t *>(s_code[w]);
    const auto put = [&](int m, float v) {
        const BlockCode bc = block_code(s_top[w][m]);
        const uint32_t n = bc.byte == 255u ? 0u : code_pair(v * bc.pre, 0.f) & 15u;
        if (n) atomicOr(&code[m * 4 + (lane >> 3)], n << (4 * (lane & 7)));
    };
    if (k >= 0 && k < c.M) put(k, bw.wR);
    if (k >= -1 && k + 1 < c.M) put(k + 1, bw.wL);
    __syncwarp();
    if (block < blocks)
        for (int m = lane; m < c.Mp; m += 32)
            *reinterpret_cast<uint4 *>(q + ((long long)b * c.Mp + m) * ld_q + block * 16) = s_code[w][m];
    __syncthreads();
    const int ktiles = (blocks + 3) / 4;
    for (int m = threadIdx.x; m < c.Mp; m += 128) {
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) bytes |= block_code(s_top[i][m]).byte << (8 * i);
        *reinterpret_cast<uint32_t *>(scale + scale_at((long long)b * c.Mp + m, blockIdx.x * 4, ktiles)) = bytes;
    }
}

cudaError_t launch_bin_mx4(const float *t, int B, int N, const LifConst &c, uint8_t *q, long long ld_q, uint8_t *scale,
                           cudaStream_t st) {
    k_bin_mx4<<<dim3((unsigned)((mx4_blocks(N) + 3) / 4), (unsigned)B), 128, 0, st>>>(t, N, c, q, ld_q, scale);
    return cudaGetLastError();
}

// row sums of the weights' values, one warp per row: a lane adds the whole
// numbers of its blocks (twice the codes' values, exact) times their powers of two
__global__ void __launch_bounds__(256) k_mx4_rowsum(const uint8_t *__restrict__ w, long long ld,
                                                    const uint8_t *__restrict__ scale, int N, int blocks,
                                                    float *rowsum) {
    const int n = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (n >= N) return;
    float sum = 0.f;
    for (int b = lane; b < blocks; b += 32) {
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(w + (long long)n * ld + (long long)b * 16));
        const uint32_t word[4] = {u.x, u.y, u.z, u.w};
        float part = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 f = pair_values((word[i >> 2] >> (8 * (i & 3))) & 255u);
            part += f.x + f.y;
        }
        sum += part * block_scale(scale[scale_at(n, b, (blocks + 3) / 4)]);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) rowsum[n] = sum;
}

cudaError_t launch_mx4_rowsum(const uint8_t *w, long long ld, const uint8_t *scale, int N, int K, float *rowsum,
                              cudaStream_t st) {
    k_mx4_rowsum<<<(N + 7) / 8, 256, 0, st>>>(w, ld, scale, N, mx4_blocks(K), rowsum);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// Product, simplest form: a block of 256 threads computes 64 channels x 64 tokens,
// one block of 32 columns at a time, values in shared memory.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(256) k_mx4_product(const Mx4Args a) {
    __shared__ float s_w[32][65], s_x[32][65];
    const int tiles = (a.N + 63) / 64;
    const long long n0 = (long long)(blockIdx.x % tiles) * 64, t0 = (long long)(blockIdx.x / tiles) * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int b = 0; b < a.blocks; ++b) {
        for (int i = threadIdx.x; i < 2 * 64 * 16; i += 256) {
            const bool tok = i >= 1024;
            const int r = (i >> 4) & 63, byte = i & 15;
            const long long row = (tok ? t0 : n0) + r;
            float2 v = make_float2(0.f, 0.f);
            if (row < (tok ? a.T : a.N)) {
                v = pair_values((tok ? a.x + row * a.ld_x : a.w + row * a.ld_w)[(long long)b * 16 + byte]);
                const float s = block_scale((tok ? a.x_scale : a.w_scale)[scale_at(row, b, (a.blocks + 3) / 4)]);
                v.x *= s;
                v.y *= s;
            }
            (tok ? s_x : s_w)[2 * byte][r] = v.x;
            (tok ? s_x : s_w)[2 * byte + 1][r] = v.y;
        }
        __syncthreads();
        for (int k = 0; k < 32; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += s_x[k][ty + 16 * i] * s_w[k][tx + 16 * j];
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long t = t0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (t >= a.T || n >= a.N) continue;
            const long long at = t * a.out.ld_t + n * a.out.ld_n;
            if (a.out.type == DSTD_TYPE_F32) ((float *)a.out.p)[at] = acc[i][j];
            else if (a.out.type == DSTD_TYPE_BF16) ((__nv_bfloat16 *)a.out.p)[at] = __float2bfloat16_rn(acc[i][j]);
            else ((__half *)a.out.p)[at] = __float2half_rn(acc[i][j]);
        }
}

cudaError_t launch_mx4_product(const Mx4Args &a, cudaStream_t st) {
    if (a.T == 0 || a.N == 0) return cudaSuccess;
    const long long grid = (((long long)a.N + 63) / 64) * (((long long)a.T + 63) / 64);
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    k_mx4_product<<<(unsigned)grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace dstd
