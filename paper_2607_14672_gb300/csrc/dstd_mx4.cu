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
    long long ld_x, ld_q, ld_v;
    uint8_t *q, *scale;
    float *values;
};

// P = 16 / sizeof(T) columns as they are in memory: the bits of the largest |x| as fp32, and codes of x pre
template <class T>
struct Quant4 {
    static constexpr int P = Pack<T>::P;
    static __device__ __forceinline__ uint32_t top(const uint4 &w) {
        if constexpr (P == 4) {
            return max(max(w.x & 0x7fffffffu, w.y & 0x7fffffffu), max(w.z & 0x7fffffffu, w.w & 0x7fffffffu));
        } else {  // two at a time: the bits without the sign order like the values, NaN on top
            const uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu),
                                        __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
            return max(m >> 16, m & 0xffffu);
        }
    }
    static __device__ __forceinline__ uint32_t fp32_bits(uint32_t top) {
        if constexpr (P == 4) {
            return top;
        } else {
            const unsigned short h = (unsigned short)top;
            return __float_as_uint(to_f32<T>(*reinterpret_cast<const T *>(&h)));
        }
    }
    // code of column i in bits 4 i
    static __device__ __forceinline__ uint32_t codes(const uint4 &w, float pre) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < P ? Pack<T>::one(w, i < P ? i : 0) * pre : 0.f;
        uint32_t word;
        asm("{\n"
            ".reg .b8 b0, b1, b2, b3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
            "mov.b32 %0, {b0, b1, b2, b3};\n"
            "}"
            : "=r"(word)
            : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
        return word;
    }
};

// 16 bytes from any address, zeros from element `left` on: the two aligned 16-byte words that hold them, shifted
// together (a word that holds an element of the row lies in its allocation; others are not read).
template <class T>
__device__ __forceinline__ uint4 load_columns(const T *p, int left) {
    constexpr int P = Pack<T>::P;
    const int r = (int)(reinterpret_cast<uintptr_t>(p) & 15);
    const uint4 *word = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(p) - r);
    const int first = (16 - r) / (int)sizeof(T);  // elements in the first word
    uint4 u = make_uint4(0, 0, 0, 0), n = u;
    if (left > 0) u = __ldg(word);
    if (left > first) n = __ldg(word + 1);
    const bool two = r & 8, one = r & 4;
    const uint32_t w0 = two ? u.z : u.x, w1 = two ? u.w : u.y, w2 = two ? n.x : u.z, w3 = two ? n.y : u.w,
                   w4 = two ? n.z : n.x;
    uint32_t v[5] = {one ? w1 : w0, one ? w2 : w1, one ? w3 : w2, one ? w4 : w3, one ? (two ? n.w : n.y) : w4};
    if constexpr (P == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], 8 * (r & 2));
    }
    constexpr int E = P / 4;  // elements of a 32-bit word
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int keep = left - E * i;
        v[i] = keep >= E ? v[i] : (keep <= 0 ? 0u : v[i] & 0xffffu);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// A lane holds P columns of a block, 32 / P lanes make a block, and a warp takes U runs of 32 P columns of one
// row, all loads first. HBM bounds large ones: 16384 x 16384 fp32 with values in 322 us (7.1 TB/s), without in 173
// (U = 2: 223), 4096 x 16384 bf16 without in 29 (U = 1: 44). Small ones take fewer runs a warp, so that
// there are warps for every SM (800 x 784 fp32 with values: 2.6 us, with U = 8 3.3).
template <class T, bool PACKED, int U, bool VALUES>
__global__ void __launch_bounds__(256) k_quantize_mx4(const T *__restrict__ x, const Quant4Args a) {
    constexpr int P = Pack<T>::P, LANES = 32 / P, RUN = 32 * P;
    let_next_launch();
    const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, runs = (int)(((long long)a.cols + U * RUN - 1) / (U * RUN));
    const long long r = item < (1ll << 31) ? (long long)((unsigned)item / (unsigned)runs) : item / runs;
    if (r >= a.rows) return;
    const int c0 = (int)(item - r * runs) * (U * RUN), left = a.cols - c0 - lane * P;  // columns from this lane's first on
    const bool whole = PACKED && a.cols - c0 >= U * RUN;
    const T *row = x + r * a.ld_x + c0 + lane * P;
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (whole || (PACKED && left - u * RUN >= P)) w[u] = __ldg(reinterpret_cast<const uint4 *>(row + u * RUN));
        else w[u] = load_columns<T>(row + u * RUN, left - u * RUN);
    }
    const int b0 = (c0 + lane * P) >> 5;  // this lane's block
    uint8_t *q = a.q + r * a.ld_q + ((c0 + lane * P) >> 1);
    uint8_t *scale = a.scale + scale_at(r, b0, (a.blocks + 3) / 4);
    const int tiles_left = (a.blocks + 3) / 4 * 4 - b0;
    float *val = VALUES ? a.values + r * a.ld_v + c0 + lane * P : nullptr;
    const bool wide = VALUES && (reinterpret_cast<uintptr_t>(val) & 15) == 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!whole && c0 + u * RUN >= a.cols + 96) break;  // no tile of the row's left (a whole warp)
        uint32_t top = Quant4<T>::top(w[u]);
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        const BlockCode k = block_code(Quant4<T>::fp32_bits(top));
        const uint32_t word = k.byte == 255u ? 0u : Quant4<T>::codes(w[u], k.pre);
        if (!whole && tiles_left <= u * P) continue;
        // P blocks a run, four of them to a tile of 512 bytes
        if ((lane & (LANES - 1)) == 0) scale[u * P / 4 * 512] = (uint8_t)k.byte;
        if (!whole && b0 + u * P >= a.blocks) continue;
        if constexpr (P == 4) *reinterpret_cast<uint16_t *>(q + u * (RUN / 2)) = (uint16_t)word;
        else *reinterpret_cast<uint32_t *>(q + u * (RUN / 2)) = word;
        if constexpr (VALUES) {
            const float s = block_scale(k.byte);
            float y[P];
#pragma unroll
            for (int i = 0; i < P; i += 2) {
                const float2 f = pair_values((word >> (4 * i)) & 255u);
                y[i] = f.x * s;
                y[i + 1] = f.y * s;
            }
            if (wide && left - u * RUN >= P) {
#pragma unroll
                for (int i = 0; i < P; i += 4)
                    *reinterpret_cast<float4 *>(val + u * RUN + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i)
                    if (u * RUN + i < left) val[u * RUN + i] = y[i];
            }
        }
    }
}

template <class T, bool PACKED, int U>
cudaError_t quantize_runs(const T *x, const Quant4Args &a, cudaStream_t st) {
    constexpr int RUN = 32 * Pack<T>::P;
    const long long items = (long long)a.rows * (((long long)a.cols + U * RUN - 1) / (U * RUN)), blocks = (items + 7) / 8;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    if (a.values) k_quantize_mx4<T, PACKED, U, true><<<(unsigned)blocks, 256, 0, st>>>(x, a);
    else k_quantize_mx4<T, PACKED, U, false><<<(unsigned)blocks, 256, 0, st>>>(x, a);
    return cudaGetLastError();
}

template <class T, bool PACKED>
cudaError_t quantize_rows4(const T *x, const Quant4Args &a, cudaStream_t st) {
    constexpr int RUN = 32 * Pack<T>::P;
    const int runs = (a.cols - 1) / RUN + 1;
    const long long all = (long long)a.rows * runs;
    constexpr int most = sizeof(T) == 4 ? 8 : 4;
    int u = 1;
    while (u < (a.values ? 2 : most) && u < runs && all >= 2 * u * 4800ll) u *= 2;
    if (u == 1) return quantize_runs<T, PACKED, 1>(x, a, st);
    if (u == 2) return quantize_runs<T, PACKED, 2>(x, a, st);
    if (u == 4) return quantize_runs<T, PACKED, 4>(x, a, st);
    return quantize_runs<T, PACKED, most>(x, a, st);
}

template <class T>
cudaError_t quantize_mx4(const T *x, const Quant4Args &a, cudaStream_t st) {
    const bool packed = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (a.ld_x * (long long)sizeof(T)) % 16 == 0;
    return packed ? quantize_rows4<T, true>(x, a, st) : quantize_rows4<T, false>(x, a, st);
}

cudaError_t launch_quantize_mx4(const void *x, dstd_type type, int rows, int cols, long long ld_x, uint8_t *q,
                                long long ld_q, uint8_t *scale, float *values, long long ld_v, cudaStream_t st) {
    if (rows == 0 || cols == 0) return cudaSuccess;
    const Quant4Args a{rows, cols, mx4_blocks(cols), ld_x, ld_q, ld_v, q, scale, values};
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

// row sums of the weights' values, one warp per row: a lane adds the codes'
// values of each of its blocks (multiples of 1/2 up to 192: exact) times its power of two
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
// Product on the 4-bit tensor cores (tcgen05, kind mxf4: a product of two codes times both powers of two, fp32
// sums), D[n, t]: a block computes 128 rows of one side (the channels, as a rule: then neighbouring lanes store
// neighbouring elements) times NT of the other. TMA brings 256 columns of K a stage, codes as they are, and the scales
// of both sides in the tiles in which they are kept; one thread copies the scales to TMEM and issues the MMAs, in that
// order; four warps take the sums out. No operand is converted on the way, so few tokens cost what reading the weights
// costs: 8 x 16384 into 16384 in 26 us, 5.4 TB/s of codes and scales (about 3 us of it before the first byte). Wide
// tiles bring 34 KB a stage from L2, which bounds them: 4096 x 16384 into 16384 took 440 us in them, 9.1 GB, 21 TB/s.
// Where there are few tiles, `parts` blocks of a cluster share K: each leaves its sums in its own shared memory, and each
// adds up its share of the columns over all, in order (no atomics: the same call gives the same bits).
// ---------------------------------------------------------------------------
__device__ unsigned int g_status_mx4 = 0;

cudaError_t mx4_status_read(unsigned int *out, int clear) {
    cudaError_t e = cudaMemcpyFromSymbol(out, g_status_mx4, sizeof(unsigned int));
    if (e != cudaSuccess || !clear) return e;
    unsigned int z = 0;
    return cudaMemcpyToSymbol(g_status_mx4, &z, sizeof(z));
}

namespace {
using namespace tc;

constexpr int kStageBlocks = 8;          // blocks of 32 along K a stage: rows of 128 bytes
constexpr int kRowBytes = 16 * kStageBlocks;
constexpr int kTileBytes = 128 * kRowBytes;
constexpr int kScaleTile = 512;          // scales of 128 rows by 4 blocks

template <int NT>
struct Mx4Cfg {
    static constexpr int B_BYTES = NT * kRowBytes;
    static constexpr int SF_BYTES = 4 * kScaleTile;  // 2 tiles along K of either side (NT divides 128 or b is one tile)
    static constexpr int STAGE = (kTileBytes + B_BYTES + SF_BYTES + 1023) / 1024 * 1024;
    static constexpr int STAGES = 216 * 1024 / STAGE;                    // a block that has an SM to itself
    static constexpr int HALF = 108 * 1024 / STAGE;                      // two to an SM
    static constexpr int smem(int slots) { return slots * STAGE + 1024 + 256; }
    static constexpr int SF_COL = NT;                    // scales: two sets of (A, B) in turn
    static constexpr int SF_SET = 16;
    static constexpr int USED = NT + 2 * SF_SET;
    static constexpr int COLS = USED <= 64 ? 64 : (USED <= 128 ? 128 : 256);
    static_assert(NT * 128 * 4 <= HALF * STAGE, "the sums of a tile fit the stages");
    static_assert(2 * STAGES * 8 + 16 <= 256, "the barriers fit");
};

// rows of one side of the product, a the side of 128-row tiles
struct Mx4Side {
    const uint8_t *scale;
    int rows;
};
struct Mx4Tc {
    Mx4Side a, b;
    int blocks, ktiles, tiles_a, tiles_b, parts, slots;  // slots: stages of a block's ring
    void *out;
    long long ld_a, ld_b;  // of out; one of them is 1
};

// tiles are taken in groups of 8 of one side, so that blocks at work at one time share both operands in L2
__device__ __forceinline__ void mx4_tile(int i, int tiles_a, int tiles_b, int &ta, int &tb) {
    const int per = 8 * tiles_a, group = i / per, r = i - group * per;
    const int left = tiles_b - group * 8, wide = left < 8 ? left : 8;
    ta = r / wide;
    tb = group * 8 + r - ta * wide;
}

__device__ __forceinline__ void mx4_timeout() { atomicOr(&g_status_mx4, STATUS_TIMEOUT); }

// The first `left` of CH columns of a lane's row to out: neighbouring lanes next to each other (ld_a = 1), or
// the lane's own columns (ld_b = 1). Whole runs without a test for each element (with one, storing took 64
// us of a product of 8192 x 32 into 8192).
template <class O, int CH>
__device__ __forceinline__ void mx4_store(O *dst, long long ld_a, long long ld_b, const float (&v)[CH], int left) {
    if (ld_b != 1 || ld_a == 1) {
        if (left >= CH) {
#pragma unroll
            for (int c = 0; c < CH; ++c, dst += ld_b) *dst = round_out<O>(v[c]);
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (c < left) dst[c * ld_b] = round_out<O>(v[c]);
        }
        return;
    }
    constexpr int P = 16 / sizeof(O);
    if (left >= CH && (reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
#pragma unroll
        for (int c = 0; c < CH; c += P) {
            alignas(16) O y[P];
#pragma unroll
            for (int u = 0; u < P; ++u) y[u] = round_out<O>(v[c + u]);
            *reinterpret_cast<uint4 *>(dst + c) = *reinterpret_cast<const uint4 *>(y);
        }
    } else if (left >= CH) {
#pragma unroll
        for (int c = 0; c < CH; ++c) dst[c] = round_out<O>(v[c]);
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c < left) dst[c] = round_out<O>(v[c]);
    }
}

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr)
                 : "memory");
    return v;
}

template <int NT, class O>
__global__ void __launch_bounds__(192) k_mx4_tc(const __grid_constant__ CUtensorMap map_a,
                                                const __grid_constant__ CUtensorMap map_b, const Mx4Tc p) {
    using C = Mx4Cfg<NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int slots = p.slots;
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + slots * C::STAGE);
    uint64_t *empty = full + slots, *done = empty + slots;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(done + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = p.parts > 1 ? (int)cluster_ctarank() : 0;
    int ta, tb;
    mx4_tile((int)(blockIdx.x / p.parts), p.tiles_a, p.tiles_b, ta, tb);
    const int stages = (p.blocks + kStageBlocks - 1) / kStageBlocks;
    const int s0 = (int)((long long)stages * part / p.parts), s1 = (int)((long long)stages * (part + 1) / p.parts);

    if (threadIdx.x == 0) {
        for (int s = 0; s < slots; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 5) tmem_alloc(tmem_slot, C::COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    wait_launch_before();

    if (warp == 4) {
        bool ok = true;
        int slot = 0;
        uint32_t turn = 0;
        for (int s = s0; s < s1; ++s) {
            ok = mbar_wait_cycles(&empty[slot], turn ^ 1u);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (elect_one()) {
                const uint32_t st = smem_u32(smem + slot * C::STAGE), sf = st + kTileBytes + C::B_BYTES;
                const int k0 = s * 2;
                const uint32_t sf_bytes = (uint32_t)min(2, p.ktiles - k0) * kScaleTile;
                mbar_expect_tx(&full[slot], (uint32_t)(kTileBytes + C::B_BYTES) + 2 * sf_bytes);
                tma_load_2d(st, &map_a, &full[slot], s * kRowBytes, ta * 128);
                tma_load_2d(st + kTileBytes, &map_b, &full[slot], s * kRowBytes, tb * NT);
                bulk_load(sf, p.a.scale + ((long long)ta * p.ktiles + k0) * kScaleTile, sf_bytes, &full[slot]);
                bulk_load(sf + 2 * kScaleTile, p.b.scale + ((long long)tb * p.ktiles + k0) * kScaleTile, sf_bytes,
                          &full[slot]);
            }
            __syncwarp();
            if (++slot == slots) slot = 0, turn ^= 1u;
        }
        // every stage released: no copy is in flight
        for (int i = 0; i < slots && ok; ++i) {
            ok = mbar_wait_cycles(&empty[slot], turn ^ 1u);
            if (++slot == slots) slot = 0, turn ^= 1u;
        }
        if (!ok) mx4_timeout();
        __syncwarp();
    } else if (warp == 5) {
        bool ok = true;
        int slot = 0;
        uint32_t turn = 0;
        for (int s = s0; s < s1; ++s) {
            ok = mbar_wait_cycles(&full[slot], turn);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t st = smem_u32(smem + slot * C::STAGE), sf = st + kTileBytes + C::B_BYTES;
                const uint32_t sfa = tmem + C::SF_COL + (s & 1) * C::SF_SET, sfb = sfa + 8;
                const uint64_t ad = sdesc_sw128(st), bd = sdesc_sw128(st + kTileBytes);
                const int left = p.blocks - s * kStageBlocks;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h * 4 >= left) break;
                    tmem_cp_scales(sfa + h * 4, sdesc_rows16(sf + h * kScaleTile));
                    tmem_cp_scales(sfb + h * 4, sdesc_rows16(sf + (2 + h) * kScaleTile));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int kk = 2 * h + i;
                        if (kk * 2 >= left) break;
                        mma_mx4(tmem, ad + kk * 2, bd + kk * 2, idesc_mx4(128, NT, 2 * i), sfa + h * 4,
                                sfb + h * 4, s > s0 || kk > 0 ? 1u : 0u);
                    }
                }
                mma_commit(&empty[slot]);
                if (s + 1 == s1) mma_commit(done);
            }
            __syncwarp();
            if (++slot == slots) slot = 0, turn ^= 1u;
        }
        if (!ok) mx4_timeout();
        __syncwarp();
    }
    bool ok = true;
    if (warp < 4) {
        const int row = warp * 32 + lane;
        const long long r = (long long)ta * 128 + row, c0 = (long long)tb * NT;
        ok = mbar_wait_cycles(done, 0);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok && lane == 0) mx4_timeout();
        tc_fence_after();
        constexpr int CH = 16;
        const uint32_t t0 = tmem + ((uint32_t)(warp * 32) << 16);
#pragma unroll 1
        for (int c = 0; c < NT && ok; c += CH) {
            float v[CH];
            tmem_ld16(t0 + c, v);
            if (p.parts > 1) {
                float *sum = reinterpret_cast<float *>(smem) + c * 128 + row;
#pragma unroll
                for (int i = 0; i < CH; ++i) sum[i * 128] = v[i];
            } else {
                const long long left = r < p.a.rows ? p.b.rows - (c0 + c) : 0;
                mx4_store<O, CH>(static_cast<O *>(p.out) + r * p.ld_a + (c0 + c) * p.ld_b, p.ld_a, p.ld_b, v,
                                 (int)max(0ll, min((long long)CH, left)));
            }
        }
    }
    if (p.parts > 1) {
        __syncwarp();
        cluster_sync();
        // this block's share of the columns, 4 rows of one at a time: all blocks' sums on their way, then added in order
        const int first = NT * part / p.parts, last = NT * (part + 1) / p.parts;
        const uint32_t base = smem_u32(smem);
        O *out = static_cast<O *>(p.out);
        const int units = (last - first) * 32;
        constexpr int U = NT >= 64 ? 4 : 1;  // a thread's units at a time
        for (int i0 = threadIdx.x; i0 < units; i0 += U * 192) {
            float4 sum[U], v[U][8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (q >= p.parts) break;
                const uint32_t from = mapa_rank(base, q);
#pragma unroll
                for (int e = 0; e < U; ++e) {
                    const int i = i0 + e * 192;
                    if (i < units) v[e][q] = ld_cluster4(from + ((first + (i >> 5)) * 128 + (i & 31) * 4) * 4);
                }
            }
#pragma unroll
            for (int e = 0; e < U; ++e) {
                sum[e] = v[e][0];
#pragma unroll
                for (int q = 1; q < 8; ++q) {
                    if (q >= p.parts) break;
                    sum[e].x += v[e][q].x;
                    sum[e].y += v[e][q].y;
                    sum[e].z += v[e][q].z;
                    sum[e].w += v[e][q].w;
                }
                const int i = i0 + e * 192;
                const long long r = (long long)ta * 128 + (i & 31) * 4, col = (long long)tb * NT + first + (i >> 5);
                if (i >= units || col >= p.b.rows) continue;
                O *dst = out + r * p.ld_a + col * p.ld_b;
                const float y[4] = {sum[e].x, sum[e].y, sum[e].z, sum[e].w};
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (r + u < p.a.rows) dst[u * p.ld_a] = round_out<O>(y[u]);
            }
        }
        __syncwarp();
        cluster_sync();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) tmem_dealloc(tmem, C::COLS);
}

// Large products: a pair of SMs computes 256 x 256, each SM its 128 rows of a and half of b's codes,
// so that a stage brings 35 KB to an SM for 391 cycles of MMAs at the 4-bit nominal rate (a block of its own, 128 x 128:
// 34 KB for half as many). The scales of b's 256 rows go to both. The pairs stay and take tiles in turn; eight warps
// take the sums out to registers, from where they are stored while the next tile is computed: two accumulators of this
// width and the scales do not fit TMEM. The tensor pipe bounds it: 4096 x 16384 into 16384 in 276 us, 8.0 PFLOP/s; 128 x 128
// tiles took 440. With few columns the stores do: 8192 x 32 into 8192 fp32 in 49 us, 5.5 TB/s.
struct PairCfg {
    static constexpr int SF_BYTES = 2 * kScaleTile * 3;  // of this SM's rows of a, of all of b's
    static constexpr int STAGE = (2 * kTileBytes + SF_BYTES + 1023) / 1024 * 1024;
    static constexpr int STAGES = 6;
    static constexpr int SMEM = STAGES * STAGE + 1024 + 256;
    static constexpr int SF_COL = 256, SF_SET = 8 + 16;
};

template <class O>
__global__ void __launch_bounds__(320, 1)
    k_mx4_pair(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb, const Mx4Tc p) {
    using C = PairCfg;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + C::STAGES * C::STAGE);  // (leader) both SMs' copies have landed
    uint64_t *empty = full + C::STAGES;                                          // the pair's MMAs have read the stage
    uint64_t *acc_full = empty + C::STAGES, *acc_empty = acc_full + 1;           // the latter at the leader
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(acc_empty + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank(), step = (int)cluster_count_x();
    const int stages = (p.blocks + kStageBlocks - 1) / kStageBlocks, tiles = p.tiles_a * p.tiles_b;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, 16);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 9) tmem_alloc_pair(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both SMs' barriers exist before any remote signal
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    wait_launch_before();

    if (warp == 8) {
        const uint32_t full0 = mapa_rank(smem_u32(&full[0]), 0);
        uint32_t it = 0;
        bool ok = true;
        for (int i = (int)cluster_id_x(); ok && i < tiles; i += step) {
            int ta, tb;
            mx4_tile(i, p.tiles_a, p.tiles_b, ta, tb);
            for (int s = 0; s < stages; ++s, ++it) {
                const int slot = it % C::STAGES;
                ok = mbar_wait_cycles(&empty[slot], ((it / C::STAGES) & 1u) ^ 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t st = smem_u32(smem + slot * C::STAGE);
                    const uint32_t bar = full0 + (uint32_t)(slot * sizeof(uint64_t));
                    if (rank == 0) mbar_expect_tx(&full[slot], (uint32_t)(2 * (2 * kTileBytes + C::SF_BYTES)));
                    tma_load_2d_pair(st, &map_a, bar, s * kRowBytes, ta * 256 + rank * 128);
                    tma_load_2d_pair(st + kTileBytes, &map_b, bar, s * kRowBytes, tb * 256 + rank * 128);
                    tma_load_2d_pair(st + 2 * kTileBytes, &map_sa, bar, s * 256, ta * 2 + rank);
                    tma_load_2d_pair(st + 2 * kTileBytes + 2 * kScaleTile, &map_sb, bar, s * 256, tb * 2);
                }
                __syncwarp();
            }
        }
        // every stage released: no copy is in flight and no commit targets this SM's stages afterwards
        for (int i = 0; i < C::STAGES && ok; ++i, ++it)
            ok = mbar_wait_cycles(&empty[it % C::STAGES], ((it / C::STAGES) & 1u) ^ 1u);
        if (!ok) mx4_timeout();
        __syncwarp();
    } else if (warp == 9) {
        if (rank == 0) {
            uint32_t it = 0, j = 0;
            bool ok = true;
            for (int i = (int)cluster_id_x(); ok && i < tiles; i += step, ++j) {
                ok = mbar_wait_cycles(acc_empty, (j & 1u) ^ 1u);
                for (int s = 0; s < stages; ++s, ++it) {
                    const int slot = it % C::STAGES;
                    ok = ok && mbar_wait_cycles(&full[slot], (it / C::STAGES) & 1u);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t st = smem_u32(smem + slot * C::STAGE), sf = st + 2 * kTileBytes;
                        const uint32_t sfa = tmem + C::SF_COL + (it & 1u) * C::SF_SET, sfb = sfa + 8;
                        const uint64_t ad = sdesc_sw128(st), bd = sdesc_sw128(st + kTileBytes);
                        const int left = p.blocks - s * kStageBlocks;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (h * 4 >= left) break;
                            tmem_cp_scales_pair(sfa + h * 4, sdesc_rows16(sf + h * kScaleTile));
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                tmem_cp_scales_pair(sfb + (h * 2 + k) * 4,
                                                    sdesc_rows16(sf + (1 + k) * 2 * kScaleTile + h * kScaleTile));
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int kk = 2 * h + k;
                                if (kk * 2 >= left) break;
                                mma_mx4_pair(tmem, ad + kk * 2, bd + kk * 2, idesc_mx4(256, 256, 2 * k), sfa + h * 4,
                                             sfb + h * 8, s > 0 || kk > 0 ? 1u : 0u);
                            }
                        }
                        mma_commit_pair(&empty[slot]);
                        if (s + 1 == stages) mma_commit_pair(acc_full);
                    }
                    __syncwarp();
                }
            }
            if (!ok) mx4_timeout();
        }
        __syncwarp();
    } else {
        // rows of quarter (warp & 3), half of the columns
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t t0 = tmem + ((uint32_t)(quarter * 32) << 16) + half * 128;
        const uint32_t acc_empty0 = mapa_rank(smem_u32(acc_empty), 0);
        uint32_t j = 0;
        for (int i = (int)cluster_id_x(); i < tiles; i += step, ++j) {
            int ta, tb;
            mx4_tile(i, p.tiles_a, p.tiles_b, ta, tb);
            if (!mbar_wait_cycles(acc_full, j & 1u)) {
                mx4_timeout();
                break;
            }
            __syncwarp();
            tc_fence_after();
            float v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(t0 + c * 32, v[c]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_pair(acc_empty0);
            const long long r = (long long)ta * 256 + rank * 128 + quarter * 32 + lane;
            const long long c0 = (long long)tb * 256 + half * 128;
            O *dst = static_cast<O *>(p.out) + r * p.ld_a + c0 * p.ld_b;
            const long long left = r < p.a.rows ? p.b.rows - c0 : 0;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                mx4_store<O, 32>(dst + c * 32 * p.ld_b, p.ld_a, p.ld_b, v[c],
                                 (int)max(0ll, min(32ll, left - c * 32)));
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // both SMs are done with TMEM, every remote arrive has landed
    if (warp == 9) tmem_dealloc_pair(tmem, 512);
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                             const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                             CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// boxes of box_rows rows of 128 bytes, swizzled; beyond the matrix zeros are read
bool code_map(CUtensorMap *m, const uint8_t *p, int rows, int blocks, long long ld, int box_rows) {
    EncodeFn enc = reinterpret_cast<EncodeFn>(tensor_map_encoder());
    if (!enc) return false;
    const cuuint64_t dim[2] = {(cuuint64_t)blocks * 16, (cuuint64_t)rows};
    const cuuint64_t stride[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kRowBytes, (cuuint32_t)box_rows};
    const cuuint32_t one[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(p), dim, stride, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// boxes of 2 tiles along K by `rows` tiles of the scales, as 32-bit words; beyond them zeros are read
bool scale_map(CUtensorMap *m, const uint8_t *p, int rows, int ktiles, int box_rows) {
    EncodeFn enc = reinterpret_cast<EncodeFn>(tensor_map_encoder());
    if (!enc) return false;
    const cuuint64_t dim[2] = {(cuuint64_t)ktiles * 128, ((cuuint64_t)rows + 127) / 128};
    const cuuint64_t stride[1] = {(cuuint64_t)ktiles * kScaleTile};
    const cuuint32_t box[2] = {256, (cuuint32_t)box_rows};
    const cuuint32_t one[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint8_t *>(p), dim, stride, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Mx4Plan {
    int nt, parts;   // nt = 0: pairs of SMs
    bool exchanged;  // the tokens are the side a
};

// the product with its sides named
Mx4Tc mx4_sides(const Mx4Args &a, const Mx4Plan &plan, int tile_a, int tile_b) {
    const bool ex = plan.exchanged;
    const int rows_a = ex ? a.T : a.N, rows_b = ex ? a.N : a.T;
    return Mx4Tc{{ex ? a.x_scale : a.w_scale, rows_a}, {ex ? a.w_scale : a.x_scale, rows_b}, a.blocks, (a.blocks + 3) / 4,
                 (rows_a - 1) / tile_a + 1, (rows_b - 1) / tile_b + 1, plan.parts, 0, a.out.p,
                 ex ? a.out.ld_t : a.out.ld_n, ex ? a.out.ld_n : a.out.ld_t};
}

template <class O>
cudaLaunchConfig_t pair_config(cudaLaunchAttribute (&attr)[2]) {
    cudaLaunchConfig_t cfg = {};
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cfg.blockDim = dim3(320);
    cfg.dynamicSmemBytes = PairCfg::SMEM;
    return cfg;
}

// SM pairs at work at a time (0: an error)
template <class O>
int mx4_pairs() {
    static PerDevice resident;
    return resident.get([](int) {
        cudaLaunchAttribute attr[2];
        cudaLaunchConfig_t cfg = pair_config<O>(attr);
        cfg.gridDim = dim3(2 * 76);
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaFuncSetAttribute(k_mx4_pair<O>, cudaFuncAttributeMaxDynamicSharedMemorySize, PairCfg::SMEM) !=
                cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, k_mx4_pair<O>, &cfg) != cudaSuccess)
            return 0;
        return n;
    });
}

template <class O>
cudaError_t launch_mx4_pair(const Mx4Args &a, const Mx4Plan &plan, cudaStream_t st) {
    const int pairs = mx4_pairs<O>();
    if (pairs < 1) return cudaErrorInvalidConfiguration;
    const Mx4Tc p = mx4_sides(a, plan, 256, 256);
    const bool ex = plan.exchanged;
    CUtensorMap map_a, map_b, map_sa, map_sb;
    if (!code_map(&map_a, ex ? a.x : a.w, p.a.rows, a.blocks, ex ? a.ld_x : a.ld_w, 128) ||
        !code_map(&map_b, ex ? a.w : a.x, p.b.rows, a.blocks, ex ? a.ld_w : a.ld_x, 128) ||
        !scale_map(&map_sa, p.a.scale, p.a.rows, p.ktiles, 1) || !scale_map(&map_sb, p.b.scale, p.b.rows, p.ktiles, 2))
        return cudaErrorInvalidValue;
    const long long tiles = (long long)p.tiles_a * p.tiles_b;
    if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = pair_config<O>(attr);
    cfg.gridDim = dim3(2 * (unsigned)std::min<long long>(tiles, pairs));
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, k_mx4_pair<O>, map_a, map_b, map_sa, map_sb, p);
}

template <int NT, class O>
cudaError_t launch_mx4_tc(const Mx4Args &a, const Mx4Plan &plan, cudaStream_t st) {
    using C = Mx4Cfg<NT>;
    static PerDevice granted;
    if (!granted.get([](int) {
            return cudaFuncSetAttribute(k_mx4_tc<NT, O>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        C::smem(C::STAGES)) == cudaSuccess ? 1 : 0;
        }))
        return cudaErrorInvalidConfiguration;
    const bool ex = plan.exchanged;
    Mx4Tc p = mx4_sides(a, plan, 128, NT);
    CUtensorMap map_a, map_b;
    if (!code_map(&map_a, ex ? a.x : a.w, p.a.rows, a.blocks, ex ? a.ld_x : a.ld_w, 128) ||
        !code_map(&map_b, ex ? a.w : a.x, p.b.rows, a.blocks, ex ? a.ld_w : a.ld_x, NT))
        return cudaErrorInvalidValue;
    const long long grid = (long long)p.tiles_a * p.tiles_b * plan.parts;
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    p.slots = grid <= 152 && plan.parts == 1 ? C::STAGES : C::HALF;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)plan.parts;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = plan.parts > 1 ? 2 : 1;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(192);
    cfg.dynamicSmemBytes = C::smem(p.slots);
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, k_mx4_tc<NT, O>, map_a, map_b, p);
}

// Which side is a: the one whose neighbouring rows are neighbours in out, unless the other way halves the padded
// tiles (5325 x 285 into 123 fp32: 5.6 us, the other way 11). Pairs from 48 tiles of 256 x 256 on (2048 x 8192 into
// 2048, 64 tiles: 17 us, in blocks of 128 x 128 21; 500 x 12000 into 3000, 24 tiles: 24 and 21).
Mx4Plan mx4_plan(const Mx4Args &q) {
    const auto width = [](int b) { return b <= 16 ? 16 : (b <= 32 ? 32 : (b <= 64 ? 64 : 128)); };
    const auto area = [&](int a, int b) {
        const long long nt = width(b);
        return (((long long)a + 127) / 128 * 128) * (((long long)b + nt - 1) / nt * nt);
    };
    Mx4Plan p{};
    const long long straight = area(q.N, q.T), exchanged = area(q.T, q.N);
    p.exchanged = q.out.ld_n == 1 ? 2 * exchanged <= straight : 2 * straight > exchanged;
    const int a = p.exchanged ? q.T : q.N, b = p.exchanged ? q.N : q.T;
    const int stages = (q.blocks + kStageBlocks - 1) / kStageBlocks;
    p.nt = width(b);
    p.parts = 1;
    const long long pair_tiles = (((long long)a + 255) / 256) * (((long long)b + 255) / 256);
    if (pair_tiles >= 48 && b > 128) {
        p.nt = 0;
        return p;
    }
    // K is shared where that is faster, by times in us of a stage and of joining 2, 4 and 8 parts (measured at 1 x
    // 4096 x 4096: 7.1 in one piece, 5.4 in four; 64 x 16384 into 2000: 22.3 and 11.0; 300 x 16384 into 130: 24.4
    // and, in eight, 12.5), and where all blocks have an SM to themselves
    const double stage = p.nt <= 32 ? 0.26 : (p.nt == 64 ? 0.29 : 0.33);
    const double join[3][3] = {{1.6, 1.6, 1.8}, {2.7, 2.4, 2.7}, {4.2, 4.3, 4.5}};
    const long long tiles = (((long long)a + 127) / 128) * (((long long)b + p.nt - 1) / p.nt);
    double best = stages * stage;
    for (int i = 0; i < 3; ++i) {
        const int parts = 2 << i;
        const double cost = stages * stage / parts + join[p.nt <= 32 ? 0 : (p.nt == 64 ? 1 : 2)][i];
        if (tiles * parts > 152 || parts > stages || cost >= best) continue;
        best = cost;
        p.parts = parts;
    }
    return p;
}

template <class O>
cudaError_t run_mx4(const Mx4Args &a, cudaStream_t st) {
    const Mx4Plan p = mx4_plan(a);
    if (p.nt == 0) return launch_mx4_pair<O>(a, p, st);
    if (p.nt == 16) return launch_mx4_tc<16, O>(a, p, st);
    if (p.nt == 32) return launch_mx4_tc<32, O>(a, p, st);
    if (p.nt == 64) return launch_mx4_tc<64, O>(a, p, st);
    return launch_mx4_tc<128, O>(a, p, st);
}

// a product of no columns
__global__ void __launch_bounds__(256) k_zero_rows(char *out, long long bytes, long long ld_bytes, int rows) {
    for (long long r = blockIdx.x; r < rows; r += gridDim.x)
        for (long long i = threadIdx.x; i < bytes; i += 256) out[r * ld_bytes + i] = 0;
}

}  // namespace

cudaError_t launch_mx4_product(const Mx4Args &a, cudaStream_t st) {
    if (a.T == 0 || a.N == 0) return cudaSuccess;
    if (a.blocks == 0) {
        const long long size = a.out.type == DSTD_TYPE_F32 ? 4 : 2;
        k_zero_rows<<<(unsigned)std::min(a.T, 4096), 256, 0, st>>>((char *)a.out.p, a.N * size, a.out.ld_t * size, a.T);
        return cudaGetLastError();
    }
    if (a.out.type == DSTD_TYPE_F32) return run_mx4<float>(a, st);
    if (a.out.type == DSTD_TYPE_BF16) return run_mx4<__nv_bfloat16>(a, st);
    return run_mx4<__half>(a, st);
}

}  // namespace dstd
