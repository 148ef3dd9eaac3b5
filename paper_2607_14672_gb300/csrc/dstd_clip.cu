// The optimiser's side of a training step over many gradient tensors: their
// global norm, clipping by it, and the clipped AdamW update.
#include "dstd_internal.cuh"

#include <math.h>

namespace dstd {

namespace {

// The tensors of one launch are cut into chunks of `chunk` elements, numbered
// through all of them; seg[i].first is tensor i's first chunk.
template <class A>
__device__ __forceinline__ int seg_of(const A &a, unsigned c) {
    int lo = 0, hi = a.count - 1;  // the last tensor whose first chunk is <= c
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.seg[mid].first <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ float load_f32(const void *p, long long i);
template <>
__device__ __forceinline__ float load_f32<float>(const void *p, long long i) { return ((const float *)p)[i]; }
template <>
__device__ __forceinline__ float load_f32<__nv_bfloat16>(const void *p, long long i) {
    return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
}
template <>
__device__ __forceinline__ float load_f32<__half>(const void *p, long long i) {
    return __half2float(((const __half *)p)[i]);
}
__device__ __forceinline__ float load_any(const void *p, long long i, int type) {
    return type == DSTD_TYPE_F32 ? load_f32<float>(p, i)
                                 : (type == DSTD_TYPE_BF16 ? load_f32<__nv_bfloat16>(p, i) : load_f32<__half>(p, i));
}
__device__ __forceinline__ void store_any(void *p, long long i, int type, float x) {
    if (type == DSTD_TYPE_F32) ((float *)p)[i] = x;
    else if (type == DSTD_TYPE_BF16) ((__nv_bfloat16 *)p)[i] = __float2bfloat16_rn(x);
    else ((__half *)p)[i] = __float2half_rn(x);
}

// sum over the block in a fixed order (every thread gets it)
__device__ __forceinline__ double block_sum(double x, double *s_part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = x;
    __syncthreads();
    double t = 0.0;
    for (int i = 0; i < (int)(blockDim.x >> 5); ++i) t += s_part[i];
    return t;
}

// Sum of squares of every chunk into its own slot (no atomics on the sums:
// the result does not depend on the order in which blocks run). The block that
// draws the last ticket then adds the slots in order, and derives from the
// total what the clipping needs.
template <int CAP>
__global__ void __launch_bounds__(256) k_sum_squares(const ClipArgs<CAP> a) {
    __shared__ double s_part[8];
    __shared__ bool s_last;
    for (unsigned c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipSeg &sg = a.seg[seg_of(a, c)];
        const long long lo = (long long)(c - sg.first) * a.chunk;
        const long long hi = lo + a.chunk < sg.n ? lo + a.chunk : sg.n;
        double s = 0.0;
        for (long long i = lo + threadIdx.x; i < hi; i += 256) {
            const double x = (double)load_any(sg.g, i, sg.type);
            s += x * x;
        }
        s = block_sum(s, s_part);
        if (threadIdx.x == 0) a.partial[c] = s;
    }
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    double s = 0.0;
    for (unsigned c = threadIdx.x; c < a.chunks; c += 256) s += a.partial[c];
    s = block_sum(s, s_part);
    if (a.norm_each) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        for (int i = warp; i < a.count; i += 8) {
            const unsigned end = i + 1 < a.count ? a.seg[i + 1].first : a.chunks;
            double e = 0.0;
            for (unsigned c = a.seg[i].first + lane; c < end; c += 32) e += a.partial[c];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) e += __shfl_xor_sync(0xffffffffu, e, o);
            if (lane == 0) a.norm_each[i] = (float)sqrt(e);
        }
    }
    if (threadIdx.x == 0) {
        *a.ticket = 0;
        const double before = a.launch == 0 ? 0.0 : a.result->sum;
        const double sum = before + s;
        a.result->sum = sum;
        if (a.last_launch) {
            const double norm = sqrt(sum);
            const bool finite = isfinite(sum);
            a.norm[0] = (float)norm;
            a.result->coef = finite && norm > a.max_norm ? (float)(a.max_norm / norm) : 1.f;
            a.result->skip = finite ? 0 : 1;
            if (a.step && finite) a.step[0] += 1;
        }
    }
}

template <int CAP>
__global__ void __launch_bounds__(256) k_clip_scale(const ClipArgs<CAP> a) {
    const float coef = a.result->coef;
    for (unsigned c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipSeg &sg = a.seg[seg_of(a, c)];
        if (coef == 1.f && sg.out == sg.g) continue;
        const long long lo = (long long)(c - sg.first) * a.chunk;
        const long long hi = lo + a.chunk < sg.n ? lo + a.chunk : sg.n;
        for (long long i = lo + threadIdx.x; i < hi; i += 256)
            store_any(sg.out, i, sg.type, load_any(sg.g, i, sg.type) * coef);
    }
}

template <int CAP>
__global__ void __launch_bounds__(256) k_adamw_clip(const ClipArgs<CAP> a) {
    if (a.result->skip) return;
    const float coef = a.result->coef;
    const float t = (float)a.step[0];
    // 1 - beta^t without the cancellation of a beta near 1
    const float bc1 = -expm1f(t * a.ln_b1), bc2 = -expm1f(t * a.ln_b2);
    const float lr = a.lr_dev ? *a.lr_dev : a.lr;
    const float decay = 1.f - lr * a.wd;
    for (unsigned c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipSeg &sg = a.seg[seg_of(a, c)];
        const long long lo = (long long)(c - sg.first) * a.chunk;
        const long long hi = lo + a.chunk < sg.n ? lo + a.chunk : sg.n;
        float *w = (float *)sg.out;
        for (long long i = lo + threadIdx.x; i < hi; i += 256) {
            const float g = load_any(sg.g, i, sg.type) * coef;
            const float m = a.b1 * sg.m[i] + a.one_b1 * g;
            const float v = a.b2 * sg.v[i] + a.one_b2 * (g * g);
            sg.m[i] = m;
            sg.v[i] = v;
            w[i] = w[i] * decay - lr * (m / bc1) / (sqrtf(v / bc2) + a.eps);
        }
    }
}

constexpr int kBlocks = 152 * 8;

// elements of a chunk: about one chunk per resident block, whole multiples of 1024
long long chunk_elements(int count, const int64_t *n) {
    long long total = 0;
    for (int i = 0; i < count; ++i) total += n[i];
    const long long c = (total + kBlocks - 1) / kBlocks;
    return c < 1024 ? 1024 : (c + 1023) / 1024 * 1024;
}

template <int CAP>
cudaError_t launch_group(const ClipTensors &t, ClipOp op, int begin, int count, ClipArgs<CAP> &a, cudaStream_t st) {
    unsigned chunks = 0;
    a.count = 0;
    for (int i = begin; i < begin + count; ++i) {
        ClipSeg &sg = a.seg[a.count++];
        sg.g = t.g[i];
        sg.out = t.out ? t.out[i] : nullptr;
        sg.m = t.m ? t.m[i] : nullptr;
        sg.v = t.v ? t.v[i] : nullptr;
        sg.n = t.n[i];
        sg.first = chunks;
        sg.type = t.type[i];
        chunks += (unsigned)((t.n[i] + a.chunk - 1) / a.chunk);
    }
    a.chunks = chunks;
    const unsigned grid = chunks < 1 ? 1 : (chunks < kBlocks ? chunks : kBlocks);
    if (op == ClipOp::Norm) k_sum_squares<CAP><<<grid, 256, 0, st>>>(a);
    else if (op == ClipOp::Scale) k_clip_scale<CAP><<<grid, 256, 0, st>>>(a);
    else k_adamw_clip<CAP><<<grid, 256, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

size_t clip_workspace_bytes(int count, const int64_t *n) {
    const long long chunk = chunk_elements(count, n);
    size_t chunks = 0;
    for (int i = 0; i < count; ++i) chunks += (size_t)((n[i] + chunk - 1) / chunk);
    return 256 + 8 * chunks;
}

cudaError_t launch_clip(const ClipTensors &t, ClipOp op, const ClipHyper &h, float *norm, float *norm_each,
                        void *workspace, cudaStream_t st) {
    auto fill = [&](auto &a) {
        a.ticket = (unsigned *)workspace;
        a.result = (ClipResult *)((char *)workspace + 64);
        a.partial = (double *)((char *)workspace + 256);
        a.norm = norm;
        a.max_norm = h.max_norm;
        a.step = op == ClipOp::Norm || op == ClipOp::Adamw ? h.step : nullptr;
        a.lr_dev = h.lr_dev;
        a.lr = (float)h.lr;
        a.b1 = (float)h.b1;
        a.b2 = (float)h.b2;
        a.one_b1 = (float)(1.0 - h.b1);
        a.one_b2 = (float)(1.0 - h.b2);
        a.ln_b1 = (float)log(h.b1);
        a.ln_b2 = (float)log(h.b2);
        a.eps = (float)h.eps;
        a.wd = (float)h.wd;
        a.chunk = chunk_elements(t.count, t.n);
    };
    for (int begin = 0, launch = 0; begin < t.count; begin += kClipMaxTensors, ++launch) {
        const int count = t.count - begin < kClipMaxTensors ? t.count - begin : kClipMaxTensors;
        cudaError_t e;
        if (count <= kClipFewTensors) {
            ClipArgs<kClipFewTensors> a{};
            fill(a);
            a.launch = launch;
            a.last_launch = begin + count == t.count;
            a.norm_each = norm_each ? norm_each + begin : nullptr;
            e = launch_group(t, op, begin, count, a, st);
        } else {
            ClipArgs<kClipMaxTensors> a{};
            fill(a);
            a.launch = launch;
            a.last_launch = begin + count == t.count;
            a.norm_each = norm_each ? norm_each + begin : nullptr;
            e = launch_group(t, op, begin, count, a, st);
        }
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace dstd
