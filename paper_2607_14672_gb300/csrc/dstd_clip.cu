// The optimiser's side of a training step over many gradient tensors: their
// global norm, clipping by it, and the clipped AdamW update. All of it is bound
// by memory: the norm has to be known before the first gradient is scaled, so
// gradients are read twice, the second time from L2 as far as they fit. Long
// lists (us a call among others): norm of 268 M bf16 gradients 83 (6.5 TB/s),
// clipped copies 274 (5.9 TB/s over three passes), their AdamW step 1229 (6.1 TB/s
// with both reads).
#include "dstd_internal.cuh"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace dstd {

__device__ unsigned int g_status_clip = 0;

namespace {

constexpr int THREADS = 256;

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

// Elements are taken four at a time (16 bytes of fp32, 8 of a 16-bit type).
template <class T>
struct Four;
template <>
struct Four<float> {
    static constexpr uintptr_t MASK = 15;
    static __device__ __forceinline__ float4 load(const float *p) { return *reinterpret_cast<const float4 *>(p); }
    static __device__ __forceinline__ void store(float *p, float4 x) { *reinterpret_cast<float4 *>(p) = x; }
    static __device__ __forceinline__ float one(float x) { return x; }
    static __device__ __forceinline__ float round(float x) { return x; }
};
template <>
struct Four<__nv_bfloat16> {
    static constexpr uintptr_t MASK = 7;
    static __device__ __forceinline__ float4 load(const __nv_bfloat16 *p) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                           __uint_as_float(u.y & 0xffff0000u));
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, float4 x) {
        uint2 u;
        *reinterpret_cast<__nv_bfloat162 *>(&u.x) = __floats2bfloat162_rn(x.x, x.y);
        *reinterpret_cast<__nv_bfloat162 *>(&u.y) = __floats2bfloat162_rn(x.z, x.w);
        *reinterpret_cast<uint2 *>(p) = u;
    }
    static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Four<__half> {
    static constexpr uintptr_t MASK = 7;
    static __device__ __forceinline__ float4 load(const __half *p) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        const float2 lo = __half22float2(*reinterpret_cast<const __half2 *>(&u.x));
        const float2 hi = __half22float2(*reinterpret_cast<const __half2 *>(&u.y));
        return make_float4(lo.x, lo.y, hi.x, hi.y);
    }
    static __device__ __forceinline__ void store(__half *p, float4 x) {
        uint2 u;
        *reinterpret_cast<__half2 *>(&u.x) = __floats2half2_rn(x.x, x.y);
        *reinterpret_cast<__half2 *>(&u.y) = __floats2half2_rn(x.z, x.w);
        *reinterpret_cast<uint2 *>(p) = u;
    }
    static __device__ __forceinline__ float one(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half round(float x) { return __float2half_rn(x); }
};

template <class T>
__device__ __forceinline__ bool fits(const T *p, int head) {
    return ((reinterpret_cast<uintptr_t>(p + head)) & Four<T>::MASK) == 0;
}

// 16 bytes of a type: P elements
template <class T>
struct Pack {
    static constexpr int P = 16 / sizeof(T);
    static __device__ __forceinline__ float one(const uint4 &u, int i) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(w[i]);
        } else {
            const unsigned short h = (unsigned short)(w[i / 2] >> (16 * (i & 1)));
            return Four<T>::one(*reinterpret_cast<const T *>(&h));
        }
    }
};

// loads that the compiler keeps together, so that a thread has all of a run's on their way at once
__device__ __forceinline__ uint4 load16(const void *p) {
    uint4 u;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
    return u;
}

// A sum as an unevaluated pair of fp32 numbers, |lo| <= ulp(hi) / 2. 64-bit
// arithmetic is slow on this part (two operations a cycle and SM: a block-wide
// sum of doubles took longer than reading the block's gradients), so only the
// chunks' results become doubles.
struct Pair {
    float hi, lo;
    __device__ __forceinline__ void add(float x) {
        const float t = hi + x, z = t - hi;
        lo += (hi - (t - z)) + (x - z);
        hi = t;
    }
    __device__ __forceinline__ void add(float h, float l) {
        add(h);
        lo += l;
    }
};

// A thread's share of the chunk's sum of squares. Squares are added in plain
// fp32 in runs of four packs (16 fp32 or 32 16-bit elements), whose sums go into
// the pair. A run whose sum leaves the range where fp32 squares are good is formed
// again in 64 bits, into `rare`, which is slow. Runs of zeros are not: silent
// neurons leave whole rows of them in a network's gradients (268 M zeros took 985
// us that way, as many other numbers 157).
template <class T>
__device__ __forceinline__ void chunk_squares(const T *g, long long n, Pair &s, double &rare) {
    constexpr int P = Pack<T>::P, RUN = 4;
    constexpr uint32_t MAGNITUDE = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
    const int tid = threadIdx.x;
    int head = 0;
    while ((reinterpret_cast<uintptr_t>(g + head) & 15) != 0) ++head;
    if (head > n) head = (int)n;
    const T *p = g + head;
    const long long packs = (n - head) / P;
    for (long long base = tid; base < packs; base += THREADS * RUN) {
        float f = 0.f;
        uint32_t bits = 0;
        if (base + THREADS * (RUN - 1) < packs) {
            uint4 u[RUN];
#pragma unroll
            for (int i = 0; i < RUN; ++i) u[i] = load16(p + P * (base + THREADS * i));
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                bits |= u[i].x | u[i].y | u[i].z | u[i].w;
#pragma unroll
                for (int e = 0; e < P; ++e) f = fmaf(Pack<T>::one(u[i], e), Pack<T>::one(u[i], e), f);
            }
        } else {
#pragma unroll
            for (int i = 0; i < RUN; ++i)
                if (base + THREADS * i < packs) {
                    const uint4 u = load16(p + P * (base + THREADS * i));
                    bits |= u.x | u.y | u.z | u.w;
#pragma unroll
                    for (int e = 0; e < P; ++e) f = fmaf(Pack<T>::one(u, e), Pack<T>::one(u, e), f);
                }
        }
        if (f > 1e-30f && f < 1e30f) {
            s.add(f);
        } else if ((bits & MAGNITUDE) != 0) {
#pragma unroll 1
            for (int i = 0; i < RUN * P; ++i) {
                const long long at = base + THREADS * (i / P);
                if (at >= packs) break;
                const float x = Four<T>::one(p[P * at + i % P]);
                if (x != 0.f) rare += (double)x * x;
            }
        }
    }
    // less than a pack at each end
    const long long done = head + P * packs;
    for (int e = 0; e < 2; ++e) {
        const long long i = e == 0 ? tid : done + tid;
        if (e == 0 ? tid < head : i < n) {
            const float x = Four<T>::one(g[i]);
            if (x != 0.f) rare += (double)x * x;
        }
    }
}

struct SumShared {
    float hi[THREADS / 32], lo[THREADS / 32];
    double rare[THREADS / 32];
};
// Sums of squares of this block's chunks (blockIdx.x, + gridDim.x, ...), each
// into its own slot: no atomics on the sums, so that the result does not depend
// on the order in which blocks run.
template <class A>
__device__ __forceinline__ void sum_chunks(const A &a, SumShared &sh) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (unsigned c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipSeg &sg = a.seg[seg_of(a, c)];
        const long long lo = (long long)(c - sg.first) * a.chunk;
        const long long n = lo + a.chunk < sg.n ? a.chunk : sg.n - lo;
        Pair s{0.f, 0.f};
        double rare = 0.0;
        if (sg.type == DSTD_TYPE_F32) chunk_squares((const float *)sg.g + lo, n, s, rare);
        else if (sg.type == DSTD_TYPE_BF16) chunk_squares((const __nv_bfloat16 *)sg.g + lo, n, s, rare);
        else chunk_squares((const __half *)sg.g + lo, n, s, rare);
        const bool any = __syncthreads_or(rare != 0.0);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            s.add(__shfl_down_sync(0xffffffffu, s.hi, o), __shfl_down_sync(0xffffffffu, s.lo, o));
        if (any) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) rare += __shfl_down_sync(0xffffffffu, rare, o);
        }
        if (lane == 0) {
            sh.hi[warp] = s.hi;
            sh.lo[warp] = s.lo;
            sh.rare[warp] = rare;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < THREADS / 32; ++w) s.add(sh.hi[w], sh.lo[w]);
            if (any)
                for (int w = 1; w < THREADS / 32; ++w) rare += sh.rare[w];
            a.partial[c] = (double)s.hi + (double)s.lo + rare;
        }
        __syncthreads();
    }
}
// the slots' sum, by one warp (lane 0 has it)
template <class A>
__device__ __forceinline__ double sum_slots(const A &a) {
    double s = 0.0;
#pragma unroll 8
    for (unsigned c = threadIdx.x & 31; c < a.chunks; c += 32) s += __ldcg(a.partial + c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
    return s;
}
__device__ __forceinline__ ClipFactor clip_factor(double norm, double max_norm) {
    if (!isfinite(norm) || !(norm > max_norm)) return ClipFactor{1.f, 1.f};
    const double c = max_norm / norm;
    return c >= 0x1p-126 ? ClipFactor{(float)c, 1.f} : ClipFactor{(float)(c * 0x1p126), 0x1p-126f};
}
// a < 1 where b is not 1: nothing overflows on the way
__device__ __forceinline__ float clipped(float g, ClipFactor c) { return g * c.a * c.b; }

// The norm by itself: the block that draws the last ticket adds the slots in
// order, and derives from the total what the clipping needs.
template <int CAP>
__global__ void __launch_bounds__(THREADS) k_sum_squares(const ClipArgs<CAP> a) {
    __shared__ SumShared sh;
    __shared__ bool s_last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // the pass that applies the norm may be launched while this one runs
    asm volatile("griddepcontrol.launch_dependents;");
    sum_chunks(a, sh);
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    if (a.norm_each) {
        for (int i = warp; i < a.count; i += THREADS / 32) {
            const unsigned end = i + 1 < a.count ? a.seg[i + 1].first : a.chunks;
            double e = 0.0;
            for (unsigned c = a.seg[i].first + lane; c < end; c += 32) e += a.partial[c];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) e += __shfl_down_sync(0xffffffffu, e, o);
            if (lane == 0) a.norm_each[i] = (float)sqrt(e);
        }
    }
    if (warp != 0) return;
    const double s = sum_slots(a);
    if (lane == 0) {
        *a.ticket = 0;
        const double sum = (a.launch == 0 ? 0.0 : a.result->sum) + s;
        a.result->sum = sum;
        if (a.last_launch) {
            const double norm = sqrt(sum);
            a.norm[0] = (float)norm;
            a.result->coef = clip_factor(norm, a.max_norm);
            a.result->skip = isfinite(norm) ? 0 : 1;
            if (a.step && isfinite(norm)) a.step[0] += 1;
        }
    }
}

// The passes after the norm take each chunk from its end: the norm read it from
// its start, so what of the gradients is still in L2 is at the ends.
template <class T>
__device__ __forceinline__ void scale_chunk(const T *g, T *out, long long n, ClipFactor coef) {
    const int tid = threadIdx.x;
    int head = 0;
    while (head < 4 && !(fits(g, head) && fits(out, head))) ++head;
    if (head == 4 || n < 4) {  // the two are placed differently (or hardly anything is there)
#pragma unroll 4
        for (long long i = tid; i < n; i += THREADS) out[i] = Four<T>::round(clipped(Four<T>::one(g[i]), coef));
        return;
    }
    const long long fours = (n - head) / 4, done = head + 4 * fours;
    if (tid < head) out[tid] = Four<T>::round(clipped(Four<T>::one(g[tid]), coef));
    if (done + tid < n) out[done + tid] = Four<T>::round(clipped(Four<T>::one(g[done + tid]), coef));
    const T *p = g + head;
    T *q = out + head;
    for (long long base = fours - 1 - tid; base >= 0; base -= THREADS * 4) {
        float4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (base - THREADS * i >= 0) x[i] = Four<T>::load(p + 4 * (base - THREADS * i));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (base - THREADS * i >= 0)
                Four<T>::store(q + 4 * (base - THREADS * i),
                               make_float4(clipped(x[i].x, coef), clipped(x[i].y, coef), clipped(x[i].z, coef),
                                           clipped(x[i].w, coef)));
    }
}

template <class A>
__device__ __forceinline__ void scale_chunks(const A &a, ClipFactor coef) {
    for (unsigned c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipSeg &sg = a.seg[seg_of(a, c)];
        if (coef.a == 1.f && coef.b == 1.f && sg.out == sg.g) continue;
        const long long lo = (long long)(c - sg.first) * a.chunk;
        const long long n = lo + a.chunk < sg.n ? a.chunk : sg.n - lo;
        if (sg.type == DSTD_TYPE_F32) scale_chunk((const float *)sg.g + lo, (float *)sg.out + lo, n, coef);
        else if (sg.type == DSTD_TYPE_BF16)
            scale_chunk((const __nv_bfloat16 *)sg.g + lo, (__nv_bfloat16 *)sg.out + lo, n, coef);
        else scale_chunk((const __half *)sg.g + lo, (__half *)sg.out + lo, n, coef);
    }
}

struct StepConst {
    ClipFactor coef;
    float b1, one_b1, b2, one_b2, bc1, bc2, lr, decay, eps;
};
__device__ __forceinline__ void adamw_one(const StepConst &c, float g, float &w, float &m, float &v) {
    g = clipped(g, c.coef);
    m = c.b1 * m + c.one_b1 * g;
    v = c.b2 * v + c.one_b2 * (g * g);
    w = w * c.decay - c.lr * (m / c.bc1) / (sqrtf(v / c.bc2) + c.eps);
}

template <class T>
__device__ __forceinline__ void adamw_chunk(const StepConst &c, const T *g, float *w, float *m, float *v, long long n) {
    const int tid = threadIdx.x;
    int head = 0;
    while (head < 4 && !(fits(g, head) && fits(w, head) && fits(m, head) && fits(v, head))) ++head;
    if (head == 4 || n < 4) {  // the four are placed differently (or hardly anything is there)
        for (long long i = tid; i < n; i += THREADS) {
            float wi = w[i], mi = m[i], vi = v[i];
            adamw_one(c, Four<T>::one(g[i]), wi, mi, vi);
            w[i] = wi;
            m[i] = mi;
            v[i] = vi;
        }
        return;
    }
    const long long fours = (n - head) / 4, done = head + 4 * fours;
    if (tid < head || done + tid < n) {  // less than four at each end
        for (int e = 0; e < 2; ++e) {
            const long long i = e == 0 ? tid : done + tid;
            if (e == 0 ? tid < head : i < n) adamw_one(c, Four<T>::one(g[i]), w[i], m[i], v[i]);
        }
    }
    for (long long base = fours - 1 - tid; base >= 0; base -= THREADS * 2) {
        float4 gx[2], wx[2], mx[2], vx[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const long long at = head + 4 * (base - THREADS * i);
            if (base - THREADS * i < 0) break;
            gx[i] = Four<T>::load(g + at);
            wx[i] = Four<float>::load(w + at);
            mx[i] = Four<float>::load(m + at);
            vx[i] = Four<float>::load(v + at);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const long long at = head + 4 * (base - THREADS * i);
            if (base - THREADS * i < 0) break;
            adamw_one(c, gx[i].x, wx[i].x, mx[i].x, vx[i].x);
            adamw_one(c, gx[i].y, wx[i].y, mx[i].y, vx[i].y);
            adamw_one(c, gx[i].z, wx[i].z, mx[i].z, vx[i].z);
            adamw_one(c, gx[i].w, wx[i].w, mx[i].w, vx[i].w);
            Four<float>::store(w + at, wx[i]);
            Four<float>::store(m + at, mx[i]);
            Four<float>::store(v + at, vx[i]);
        }
    }
}

// t: updates done with this one
template <class A>
__device__ __forceinline__ void adamw_chunks(const A &a, ClipFactor coef, float t) {
    StepConst k;
    k.coef = coef;
    k.b1 = a.b1;
    k.one_b1 = a.one_b1;
    k.b2 = a.b2;
    k.one_b2 = a.one_b2;
    // 1 - beta^t without the cancellation of a beta near 1
    k.bc1 = -expm1f(t * a.ln_b1);
    k.bc2 = -expm1f(t * a.ln_b2);
    k.lr = a.lr_dev ? *a.lr_dev : a.lr;
    k.decay = 1.f - k.lr * a.wd;
    k.eps = a.eps;
    for (unsigned c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipSeg &sg = a.seg[seg_of(a, c)];
        const long long lo = (long long)(c - sg.first) * a.chunk;
        const long long n = lo + a.chunk < sg.n ? a.chunk : sg.n - lo;
        float *w = (float *)sg.out + lo, *m = sg.m + lo, *v = sg.v + lo;
        if (sg.type == DSTD_TYPE_F32) adamw_chunk(k, (const float *)sg.g + lo, w, m, v, n);
        else if (sg.type == DSTD_TYPE_BF16)
            adamw_chunk(k, (const __nv_bfloat16 *)sg.g + lo, w, m, v, n);
        else adamw_chunk(k, (const __half *)sg.g + lo, w, m, v, n);
    }
}

// The passes after k_sum_squares.
template <int CAP, bool STEP>
__global__ void __launch_bounds__(THREADS) k_clip_apply(const ClipArgs<CAP> a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");  // for the norm
    if constexpr (STEP) {
        if (!a.result->skip) adamw_chunks(a, a.result->coef, (float)a.step[0]);
    } else {
        scale_chunks(a, a.result->coef);
    }
}

// Short lists: norm and pass in one cooperative launch. Every block leaves its
// sums, waits for the others', and adds up all slots itself, in the same order:
// no ticket, no last block that the rest waits for, and no second launch
// (asking for the update's other operands in L2 before the wait made it slower).
// The wait ends by itself after about 2 s; a block whose wait ran out changes
// nothing and sets the status word.
template <int CAP, bool STEP>
__global__ void __launch_bounds__(THREADS, 2) k_clip_once(const ClipArgs<CAP> a) {
    __shared__ SumShared sh;
    __shared__ ClipFactor s_coef;
    __shared__ int s_go;
    unsigned *arrived = a.ticket + 1, *left = a.ticket + 2;
    const float t = STEP ? (float)(a.step[0] + 1) : 0.f;
    sum_chunks(a, sh);
    if (threadIdx.x == 0) {
        __threadfence();
        atomicAdd(arrived, 1u);
        int go = 1;
        const long long t0 = clock64();
        for (;;) {
            unsigned n;
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(n) : "l"(arrived) : "memory");
            if (n >= gridDim.x) break;
            if (clock64() - t0 > 4000000000ll) {
                go = 0;
                atomicOr(&g_status_clip, STATUS_TIMEOUT);
                break;
            }
        }
        s_go = go;
    }
    __syncthreads();
    if (s_go && threadIdx.x < 32) {
        const double sum = sum_slots(a);
        if (threadIdx.x == 0) {
            const double norm = sqrt(sum);
            s_coef = clip_factor(norm, a.max_norm);
            if (STEP && !isfinite(norm)) s_go = 0;
            if (blockIdx.x == 0) a.norm[0] = (float)norm;
        }
    }
    __syncthreads();
    if (s_go) {
        if constexpr (STEP) adamw_chunks(a, s_coef, t);
        else scale_chunks(a, s_coef);
    }
    if (threadIdx.x == 0) {
        // the last block to leave: every other one has read the count and the slots
        if (atomicAdd(left, 1u) == gridDim.x - 1) {
            *arrived = 0;
            *left = 0;
            if (STEP && s_go) a.step[0] += 1;
        }
    }
}

constexpr int kBlocks = 152 * 6;
constexpr int kOnceBlocks = 152 * 4;                    // at most, of the one-launch form
// longer lists take two launches: of a step, and of a clipping (whose second pass is too short to gain by it)
constexpr long long kOnceStep = 1ll << 24, kOnceClip = 1ll << 19;

// elements of a chunk: about one chunk per resident block. For the norm in
// multiples of 4096 (four 16-byte loads of fp32 a thread): small lists take
// fewer blocks, since the last one has to collect what the others leave. The
// passes after it take 2048 at least (one step of the update).
long long chunk_elements(int count, const int64_t *n, int least) {
    long long total = 0;
    for (int i = 0; i < count; ++i) total += n[i];
    const long long c = (total + kBlocks - 1) / kBlocks;
    return c < least ? least : (c + least - 1) / least * least;
}

template <int CAP>
void fill_segments(const ClipTensors &t, int begin, int count, ClipArgs<CAP> &a) {
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
}

template <int CAP>
cudaError_t launch_group(const ClipTensors &t, ClipOp op, int begin, int count, ClipArgs<CAP> &a, cudaStream_t st) {
    fill_segments(t, begin, count, a);
    const unsigned chunks = a.chunks;
    const unsigned grid = chunks < 1 ? 1 : (chunks < kBlocks ? chunks : kBlocks);
    if (op == ClipOp::Norm) {
        k_sum_squares<CAP><<<grid, THREADS, 0, st>>>(a);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = begin == 0 ? 1 : 0;  // the launch before this one is the norm's last
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, op == ClipOp::Scale ? k_clip_apply<CAP, false> : k_clip_apply<CAP, true>, a);
}

// blocks of the one-launch form that are resident at once (0: an error)
template <int CAP, bool STEP>
unsigned once_blocks() {
    static PerDevice blocks;
    return (unsigned)blocks.get([](int dev) {
        int sms = 0, each = 0;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, k_clip_once<CAP, STEP>, THREADS, 0) != cudaSuccess)
            return 0;
        return sms * std::min(each, kOnceBlocks / 152);
    });
}

template <int CAP, bool STEP>
cudaError_t launch_once(const ClipTensors &t, long long total, ClipArgs<CAP> &a, cudaStream_t st) {
    const unsigned blocks = std::min(once_blocks<CAP, STEP>(), (unsigned)kOnceBlocks);
    if (blocks == 0) return cudaErrorInvalidConfiguration;
    // one chunk a block where the list allows it: every tensor's last chunk may be a short one
    const long long share = blocks > 2u * t.count ? (total + blocks - t.count - 1) / (blocks - t.count)
                                                  : 2 * ((total + blocks - 1) / blocks);
    a.chunk = std::max(1024ll, (share + 63) / 64 * 64);
    fill_segments(t, 0, t.count, a);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(std::max(1u, std::min(a.chunks, blocks)));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, k_clip_once<CAP, STEP>, a);
}

}  // namespace

size_t clip_workspace_bytes(int count, const int64_t *n) {
    const long long chunk = chunk_elements(count, n, 4096);
    size_t chunks = 0;
    for (int i = 0; i < count; ++i) chunks += (size_t)((n[i] + chunk - 1) / chunk);
    // the one-launch form has at most a chunk a block and one more a tensor
    return 256 + 8 * std::max(chunks, (size_t)kOnceBlocks + (size_t)std::min(count, kClipMaxTensors));
}

cudaError_t clip_status_read(unsigned int *out, int clear) {
    cudaError_t e = cudaMemcpyFromSymbol(out, g_status_clip, sizeof(unsigned int));
    if (e != cudaSuccess || !clear) return e;
    unsigned int z = 0;
    return cudaMemcpyToSymbol(g_status_clip, &z, sizeof(z));
}

cudaError_t launch_clip(const ClipTensors &t, ClipOp op, const ClipHyper &h, float *norm, float *norm_each,
                        void *workspace, int &launches, cudaStream_t st) {
    auto fill = [&](auto &a, ClipOp pass) {
        a.ticket = (unsigned *)workspace;
        a.result = (ClipResult *)((char *)workspace + 64);
        a.partial = (double *)((char *)workspace + 256);
        a.norm = norm;
        a.max_norm = h.max_norm;
        a.step = h.step;
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
        a.chunk = chunk_elements(t.count, t.n, pass == ClipOp::Norm ? 4096 : 2048);
    };
    long long total = 0;
    for (int i = 0; i < t.count; ++i) total += t.n[i];
    // one launch against two, cold caches, without what any launch costs (us): a step of 100 thousand weights 6.5
    // and 8.5, 1.3 M 12.6 and 14.6, 4.7 M 26.9 and 29.0, 16 M 82 and 83, 67 M 343 and 333; clipping 100 thousand
    // gradients 4.4 and 5.4, 1.3 M 8.5 and 7.5
    if (op != ClipOp::Norm && t.count <= kClipMaxTensors && total <= (op == ClipOp::Adamw ? kOnceStep : kOnceClip)) {
        launches = 1;
        auto once = [&](auto &a) {
            fill(a, op);
            return op == ClipOp::Scale ? launch_once<std::extent_v<decltype(a.seg)>, false>(t, total, a, st)
                                       : launch_once<std::extent_v<decltype(a.seg)>, true>(t, total, a, st);
        };
        if (t.count <= kClipFewTensors) {
            ClipArgs<kClipFewTensors> a{};
            return once(a);
        }
        ClipArgs<kClipMaxTensors> a{};
        return once(a);
    }
    // the norm (whose last launch counts the update), then the pass
    launches = 0;
    for (int pass = 0; pass < (op == ClipOp::Norm ? 1 : 2); ++pass) {
        const ClipOp now = pass == 0 ? ClipOp::Norm : op;
        for (int begin = 0, launch = 0; begin < t.count; begin += kClipMaxTensors, ++launch) {
            const int count = std::min(t.count - begin, kClipMaxTensors);
            auto group = [&](auto &a) {
                fill(a, now);
                a.launch = launch;
                a.last_launch = begin + count == t.count;
                a.norm_each = norm_each ? norm_each + begin : nullptr;
                return launch_group(t, now, begin, count, a, st);
            };
            ++launches;
            cudaError_t e;
            if (count <= kClipFewTensors) {
                ClipArgs<kClipFewTensors> a{};
                e = group(a);
            } else {
                ClipArgs<kClipMaxTensors> a{};
                e = group(a);
            }
            if (e != cudaSuccess) return e;
        }
    }
    return cudaSuccess;
}

}  // namespace dstd
