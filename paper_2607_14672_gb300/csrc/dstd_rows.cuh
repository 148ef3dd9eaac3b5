// What the kernels over rows of several element types share: dependent launches,
// conversion to fp32, 16-byte pieces.
#pragma once

#include "dstd_internal.cuh"

namespace dstd {

// Dependent launch. A grid launched with launch_dependent may start while the
// one before it in the stream still runs, from when all of that one's blocks
// have called let_next_launch (or ended); what that one writes, and what was
// there before it, is there after wait_launch_before. A grid that lets the next
// one start was launched without this, or has itself waited first: nothing older
// is still running then.
__device__ __forceinline__ void wait_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <class... P, class... A>
cudaError_t launch_dependent(void (*kernel)(P...), unsigned grid, unsigned block, cudaStream_t st, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <class T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }

template <class O>
__device__ __forceinline__ O round_out(float y);
template <>
__device__ __forceinline__ float round_out<float>(float y) { return y; }
template <>
__device__ __forceinline__ __nv_bfloat16 round_out<__nv_bfloat16>(float y) { return __float2bfloat16_rn(y); }
template <>
__device__ __forceinline__ __half round_out<__half>(float y) { return __float2half_rn(y); }

// 16 bytes of a type, kept as they are until used (a 16-bit row takes half the registers)
template <class T>
struct Pack {
    static constexpr int P = 16 / sizeof(T);
    static __device__ __forceinline__ float one(const uint4 &u, int i) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(w[i]);
        } else {
            const unsigned short h = (unsigned short)(w[i / 2] >> (16 * (i & 1)));
            return to_f32<T>(*reinterpret_cast<const T *>(&h));
        }
    }
};

}  // namespace dstd
