// A CUDA runtime of several devices that runs nothing: the library's objects
// linked against it show, on a machine without a GPU, what their host code asks
// for. Every launch is written down (the kernel's name, grid, block, dynamic
// shared memory, device); one that asks for more dynamic shared memory than the
// kernel has been granted on the present device fails, as it does in earnest.
#include <cuda_runtime_api.h>
#include <string.h>

#include <map>
#include <string>
#include <utility>
#include <vector>

namespace {

constexpr int DEVICES = 3;
constexpr int kSms[DEVICES] = {152, 152, 100}, kClusters[DEVICES] = {76, 76, 50}, kBlocks[DEVICES] = {4, 4, 3};

struct Launch {
    const void *func;
    dim3 grid, block;
    size_t shared;
    int device, cooperative;
    unsigned char arg2[64];  // the start of the third argument, where it was asked for
};

struct State {
    std::map<const void *, std::string> names;
    std::map<std::pair<int, const void *>, int> granted;
    std::vector<Launch> launches;
    std::string keep_arg2_of;
    int device = 0, refuse_attribute = 0, refuse_occupancy = 0;
    dim3 grid, block;
    size_t shared = 0;
    cudaStream_t stream = nullptr;
};
State &st() {
    static State s;
    return s;
}

cudaError_t launch(const void *func, dim3 grid, dim3 block, size_t shared, void **args, int cooperative) {
    State &s = st();
    if (shared > 48 * 1024) {
        const auto it = s.granted.find({s.device, func});
        if (it == s.granted.end() || (size_t)it->second < shared) return cudaErrorInvalidValue;
    }
    if (grid.x < 1 || grid.x > 0x7fffffffu) return cudaErrorInvalidConfiguration;
    Launch l{func, grid, block, shared, s.device, cooperative, {}};
    if (args && !s.keep_arg2_of.empty() && s.names[func].find(s.keep_arg2_of) != std::string::npos)
        memcpy(l.arg2, args[2], sizeof(l.arg2));
    s.launches.push_back(l);
    return cudaSuccess;
}

int encode_tiled() { return 0; }

}  // namespace

extern "C" {

// what a test says and asks
void fake_reset() {
    st().launches.clear();
    st().device = st().refuse_attribute = st().refuse_occupancy = 0;
    st().keep_arg2_of.clear();
}
void fake_device(int d) { st().device = d; }
void fake_refuse_attributes(int calls) { st().refuse_attribute = calls; }
void fake_refuse_occupancy(int calls) { st().refuse_occupancy = calls; }
void fake_keep_arg2_of(const char *name) { st().keep_arg2_of = name; }
int fake_launches() { return (int)st().launches.size(); }
const char *fake_name(int i) { return st().names[st().launches[i].func].c_str(); }
unsigned fake_grid(int i) { return st().launches[i].grid.x; }
unsigned fake_block(int i) { return st().launches[i].block.x; }
int fake_launch_device(int i) { return st().launches[i].device; }
int fake_cooperative(int i) { return st().launches[i].cooperative; }
const unsigned char *fake_arg2(int i) { return st().launches[i].arg2; }

// the compiler's registration and launch calls
void **__cudaRegisterFatBinary(void *) {
    static void *handle;
    return &handle;
}
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterVar(void **, char *, char *, const char *, int, size_t, int, int) {}
void __cudaRegisterFunction(void **, const char *host, char *, const char *name, int, uint3 *, uint3 *, dim3 *, dim3 *,
                            int *) {
    st().names[host] = name;
}
unsigned __cudaPushCallConfiguration(dim3 grid, dim3 block, size_t shared, CUstream_st *stream) {
    st().grid = grid;
    st().block = block;
    st().shared = shared;
    st().stream = stream;
    return 0;
}
cudaError_t __cudaPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, void *stream) {
    *grid = st().grid;
    *block = st().block;
    *shared = st().shared;
    *static_cast<cudaStream_t *>(stream) = st().stream;
    return cudaSuccess;
}
cudaError_t __cudaGetKernel(cudaKernel_t *kernel, const void *func) {
    *kernel = (cudaKernel_t)func;
    return cudaSuccess;
}
cudaError_t __cudaLaunchKernel(cudaKernel_t kernel, dim3 grid, dim3 block, void **args, size_t shared, cudaStream_t) {
    return launch(kernel, grid, block, shared, args, 0);
}

// the runtime
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *func, void **args) {
    int cooperative = 0;
    for (unsigned i = 0; i < c->numAttrs; ++i)
        if (c->attrs[i].id == cudaLaunchAttributeCooperative) cooperative = c->attrs[i].val.cooperative;
    return launch(func, c->gridDim, c->blockDim, c->dynamicSmemBytes, args, cooperative);
}
cudaError_t cudaGetDevice(int *d) {
    *d = st().device;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr a, int d) {
    if (d < 0 || d >= DEVICES) return cudaErrorInvalidDevice;
    *v = a == cudaDevAttrComputeCapabilityMajor ? 10
         : a == cudaDevAttrComputeCapabilityMinor ? 3
         : a == cudaDevAttrMultiProcessorCount ? kSms[d] : 0;
    return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void *func, cudaFuncAttribute a, int value) {
    if (st().refuse_attribute > 0) {
        --st().refuse_attribute;
        return cudaErrorUnknown;
    }
    if (a == cudaFuncAttributeMaxDynamicSharedMemorySize) st().granted[{st().device, func}] = value;
    return cudaSuccess;
}
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes *a, const void *) {
    memset(a, 0, sizeof(*a));
    a->numRegs = 96;
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *, const cudaLaunchConfig_t *) {
    if (st().refuse_occupancy > 0) {
        --st().refuse_occupancy;
        return cudaErrorUnknown;
    }
    *n = kClusters[st().device];
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int *n, const void *, int, size_t, unsigned) {
    if (st().refuse_occupancy > 0) {
        --st().refuse_occupancy;
        return cudaErrorUnknown;
    }
    *n = kBlocks[st().device];
    return cudaSuccess;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **f, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult *q) {
    *f = (void *)encode_tiled;
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaDeviceSynchronize() { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemcpyFromSymbol(void *to, const void *, size_t n, size_t, cudaMemcpyKind) {
    memset(to, 0, n);
    return cudaSuccess;
}
cudaError_t cudaMemcpyToSymbol(const void *, const void *, size_t, size_t, cudaMemcpyKind) { return cudaSuccess; }
cudaError_t cudaGetSymbolAddress(void **p, const void *) {
    *p = (void *)256;
    return cudaSuccess;
}
cudaError_t cudaEventCreate(cudaEvent_t *e) {
    *e = (cudaEvent_t)256;
    return cudaSuccess;
}
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *, unsigned) { return cudaErrorUnknown; }
cudaError_t cudaEventElapsedTime(float *ms, cudaEvent_t, cudaEvent_t) {
    *ms = 1.0f;
    return cudaSuccess;
}
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventRecordWithFlags(cudaEvent_t, cudaStream_t, unsigned) { return cudaErrorUnknown; }
cudaError_t cudaStreamCreateWithFlags(cudaStream_t *, unsigned) { return cudaErrorUnknown; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus *s) {
    *s = cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaErrorUnknown; }

}  // extern "C"
