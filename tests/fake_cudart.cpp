// Stands in for the CUDA runtime's calls that the cache's entry points make on the host, so that
// their set-up can be watched without a GPU: loaded before libfdllm.so, its definitions come first.
// Kernels are not run; a launch is refused as the runtime would refuse it, where its shared memory
// was not asked for on the current device.
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstring>
#include <map>
#include <utility>
#include <vector>

namespace {
int device = 0;       // the current device
int fail_in = 0;      // the so manieth of the next set-up calls fails (0: none)
int launches = 0;
int programmatic = 0;          // of them, programmatic dependents, since the last capture began
bool reject_programmatic = false;
int instantiated = 0;
bool maps_fail = false;
std::map<std::pair<int, const void *>, int> shared_limit;  // of (device, kernel)
struct Map {
    int rank;
    unsigned long long dims[5], strides[5];
    unsigned box[5];
};
std::vector<Map> maps;  // tensor maps encoded so far

bool fails() { return fail_in > 0 && --fail_in == 0; }

CUresult encode(CUtensorMap *m, CUtensorMapDataType, cuuint32_t rank, void *, const cuuint64_t *dims,
                const cuuint64_t *strides, const cuuint32_t *box, const cuuint32_t *,
                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                CUtensorMapFloatOOBfill)
{
    if (maps_fail)
        return CUDA_ERROR_INVALID_VALUE;
    Map r = {};
    r.rank = (int)rank;
    for (unsigned i = 0; i < rank; ++i) {
        // the driver's own limits
        if (dims[i] < 1 || dims[i] > (1ull << 32) || box[i] < 1 || box[i] > 256)
            return CUDA_ERROR_INVALID_VALUE;
        if (i + 1 < rank && (strides[i] % 16 != 0 || strides[i] >= (1ull << 40)))
            return CUDA_ERROR_INVALID_VALUE;
        r.dims[i] = dims[i];
        r.box[i] = box[i];
        r.strides[i] = i + 1 < rank ? strides[i] : 0;
    }
    maps.push_back(r);
    std::memset(m, 0, sizeof *m);
    return CUDA_SUCCESS;
}
}  // namespace

extern "C" {

void fake_set_device(int d) { device = d; }
void fake_fail(int n) { fail_in = n; }
int fake_failed() { return fail_in == 0; }
void fake_maps_fail(int x) { maps_fail = x != 0; }
int fake_launches() { return launches; }
int fake_programmatic() { return programmatic; }
void fake_reject_programmatic(int x) { reject_programmatic = x != 0; }
int fake_instantiated() { return instantiated; }
int fake_maps() { return (int)maps.size(); }
unsigned long long fake_map(int i, int what, int axis)
{
    const Map &m = maps[i];
    return what == 0 ? m.rank : what == 1 ? m.dims[axis] : what == 2 ? m.strides[axis] : m.box[axis];
}

cudaError_t cudaGetDevice(int *d)
{
    *d = device;
    return cudaSuccess;
}
cudaError_t cudaSetDevice(int d)
{
    device = d;
    return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int *value, cudaDeviceAttr, int)
{
    *value = 152;
    return cudaSuccess;
}
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes *a, const void *)
{
    std::memset(a, 0, sizeof *a);
    a->numRegs = 255;
    return fails() ? cudaErrorUnknown : cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void *f, cudaFuncAttribute what, int value)
{
    if (fails())
        return cudaErrorUnknown;
    if (what == cudaFuncAttributeMaxDynamicSharedMemorySize)
        shared_limit[{device, f}] = value;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *f, void **)
{
    const auto at = shared_limit.find({device, f});
    const int limit = at == shared_limit.end() ? 48 * 1024 : at->second;
    if ((long long)c->dynamicSmemBytes > limit)
        return cudaErrorInvalidValue;
    ++launches;
    for (unsigned i = 0; i < c->numAttrs; ++i)
        programmatic += c->attrs[i].id == cudaLaunchAttributeProgrammaticStreamSerialization &&
                        c->attrs[i].val.programmaticStreamSerializationAllowed;
    return cudaSuccess;
}
cudaError_t cudaGetSymbolAddress(void **p, const void *)
{
    static unsigned words[64];
    *p = &words[device];
    return fails() ? cudaErrorUnknown : cudaSuccess;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **f, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult *q)
{
    if (fails())
        return cudaErrorUnknown;
    *f = reinterpret_cast<void *>(&encode);
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

// What a device-resident loop needs besides: a graph that is refused, where it has programmatic
// edges, and memory that reads as 0.
cudaError_t __cudaGetKernel(cudaKernel_t *k, const void *f)
{
    *k = static_cast<cudaKernel_t>(const_cast<void *>(f));
    return cudaSuccess;
}
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void **, size_t, cudaStream_t)
{
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int *n, const void *, int, size_t, unsigned)
{
    *n = 1;
    return cudaSuccess;
}
cudaError_t cudaMalloc(void **p, size_t)
{
    static char memory[1 << 20];
    *p = memory;
    return cudaSuccess;
}
cudaError_t cudaFree(void *) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *, int, size_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void *to, const void *, size_t n, cudaMemcpyKind, cudaStream_t)
{
    std::memset(to, 0, n);
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamCreateWithFlags(cudaStream_t *s, unsigned)
{
    *s = reinterpret_cast<cudaStream_t>(0x1000);
    return cudaSuccess;
}
cudaError_t cudaStreamDestroy(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGraphCreate(cudaGraph_t *g, unsigned)
{
    *g = reinterpret_cast<cudaGraph_t>(0x2000);
    return cudaSuccess;
}
cudaError_t cudaGraphConditionalHandleCreate(cudaGraphConditionalHandle *h, cudaGraph_t, unsigned, unsigned)
{
    *h = 1;
    return cudaSuccess;
}
cudaError_t cudaGraphAddNode(cudaGraphNode_t *, cudaGraph_t, const cudaGraphNode_t *,
                             const cudaGraphEdgeData *, size_t, cudaGraphNodeParams *p)
{
    static cudaGraph_t body[1] = {reinterpret_cast<cudaGraph_t>(0x3000)};
    p->conditional.phGraph_out = body;
    return cudaSuccess;
}
cudaError_t cudaStreamBeginCaptureToGraph(cudaStream_t, cudaGraph_t, const cudaGraphNode_t *,
                                          const cudaGraphEdgeData *, size_t, cudaStreamCaptureMode)
{
    programmatic = 0;
    return cudaSuccess;
}
cudaError_t cudaStreamEndCapture(cudaStream_t, cudaGraph_t *) { return cudaSuccess; }
cudaError_t cudaGraphInstantiate(cudaGraphExec_t *e, cudaGraph_t, unsigned long long)
{
    if (reject_programmatic && programmatic > 0)
        return cudaErrorNotSupported;
    ++instantiated;
    *e = reinterpret_cast<cudaGraphExec_t>(0x4000);
    return cudaSuccess;
}
cudaError_t cudaGraphExecDestroy(cudaGraphExec_t) { return cudaSuccess; }
cudaError_t cudaGraphDestroy(cudaGraph_t) { return cudaSuccess; }
cudaError_t cudaGraphLaunch(cudaGraphExec_t, cudaStream_t) { return cudaSuccess; }

}  // extern "C"
