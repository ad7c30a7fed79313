// A CUDA runtime for host tests: memory is host memory, nothing is launched, and the calls that order work
// (launches, events, waits) are written to a log.  The n-th launch can be made to fail.
#include <cuda.h>
#include <cuda_runtime_api.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

namespace {

enum Op : uint32_t { LAUNCH = 1, LAUNCH_FAILED = 2, RECORD = 3, WAIT = 4 };
struct Entry {
    uint32_t op, unused;
    uint64_t stream, event;
};
std::vector<Entry> entries;
int64_t fail_at = 0, launches = 0;
cudaError_t last_error = cudaSuccess;
cudaStream_t pushed_stream = nullptr;
uint64_t next_handle = 0x1000;

void note(Op op, const void *stream, const void *event)
{
    entries.push_back({op, 0, reinterpret_cast<uint64_t>(stream), reinterpret_cast<uint64_t>(event)});
}
cudaError_t launch(cudaStream_t s)
{
    launches += 1;
    if (launches != fail_at) {
        note(LAUNCH, s, nullptr);
        return cudaSuccess;
    }
    note(LAUNCH_FAILED, s, nullptr);
    return last_error = cudaErrorLaunchOutOfResources;
}
CUresult encode(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                CUtensorMapL2promotion, CUtensorMapFloatOOBfill)
{
    return CUDA_SUCCESS;
}

}  // namespace

extern "C" {

void fake_reset(int64_t fail_launch)
{
    entries.clear();
    launches = 0;
    fail_at = fail_launch;
}
uint64_t fake_log(Entry *out, uint64_t room)
{
    for (uint64_t i = 0; i < entries.size() && i < room; ++i) out[i] = entries[i];
    return entries.size();
}

void **__cudaRegisterFatBinary(void *) { return reinterpret_cast<void **>(&next_handle); }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *, char *, const char *, int, uint3 *, uint3 *, dim3 *, dim3 *, int *) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, struct CUstream_st *stream)
{
    pushed_stream = stream;
    return 0;
}
cudaError_t __cudaPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, void *stream)
{
    *grid = *block = dim3(1);
    *shared = 0;
    *static_cast<cudaStream_t *>(stream) = pushed_stream;
    return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void *, dim3, dim3, void **, size_t, cudaStream_t s) { return launch(s); }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *, void **) { return launch(c->stream); }
cudaError_t cudaGetLastError()
{
    const cudaError_t e = last_error;
    last_error = cudaSuccess;
    return e;
}
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr, int)
{
    *v = 148;
    return cudaSuccess;
}
cudaError_t cudaDeviceSynchronize() { return cudaSuccess; }
cudaError_t cudaGetDevice(int *d)
{
    *d = 0;
    return cudaSuccess;
}
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaMalloc(void **p, size_t n)
{
    *p = malloc(n);
    return cudaSuccess;
}
cudaError_t cudaFree(void *p)
{
    free(p);
    return cudaSuccess;
}
cudaError_t cudaMemset(void *p, int v, size_t n)
{
    memset(p, v, n);
    return cudaSuccess;
}
cudaError_t cudaMemcpy(void *to, const void *from, size_t n, cudaMemcpyKind)
{
    memcpy(to, from, n);
    return cudaSuccess;
}
cudaError_t cudaMemcpyAsync(void *to, const void *from, size_t n, cudaMemcpyKind, cudaStream_t)
{
    memcpy(to, from, n);
    return cudaSuccess;
}
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes *a, const void *)
{
    memset(a, 0, sizeof(*a));
    return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void *, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **fn, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult *found)
{
    *fn = reinterpret_cast<void *>(&encode);
    *found = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaStreamCreateWithFlags(cudaStream_t *s, unsigned)
{
    *s = reinterpret_cast<cudaStream_t>(next_handle += 16);
    return cudaSuccess;
}
cudaError_t cudaStreamDestroy(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *e, unsigned)
{
    *e = reinterpret_cast<cudaEvent_t>(next_handle += 16);
    return cudaSuccess;
}
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t e, cudaStream_t s)
{
    note(RECORD, s, e);
    return cudaSuccess;
}
cudaError_t cudaStreamWaitEvent(cudaStream_t s, cudaEvent_t e, unsigned)
{
    note(WAIT, s, e);
    return cudaSuccess;
}

}  // extern "C"
