// A CUDA runtime without a device: what the host side of the operators asks of it is written into a
// log, so that tests on a machine without a GPU see the order of a call's allocations, waits, launches
// and records, on several devices and streams.  Device memory is addresses only.  Linked with the
// library's object files in place of the CUDA runtime.
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <new>
#include <string>
#include <utility>

namespace {

struct Stream { unsigned long long id; bool capturing; };
std::string events, given;
std::map<void *, Stream> streams;
std::map<const void *, std::string> kernels;
std::map<std::pair<const void *, int>, int> granted;          // dynamic shared memory of (kernel, device)
std::map<void *, size_t> blocks;
uintptr_t next_address = 0x100000000000;
int device = 0, launches_until_failure = -1, clusters = 10, allocations_until_failure = -1;

struct Own {                                                  // while it lives allocations are the fake runtime's and succeed
    int kept = allocations_until_failure;
    Own() { allocations_until_failure = -1; }
    ~Own() { allocations_until_failure = kept; }
};

void note(const char *format, ...)
{
    const Own own;
    char line[512];
    va_list a;
    va_start(a, format);
    vsnprintf(line, sizeof line, format, a);
    va_end(a);
    events += line;
    events += '\n';
}

cudaError_t launch(const void *kernel, cudaStream_t stream, size_t smem)
{
    if (launches_until_failure == 0) { launches_until_failure = -1; return cudaErrorLaunchFailure; }
    if (launches_until_failure > 0) --launches_until_failure;
    const auto g = granted.find({kernel, device});
    if (smem > 48 * 1024 && (g == granted.end() || (int)smem > g->second)) return cudaErrorInvalidValue;
    note("launch device=%d stream=%p kernel=%s smem=%zu", device, (void *)stream, kernels[kernel].c_str(), smem);
    return cudaSuccess;
}

CUresult encode(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill)
{
    return CUDA_SUCCESS;
}

}  // namespace

// The library's own allocations (those within the C++ library are its own).
void *operator new(size_t n)
{
    if (allocations_until_failure == 0) throw std::bad_alloc();
    if (allocations_until_failure > 0) --allocations_until_failure;
    if (void *p = malloc(n)) return p;
    throw std::bad_alloc();
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

extern "C" {

// ---- what tests call -------------------------------------------------------------------------

const char *fake_log()                                       // the events since the last call
{
    given.swap(events);
    events.clear();
    return given.c_str();
}
void fake_stream(void *handle, unsigned long long id, int capturing) { streams[handle] = Stream{id, capturing != 0}; }
void fake_fail_launch(int after) { launches_until_failure = after; }
void fake_clusters(int n) { clusters = n; }                  // that the present device holds at a time
void fake_fail_allocations(int after) { allocations_until_failure = after; }       // -1: no more
int fake_blocks() { return (int)blocks.size(); }

// ---- the runtime -----------------------------------------------------------------------------

cudaError_t cudaGetDeviceCount(int *n) { *n = 2; return cudaSuccess; }
cudaError_t cudaGetDevice(int *d) { *d = device; return cudaSuccess; }
cudaError_t cudaSetDevice(int d) { device = d; return cudaSuccess; }
cudaError_t cudaGetDeviceProperties_v2(cudaDeviceProp *p, int)
{
    memset(p, 0, sizeof *p);
    p->major = 10;
    p->multiProcessorCount = 148;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr a, int)
{
    *v = a == cudaDevAttrMultiProcessorCount ? 148 : 0;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetStreamPriorityRange(int *lo, int *hi) { *lo = *hi = 0; return cudaSuccess; }
cudaError_t cudaMalloc(void **p, size_t bytes)
{
    const Own own;
    *p = reinterpret_cast<void *>(next_address);
    next_address += (bytes + 4095) / 4096 * 4096 + 4096;
    blocks[*p] = bytes;
    note("malloc device=%d block=%p bytes=%zu", device, *p, bytes);
    return cudaSuccess;
}
cudaError_t cudaFree(void *p)
{
    if (p && !blocks.erase(p)) note("free of no block %p", p);
    else if (p) note("free block=%p", p);
    return cudaSuccess;
}
cudaError_t cudaHostAlloc(void **p, size_t bytes, unsigned) { *p = calloc(1, bytes); return cudaSuccess; }
cudaError_t cudaFreeHost(void *p) { free(p); return cudaSuccess; }
cudaError_t cudaHostGetDevicePointer(void **d, void *h, unsigned) { *d = h; return cudaSuccess; }
cudaError_t cudaMemset(void *, int, size_t) { return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *, int, size_t, cudaStream_t s) { note("memset stream=%p", (void *)s); return cudaSuccess; }
cudaError_t cudaMemcpy(void *, const void *, size_t, cudaMemcpyKind) { return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void *, const void *, size_t, cudaMemcpyKind, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventCreate(cudaEvent_t *e) { *e = reinterpret_cast<cudaEvent_t>(malloc(1)); return cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *e, unsigned) { return cudaEventCreate(e); }
cudaError_t cudaEventDestroy(cudaEvent_t e) { free(e); return cudaSuccess; }
cudaError_t cudaEventElapsedTime(float *ms, cudaEvent_t, cudaEvent_t) { *ms = 0.f; return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t s) { note("record stream=%p", (void *)s); return cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaStreamCreateWithPriority(cudaStream_t *s, unsigned, int) { *s = reinterpret_cast<cudaStream_t>(malloc(1)); return cudaSuccess; }
cudaError_t cudaStreamDestroy(cudaStream_t s) { free(s); return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t s) { note("synchronize device=%d stream=%p", device, (void *)s); return cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t s, cudaEvent_t, unsigned) { note("wait stream=%p", (void *)s); return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t s, cudaStreamCaptureStatus *status)
{
    *status = streams.count(s) && streams[s].capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t cudaStreamGetId(cudaStream_t s, unsigned long long *id)
{
    *id = streams.count(s) ? streams[s].id : reinterpret_cast<uintptr_t>(s);
    return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void *kernel, cudaFuncAttribute a, int v)
{
    const Own own;
    if (a == cudaFuncAttributeMaxDynamicSharedMemorySize) granted[{kernel, device}] = v;
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveBlocksPerMultiprocessorWithFlags(int *n, const void *, int, size_t, unsigned) { *n = 2; return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *, const cudaLaunchConfig_t *) { *n = clusters; return cudaSuccess; }
cudaError_t cudaLaunchKernel(const void *kernel, dim3, dim3, void **, size_t smem, cudaStream_t s) { return launch(kernel, s, smem); }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *kernel, void **) { return launch(kernel, c->stream, c->dynamicSmemBytes); }
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char *cudaGetErrorString(cudaError_t) { return "an error of the fake runtime"; }
cudaError_t cudaGetSymbolAddress(void **p, const void *) { return cudaMalloc(p, 4096); }
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **f, unsigned, unsigned long long, cudaDriverEntryPointQueryResult *r)
{
    *f = reinterpret_cast<void *>(&encode);
    *r = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}

// ---- what the compiler's host code calls --------------------------------------------------------

void **__cudaRegisterFatBinary(void *) { static void *handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction(void **, const char *host, char *, const char *name, int, uint3 *, uint3 *, dim3 *, dim3 *, int *) { kernels[host] = name; }
void __cudaRegisterVar(void **, char *, char *, const char *, int, size_t, int, int) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void *) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3 *, dim3 *, size_t *, void *) { return cudaSuccess; }

}  // extern "C"
