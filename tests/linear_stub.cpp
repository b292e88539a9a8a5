// The host side of cb_linear_* (linear.cu) over stand-ins for the CUDA runtime and
// the kernel launchers, for the CPU tests of its choices and of its error paths
// (test_block_dispatch_cpu.py). Nothing here runs a kernel: a launcher notes what it
// was given. Device properties are a GB300's.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdio>
#include <cstring>
#include <string>

#include "../paper_2608_23429_gb300/csrc/linear.cuh"

namespace {
std::string g_log;         // one line per call noted
std::string g_fail;        // the next call of this name fails
int g_pairs = 76;          // pairs of CTAs that run at once
bool g_capturing = false;

cudaError_t call(const char* name, const std::string& note = "") {
    const bool bad = g_fail == name;
    g_log += std::string(name) + (bad ? " FAILED" : "") + " " + note + "\n";
    if (!bad) return cudaSuccess;
    g_fail.clear();
    return cudaErrorMemoryAllocation;
}

CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t*,
                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    char b[128];
    std::snprintf(b, sizeof b, "wide=%llu rows=%llu stride=%llu", (unsigned long long)dims[0], (unsigned long long)dims[1],
                  (unsigned long long)strides[0]);
    (void)call("map", b);
    return dims[0] < 1ull << 32 ? CUDA_SUCCESS : CUDA_ERROR_INVALID_VALUE;
}
}  // namespace

extern "C" {
const char* stub_log() { return g_log.c_str(); }
void stub_reset() {
    g_log.clear();
    g_fail.clear();
    g_capturing = false;
}
void stub_fail(const char* name) { g_fail = name; }
void stub_pairs(int n) { g_pairs = n; }  // before the first call: the device is looked at once
void stub_capturing(int on) { g_capturing = on != 0; }

cudaError_t cudaGetDevice(int* d) { return *d = 0, cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) {
    *v = a == cudaDevAttrMultiProcessorCount ? 152 : a == cudaDevAttrMaxSharedMemoryPerBlockOptin ? 232448 : 0;
    return cudaSuccess;
}
cudaError_t cudaGetSymbolAddress(void** p, const void* symbol) { return *p = const_cast<void*>(symbol), cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode*) { return cudaSuccess; }
cudaError_t cudaMemPoolCreate(cudaMemPool_t* pool, const cudaMemPoolProps*) { return *pool = nullptr, cudaSuccess; }
cudaError_t cudaMemPoolSetAttribute(cudaMemPool_t, cudaMemPoolAttr, void*) { return cudaSuccess; }
cudaError_t cudaMemPoolDestroy(cudaMemPool_t) { return cudaSuccess; }
cudaError_t cudaMemPoolTrimTo(cudaMemPool_t, size_t) { return call("trim"); }
cudaError_t cudaMallocFromPoolAsync(void** p, size_t n, cudaMemPool_t, cudaStream_t) {
    *p = reinterpret_cast<void*>(1ull << 45);
    return call("malloc", "bytes=" + std::to_string(n));
}
cudaError_t cudaFreeAsync(void*, cudaStream_t) { return call("free"); }
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** fn, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* found) {
    *fn = reinterpret_cast<void*>(encode);
    *found = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
    *s = g_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t cudaMemcpyAsync(void* dst, const void*, size_t n, cudaMemcpyKind, cudaStream_t) {
    std::memset(dst, 0, n);
    return call("memcpy");
}
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return call("memset"); }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return call("synchronize"); }
}

namespace cbk {
int cuda_error(cudaError_t, const char*) { return CB_ERR_CUDA; }
size_t linear_stage_bytes(int cg, int tile_n) { return (size_t)(128 + tile_n / cg) * 128; }
size_t linear_fixed_bytes(Results, int more_boxes) { return 6144 + (size_t)8 * (4096 + more_boxes * kBox); }
cudaError_t prepare_linear(size_t, int* pairs) { return *pairs = g_pairs, cudaSuccess; }
cudaError_t launch_linear(const LinearArgs& a, int cg, bool fp8, int grid, cudaStream_t) {
    char b[256];
    std::snprintf(b, sizeof b, "results=%d cg=%d fp8=%d grid=%d tile_n=%d parts=%d passes=%d overlap=%d", (int)a.results, cg, fp8, grid, a.tile_n,
                  a.parts, a.passes, a.overlap);
    return call("tc", b);
}
cudaError_t launch_linear_few(const LinearFewArgs&, bool, bool shift, int, cudaStream_t) { return call("few", "shift=" + std::to_string(shift)); }
cudaError_t launch_linear_pack(LinearPackArgs& a, cudaStream_t) { return call("pack", "overlap=" + std::to_string(a.overlap)); }
cudaError_t launch_linear_join(const LinearJoinArgs& a, cudaStream_t) { return call("join", "parts=" + std::to_string(a.parts)); }
cudaError_t take_status(int* word, int* status, cudaStream_t) {
    const cudaError_t e = call("take_status");
    (void)word, (void)status;  // device memory
    return e;
}
}  // namespace cbk
