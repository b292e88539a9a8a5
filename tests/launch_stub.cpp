// The launch of the tensor-core kernels (linear_tc.cu) over stand-ins for the CUDA runtime and the kernels, for test_linear_prepare_cpu.py.
// Nothing here runs a kernel: what is prepared and launched is noted.
#include <cuda.h>
#include <cuda_runtime.h>

#include <string>

#include "../paper_2608_23429_gb300/csrc/linear.cuh"

namespace {
std::string g_log;
int g_device = 0, g_fail_at = -1, g_prepared = 0;
cbk::LinearKernel kernel(int i) { return reinterpret_cast<cbk::LinearKernel>(static_cast<size_t>(0x1000 + i)); }
}  // namespace

namespace cbk {
LinearKernel linear_out_kernel(int cg, bool fp8, bool passes) { return kernel(cg + 2 * fp8 + 4 * passes); }
LinearKernel linear_hidden_kernel(int cg, bool fp8, bool passes) { return kernel(16 + cg + 2 * fp8 + 4 * passes); }
LinearKernel linear_direct_kernel(int cg, bool fp8, bool passes) { return kernel(32 + cg + 2 * fp8 + 4 * passes); }
LinearKernel linear_mx_kernel(Results r, int cg, bool passes) { return kernel(256 + 8 * (int)r + cg + 2 * passes); }
}  // namespace cbk

extern "C" {
cudaError_t cudaFuncSetAttribute(const void* f, cudaFuncAttribute, int) {
    if (g_prepared++ == g_fail_at) return cudaErrorMemoryAllocation;
    g_log += "set " + std::to_string(reinterpret_cast<size_t>(f) - 0x1000) + "\n";
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) { return *n = 76, cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void* f, void**) {
    g_log += "launch " + std::to_string(reinterpret_cast<size_t>(f) - 0x1000) + "\n";
    return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { return *d = g_device, cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { return *v = 232448, cudaSuccess; }
cudaError_t cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode* m) {
    g_log += *m == cudaStreamCaptureModeRelaxed ? "relaxed\n" : "as before\n";
    *m = cudaStreamCaptureModeGlobal;
    return cudaSuccess;
}

const char* stub_log() { return g_log.c_str(); }
void stub_reset(int device, int fail_at) { g_log.clear(), g_device = device, g_fail_at = fail_at, g_prepared = 0; }
int stub_prepare() {
    int pairs = 0;
    return cbk::prepare_linear(232448, &pairs) == cudaSuccess && pairs == 76 ? 0 : -1;
}
int stub_launch(int mx, int results, int cg) {
    cbk::LinearArgs a{};
    a.operands = mx ? cbk::Operands::kMx : cbk::Operands::kBf16, a.results = (cbk::Results)results;
    a.tile_n = 128, a.stages = 4, a.out_boxes = 2, a.passes = 1;
    return (int)cbk::launch_linear(a, cg, false, 8, nullptr);
}
}
