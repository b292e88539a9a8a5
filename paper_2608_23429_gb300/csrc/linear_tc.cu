// The launch of the tensor-core kernels (see linear_tc.cuh).
#include <atomic>

#include "linear_tc.cuh"

namespace cbk {
namespace {

// Devices on which the kernels for 4 bits are prepared: their first product there does it, which loads them, so that programs without one do not (GB300,
// a process's first bf16 product 2.92 -> 1.77 ms and 2.1 MB of device memory less; the first one in 4 bits 1.3 ms).
std::atomic<bool> g_mx_prepared[kMaxStatusDevices];

cudaError_t prepare_mx() {
    int d = 0, smem = 0;
    cudaError_t e = cudaGetDevice(&d);
    if (e != cudaSuccess || g_mx_prepared[d].load(std::memory_order_acquire)) return e;  // (d: looked at by cb_linear_run)
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;  // this call, or another stream's, may be captured
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
    e = cudaDeviceGetAttribute(&smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, d);
    for (int i = 0; i < 4; ++i)
        for (Results r : {Results::kOut, Results::kHidden, Results::kDirect, Results::kQuant, Results::kHiddenLong})
            if (e == cudaSuccess)
                e = cudaFuncSetAttribute(linear_mx_kernel(r, 1 + i % 2, i & 2), cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
    if (e == cudaSuccess) g_mx_prepared[d].store(true, std::memory_order_release);
    else (void)cudaGetLastError();  // returned here
    return e;
}

}  // namespace

size_t linear_stage_bytes(int cg, int tile_n) { return (size_t)(kRows + tile_n / cg) * kSlab; }

size_t linear_fixed_bytes(Results r, int more_boxes) { return kTailBytes + (size_t)epi_warps(r) * (kTurnBytes + more_boxes * kBox); }

cudaError_t prepare_linear(size_t smem, int* pairs) {
    for (int i = 0; i < 8; ++i)
        for (auto of : {linear_out_kernel, linear_hidden_kernel, linear_direct_kernel}) {
            const cudaError_t e = cudaFuncSetAttribute(of(1 + i % 2, i & 2, i & 4), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return e;
        }
    // pairs of CTAs that run at once
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(2);
    c.blockDim = dim3(linear_threads(Results::kOut));
    c.dynamicSmemBytes = smem;
    c.attrs = &at;
    c.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(pairs, reinterpret_cast<const void*>(linear_out_kernel(2, false, false)), &c);
}

cudaError_t launch_linear(const LinearArgs& a, int cg, bool fp8, int grid, cudaStream_t s) {
    const bool mx = a.operands == Operands::kMx;
    if (mx) {
        const cudaError_t e = prepare_mx();
        if (e != cudaSuccess) return e;
    }
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = a.overlap;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cg, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid);
    c.blockDim = dim3(linear_threads(a.results, mx));
    const size_t stage = linear_stage_bytes(cg, a.tile_n) + (mx ? mx_scale_bytes(a.tile_n) : 0);
    c.dynamicSmemBytes = (size_t)a.stages * stage + linear_fixed_bytes(a.results, a.more_boxes) + (mx ? mx_more_bytes(a.results, a.more_boxes, a.out_boxes) : 0);
    c.stream = s;
    c.attrs = at;
    c.numAttrs = cg == 2 ? 2 : 1;
    const auto of = a.results == Results::kOut ? linear_out_kernel : a.results == Results::kHidden ? linear_hidden_kernel : linear_direct_kernel;
    const LinearKernel k = mx ? linear_mx_kernel(a.results, cg, a.passes > 1) : of(cg, fp8, a.passes > 1);
    void* args[] = {const_cast<void*>(static_cast<const void*>(&a))};
    const cudaError_t e = cudaLaunchKernelExC(&c, reinterpret_cast<const void*>(k), args);
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e;
}

}  // namespace cbk
