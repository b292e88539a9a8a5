// The launch of the tensor-core kernels (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {

size_t linear_stage_bytes(int cg, int tile_n) { return (size_t)(kRows + tile_n / cg) * kSlab; }

size_t linear_fixed_bytes(Results r, int more_boxes) { return kTailBytes + (size_t)epi_warps(r) * (kTurnBytes + more_boxes * kBox); }

cudaError_t prepare_linear(size_t smem, int* pairs) {
    for (int i = 0; i < 8; ++i)
        for (auto of : {linear_out_kernel, linear_hidden_kernel, linear_direct_kernel}) {
            const cudaError_t e = cudaFuncSetAttribute(of(1 + i % 2, i & 2, i & 4), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return e;
        }
    for (int i = 0; i < 4; ++i)
        for (Results r : {Results::kOut, Results::kHidden, Results::kDirect, Results::kQuant, Results::kHiddenLong}) {
            const cudaError_t e = cudaFuncSetAttribute(linear_mx_kernel(r, 1 + i % 2, i & 2), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
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
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = a.overlap;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cg, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid);
    c.blockDim = dim3(linear_threads(a.results, a.operands == Operands::kMx));
    const bool mx = a.operands == Operands::kMx;
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
