// The tensor-core kernels whose sums stay in one accumulator, and the launch of all of them (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {

size_t linear_stage_bytes(int cg, int tile_n) { return (size_t)(kRows + tile_n / cg) * kSlab; }

size_t linear_fixed_bytes(bool shift, int tile_n) {
    return sizeof(Tail) + (shift ? (size_t)kRawSlabs * kRawRow * (kRows + tile_n) : 0);
}

cudaError_t prepare_linear(size_t smem, int* pairs) {
    for (int fp8 = 0; fp8 < 2; ++fp8)
        for (LinearKernel k : {kernel_of<false>(2, fp8, 0), kernel_of<false>(1, fp8, 0), kernel_of<false>(1, fp8, kFewLoaders),
                               kernel_of<false>(1, fp8, kManyLoaders), linear_passes_kernel(2, fp8, 0), linear_passes_kernel(1, fp8, 0),
                               linear_passes_kernel(1, fp8, kFewLoaders), linear_passes_kernel(1, fp8, kManyLoaders)}) {
            const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return e;
        }
    // pairs of CTAs that run at once
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(2);
    c.blockDim = dim3(linear_threads(0));
    c.dynamicSmemBytes = smem;
    c.attrs = &at;
    c.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(pairs, reinterpret_cast<const void*>(kernel_of<false>(2, false, 0)), &c);
}

cudaError_t launch_linear(const LinearArgs& a, int cg, bool fp8, int grid, cudaStream_t s) {
    const bool shift = a.grid_bytes < 16;
    const int loaders = !shift ? 0 : a.k_blocks >= kManyFrom ? kManyLoaders : kFewLoaders;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = a.overlap;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cg, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid);
    c.blockDim = dim3(linear_threads(loaders));
    c.dynamicSmemBytes = (size_t)a.stages * linear_stage_bytes(cg, a.tile_n) + linear_fixed_bytes(shift, a.tile_n);
    c.stream = s;
    c.attrs = at;
    c.numAttrs = cg == 2 ? 2 : 1;
    const LinearKernel k = a.passes > 1 ? linear_passes_kernel(cg, fp8, loaders) : kernel_of<false>(cg, fp8, loaders);
    void* args[] = {const_cast<void*>(static_cast<const void*>(&a))};
    const cudaError_t e = cudaLaunchKernelExC(&c, reinterpret_cast<const void*>(k), args);
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e;
}

}  // namespace cbk
