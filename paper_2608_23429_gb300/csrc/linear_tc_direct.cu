// The tensor-core kernels of cb_linear_run for results off the 16-byte grid, which the threads store (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {

LinearKernel linear_direct_kernel(int cg, bool fp8, bool passes) {
    return passes ? kernel_of<Results::kDirect, true>(cg, fp8) : kernel_of<Results::kDirect, false>(cg, fp8);
}

}  // namespace cbk
