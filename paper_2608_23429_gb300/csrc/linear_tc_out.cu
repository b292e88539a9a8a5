// The tensor-core kernels of cb_linear_run for an output alone, which leaves by TMA (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {

LinearKernel linear_out_kernel(int cg, bool fp8, bool passes) {
    return passes ? kernel_of<Results::kOut, true>(cg, fp8) : kernel_of<Results::kOut, false>(cg, fp8);
}

}  // namespace cbk
