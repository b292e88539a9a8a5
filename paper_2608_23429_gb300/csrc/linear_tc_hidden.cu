// The tensor-core kernels of cb_linear_run for a hidden state, which comes and leaves by TMA, with or without an output (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {

LinearKernel linear_hidden_kernel(int cg, bool fp8, bool passes) {
    return passes ? kernel_of<Results::kHidden, true>(cg, fp8) : kernel_of<Results::kHidden, false>(cg, fp8);
}

}  // namespace cbk
