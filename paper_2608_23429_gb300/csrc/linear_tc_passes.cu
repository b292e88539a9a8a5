// The tensor-core kernels that sum in passes over K (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {

void (*linear_passes_kernel(int cg, bool fp8))(LinearArgs) { return kernel_of<true>(cg, fp8); }

}  // namespace cbk
