// The tensor-core kernels that sum in passes over K (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {

void (*linear_passes_kernel(int cg, bool fp8, int loaders))(LinearArgs) { return kernel_of<true>(cg, fp8, loaders); }

}  // namespace cbk
