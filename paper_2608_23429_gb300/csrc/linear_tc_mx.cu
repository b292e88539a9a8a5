// The tensor-core kernels of cb_linear_run for operands in 4 bits (see linear_tc.cuh).
#include "linear_tc.cuh"

namespace cbk {
namespace {

template <Results RESULTS>
LinearKernel of(int cg, bool passes) {
    constexpr Operands M = Operands::kMx;
    if (cg == 2) return passes ? linear_kernel<2, M, true, RESULTS> : linear_kernel<2, M, false, RESULTS>;
    return passes ? linear_kernel<1, M, true, RESULTS> : linear_kernel<1, M, false, RESULTS>;
}

}  // namespace

LinearKernel linear_mx_kernel(Results r, int cg, bool passes) {
    return r == Results::kOut      ? of<Results::kOut>(cg, passes)
           : r == Results::kHidden ? of<Results::kHidden>(cg, passes)
           : r == Results::kHiddenLong ? of<Results::kHiddenLong>(cg, passes)
           : r == Results::kDirect ? of<Results::kDirect>(cg, passes)
                                   : of<Results::kQuant>(cg, passes);
}

}  // namespace cbk
