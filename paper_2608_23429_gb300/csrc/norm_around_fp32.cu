// cb_norm_around's rows reached by vectors, with lines in fp32 (see norm_around_rows.cuh).
#include "norm_around_rows.cuh"

namespace cbk {

cudaError_t launch_around_fp32_lines(AroundArgs& a, int sms, cudaStream_t s) { return launch_around_lines<false>(a, sms, s); }

}  // namespace cbk
