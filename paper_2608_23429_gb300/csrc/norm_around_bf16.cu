// cb_norm_around's rows reached by vectors, with lines in bf16 (see norm_around_rows.cuh).
#include "norm_around_rows.cuh"

namespace cbk {

cudaError_t launch_around_bf16_lines(AroundArgs& a, int sms, cudaStream_t s) { return launch_around_lines<true>(a, sms, s); }

}  // namespace cbk
