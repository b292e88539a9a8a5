// The RMS norm's vector kernels with gate, weight, scale and shift in fp32.
#include "norm_rows.cuh"

namespace cbk {

cudaError_t launch_norm_fp32_lines(NormArgs& a, int sms, cudaStream_t s) { return launch_lines<false>(a, sms, s); }

}  // namespace cbk
