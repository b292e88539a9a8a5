// The RMS norm's vector kernels with gate, weight, scale and shift in bf16.
#include "norm_rows.cuh"

namespace cbk {

cudaError_t launch_norm_bf16_lines(NormArgs& a, int sms, cudaStream_t s) { return launch_lines<true>(a, sms, s); }

}  // namespace cbk
