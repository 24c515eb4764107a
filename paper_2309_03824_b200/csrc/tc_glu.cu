// Gated feed-forward blocks with bf16 operands (the kernel: tc_glu.cuh).
#include "tc_glu.cuh"

namespace lrd {

lrd_status_t tc_glu_bf16(const GluArgs& g, cudaStream_t s) { return glu::launch_shape<false, true, __nv_bfloat16>(g, s); }

}  // namespace lrd
