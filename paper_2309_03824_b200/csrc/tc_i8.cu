// Products in 8-bit integers, plain and gated (the kernel: tc_glu.cuh).
#include "tc_glu.cuh"

namespace lrd {

lrd_status_t tc_glu_i8(const GluArgs& g, cudaStream_t s) {
    if (g.dtype == LRD_BF16) return g.gated ? glu::launch_shape<true, true, __nv_bfloat16>(g, s) : glu::launch_shape<true, false, __nv_bfloat16>(g, s);
    return g.gated ? glu::launch_shape<true, true, float>(g, s) : glu::launch_shape<true, false, float>(g, s);
}

}  // namespace lrd
