// Backward passes of the layer norm whose du is f32.
#include "norm_bwd.h"

namespace dc {

hipError_t launch_norm_bwd_f32(const NormArgs& a, hipStream_t s) {
    if (a.q)
        DC_NORM_LAUNCH(norm_bwd_kernel, 1, a, s, char, float);
    else if (a.x.dt == DC_F32)
        DC_NORM_LAUNCH(norm_bwd_kernel, 1, a, s, float, float);
    else
        DC_NORM_LAUNCH(norm_bwd_kernel, 1, a, s, __bf16, float);
    return hipGetLastError();
}

}  // namespace dc
