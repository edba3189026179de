// Backward passes of the layer norm whose du is bf16.
#include "norm_bwd.h"

namespace dc {

hipError_t launch_norm_bwd_bf16(const NormArgs& a, hipStream_t s) {
    if (a.q)
        DC_NORM_LAUNCH(norm_bwd_kernel, 1, a, s, char, __bf16);
    else if (a.x.dt == DC_F32)
        DC_NORM_LAUNCH(norm_bwd_kernel, 1, a, s, float, __bf16);
    else
        DC_NORM_LAUNCH(norm_bwd_kernel, 1, a, s, __bf16, __bf16);
    return hipGetLastError();
}

}  // namespace dc
