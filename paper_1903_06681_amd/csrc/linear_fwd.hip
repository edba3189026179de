// Forward pass of a product over channels, both types.
#include "linear_pass.h"

namespace dc {

hipError_t launch_linear_fwd(const LinearArgs& a, bool f32, hipStream_t s) {
    return f32 ? launch_linear<float, false>(a, s) : launch_linear<__bf16, false>(a, s);
}

}  // namespace dc
