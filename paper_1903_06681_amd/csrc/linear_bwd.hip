// Input gradient of a product over channels, both types.
#include "linear_pass.h"

namespace dc {

hipError_t launch_linear_bwd(const LinearArgs& a, bool f32, hipStream_t s) {
    return f32 ? launch_linear<float, true>(a, s) : launch_linear<__bf16, true>(a, s);
}

}  // namespace dc
