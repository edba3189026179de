// Gradient at the sums of the gated product, both types.
#include "gate.h"

namespace dc {

hipError_t launch_gate_bwd(const GateArgs& a, bool f32, hipStream_t s) {
    return f32 ? launch_gate<float, true>(a, s) : launch_gate<__bf16, true>(a, s);
}

}  // namespace dc
