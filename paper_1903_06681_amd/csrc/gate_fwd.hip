// Forward pass of the gated product, both types.
#include "gate.h"

namespace dc {

hipError_t launch_gate_fwd(const GateArgs& a, bool f32, hipStream_t s) {
    return f32 ? launch_gate<float, false>(a, s) : launch_gate<__bf16, false>(a, s);
}

}  // namespace dc
