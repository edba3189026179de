// The second launch of the layer norm's backward pass: the workgroups' parameter
// sums, added in order.
#include <algorithm>

#include "norm.h"

namespace dc {

hipError_t launch_norm_bwd_f32(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_bwd_bf16(const NormArgs& a, hipStream_t s);

// 64 sums of consecutive parameters and 16 shares of the rows a workgroup
__global__ __launch_bounds__(1024) void norm_params_kernel(NormArgs a, int rows) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6;
    const int width = 2 * a.blocks * 32, v = blockIdx.x * 64 + lane;
    float s = 0;
#pragma unroll 8
    for (int i = share; i < rows; i += 16) s += a.part[int64_t(i) * width + v];
    red[share][lane] = s;
    __syncthreads();
    if (share != 0) return;
    s = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += red[i][lane];
    const bool second = v >= a.blocks * 32;
    const int c = v - (second ? a.blocks * 32 : 0);
    float* out = second ? a.dbeta : a.dgamma;
    if (out && c < a.C) out[c] = a.accumulate ? out[c] + s : s;
}

static size_t part_bytes(const NormArgs& a) { return size_t(a.grid) * 2 * a.blocks * 32 * sizeof(float); }

// the larger of the two layouts' (rows of channels or tiles): the workspace does
// not depend on the other views' strides
size_t norm_bwd_part_bytes(int M, int C) {
    size_t need = 0;
    for (int cl = 0; cl < 2; ++cl) {
        NormArgs a{};
        a.px.M = M;
        a.C = C;
        a.cl = cl;
        norm_plan(a, true);
        need = std::max(need, part_bytes(a));
    }
    return need;
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s) {
    const hipError_t e = a.du.dt == DC_F32 ? launch_norm_bwd_f32(a, s) : launch_norm_bwd_bf16(a, s);
    if (e != hipSuccess || (!a.dgamma && !a.dbeta)) return e;
    hipLaunchKernelGGL(norm_params_kernel, dim3(a.blocks), dim3(1024), 0, s, a, a.grid);
    return hipGetLastError();
}

}  // namespace dc
