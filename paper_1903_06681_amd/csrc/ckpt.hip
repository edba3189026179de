// Activations in 8 bits: 32 channels of a pixel share a power of two.
//
// A lane takes one pixel's block: its 32 values are accesses contiguous over the
// wave's pixels, the largest magnitude and the rounding are its own registers'
// work, and its 32 bytes lie together (two 16-byte accesses).  Bound: memory: 4 x 64 x
// 256 x 256 in bf16 (51 MB each way) is saved in 10 to 12 us and loaded in 10, partly from
// the Infinity Cache.
#include "act.h"
#include "act_kernels.h"

namespace dc {

template <typename T, bool CL>
__global__ __launch_bounds__(256) void ckpt_save_kernel(CkptArgs a) {
    const int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int cb = blockIdx.y;
    if (e >= a.px.M) return;
    const Pixel p = pixel_of(a.px, int(e));
    float v[32];
    load_block<T, CL>(v, a.x, p, cb * 32, a.C);
    q8_store_block(a.q, a.qm, p, cb, v);
}

template <typename T, bool CL, int ACT>
__global__ __launch_bounds__(256) void ckpt_load_kernel(CkptArgs a) {
    const int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int cb = blockIdx.y;
    if (e >= a.px.M) return;
    const Pixel p = pixel_of(a.px, int(e));
    float v[32];
    q8_load_block(v, a.q, a.qm, p, cb);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = act_fwd<ACT>(v[j]);
    store_block<T, CL>(a.x, p, cb * 32, a.C, v);
}

template <typename T, bool CL>
static void load_act(const CkptArgs& a, dim3 g, hipStream_t s) {
    constexpr int kGelu = sizeof(T) == 4 ? int(ACT_GELU_F32) : int(DC_ACT_GELU);
    switch (a.act) {
        case DC_ACT_RELU: hipLaunchKernelGGL((ckpt_load_kernel<T, CL, DC_ACT_RELU>), g, dim3(256), 0, s, a); break;
        case DC_ACT_GELU: hipLaunchKernelGGL((ckpt_load_kernel<T, CL, kGelu>), g, dim3(256), 0, s, a); break;
        case DC_ACT_SILU: hipLaunchKernelGGL((ckpt_load_kernel<T, CL, DC_ACT_SILU>), g, dim3(256), 0, s, a); break;
        default: hipLaunchKernelGGL((ckpt_load_kernel<T, CL, DC_ACT_NONE>), g, dim3(256), 0, s, a);
    }
}

hipError_t launch_ckpt(const CkptArgs& a, bool save, hipStream_t s) {
    const dim3 g((a.px.M - 1) / 256 + 1, (a.C + 31) / 32);
    const bool f = a.x.dt == DC_F32;
    if (save) {
        if (f && a.cl) hipLaunchKernelGGL((ckpt_save_kernel<float, true>), g, dim3(256), 0, s, a);
        else if (f) hipLaunchKernelGGL((ckpt_save_kernel<float, false>), g, dim3(256), 0, s, a);
        else if (a.cl) hipLaunchKernelGGL((ckpt_save_kernel<__bf16, true>), g, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((ckpt_save_kernel<__bf16, false>), g, dim3(256), 0, s, a);
    } else {
        if (f && a.cl) load_act<float, true>(a, g, s);
        else if (f) load_act<float, false>(a, g, s);
        else if (a.cl) load_act<__bf16, true>(a, g, s);
        else load_act<__bf16, false>(a, g, s);
    }
    return hipGetLastError();
}

}  // namespace dc
