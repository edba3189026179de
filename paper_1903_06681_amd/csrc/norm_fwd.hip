// Layer norm over the channels of each pixel, forward.
//
//   u = gamma (x - mu) r + beta,  mu = mean x,  r = (mean (x - mu)^2 + eps)^-1/2
//
// Bound: memory (about ten operations per value).  A lane holds one pixel's block
// of 32 channels in registers: every channel's access is contiguous over the
// wave's pixels, the sums over channels are the lane's own plus one exchange
// through LDS with the other blocks of the pixel, and the 8-bit form's scale needs
// no exchange at all.  One pass over the data: the variance comes from the
// centred registers, not from a difference of large sums.  4 x 64 x 256 x 256 fp32 to a
// bf16 tile with statistics and checkpoint (118 MB): 33.5 us, 3.5 TB/s.  Rows of more than
// 4096 channels (tiles of more than 2048) are read again for each sum: 2048 rows of 8192 in
// bf16 35.6 us, of 4096 15.6.
#include <algorithm>

#include "norm.h"

namespace dc {

template <typename XT, int LPX, int R, bool CL>
__global__ __launch_bounds__(512) void norm_fwd_kernel(NormArgs a) {
    __shared__ float red[2][1][kNormWaves * LPX];
    const NormLane l = norm_lane<LPX>(a);
    // workgroups past what one dimension of a grid counts lie in the second
    const int wg = int(blockIdx.y * gridDim.x + blockIdx.x);
    if (wg >= a.grid) return;
    const int m = (xcd_range(wg, a.grid) * a.pg + l.pg) * LPX + l.px;
    const bool in = m < a.px.M;
    const Pixel p = pixel_of(a.px, m);
    float v[R ? R : 1][32];
    float s[1] = {0};
    each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
        load_block<XT, CL>(v[i], a.x, p, cb * 32, a.C);
    });
    each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
        if constexpr (!R) load_block<XT, CL>(v[0], a.x, p, cb * 32, a.C);
#pragma unroll
        for (int j = 0; j < 32; ++j) s[0] += v[i][j];
    });
    pixel_sum<LPX>(s, a, l, red[0]);
    const float mu = s[0] * a.invC;
    s[0] = 0;
    each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
        if constexpr (!R) load_block<XT, CL>(v[0], a.x, p, cb * 32, a.C);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float d = cb * 32 + j < a.C ? v[i][j] - mu : 0.0f;
            s[0] = fmaf(d, d, s[0]);
        }
    });
    pixel_sum<LPX>(s, a, l, red[1]);
    const float r = 1.0f / sqrtf(s[0] * a.invC + a.eps);
    if (!in) return;
    if (a.stat && l.unit == 0) {
        a.stat[m] = mu;
        a.stat[int64_t(a.px.M) + m] = r;
    }
    each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
        if constexpr (!R) load_block<XT, CL>(v[0], a.x, p, cb * 32, a.C);
        if (a.q) q8_store_block(a.q, a.qm, p, cb, v[i]);
        float g[32], b[32];
        load_params<LPX>(g, a.gamma, cb * 32, a.C, 1.0f);
        load_params<LPX>(b, a.beta, cb * 32, a.C, 0.0f);
#pragma unroll
        for (int j = 0; j < 32; ++j) g[j] = fmaf(g[j], (v[i][j] - mu) * r, b[j]);
        store_any<CL>(a.u, p, cb * 32, a.C, g);
    });
}

// Which pixels and blocks go side by side.  Rows of channels (cl): the lanes of a
// pixel lie next to each other, so that a wave reads whole rows.  Else 64 pixels
// a wave, or 16 where that leaves the chip without work (fewer than 2048 waves of
// 64 pixels and 32 channels) or the channels do not fit a workgroup's registers.
void norm_plan(NormArgs& a, bool backward) {
    a.blocks = (a.C + 31) / 32;
    a.invC = 1.0f / float(a.C);
    const int64_t waves = (int64_t(a.px.M) + 63) / 64 * a.blocks;
    if (a.cl)
        a.lpx = a.blocks >= 16 ? 4 : 16;
    else
        a.lpx = a.blocks <= 2 * kNormWaves && waves >= 2048 ? 64 : 16;
    const int sb = 64 / a.lpx;
    a.nw = std::min((a.blocks + sb - 1) / sb, kNormWaves);
    const int held = (a.blocks + a.nw * sb - 1) / (a.nw * sb);
    a.held = held <= 1 ? 1 : held == 2 && !a.cl && !(backward && a.lpx == 16) ? 2 : 0;   // as registers allow
    a.groups = int((int64_t(a.px.M) + a.lpx - 1) / a.lpx);
    // enough workgroups for the chip first, then up to four waves each (more would not fit
    // the registers evenly).  Backward launches only what is resident and a turn more costs a
    // whole one, so it rounds up: 56 channels on 3 x 198 x 47 bf16 in one turn 17.5 us, in
    // two 26.8; 64 on 1 x 150 x 160 11.7 and 17.2
    a.pg = std::max(1, std::min(4 / a.nw, backward ? (a.groups + 511) / 512 : a.groups / 512));
    a.grid = (a.groups + a.pg - 1) / a.pg;
    // What is resident at a time: 12 or 8 waves a compute unit.  Eight-wave workgroups of 256
    // channels on 4 x 128 x 128: 256 of them 45.5 us, 512 49.2.  No more than three workgroups:
    // four of three waves (96 channels, 4 x 200 x 200) 48.4 us, three 41.0.
    const int waves_cu = a.lpx == 64 && a.held == 1 ? 12 : 8;
    if (backward) a.grid = std::min(a.grid, 256 * std::clamp(waves_cu / (a.nw * a.pg), 1, 3));
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
    if (a.x.dt == DC_F32)
        DC_NORM_LAUNCH(norm_fwd_kernel, 2, a, s, float);
    else
        DC_NORM_LAUNCH(norm_fwd_kernel, 2, a, s, __bf16);
    return hipGetLastError();
}

}  // namespace dc
