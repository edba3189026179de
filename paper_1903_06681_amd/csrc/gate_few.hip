// The gated product and the gradient at its sums where the tile loop has too few blocks for
// the chip: single tokens, a few dozen rows, small images with many channels.
//
// Bound: the weights, each read once: memory latency first.  As for the plain product
// (linear_few.hip) a workgroup deals k out to sixteen waves, whose sums meet in LDS in order;
// forward, eight channels a workgroup: eight rows of Wg and eight of Wu fill the matrix
// instruction's sixteen.  Forward on up to 16 pixels with two workgroups or more a compute unit,
// eight waves: one pixel, 1024 to twice 4096 in bf16, 6.4 us (16.8 MB: 3.4 at a copy's rate), with
// sixteen 7.5; 2048 to twice 8192 14.5 (4.6 TB/s) and 17.6.  Backward and below 512 workgroups
// (no difference) sixteen.  Backward, a workgroup reads 32 or 64 bytes of a weight row: those that
// read the rest of a line run on the same XCD, whose L2 has it by then (one pixel, 2048 from 8192 in
// bf16, with the product's gradient in turn: 9.5 us, dealt out over the XCDs 23.6).
#include <algorithm>

#include "gate.h"
#include "linear_few.h"

namespace dc {

template <typename T, bool BWD, bool CL, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void gate_few_kernel(GateArgs a, int M) {
    constexpr int CH = BWD ? 16 : 8;       // channels of a workgroup
    __shared__ float sums[WAVES][NT * 256];
    const LinearArgs& l = a.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int o0 = (BWD ? xcd_range(blockIdx.x, gridDim.x) : int(blockIdx.x)) * CH, m0 = blockIdx.y * NT * 16;
    const int hw = int(l.s.dsample.d) / l.s.cpr * l.s.len;
    int row;
    if constexpr (BWD) row = min(o0 + (lane & 15), l.rows - 1);
    else row = min(o0 + (lane & 7), l.rows - 1) + (lane & 8 ? l.rows : 0);
    few_sums<T, BWD, CL, NT>(sums, l, row, m0, M, hw, lane, wave);
    for (int e = threadIdx.x; e < NT * 16 * CH; e += 64 * WAVES) {
        const int in = e % (16 * CH), t = e / (16 * CH);
        // channels next to each other in memory (rows of channels) lie next to each other on the lanes
        const int ch = CL ? in % CH : in / 16, mt = CL ? in / CH : in % 16;
        const int o = o0 + ch, m = m0 + t * 16 + mt;
        if (o >= l.rows || m >= M) continue;
        const int at = t * 256 + ch * 16 + mt;
        const int n = m / hw, pix = m - n * hw;
        float v = 0, u[1] = {0};
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += sums[i][at];
        auto index = [&](const View& w, int c) __attribute__((always_inline)) {
            const int r = pix / l.s.len;
            return n * w.sn + r * w.sh + (pix - r * l.s.len) + c * w.sc;
        };
        auto put = [&](const View& w, int c, float f) __attribute__((always_inline)) {
            if (w.dt == DC_F32) store1(reinterpret_cast<float*>(w.p) + index(w, c), f);
            else store1(reinterpret_cast<__bf16*>(w.p) + index(w, c), f);
        };
        auto get = [&](const View& w, int c) __attribute__((always_inline)) {
            if (w.dt == DC_Q8) {
                const int64_t blk = int64_t(c / 32) * l.qm.HW + pix;
                const uint32_t s = reinterpret_cast<const uint8_t*>(w.p)[l.qm.s0 + n * l.qm.sn + blk];
                return float(reinterpret_cast<const int8_t*>(w.p)[n * l.qm.qn + blk * 32 + c % 32]) * q8_step(s);
            }
            return w.dt == DC_F32 ? load1(reinterpret_cast<const float*>(w.p) + index(w, c))
                                  : load1(reinterpret_cast<const __bf16*>(w.p) + index(w, c));
        };
        float factor = 1.0f;
        bool stays = true;
        if (a.drop.t) {
            const DropPixel dp = drop_pixel(a.drop, n, pix);
            const Philox w = philox(dp.pos + uint64_t(o / 8) * uint64_t(a.drop.plane), dp.ctr, a.drop.seed);
            const uint32_t two = o & 4 ? (o & 2 ? w.w[3] : w.w[2]) : (o & 2 ? w.w[1] : w.w[0]);
            stays = (o & 1 ? two >> 16 : two & 0xffffu) >= uint32_t(a.drop.t);
            factor = a.drop.scale;
        }
        if constexpr (BWD) {
            float f[1] = {get(l.z, o)}, g[1];
            const float zu = get(a.zu, o);
            v = stays ? v * factor : 0.0f;
            g[0] = v * zu;
            apply_slope(f, g, l.act);
            put(l.out, o, g[0]);
            put(l.out, o + l.rows, v * f[0]);
            if (l.h.dt >= 0) put(l.h, o, stays ? f[0] * zu * factor : 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < WAVES; ++i) u[0] += sums[i][at + 128];
            float f[1] = {v};
            if (l.bias) {
                f[0] += l.bias[o];
                u[0] += l.bias[o + l.rows];
            }
            if (l.z.dt >= 0) {
                put(l.z, o, f[0]);
                put(a.zu, o, u[0]);
            }
            apply_act(f, l.act);
            put(l.out, o, stays ? f[0] * u[0] * factor : 0.0f);
        }
    }
}

// As for the plain product; z in 8 bits is written 32 channels at a time: the tile loop's.
bool gate_few(const GateArgs& a, bool bwd, bool f32) {
    if (!bwd && a.l.z.dt == DC_Q8) return false;
    const int64_t M = few_pixels(a.l), rows = int64_t(a.l.rows) * (bwd ? 1 : 2);
    const int limit = !bwd && (f32 || !a.l.direct) ? 64 : 31;
    return M <= 64 || (a.l.a.red >= 256 && (rows + 63) / 64 * ((M + 63) / 64) <= limit);
}

template <typename T, bool BWD, bool CL>
static void launch(const GateArgs& a, int M, hipStream_t s) {
    const int ch = BWD ? 16 : 8;
    const dim3 g((a.l.rows + ch - 1) / ch, (M + 63) / 64), t(64 * kFewWaves);
    if constexpr (!BWD) {
        if (M <= 16 && g.x >= 512) {
            hipLaunchKernelGGL((gate_few_kernel<T, BWD, CL, 1, 8>), g, dim3(64 * 8), 0, s, a, M);
            return;
        }
    }
    if (M <= 16) hipLaunchKernelGGL((gate_few_kernel<T, BWD, CL, 1, kFewWaves>), g, t, 0, s, a, M);
    else if (M <= 32) hipLaunchKernelGGL((gate_few_kernel<T, BWD, CL, 2, kFewWaves>), g, t, 0, s, a, M);
    else hipLaunchKernelGGL((gate_few_kernel<T, BWD, CL, 4, kFewWaves>), g, t, 0, s, a, M);
}

template <typename T, bool BWD>
static void launch(const GateArgs& a, int M, hipStream_t s) {
    a.l.cl ? launch<T, BWD, true>(a, M, s) : launch<T, BWD, false>(a, M, s);
}

hipError_t launch_gate_few(const GateArgs& a, bool bwd, bool f32, hipStream_t s) {
    const int M = few_pixels(a.l);
    if (f32) bwd ? launch<float, true>(a, M, s) : launch<float, false>(a, M, s);
    else bwd ? launch<__bf16, true>(a, M, s) : launch<__bf16, false>(a, M, s);
    return hipGetLastError();
}

}  // namespace dc
