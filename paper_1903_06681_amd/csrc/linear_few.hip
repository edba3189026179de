// Products over channels where the tile loop has too few blocks for the chip: a classifier
// on pooled samples, single rows of channels, small images with many channels.
//
// Bound: the weights, each read once: memory latency first (4 MB over the chip is a
// microsecond).  A workgroup takes 16 channels of the result and up to 64 pixels and deals
// k out to its sixteen waves, so that a wave's loads are few and all in flight at once;
// fragments come straight from memory (16 x 16 blocks of the result), and the waves' sums
// meet in LDS, in order.  2048 -> 1000 channels on four rows (bf16): 5.8 us, the tile
// loop's 32 slices one after the other 16 us.  Backward, the workgroups that share a line of
// the weights run on the same XCD: one pixel, 2048 from 8192 channels (bf16) 10.6 us, dealt out
// over the XCDs 22.7.
#include <algorithm>

#include "linear_few.h"

namespace dc {

// NT: tiles of 16 pixels.  BWD: weights [k][row], and the activation's slope.  DEEP: see deep_pays.
template <typename T, bool BWD, bool CL, int NT, bool DEEP>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(LinearArgs a, int M) {
    __shared__ float sums[kFewWaves][NT * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int o0 = (BWD ? xcd_range(blockIdx.x, gridDim.x) : int(blockIdx.x)) * 16, m0 = blockIdx.y * NT * 16;
    const int hw = int(a.s.dsample.d) / a.s.cpr * a.s.len;
    const int row = min(o0 + (lane & 15), a.rows - 1);
    few_sums<T, BWD, CL, NT, kFewWaves, DEEP>(sums, a, row, m0, M, hw, lane, wave);
    // channels next to each other in memory (rows of channels) lie next to each other on the lanes
    for (int e = threadIdx.x; e < NT * 256; e += 64 * kFewWaves) {
        const int in = e & 255, o = o0 + (CL ? in & 15 : in >> 4), mt = CL ? in >> 4 : in & 15, m = m0 + (e >> 8) * 16 + mt;
        if (o >= a.rows || m >= M) continue;
        const int at = (e & ~255) + (o - o0) * 16 + mt;
        float v[1] = {0};
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) v[0] += sums[i][at];
        auto put = [&](const View& t, float f) __attribute__((always_inline)) {
            const int64_t k = few_offset(a.s, hw, m, t) + o * t.sc;
            if (t.dt == DC_F32) store1(reinterpret_cast<float*>(t.p) + k, f);
            else store1(reinterpret_cast<__bf16*>(t.p) + k, f);
        };
        auto get = [&](const View& t) __attribute__((always_inline)) {
            const int64_t k = few_offset(a.s, hw, m, t) + o * t.sc;
            return t.dt == DC_F32 ? load1(reinterpret_cast<const float*>(t.p) + k) : load1(reinterpret_cast<const __bf16*>(t.p) + k);
        };
        if constexpr (BWD) {
            if (a.act != DC_ACT_NONE) {
                float z[1];
                if (a.z.dt == DC_Q8) {
                    const int n = m / hw;
                    const int64_t blk = int64_t(o / 32) * a.qm.HW + (m - n * hw);
                    const uint32_t s = reinterpret_cast<const uint8_t*>(a.z.p)[a.qm.s0 + n * a.qm.sn + blk];
                    z[0] = float(reinterpret_cast<const int8_t*>(a.z.p)[n * a.qm.qn + blk * 32 + o % 32]) * q8_step(s);
                } else {
                    z[0] = get(a.z);
                }
                apply_slope(z, v, a.act);
                if (a.h.dt >= 0) put(a.h, z[0]);
            }
        } else {
            if (a.bias) v[0] += a.bias[o];
            if (a.z.dt >= 0) put(a.z, v[0]);
            apply_act(v, a.act);
            if (a.res.dt >= 0) v[0] += get(a.res);
        }
        put(a.out, v[0]);
    }
}

// Up to 64 pixels, or a long sum with few blocks of the tile loop to share it.  Forward
// where the loop's slices are dear (fp32's matrix rate, operands staged through registers):
// up to 64 blocks, a workgroup a compute unit here.  fp32, 1024 channels to 256 on 32 x 32
// 14.3 us, the tile loop's 24.6; 512 to 128 on 4096 pixels (128 blocks) 18.6 and 14.5.  bf16,
// 1024 to 128 on 8 x 14 x 15 (not on 16 bytes) 11.3 and 14.5, but 2048 to 256 on 32 x 32
// 16.4 and 13.0.  z in 8 bits is written 32 channels at a time: the tile loop's.
bool linear_few(const LinearArgs& a, bool bwd, bool f32) {
    if (!bwd && a.z.dt == DC_Q8) return false;
    const int64_t M = few_pixels(a);
    const int limit = !bwd && (f32 || !a.direct) ? 64 : 31;
    return M <= 64 || (a.a.red >= 256 && (a.rows + 63) / 64 * ((M + 63) / 64) <= limit);
}

// Whether a wave's steps of k (per of them) go out several at once, in up to 128 registers, or one after the
// other as the compiler arranges them, in about half.  us, several at once against one after the other:
//   one step a wave: nothing to gain, and the longer code costs (64 to 1000 channels, 48 pixels, fp32 4.8
//     against 4.1; 512 to 16384, 24 pixels, bf16 13.4 and 11.7)
//   from two steps on: one pixel, 4096 to 4096, bf16 9.0 and 11.4, fp32 14.0 and 18.5; 64 pixels, 1024 to
//     1024, rows, fp32 13.8 and 15.9; 24 pixels, planes, bf16 6.4 and 7.4
//   more workgroups than compute units where it takes the registers of a second one: gradient of 24 rows,
//     1024 to 8192, bf16 11.9 and 10.0, 1536 to 8192 15.2 and 13.0; 24 rows, 512 to 16384, fp32 20.4 and
//     18.4 (sums over 4096 the same within 5%)
//   fp32 planes, two tiles or four, whose loads are 4 bytes each: 768 to 1024, 64 pixels 10.2 and 10.3,
//     4096 to 1024 44 and 38; gradient 768 to 4096 9.9 and 11.1, 1024 to 2048 10.4 and 12.5, to 4096 15.0 and 13.8
template <typename T, bool BWD, bool CL, int NT>
static bool deep_pays(int per, int64_t workgroups) {
    constexpr bool f32 = sizeof(T) == 4;
    constexpr bool second = f32 ? NT == 2 || (NT == 4 && CL) : NT < 4 && (BWD || !CL);
    if (per < 2 || (second && workgroups > 256)) return false;
    return !f32 || CL || NT == 1 || per <= 3 || (BWD && per == 4 && workgroups <= 128);
}

template <typename T, bool BWD, bool CL, int NT>
static void launch(const LinearArgs& a, int M, dim3 g, hipStream_t s) {
    const int steps = (a.a.red + 64 / int(sizeof(T)) - 1) / (64 / int(sizeof(T))), per = (steps + kFewWaves - 1) / kFewWaves;
    if (deep_pays<T, BWD, CL, NT>(per, int64_t(g.x) * g.y))
        hipLaunchKernelGGL((linear_few_kernel<T, BWD, CL, NT, true>), g, dim3(64 * kFewWaves), 0, s, a, M);
    else
        hipLaunchKernelGGL((linear_few_kernel<T, BWD, CL, NT, false>), g, dim3(64 * kFewWaves), 0, s, a, M);
}

template <typename T, bool BWD, bool CL>
static void launch(const LinearArgs& a, int M, hipStream_t s) {
    const dim3 g((a.rows + 15) / 16, (M + 63) / 64);
    if (M <= 16) launch<T, BWD, CL, 1>(a, M, g, s);
    else if (M <= 32) launch<T, BWD, CL, 2>(a, M, g, s);
    else launch<T, BWD, CL, 4>(a, M, g, s);
}

template <typename T, bool BWD>
static void launch(const LinearArgs& a, int M, hipStream_t s) {
    a.cl ? launch<T, BWD, true>(a, M, s) : launch<T, BWD, false>(a, M, s);
}

hipError_t launch_linear_few(const LinearArgs& a, bool bwd, bool f32, hipStream_t s) {
    const int M = few_pixels(a);
    if (f32) bwd ? launch<float, true>(a, M, s) : launch<float, false>(a, M, s);
    else bwd ? launch<__bf16, true>(a, M, s) : launch<__bf16, false>(a, M, s);
    return hipGetLastError();
}

}  // namespace dc
