// Products over channels where the tile loop has too few blocks for the chip: a classifier
// on pooled samples, single rows of channels, small images with many channels.
//
// Bound: the weights, each read once: memory latency first (4 MB over the chip is a
// microsecond).  A workgroup takes 16 channels of the result and up to 64 pixels and deals
// k out to its sixteen waves, so that a wave's loads are few and all in flight at once;
// fragments come straight from memory (16 x 16 blocks of the result), and the waves' sums
// meet in LDS, in order.  2048 -> 1000 channels on four rows (bf16): 5.8 us, the tile
// loop's 32 slices one after the other 16 us.
#include <algorithm>

#include "linear_pass.h"

namespace dc {

static constexpr int kFewWaves = 16;
typedef float f32x4_acc __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ void multiply16(f32x4_acc& acc, const uint4& a, const uint4& b) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0,
                                                      0, 0);
    } else {
        const f32x4_t fa = __builtin_bit_cast(f32x4_t, a), fb = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[i], fb[i], acc, 0, 0, 0);
    }
}

// NT: tiles of 16 pixels.  BWD: weights [k][row], and the activation's slope.
template <typename T, bool BWD, bool CL, int NT>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(LinearArgs a, int M) {
    constexpr int E = 16 / int(sizeof(T)), STEP = 4 * E;      // k of a lane's chunk, of a wave's step
    __shared__ float sums[kFewWaves][NT * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int o0 = blockIdx.x * 16, m0 = blockIdx.y * NT * 16, red = a.a.red;
    const int hw = int(a.s.dsample.d) / a.s.cpr * a.s.len;
    auto offset = [&](int m, const auto& v) __attribute__((always_inline)) {   // of channel 0 of pixel m
        const int n = m / hw, pix = m - n * hw, r = pix / a.s.len;
        return n * v.sn + r * v.sh + (pix - r * a.s.len);
    };
    const T* w = reinterpret_cast<const T*>(a.a.p);
    const T* x = reinterpret_cast<const T*>(a.b.p);
    const int row = min(o0 + (lane & 15), a.rows - 1);
    int64_t xo[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) xo[t] = offset(min(m0 + t * 16 + (lane & 15), M - 1), a.b);
    // eight (four) values of k of which n count, `step` elements apart; past the end the last one's address
    auto gather = [&](const T* p, int64_t step, int n) __attribute__((always_inline)) {
        T e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const T f = p[max(min(i, n - 1), 0) * step];
            e[i] = i < n ? f : T(0);
        }
        uint4 r;
        __builtin_memcpy(&r, e, 16);
        return r;
    };
    // this wave's steps of k
    const int steps = (red + STEP - 1) / STEP, per = (steps + kFewWaves - 1) / kFewWaves;
    const int s1 = min((wave + 1) * per, steps);
    f32x4_acc acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4_acc{0, 0, 0, 0};
#pragma unroll 4
    for (int s = wave * per; s < s1; ++s) {
        const int k = s * STEP + (lane >> 4) * E, n = red - k, kk = min(k, red - 1);
        uint4 fa = make_uint4(0, 0, 0, 0), fb[NT];
        if constexpr (BWD) fa = gather(w + int64_t(kk) * a.a.ld + row, a.a.ld, n);
        else if (n > 0) fa = keep16<T>(load16(w, row * a.a.ld + k, a.a.end), n);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            fb[t] = make_uint4(0, 0, 0, 0);
            if constexpr (CL) {
                if (n > 0) fb[t] = keep16<T>(load16(x, xo[t] + k, a.b.end), n);
            } else {
                fb[t] = gather(x + xo[t] + kk * a.b.sc, a.b.sc, n);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) multiply16<T>(acc[t], fa, fb[t]);
    }
    // lane: pixel lane % 16, channels 4 (lane / 16) .. + 3
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][t * 256 + (4 * (lane >> 4) + r) * 16 + (lane & 15)] = acc[t][r];
    __syncthreads();
    // channels next to each other in memory (rows of channels) lie next to each other on the lanes
    for (int e = threadIdx.x; e < NT * 256; e += 64 * kFewWaves) {
        const int in = e & 255, o = o0 + (CL ? in & 15 : in >> 4), mt = CL ? in >> 4 : in & 15, m = m0 + (e >> 8) * 16 + mt;
        if (o >= a.rows || m >= M) continue;
        const int at = (e & ~255) + (o - o0) * 16 + mt;
        float v[1] = {0};
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) v[0] += sums[i][at];
        auto put = [&](const View& t, float f) __attribute__((always_inline)) {
            const int64_t k = offset(m, t) + o * t.sc;
            if (t.dt == DC_F32) store1(reinterpret_cast<float*>(t.p) + k, f);
            else store1(reinterpret_cast<__bf16*>(t.p) + k, f);
        };
        auto get = [&](const View& t) __attribute__((always_inline)) {
            const int64_t k = offset(m, t) + o * t.sc;
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

static int pixels_in(const LinearArgs& a) {
    return a.s.chunks / int(a.s.dsample.d) * (int(a.s.dsample.d) / a.s.cpr * a.s.len);
}

// Up to 64 pixels, or a long sum with few blocks of the tile loop to share it.  Forward
// where the loop's slices are dear (fp32's matrix rate, operands staged through registers):
// up to 64 blocks, a workgroup a compute unit here.  fp32, 1024 channels to 256 on 32 x 32
// 14.3 us, the tile loop's 24.6; 512 to 128 on 4096 pixels (128 blocks) 18.6 and 14.5.  bf16,
// 1024 to 128 on 8 x 14 x 15 (not on 16 bytes) 11.3 and 14.5, but 2048 to 256 on 32 x 32
// 16.4 and 13.0.  z in 8 bits is written 32 channels at a time: the tile loop's.
bool linear_few(const LinearArgs& a, bool bwd, bool f32) {
    if (!bwd && a.z.dt == DC_Q8) return false;
    const int64_t M = pixels_in(a);
    const int limit = !bwd && (f32 || !a.direct) ? 64 : 31;
    return M <= 64 || (a.a.red >= 256 && (a.rows + 63) / 64 * ((M + 63) / 64) <= limit);
}

template <typename T, bool BWD, bool CL>
static void launch(const LinearArgs& a, int M, hipStream_t s) {
    const dim3 g((a.rows + 15) / 16, (M + 63) / 64), t(64 * kFewWaves);
    if (M <= 16) hipLaunchKernelGGL((linear_few_kernel<T, BWD, CL, 1>), g, t, 0, s, a, M);
    else if (M <= 32) hipLaunchKernelGGL((linear_few_kernel<T, BWD, CL, 2>), g, t, 0, s, a, M);
    else hipLaunchKernelGGL((linear_few_kernel<T, BWD, CL, 4>), g, t, 0, s, a, M);
}

template <typename T, bool BWD>
static void launch(const LinearArgs& a, int M, hipStream_t s) {
    a.cl ? launch<T, BWD, true>(a, M, s) : launch<T, BWD, false>(a, M, s);
}

hipError_t launch_linear_few(const LinearArgs& a, bool bwd, bool f32, hipStream_t s) {
    const int M = pixels_in(a);
    if (f32) bwd ? launch<float, true>(a, M, s) : launch<float, false>(a, M, s);
    else bwd ? launch<__bf16, true>(a, M, s) : launch<__bf16, false>(a, M, s);
    return hipGetLastError();
}

}  // namespace dc
