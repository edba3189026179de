// What both passes of the layer norm share: which pixel and which blocks of 32
// channels a lane holds, the sums over a pixel's channels, types chosen at run time.
#pragma once

#include "act.h"
#include "act_kernels.h"

namespace dc {

static constexpr int kNormWaves = 8;    // most waves of a workgroup

struct NormLane {
    int px, unit, ng, pg, wave;
};
// A: the arguments of the norm, or of the join of a branch (join.h)
template <int LPX, typename A>
__device__ __forceinline__ NormLane norm_lane(const A& a) {
    const int lane = threadIdx.x & 63;
    NormLane l;
    l.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    l.pg = l.wave / a.nw;
    l.px = lane % LPX;
    l.unit = (l.wave - l.pg * a.nw) * (64 / LPX) + lane / LPX;   // uniform where LPX is 64
    l.ng = a.nw * (64 / LPX);
    return l;
}

// Sums of K values over the units of a pixel, in all of them.  Fixed order: the
// lanes of the wave that share the pixel, then the waves.
template <int LPX, int K, typename A>
__device__ __forceinline__ void pixel_sum(float (&v)[K], const A& a, const NormLane& l,
                                          float (&red)[K][kNormWaves * LPX]) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int d = LPX; d < 64; d *= 2) v[k] += __shfl_xor(v[k], d);
    if (a.nw == 1) return;
#pragma unroll
    for (int k = 0; k < K; ++k) red[k][l.wave * LPX + l.px] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float s = 0;
        for (int w = 0; w < a.nw; ++w) s += red[k][(l.pg * a.nw + w) * LPX + l.px];
        v[k] = s;
    }
}

// gamma or beta of a block; where there is none, `none`.  One block a wave: scalar loads.
// Else vector loads whose address is formed here (ahead of a loop it, or the values, would
// take the registers).
template <int LPX>
__device__ __forceinline__ void load_params(float (&v)[32], const float* p, int c0, int C, float none) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = none;
    } else if constexpr (LPX == 64) {
        if (c0 + 32 <= C) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = p[c0 + j];
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = p[min(c0 + j, C - 1)];
        }
    } else {
        char* a = reinterpret_cast<char*>(const_cast<float*>(p + c0));
        if (C % 32 == 0) {
            next(a, 0);
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 f = *reinterpret_cast<const float4*>(a + 4 * j);
                v[j] = f.x;
                v[j + 1] = f.y;
                v[j + 2] = f.z;
                v[j + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                v[j] = *reinterpret_cast<const float*>(a);
                next(a, c0 + j + 1 < C ? 4 : 0);
            }
        }
    }
}

// a block of a view whose type is a (uniform) run-time choice
template <bool CL>
__device__ __forceinline__ void load_any(float (&v)[32], const View& t, const Pixel& p, int c0, int C) {
    if (t.dt == DC_F32)
        load_block<float, CL>(v, t, p, c0, C);
    else
        load_block<__bf16, CL>(v, t, p, c0, C);
}
template <bool CL>
__device__ __forceinline__ void store_any(const View& t, const Pixel& p, int c0, int C, const float (&v)[32]) {
    if (t.dt == DC_F32)
        store_block<float, CL>(t, p, c0, C, v);
    else
        store_block<__bf16, CL>(t, p, c0, C, v);
}

// f(slot, block) for the blocks of a unit: R of them held in registers, or (R = 0)
// any number, one after the other in slot 0
template <int R, typename A, typename F>
__device__ __forceinline__ void each_block(const A& a, const NormLane& l, F&& f) {
    if constexpr (R) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (l.unit + i * l.ng < a.blocks) f(i, l.unit + i * l.ng);
    } else {
        for (int cb = l.unit; cb < a.blocks; cb += l.ng) f(0, cb);
    }
}

// Sums of V values over the LPX pixel lanes of a wave, by halving: each step a lane gives away
// half of its values.  Lane px ends with those of values px * V / LPX + e, in v[e]; where
// there are fewer values than lanes, neighbours hold the same one.
template <int D, int N, int V>
__device__ __forceinline__ void sum_step(float (&v)[V], int lane) {
    if constexpr (D >= 1 && N >= 1) {
        const bool hi = lane & D;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float keep = hi ? v[k + N] : v[k], give = hi ? v[k] : v[k + N];
            v[k] = keep + __shfl_xor(give, D);
        }
        sum_step<D / 2, N / 2>(v, lane);
    } else if constexpr (D >= 1) {
        v[0] += __shfl_xor(v[0], D);
        sum_step<D / 2, N>(v, lane);
    }
}
template <int LPX, int V>
__device__ __forceinline__ void sum_lanes(float (&v)[V], int lane) {
    sum_step<LPX / 2, V / 2>(v, lane);
}

// Launch K<type, LPX, R, CL> as planned (norm_plan keeps to these).  HELD16: blocks that a
// lane of a 16-pixel wave holds at most, 2 forward, 1 backward (which has twice the values).
#define DC_NORM_LAUNCH(KERNEL, HELD16, a, s, ...)                                                               \
    do {                                                                                                        \
        const unsigned x_ = (a).grid < (1 << 22) ? (a).grid : 1 << 22;  /* threads of a dimension: 32 bits */   \
        const dim3 g_(x_, ((a).grid + x_ - 1) / x_), b_(64 * (a).nw * (a).pg);                                  \
        if ((a).lpx == 64 && (a).held == 1) hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 64, 1, false>), g_, b_, 0, s, a);      \
        else if ((a).lpx == 64) hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 64, 2, false>), g_, b_, 0, s, a);       \
        else if ((a).lpx == 16 && !(a).cl && (a).held == 1)                                                     \
            hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 16, 1, false>), g_, b_, 0, s, a);                           \
        else if ((a).lpx == 16 && !(a).cl && (a).held == HELD16)                                                \
            hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 16, HELD16, false>), g_, b_, 0, s, a);                      \
        else if ((a).lpx == 16 && !(a).cl) hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 16, 0, false>), g_, b_, 0, s, a);       \
        else if ((a).lpx == 16) hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 16, 1, true>), g_, b_, 0, s, a);        \
        else if ((a).held == 1) hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 4, 1, true>), g_, b_, 0, s, a);         \
        else hipLaunchKernelGGL((KERNEL<__VA_ARGS__, 4, 0, true>), g_, b_, 0, s, a);                            \
    } while (0)

}  // namespace dc
