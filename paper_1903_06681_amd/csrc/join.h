// The join of a block's branch with its residual stream, what both passes share:
//
//   o = x + scale gate drop(post(y)),  u = pre(o)
//
// post and pre are norms of a pixel over its channels (layer, root mean square, or none).
// As in the layer norm (norm.h) a lane holds one pixel's block of 32 channels.  The tensors'
// types are known at run time: a block is loaded as it lies in memory, and widened when all
// loads are on their way.
#pragma once

#include "drop.h"
#include "norm.h"

namespace dc {

struct JoinNorm {
    const float *gamma, *beta;     // null: 1 and 0
    float eps;
    int32_t kind;                  // dc_norm_kind; DC_NORM_NONE: no norm
};

struct JoinArgs {
    View y, x, o, u;               // branch, residual, their sum, its norm
    View du, dr, dx, dy;           // backward: gradients at u and o; of the residual and the branch
    char* q;                       // o in 8 bits, written (forward); null: not
    Q8Map qm;
    Pixels px;
    JoinNorm post, pre;
    const float *scale, *gate;     // [C], [N][C]; null: 1
    DropArgs drop;
    float* stat;                   // [4][pixels]: mean and 1 / deviation of y, of o; null (forward): not kept
    float invC;
    int32_t C, blocks;
    int32_t lpx, nw, pg, held;     // as in NormArgs
    int32_t grid, cl;
    int32_t groups;                // pixel groups of a sample (of all pixels where there is no gate)
    // backward: parameters' gradients
    float *dscale, *dgate, *dgpost, *dbpost, *dgpre, *dbpre;   // null: not wanted
    float *part, *spart;           // workspace: [walker][4][32 blocks], [unit][32 blocks]
    int32_t samples, span;         // samples that sums are kept apart for; pixels of one
    int32_t slices, units;         // a sample's pixel groups are dealt to so many units; units in all
    int32_t accumulate;
    FastDiv dslices;
};
void join_plan(JoinArgs& a, bool backward);
size_t join_bwd_part_bytes(int N, int HW, int C, bool gate);
hipError_t launch_join_fwd(const JoinArgs& a, hipStream_t s);
hipError_t launch_join_bwd(const JoinArgs& a, hipStream_t s);

// a block as it lies in memory; channels past C repeat the last one
template <bool CL>
__device__ __forceinline__ void load_raw(uint32_t (&w)[32], const View& t, const Q8Map& qm, const Pixel& p, int c0, int C) {
    if (t.dt == DC_Q8) {
        const int64_t at = int64_t(c0 / 32) * qm.HW + p.pix;
        const uint4* d = reinterpret_cast<const uint4*>(t.p + p.n * qm.qn + at * 32);
        const uint4 a = d[0], b = d[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
        w[8] = reinterpret_cast<const uint8_t*>(t.p)[qm.s0 + p.n * qm.sn + at];
        return;
    }
    const int es = t.dt == DC_F32 ? 4 : 2;
    char* a = t.p + (p.n * t.sn + p.h * t.sh + p.w + c0 * (CL ? 1 : t.sc)) * es;
    if constexpr (CL) {
        if (c0 + 32 <= C) {
            const int n = es == 4 ? 8 : 4;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) {
                    const u32x4_any u = *reinterpret_cast<const u32x4_any*>(a + 16 * j);
                    w[4 * j] = u.x, w[4 * j + 1] = u.y, w[4 * j + 2] = u.z, w[4 * j + 3] = u.w;
                }
        } else if (es == 4) {
#pragma unroll
            for (int j = 0; j < 32; ++j) w[j] = reinterpret_cast<const uint32_t*>(a)[min(j, C - 1 - c0)];
        } else {
            const uint16_t* e = reinterpret_cast<const uint16_t*>(a);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                w[j] = e[min(2 * j, C - 1 - c0)] | uint32_t(e[min(2 * j + 1, C - 1 - c0)]) << 16;
        }
    } else {
        const int64_t step = t.sc * es;
        if (es == 4) {
#pragma unroll
            for (int j = 0; j < 32; ++j, next(a, c0 + j < C ? step : 0)) w[j] = *reinterpret_cast<const uint32_t*>(a);
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j, next(a, c0 + j < C ? step : 0)) w[j] = *reinterpret_cast<const uint16_t*>(a);
        }
    }
}

// its values; channels past C are zero
template <bool CL>
__device__ __forceinline__ void raw_values(float (&v)[32], const uint32_t (&w)[32], const View& t, int c0, int C) {
    if (t.dt == DC_Q8) {
        const float step = q8_step(w[8]);
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = q8_value(w[j / 4], j % 4, step);
    } else if (t.dt == DC_F32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __builtin_bit_cast(float, w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if constexpr (CL) v[j] = __builtin_bit_cast(float, j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
            else v[j] = __builtin_bit_cast(float, w[j] << 16);
        }
    }
    if (c0 + 32 > C) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = c0 + j < C ? v[j] : 0.0f;
    }
}

// what channel c0 + j of pixel p's sample is multiplied by
template <int LPX>
__device__ __forceinline__ void load_factor(float (&f)[32], const JoinArgs& a, const Pixel& p, int c0) {
    load_params<LPX>(f, a.scale, c0, a.C, 1.0f);
    if (a.gate) {
        float g[32];
        load_params<16>(g, a.gate + int64_t(p.n) * a.C, c0, a.C, 1.0f);
#pragma unroll
        for (int j = 0; j < 32; ++j) f[j] *= g[j];
    }
}

#define DC_JOIN_LAUNCH(KERNEL, HELD, a, g, s)                                                                     \
    do {                                                                                                          \
        const dim3 b_(64 * (a).nw * (a).pg);                                                                      \
        if ((a).lpx == 64 && (a).held == 1) hipLaunchKernelGGL((KERNEL<64, 1, false>), g, b_, 0, s, a);            \
        else if ((a).lpx == 64) hipLaunchKernelGGL((KERNEL<64, HELD, false>), g, b_, 0, s, a);                     \
        else if ((a).lpx == 16 && !(a).cl && (a).held == 1) hipLaunchKernelGGL((KERNEL<16, 1, false>), g, b_, 0, s, a);   \
        else if ((a).lpx == 16 && !(a).cl) hipLaunchKernelGGL((KERNEL<16, 0, false>), g, b_, 0, s, a);             \
        else if ((a).lpx == 16) hipLaunchKernelGGL((KERNEL<16, 1, true>), g, b_, 0, s, a);                         \
        else if ((a).held == 1) hipLaunchKernelGGL((KERNEL<4, 1, true>), g, b_, 0, s, a);                          \
        else hipLaunchKernelGGL((KERNEL<4, 0, true>), g, b_, 0, s, a);                                             \
    } while (0)

}  // namespace dc
