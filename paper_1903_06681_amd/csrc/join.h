// The join of a block's branch with its residual stream, what both passes share:
//
//   o = x + scale gate drop(post(y)),  u = pre(o)
//
// post and pre are norms of a pixel over its channels (layer, root mean square, or none).  The
// tensors' types are known at run time: channels are loaded as they lie in memory, and widened
// when all loads are on their way.
#pragma once

#include "drop.h"
#include "eight.h"
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
    int32_t form_o;                // backward: o is formed from y and x; else x is o
    char* q;                       // o in 8 bits, written (forward); null: not
    Q8Map qm;
    Pixels px;
    JoinNorm post, pre;
    const float *scale, *gate;     // [C], [N][C]; null: 1
    DropArgs drop;
    float* stat;                   // [4][pixels]: mean and 1 / deviation of y, of o; null (forward): not kept
    float invC;
    int32_t C, blocks;
    int32_t eights;                // lanes of eight channels, else of 32
    int32_t lpx, nw, pg, held;     // as in NormArgs; held: eights, or blocks of 32 channels
    int32_t grid, cl;
    int32_t groups;                // pixel groups (backward: of a sample, or of all pixels where there is no gate)
    // backward: parameters' gradients
    float *dscale, *dgate, *dgpost, *dbpost, *dgpre, *dbpre;   // null: not wanted
    float *part, *spart;           // workspace: [workgroup][4][32 blocks], [unit][32 blocks]
    int32_t samples, span;         // samples that sums are kept apart for; pixels of one
    int32_t slices, units;         // a sample's pixel groups are dealt to so many units; units in all
    int32_t accumulate;
    FastDiv dslices;
};
void join_plan(JoinArgs& a, bool backward);
size_t join_bwd_part_bytes(int N, int HW, int C, bool gate);
hipError_t launch_join_fwd(const JoinArgs& a, hipStream_t s);
hipError_t launch_join_bwd(const JoinArgs& a, hipStream_t s);

// Planes: a block of 32 channels as it lies in memory; channels past C repeat the last one
__device__ __forceinline__ void load_raw(uint32_t (&w)[32], const View& t, const Pixel& p, int c0, int C) {
    const int es = t.dt == DC_F32 ? 4 : 2;
    char* a = t.p + (p.n * t.sn + p.h * t.sh + p.w + c0 * t.sc) * es;
    const int64_t step = t.sc * es;
    if (es == 4) {
#pragma unroll
        for (int j = 0; j < 32; ++j, next(a, c0 + j < C ? step : 0)) w[j] = *reinterpret_cast<const uint32_t*>(a);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j, next(a, c0 + j < C ? step : 0)) w[j] = *reinterpret_cast<const uint16_t*>(a);
    }
}

// its values; channels past C are zero
__device__ __forceinline__ void raw_values(float (&v)[32], const uint32_t (&w)[32], const View& t, int c0, int C) {
    if (t.dt == DC_F32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __builtin_bit_cast(float, w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __builtin_bit_cast(float, w[j] << 16);
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

// ---- lanes of eight channels: what a call of the generator serves, and 16 bytes of bf16.
//
// Planes: a wave takes LPX pixels next to each other, and 64 / LPX eights of channels.  Rows
// of channels (CL): 64 / LPX neighbouring lanes a row.  A lane holds R eights of one pixel, or
// (R = 0) goes through any number of them one by one, and the row again for every sum.

static constexpr int kJoinWaves = 8;    // most waves of a workgroup

struct JoinLane { int px, unit, ng, pg, wave; };
template <int LPX, bool CL>
__device__ __forceinline__ JoinLane join_lane(const JoinArgs& a) {
    constexpr int U = 64 / LPX;
    const int lane = threadIdx.x & 63;
    JoinLane l;
    l.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    l.pg = l.wave / a.nw;
    l.px = CL ? lane / U : lane % LPX;
    l.unit = (l.wave - l.pg * a.nw) * U + (CL ? lane % U : lane / LPX);     // uniform where LPX is 64
    l.ng = a.nw * U;
    return l;
}

// f(slot, eight) for the eights of a lane
template <int R, typename F>
__device__ __forceinline__ void each_eight(const JoinArgs& a, const JoinLane& l, F&& f) {
    const int eights = (a.C + 7) / 8;
    if constexpr (R) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (l.unit + i * l.ng < eights) f(i, l.unit + i * l.ng);
    } else {
        for (int e = l.unit; e < eights; e += l.ng) f(0, e);
    }
}

// v plus the value of the lane D on or back, D = 1, 2, 4 .. in turn: no trip through LDS.  D = 4
// and 8 mirror the lanes, whose values agree below D by then.
template <int D>
__device__ __forceinline__ float add_across(float v) {
    const int b = __builtin_bit_cast(int, v);
    if constexpr (D <= 8) {
        constexpr int ctrl = D == 1 ? 0xb1 : D == 2 ? 0x4e : D == 4 ? 0x141 : 0x140;   // quad_perm, row_half_mirror, row_mirror
        return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, b, ctrl, 0xf, 0xf, true));
    } else if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        return __builtin_bit_cast(float, int(r[0])) + __builtin_bit_cast(float, int(r[1]));
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        return __builtin_bit_cast(float, int(r[0])) + __builtin_bit_cast(float, int(r[1]));
    }
}
// over the lanes that are equal modulo LPX (planes)
template <int N>
__device__ __forceinline__ float add_rotated(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, true));
}
template <int LPX, bool CL>
__device__ __forceinline__ float add_lanes(float v) {
    constexpr int U = 64 / LPX;
    if constexpr (CL) {
        if constexpr (U > 1) v = add_across<1>(v);
        if constexpr (U > 2) v = add_across<2>(v);
        if constexpr (U > 4) v = add_across<4>(v);
        if constexpr (U > 8) v = add_across<8>(v);
        if constexpr (U > 16) v = add_across<16>(v);
        if constexpr (U > 32) v = add_across<32>(v);
    } else {
        if constexpr (LPX <= 8) v = add_rotated<8>(v);
        if constexpr (LPX <= 4) v = add_rotated<4>(v);
        if constexpr (LPX <= 16) v = add_across<16>(v);
        if constexpr (LPX <= 32) v = add_across<32>(v);
    }
    return v;
}

// Sums of K values over the lanes of a pixel, in all of them, in a fixed order.
template <int LPX, bool CL, int K>
__device__ __forceinline__ void lane_sum(float (&v)[K], const JoinArgs& a, const JoinLane& l, float (&red)[K][kJoinWaves * LPX]) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = add_lanes<LPX, CL>(v[k]);
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

template <bool UNIFORM>
__device__ __forceinline__ void factor8(float (&f)[8], const JoinArgs& a, const Pixel& p, int c0) {
    params8<UNIFORM>(f, a.scale, c0, a.C, 1.0f);
    if (a.gate) {
        float g[8];
        params8<false>(g, a.gate + int64_t(p.n) * a.C, c0, a.C, 1.0f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= g[j];
    }
}

}  // namespace dc
