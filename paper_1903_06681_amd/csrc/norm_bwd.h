// Layer norm over the channels of each pixel, backward.
//
//   xh = (x - mu) r,  g = gamma du,  dx = r (g - mean g - xh mean(g xh)) + res
//   dgamma = sum over pixels of du xh,  dbeta = sum over pixels of du
//
// Bound: memory.  As in the forward pass a lane holds one pixel's block of 32
// channels of x (or of its 8-bit form) and of du, read once.  The parameters'
// sums: the 64 products of a block are summed over the wave's pixels by halving
// (each step a lane gives away half of its values), 63 exchanges for 64 sums, which
// leaves one register a block to carry along a workgroup's pixels; the workgroups'
// sums are added in order by a second launch.  No atomics.  4 x 64 x 256 x 256
// from the checkpoint, skip path added, u formed again (151 MB): 46 to 50 us and 5 for the
// second launch; three waves a SIMD with 8 to 40 bytes of scratch a lane (four do not fit the
// registers: 111 us).  Rows of more than 4096 channels (tiles of more than 1024) are read
// again for each sum: 2048 rows of 8192 in bf16 69.5 us, of 4096 29.6.
#pragma once

#include "norm.h"

namespace dc {

// XT: float or __bf16 of the tile, or char: the checkpoint.
template <typename XT, typename DT, int LPX, int R, bool CL>
__global__ __launch_bounds__(512, LPX == 64 && R == 1 ? 3 : 2) void norm_bwd_kernel(NormArgs a) {
    constexpr bool Q = sizeof(XT) == 1;
    constexpr int H = R ? R : 1, E = 64 / LPX;
    __shared__ float red[2][2][kNormWaves * LPX];
    __shared__ float psum[R ? kNormWaves : 1][H * E * 64];
    const NormLane l = norm_lane<LPX>(a);
    const int lane = threadIdx.x & 63;
    const bool params = a.dgamma || a.dbeta;
    // value e of this lane's parameter sums of block cb lies here
    auto part_at = [&](int cb, int e) __attribute__((always_inline)) {
        const int v = l.px * E + e;
        return a.part + (int64_t(blockIdx.x) * 2 + v / 32) * a.blocks * 32 + cb * 32 + v % 32;
    };
    float acc[H][E];
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[i][e] = 0;
    if (!R && params)
        each_block<R>(a, l, [&](int, int cb) {
            for (int e = 0; e < E; ++e) *part_at(cb, e) = 0;
        });
    int par = 0;
    // Every wave of a workgroup takes the same number of turns.  Where a wave's rows are short,
    // neighbours share an XCD, and their lines meet in its L2 (1024 channels on 32 x 14 x 14
    // read 129 MB of memory for 32 MB otherwise: 48 us against 38).
    const int first = LPX == 64 ? int(blockIdx.x) : xcd_range(blockIdx.x, a.grid);
    for (int g0 = first * a.pg; g0 < a.groups; g0 += a.grid * a.pg, par ^= 1) {
        const int m = (g0 + l.pg) * LPX + l.px;
        const bool in = m < a.px.M;
        const int mm = min(m, a.px.M - 1);
        const Pixel p = pixel_of<true>(a.px, m);
        const float mu = a.stat[mm], r = a.stat[int64_t(a.px.M) + mm];
        float vx[H][32], vd[H][32];
        auto load = [&](int i, int cb) __attribute__((always_inline)) {
            if constexpr (Q)
                q8_load_block(vx[i], a.q, a.qm, p, cb);
            else
                load_block<XT, CL>(vx[i], a.x, p, cb * 32, a.C);
            load_block<DT, CL>(vd[i], a.du, p, cb * 32, a.C);
        };
        auto centre = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 32; ++j) vx[i][j] = (vx[i][j] - mu) * r;
        };
        float s[2] = {0, 0};
        if constexpr (R) each_block<R>(a, l, load);
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
            if constexpr (!R) load(0, cb);
            centre(i);
            float gm[32];
            load_params<LPX>(gm, a.gamma, cb * 32, a.C, 1.0f);
#pragma unroll
            for (int j = 0; j < 32; ++j) {     // du is zero past C, x finite there or NaN with the pixel
                const float g = gm[j] * vd[i][j];
                s[0] += g;
                s[1] = fmaf(g, cb * 32 + j < a.C ? vx[i][j] : 0.0f, s[1]);
            }
        });
        pixel_sum<LPX>(s, a, l, red[par]);
        const float m1 = s[0] * a.invC, m2 = s[1] * a.invC;
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
            if constexpr (!R) {
                load(0, cb);
                centre(0);
            }
            if (params) {
                float t[64];
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    t[j] = in ? vd[i][j] * vx[i][j] : 0.0f;
                    t[32 + j] = in ? vd[i][j] : 0.0f;
                }
                sum_lanes<LPX>(t, lane);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (R)
                        acc[i][e] += t[e];
                    else
                        *part_at(cb, e) += t[e];
                }
            }
            if (!in) return;
            float gm[32], o[32];
            load_params<LPX>(gm, a.gamma, cb * 32, a.C, 1.0f);
            if (a.res.p) load_any<CL>(o, a.res, p, cb * 32, a.C);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float d = fmaf(-vx[i][j], m2, fmaf(gm[j], vd[i][j], -m1));
                o[j] = a.res.p ? fmaf(r, d, o[j]) : r * d;
            }
            store_any<CL>(a.dx, p, cb * 32, a.C, o);
            if (a.u.p) {
                load_params<LPX>(o, a.beta, cb * 32, a.C, 0.0f);
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = fmaf(gm[j], vx[i][j], o[j]);
                store_any<CL>(a.u, p, cb * 32, a.C, o);
            }
        });
    }
    if constexpr (R) {
        if (!params) return;
        if (a.pg > 1) {     // the workgroup's pixel groups, in order
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) psum[l.wave][(i * E + e) * 64 + lane] = acc[i][e];
            __syncthreads();
            if (l.pg != 0) return;
            for (int g = 1; g < a.pg; ++g)
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[i][e] += psum[g * a.nw + l.wave][(i * E + e) * 64 + lane];
        }
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < E; ++e) *part_at(cb, e) = acc[i][e];
        });
    }
}

}  // namespace dc
