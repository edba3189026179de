// The join of a branch with its residual stream, forward.
//
//   v = post(y),  o = x + scale gate drop(v),  u = pre(o)
//
// Bound: memory.  One pass: y and x are held in registers, the variances come from centred
// values, o goes from the registers where it is formed (before its rounding) into u.  4 x 64 x 256 x
// 256 with fp32 x 52 us (3.9 TB/s), 8192 rows of 1024 bf16 24 (2.8; 15 us of vector operations).
#include <algorithm>

#include "join.h"

namespace dc {

// Planes: as in the layer norm (norm.h) a lane holds one pixel's blocks of 32 channels.
template <int LPX, int R>
__global__ __launch_bounds__(512) void join_fwd_kernel(JoinArgs a) {
    constexpr int H = R ? R : 1;
    __shared__ float red[4][1][kNormWaves * LPX];
    const NormLane l = norm_lane<LPX>(a);
    const int wg = int(blockIdx.y * gridDim.x + blockIdx.x);
    if (wg >= a.grid) return;
    const int m = (xcd_range(wg, a.grid) * a.pg + l.pg) * LPX + l.px;
    const bool in = m < a.px.M;
    const Pixel p = pixel_of(a.px, m);
    float v[H][32];
    uint32_t wx[H][32];
    auto load_y = [&](int i, int cb) __attribute__((always_inline)) {
        uint32_t w[32];
        load_raw(w, a.y, p, cb * 32, a.C);
        raw_values(v[i], w, a.y, cb * 32, a.C);
    };
    if constexpr (R) {
        uint32_t wy[H][32];
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
            load_raw(wy[i], a.y, p, cb * 32, a.C);
            if (a.x.p) load_raw(wx[i], a.x, p, cb * 32, a.C);
        });
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) { raw_values(v[i], wy[i], a.y, cb * 32, a.C); });
    }
    // mean and 1 / deviation of what `form` leaves in v
    auto moments = [&](const JoinNorm& k, int at, float& mu, float& r, auto&& form) __attribute__((always_inline)) {
        float s[1] = {0};
        mu = 0;
        if (k.kind == DC_NORM_LAYER) {
            each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
                if constexpr (!R) form(i, cb);
#pragma unroll
                for (int j = 0; j < 32; ++j) s[0] += v[i][j];
            });
            pixel_sum<LPX>(s, a, l, red[at]);
            mu = s[0] * a.invC;
            s[0] = 0;
        }
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
            if constexpr (!R) form(i, cb);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float d = cb * 32 + j < a.C ? v[i][j] - mu : 0.0f;
                s[0] = fmaf(d, d, s[0]);
            }
        });
        pixel_sum<LPX>(s, a, l, red[at + 1]);
        r = 1.0f / sqrtf(s[0] * a.invC + k.eps);
    };
    auto keep = [&](int at, float mu, float r) __attribute__((always_inline)) {
        if (a.stat && in && l.unit == 0) {
            a.stat[int64_t(at) * a.px.M + m] = mu;
            a.stat[int64_t(at + 1) * a.px.M + m] = r;
        }
    };
    float mu1 = 0, r1 = 0;
    if (a.post.kind) {
        moments(a.post, 0, mu1, r1, load_y);
        keep(0, mu1, r1);
    }
    DropPixel dp{};
    if (a.drop.t) dp = drop_pixel(a.drop, p.n, p.pix);
    // y in v -> o
    auto join = [&](int i, int cb) __attribute__((always_inline)) {
        const int c0 = cb * 32;
        if constexpr (!R) {
            load_y(0, cb);
            if (a.x.p) load_raw(wx[0], a.x, p, c0, a.C);
        }
        if (a.post.kind) {
            float g[32], b[32];
            load_params<LPX>(g, a.post.gamma, c0, a.C, 1.0f);
            load_params<LPX>(b, a.post.beta, c0, a.C, 0.0f);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[i][j] = fmaf(g[j], (v[i][j] - mu1) * r1, b[j]);
        }
        if (a.drop.t) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float keep[8];
                keep8(keep, a.drop, dp, cb * 4 + k);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][8 * k + j] = dropped(v[i][8 * k + j], keep[j]);
            }
        }
        float f[32], x[32];
        load_factor<LPX>(f, a, p, c0);
        if (a.x.p) raw_values(x, wx[i], a.x, c0, a.C);
#pragma unroll
        for (int j = 0; j < 32; ++j) v[i][j] = fmaf(v[i][j], f[j], a.x.p ? x[j] : 0.0f);
        if (c0 + 32 > a.C) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[i][j] = c0 + j < a.C ? v[i][j] : 0.0f;
        }
    };
    if constexpr (R) each_block<R>(a, l, join);
    float mu2 = 0, r2 = 0;
    if (a.pre.kind) {
        moments(a.pre, 2, mu2, r2, join);
        keep(2, mu2, r2);
    }
    if (!in) return;
    each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
        const int c0 = cb * 32;
        if constexpr (!R) join(0, cb);
        store_any<false>(a.o, p, c0, a.C, v[i]);
        if (a.q) q8_store_block(a.q, a.qm, p, cb, v[i]);
        if (a.pre.kind && a.u.p) {
            float g[32], b[32];
            load_params<LPX>(g, a.pre.gamma, c0, a.C, 1.0f);
            load_params<LPX>(b, a.pre.beta, c0, a.C, 0.0f);
#pragma unroll
            for (int j = 0; j < 32; ++j) g[j] = fmaf(g[j], (v[i][j] - mu2) * r2, b[j]);
            store_any<false>(a.u, p, c0, a.C, g);
        }
    });
}

// Rows of channels (CL), a row's lanes next to each other, and planes of few channels: eight
// channels a lane.
template <int LPX, int R, bool CL>
__global__ __launch_bounds__(512) void join_eights_fwd_kernel(JoinArgs a) {
    constexpr int H = R ? R : 1;
    __shared__ float red[4][1][kJoinWaves * LPX];
    const JoinLane l = join_lane<LPX, CL>(a);
    const int wg = int(blockIdx.y * gridDim.x + blockIdx.x);
    if (wg >= a.grid) return;
    const int m = (wg * a.pg + l.pg) * LPX + l.px;
    const bool in = m < a.px.M;
    const Pixel p = pixel_of(a.px, m);
    float v[H][8];
    u32x8 wx[H];
    auto load_y = [&](int i, int e) __attribute__((always_inline)) {
        values8<CL>(v[i], load8<CL>(a.y, a.qm, p, 8 * e, a.C), a.y, 8 * e, a.C);
    };
    if constexpr (R) {
        u32x8 wy[H];
        each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
            wy[i] = load8<CL>(a.y, a.qm, p, 8 * e, a.C);
            if (a.x.p) wx[i] = load8<CL>(a.x, a.qm, p, 8 * e, a.C);
        });
        each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) { values8<CL>(v[i], wy[i], a.y, 8 * e, a.C); });
    }
    // mean and 1 / deviation of what `form` leaves in v
    auto moments = [&](const JoinNorm& k, int at, float& mu, float& r, auto&& form) __attribute__((always_inline)) {
        float s[1] = {0};
        mu = 0;
        if (k.kind == DC_NORM_LAYER) {
            each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
                if constexpr (!R) form(i, e);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[0] += v[i][j];
            });
            lane_sum<LPX, CL>(s, a, l, red[at]);
            mu = s[0] * a.invC;
            s[0] = 0;
        }
        each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
            if constexpr (!R) form(i, e);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = 8 * e + j < a.C ? v[i][j] - mu : 0.0f;
                s[0] = fmaf(d, d, s[0]);
            }
        });
        lane_sum<LPX, CL>(s, a, l, red[at + 1]);
        r = 1.0f / sqrtf(s[0] * a.invC + k.eps);
        if (a.stat && in && l.unit == 0) {
            a.stat[int64_t(at) * a.px.M + m] = mu;
            a.stat[int64_t(at + 1) * a.px.M + m] = r;
        }
    };
    float mu1 = 0, r1 = 0;
    if (a.post.kind) moments(a.post, 0, mu1, r1, load_y);
    DropPixel dp{};
    if (a.drop.t) dp = drop_pixel(a.drop, p.n, p.pix);
    // y in v -> o
    auto join = [&](int i, int e) __attribute__((always_inline)) {
        const int c0 = 8 * e;
        if constexpr (!R) {
            load_y(0, e);
            if (a.x.p) wx[0] = load8<CL>(a.x, a.qm, p, c0, a.C);
        }
        if (a.post.kind) {
            float g[8], b[8];
            params8<LPX == 64>(g, a.post.gamma, c0, a.C, 1.0f);
            params8<LPX == 64>(b, a.post.beta, c0, a.C, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = fmaf(g[j], (v[i][j] - mu1) * r1, b[j]);
        }
        float f[8], k[8], x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        keep8(k, a.drop, dp, e);
        factor8<LPX == 64>(f, a, p, c0);
        if (a.x.p) values8<CL>(x, wx[i], a.x, c0, a.C);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = fmaf(dropped(v[i][j], k[j]), f[j], x[j]);
        clear8(v[i], c0, a.C);
    };
    if constexpr (R) each_eight<R>(a, l, join);
    float mu2 = 0, r2 = 0;
    if (a.pre.kind) moments(a.pre, 2, mu2, r2, join);
    if (CL && a.q) { // the four lanes of a block of 32 channels together, also those past the last eight
        for (int i = 0, e = l.unit; e < a.blocks * 4; e += l.ng, ++i) {
            float o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (8 * e < a.C) {
                if constexpr (!R) join(0, e);
#pragma unroll
                for (int k = 0; k < H; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = k == i || !R ? v[k][j] : o[j];
            }
            q8_store_eight(a.q, a.qm, p, e, in, a.C, o);
        }
    }
    each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
        const int c0 = 8 * e;
        if constexpr (!R) join(0, e);
        if (in) store8<CL>(a.o, p, c0, a.C, v[i]);
        if (a.pre.kind && a.u.p) {
            float g[8], b[8];
            params8<LPX == 64>(g, a.pre.gamma, c0, a.C, 1.0f);
            params8<LPX == 64>(b, a.pre.beta, c0, a.C, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = fmaf(g[j], (v[i][j] - mu2) * r2, b[j]);
            if (in) store8<CL>(a.u, p, c0, a.C, g);
        }
    });
}

// Rows of channels: eight channels a lane, as many lanes as a row has eights, up to 64, then up to
// eight waves, then two eights a lane.  Planes, backward: 16 pixels a wave and four eights side by
// side, 64 and one where there are three eights at most (4 x 64 x 256 x 256: two waves of 16
// pixels 96 us, eight of 64, which meet at a barrier twice a step, 101), 4 for 257 to 2048 channels.
// Above that 16 again, and the eights one by one (held = 0: read again for every sum), as in rows of
// more than 8192 channels.  Planes, forward: up to three eights likewise (2 x 8 x 16 x 16 fp32 8 us, in lanes of 32
// channels 13); else as the layer norm's (norm_fwd.hip), 32 channels a lane, 64 pixels a
// wave, or 16 where there are few or many channels.
void join_plan(JoinArgs& a, bool backward) {
    a.blocks = (a.C + 31) / 32;
    a.invC = 1.0f / float(a.C);
    const int eights = (a.C + 7) / 8;
    const int64_t M = a.px.M, waves = (M + 63) / 64 * a.blocks;
    a.eights = a.cl || backward || (eights <= 3 && !a.q);
    if (a.eights) {
        if (a.cl) {
            a.lpx = 16;
            while (64 / a.lpx < eights && a.lpx > 1) a.lpx /= 2;
        } else {
            a.lpx = eights <= 3 ? 64 : eights <= 32 || eights > 256 ? 16 : 4;
        }
        const int u = 64 / a.lpx;
        a.held = eights <= 8 * u ? 1 : eights <= 16 * u ? 2 : 0;
        a.nw = std::min((eights + u * std::max(a.held, 1) - 1) / (u * std::max(a.held, 1)), kJoinWaves);
    } else {
        a.lpx = a.blocks <= 2 * kNormWaves && waves >= 2048 ? 64 : 16;
        const int sb = 64 / a.lpx;
        a.nw = std::min((a.blocks + sb - 1) / sb, kNormWaves);
        const int held = (a.blocks + a.nw * sb - 1) / (a.nw * sb);
        a.held = held <= 1 ? 1 : held == 2 && a.lpx == 64 ? 2 : 0;
    }
    if (!backward) {
        a.groups = int((M + a.lpx - 1) / a.lpx);
        a.pg = std::max(1, std::min(4 / a.nw, a.groups / 512));
        a.grid = (a.groups + a.pg - 1) / a.pg;
        return;
    }
    // Where there is a gate its sums are kept apart for each sample.
    a.samples = a.gate ? a.px.M / a.px.HW : 1;
    a.span = a.gate ? a.px.HW : a.px.M;
    a.groups = int((int64_t(a.span) + a.lpx - 1) / a.lpx);
    // Units: slices of a sample's groups.  Workgroups take them in turns; of one to four times as
    // many units as workgroups, what leaves the least idle.
    const int64_t all = int64_t(a.groups) * a.samples;
    a.pg = int(std::max<int64_t>(1, std::min<int64_t>(std::max(1, (a.cl ? 8 : 4) / a.nw), (all + 511) / 512)));
    a.grid = int(std::min<int64_t>((all + a.pg - 1) / a.pg, 256 * std::clamp(8 / (a.nw * a.pg), 1, 4)));
    const int most = (a.groups + a.pg - 1) / a.pg;
    a.slices = std::min(a.grid, most);
    if (a.gate) {
        int64_t best = 0;
        for (int k = 1; k <= 4; ++k) {
            const int64_t s = std::max<int64_t>(1, std::min<int64_t>(most, int64_t(k) * a.grid / a.samples));
            const int64_t turns = (s * a.samples + a.grid - 1) / a.grid * ((most + s - 1) / s);
            if (!best || turns < best) {
                best = turns;
                a.slices = int(s);
            }
        }
    }
    a.units = a.slices * a.samples;
    a.dslices = fast_div(uint32_t(a.slices));
}

hipError_t launch_join_fwd(const JoinArgs& a, hipStream_t s) {
    const unsigned x = unsigned(std::min(a.grid, 1 << 22));     // threads of a dimension: 32 bits
    const dim3 g(x, (unsigned(a.grid) + x - 1) / x), b(64 * a.nw * a.pg);
    if (a.cl) {
        if (a.lpx == 16) hipLaunchKernelGGL((join_eights_fwd_kernel<16, 1, true>), g, b, 0, s, a);
        else if (a.lpx == 8) hipLaunchKernelGGL((join_eights_fwd_kernel<8, 1, true>), g, b, 0, s, a);
        else if (a.lpx == 4) hipLaunchKernelGGL((join_eights_fwd_kernel<4, 1, true>), g, b, 0, s, a);
        else if (a.lpx == 2) hipLaunchKernelGGL((join_eights_fwd_kernel<2, 1, true>), g, b, 0, s, a);
        else if (a.held == 1) hipLaunchKernelGGL((join_eights_fwd_kernel<1, 1, true>), g, b, 0, s, a);
        else if (a.held == 2) hipLaunchKernelGGL((join_eights_fwd_kernel<1, 2, true>), g, b, 0, s, a);
        else hipLaunchKernelGGL((join_eights_fwd_kernel<1, 0, true>), g, b, 0, s, a);
    } else if (a.eights) {
        hipLaunchKernelGGL((join_eights_fwd_kernel<64, 1, false>), g, b, 0, s, a);
    } else if (a.lpx == 64) {
        if (a.held == 1) hipLaunchKernelGGL((join_fwd_kernel<64, 1>), g, b, 0, s, a);
        else hipLaunchKernelGGL((join_fwd_kernel<64, 2>), g, b, 0, s, a);
    } else {
        if (a.held == 1) hipLaunchKernelGGL((join_fwd_kernel<16, 1>), g, b, 0, s, a);
        else hipLaunchKernelGGL((join_fwd_kernel<16, 0>), g, b, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace dc
