// The join of a branch with its residual stream, forward.
//
//   v = post(y),  o = x + scale gate drop(v),  u = pre(o)
//
// Bound: memory.  One pass: y and x are held in registers, the variances come from centred
// values, o goes from the registers where it is formed (before its rounding) into u.
#include <algorithm>

#include "join.h"

namespace dc {

template <int LPX, int R, bool CL>
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
        load_raw<CL>(w, a.y, a.qm, p, cb * 32, a.C);
        raw_values<CL>(v[i], w, a.y, cb * 32, a.C);
    };
    if constexpr (R) {
        uint32_t wy[H][32];
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
            load_raw<CL>(wy[i], a.y, a.qm, p, cb * 32, a.C);
            if (a.x.p) load_raw<CL>(wx[i], a.x, a.qm, p, cb * 32, a.C);
        });
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) { raw_values<CL>(v[i], wy[i], a.y, cb * 32, a.C); });
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
            if (a.x.p) load_raw<CL>(wx[0], a.x, a.qm, p, c0, a.C);
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
                const Philox w = philox(dp.pos + uint64_t(cb * 4 + k) * uint64_t(a.drop.plane), dp.ctr, a.drop.seed);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v[i][8 * k + j] = kept(w, j, a.drop.t) ? v[i][8 * k + j] * a.drop.scale : 0.0f;
            }
        }
        if (a.scale || a.gate) {
            float f[32];
            load_factor<LPX>(f, a, p, c0);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[i][j] *= f[j];
        }
        if (a.x.p) {
            float x[32];
            raw_values<CL>(x, wx[i], a.x, c0, a.C);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[i][j] += x[j];
        }
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
        store_any<CL>(a.o, p, c0, a.C, v[i]);
        if (a.q) q8_store_block(a.q, a.qm, p, cb, v[i]);
        if (a.pre.kind && a.u.p) {
            float g[32], b[32];
            load_params<LPX>(g, a.pre.gamma, c0, a.C, 1.0f);
            load_params<LPX>(b, a.pre.beta, c0, a.C, 0.0f);
#pragma unroll
            for (int j = 0; j < 32; ++j) g[j] = fmaf(g[j], (v[i][j] - mu2) * r2, b[j]);
            store_any<CL>(a.u, p, c0, a.C, g);
        }
    });
}

// As the layer norm's (norm_fwd.hip): rows of channels with a pixel's lanes next to each
// other, tiles with 64 pixels a wave, or 16 where there are few or many channels.
void join_plan(JoinArgs& a, bool backward) {
    a.blocks = (a.C + 31) / 32;
    a.invC = 1.0f / float(a.C);
    const int64_t waves = (int64_t(a.px.M) + 63) / 64 * a.blocks;
    if (a.cl)
        a.lpx = a.blocks >= 16 ? 4 : 16;
    else
        a.lpx = a.blocks <= (backward ? 1 : 2) * kNormWaves && waves >= 2048 ? 64 : 16;
    const int sb = 64 / a.lpx;
    a.nw = std::min((a.blocks + sb - 1) / sb, kNormWaves);
    const int held = (a.blocks + a.nw * sb - 1) / (a.nw * sb);
    a.held = held <= 1 ? 1 : held == 2 && a.lpx == 64 ? 2 : 0;
    if (!backward) {
        a.groups = int((int64_t(a.px.M) + a.lpx - 1) / a.lpx);
        a.pg = std::max(1, std::min(4 / a.nw, a.groups / 512));
        a.grid = (a.groups + a.pg - 1) / a.pg;
        return;
    }
    // Where there is a gate its sums are kept apart for each sample.
    a.samples = a.gate ? a.px.M / a.px.HW : 1;
    a.span = a.gate ? a.px.HW : a.px.M;
    a.groups = int((int64_t(a.span) + a.lpx - 1) / a.lpx);
    const int64_t all = int64_t(a.groups) * a.samples;
    a.pg = int(std::max<int64_t>(1, std::min<int64_t>(4 / a.nw, (all + 511) / 512)));
    const int64_t grid = (all + a.pg - 1) / a.pg;
    a.grid = int(std::min<int64_t>(grid, 256 * std::clamp(8 / (a.nw * a.pg), 1, 2)));
    // Units: slices of a sample's groups.  Walkers take them in turns; of one to four times as
    // many units as walkers, what leaves the least idle.
    const int walkers = a.grid * a.pg;
    a.slices = std::min(walkers, a.groups);
    if (a.gate) {
        int64_t best = 0;
        for (int k = 1; k <= 4; ++k) {
            const int64_t s = std::max<int64_t>(1, std::min<int64_t>(a.groups, int64_t(k) * walkers / a.samples));
            const int64_t turns = (s * a.samples + walkers - 1) / walkers * ((a.groups + s - 1) / s);
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
    DC_JOIN_LAUNCH(join_fwd_kernel, 2, a, dim3(x, (unsigned(a.grid) + x - 1) / x), s);
    return hipGetLastError();
}

}  // namespace dc
