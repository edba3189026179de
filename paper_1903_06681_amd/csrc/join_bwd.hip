// The join of a branch with its residual stream, backward.
//
//   dO = dr + pre'(du),  dx = dO,  dv = dO scale gate drop,  dy = post'(dv)
//
// with norm'(g) = r (gamma g - mean(gamma g) - xh mean(gamma g xh)) (no first mean for the
// root mean square), and the sums over pixels  dgamma = g xh,  dbeta = g  of both norms and
// t = dO drop(v) a sample, from which dgate = scale t and dscale = sum of gate t.
//
// Bound: memory.  One pass: y, x, du and dr are held in registers, and o is formed from the
// first two as the forward pass formed it, before its rounding (or read, where it is given).  The sums over pixels
// halve across a wave's lanes and are carried in registers along the pixel groups that
// a walker (the waves that share a pixel) takes; a second launch adds the walkers' sums in
// order.  No atomics.
#include <algorithm>

#include "join.h"

namespace dc {

// v where the mask's bit j is set, else 0
__device__ __forceinline__ float masked(float v, uint32_t bits, int j) {
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) & uint32_t(int32_t(bits << (31 - j)) >> 31));
}
__device__ __forceinline__ float dropped(float v, uint32_t bits, int j, const DropArgs& d) {
    return d.t ? masked(v * d.scale, bits, j) : v;
}

template <int LPX, int R, bool CL>
__global__ __launch_bounds__(512, 2) void join_bwd_kernel(JoinArgs a) {
    constexpr int H = R ? R : 1, E = 64 / LPX, ES = E > 1 ? E / 2 : 1;
    __shared__ float red[2][2][2][kNormWaves * LPX];
    const NormLane l = norm_lane<LPX>(a);
    const int lane = threadIdx.x & 63;
    const bool has_pre = a.pre.kind && a.du.p, has_post = a.post.kind != DC_NORM_NONE, has_y = a.y.p != nullptr;
    const bool want_pre = has_pre && (a.dgpre || a.dbpre), want_post = has_post && (a.dgpost || a.dbpost);
    const bool want_scale = a.dscale || a.dgate;
    const int width = a.blocks * 32, walkers = a.grid * a.pg;
    const int walker = xcd_range(blockIdx.x, a.grid) * a.pg + l.pg;
    // where value e of this lane's sums lies: of a norm's 64 (which: 0 pre, 1 post), of the 32 of t
    auto part_at = [&](int which, int cb, int e) __attribute__((always_inline)) {
        const int v = l.px * E + e;
        return a.part + (int64_t(walker) * 4 + which * 2 + v / 32) * width + cb * 32 + v % 32;
    };
    auto spart_at = [&](int unit, int cb, int e) __attribute__((always_inline)) {
        return a.spart + int64_t(unit) * width + cb * 32 + (LPX == 64 ? l.px / 2 : l.px * ES + e);
    };
    float acc[2][H][E], sacc[H][ES];
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[0][i][e] = acc[1][i][e] = 0;
    if constexpr (!R) {
        each_block<R>(a, l, [&](int, int cb) {
            for (int e = 0; e < E; ++e) {
                if (want_pre) *part_at(0, cb, e) = 0;
                if (want_post) *part_at(1, cb, e) = 0;
            }
        });
    }
    const int turns = (a.units + walkers - 1) / walkers, steps = (a.groups + a.slices - 1) / a.slices;
    int par = 0;
    // every wave takes the same number of turns and steps: barriers
    for (int turn = 0; turn < turns; ++turn) {
        const int unit = walker + turn * walkers, uu = min(unit, a.units - 1);
        const int smp = int(a.dslices.div(uint32_t(uu))), slice = uu - smp * a.slices;
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int e = 0; e < ES; ++e) sacc[i][e] = 0;
        if constexpr (!R) {
            if (want_scale && unit < a.units)
                each_block<R>(a, l, [&](int, int cb) {
                    for (int e = 0; e < ES; ++e) *spart_at(unit, cb, e) = 0;
                });
        }
        for (int st = 0; st < steps; ++st, par ^= 1) {
            const int64_t q = int64_t(slice + st * a.slices) * LPX + l.px;
            const bool in = unit < a.units && q < a.span;
            const int m = int(smp * int64_t(a.span) + min(q, int64_t(a.span) - 1));
            const Pixel p = pixel_of(a.px, m);
            float mu1 = 0, r1 = 0, mu2 = 0, r2 = 0;
            if (has_post) {
                mu1 = a.stat[m];
                r1 = a.stat[int64_t(a.px.M) + m];
            }
            if (has_pre) {
                mu2 = a.stat[2 * int64_t(a.px.M) + m];
                r2 = a.stat[3 * int64_t(a.px.M) + m];
            }
            DropPixel dp{};
            if (a.drop.t) dp = drop_pixel(a.drop, p.n, p.pix);
            // o's normed value; du, then dO, then dv; y's normed value (y without a norm); drop of what the
            // factor multiplies; the mask
            float vo[H][32], vd[H][32], vy[H][32], vt[H][32];
            uint32_t wr[H][32], bits[H];
            auto load = [&](int i, int cb) __attribute__((always_inline)) {
                const int c0 = cb * 32;
                uint32_t wo[32], wd[32], wy[32];
                if (has_pre) {
                    load_raw<CL>(wo, a.o.p ? a.o : a.x, a.qm, p, c0, a.C);
                    load_raw<CL>(wd, a.du, a.qm, p, c0, a.C);
                }
                if (has_y) load_raw<CL>(wy, a.y, a.qm, p, c0, a.C);
                if (a.dr.p) load_raw<CL>(wr[i], a.dr, a.qm, p, c0, a.C);
                bits[i] = ~0u;
                if (a.drop.t) {
                    bits[i] = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const Philox w = philox(dp.pos + uint64_t(cb * 4 + k) * uint64_t(a.drop.plane), dp.ctr, a.drop.seed);
#pragma unroll
                        for (int j = 0; j < 8; ++j) bits[i] |= kept(w, j, a.drop.t) ? 1u << (8 * k + j) : 0u;
                    }
                }
                if (has_y) {
                    raw_values<CL>(vy[i], wy, a.y, c0, a.C);
                    float g[32], b[32];
                    if (has_post) {
                        load_params<LPX>(g, a.post.gamma, c0, a.C, 1.0f);
                        load_params<LPX>(b, a.post.beta, c0, a.C, 0.0f);
#pragma unroll
                        for (int j = 0; j < 32; ++j) vy[i][j] = (vy[i][j] - mu1) * r1;
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) vt[i][j] = dropped(has_post ? fmaf(g[j], vy[i][j], b[j]) : vy[i][j], bits[i], j, a.drop);
                }
                if (has_pre) {
                    raw_values<CL>(vo[i], wo, a.o.p ? a.o : a.x, c0, a.C);
                    raw_values<CL>(vd[i], wd, a.du, c0, a.C);
                    if (!a.o.p) {      // o as the forward pass formed it
                        float f[32];
                        load_factor<LPX>(f, a, p, c0);
#pragma unroll
                        for (int j = 0; j < 32; ++j) vo[i][j] += f[j] * vt[i][j];
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j) vo[i][j] = (vo[i][j] - mu2) * r2;
                }
            };
            if constexpr (R) each_block<R>(a, l, load);
            float m1 = 0, m2 = 0;
            if (has_pre) {
                float s[2] = {0, 0};
                each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
                    if constexpr (!R) load(0, cb);
                    float gm[32];
                    load_params<LPX>(gm, a.pre.gamma, cb * 32, a.C, 1.0f);
#pragma unroll
                    for (int j = 0; j < 32; ++j) {     // du is zero past C, the normed value finite there or NaN with the pixel
                        const float g = gm[j] * vd[i][j];
                        s[0] += g;
                        s[1] = fmaf(g, cb * 32 + j < a.C ? vo[i][j] : 0.0f, s[1]);
                    }
                });
                pixel_sum<LPX>(s, a, l, red[par][0]);
                m1 = a.pre.kind == DC_NORM_LAYER ? s[0] * a.invC : 0.0f;
                m2 = s[1] * a.invC;
            }
            // sums over pixels of 64 values, f(j) and g(j)
            auto sums = [&](int which, int i, int cb, auto&& f, auto&& g) __attribute__((always_inline)) {
                float t[64];
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    t[j] = in ? f(j) : 0.0f;
                    t[32 + j] = in ? g(j) : 0.0f;
                }
                sum_lanes<LPX>(t, lane);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (R) acc[which][i][e] += t[e];
                    else *part_at(which, cb, e) += t[e];
                }
            };
            auto pre_sums = [&](int i, int cb) __attribute__((always_inline)) {
                if (want_pre) sums(0, i, cb, [&](int j) { return vd[i][j] * vo[i][j]; }, [&](int j) { return vd[i][j]; });
            };
            // dO in vd
            auto through_pre = [&](int i, int cb) __attribute__((always_inline)) {
                float e[32];
                if (a.dr.p) raw_values<CL>(e, wr[i], a.dr, cb * 32, a.C);
                if (has_pre) {
                    float gm[32];
                    load_params<LPX>(gm, a.pre.gamma, cb * 32, a.C, 1.0f);
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const float d = fmaf(-vo[i][j], m2, fmaf(gm[j], vd[i][j], -m1));
                        vd[i][j] = a.dr.p ? fmaf(r2, d, e[j]) : r2 * d;
                    }
                    if (cb * 32 + 32 > a.C) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) vd[i][j] = cb * 32 + j < a.C ? vd[i][j] : 0.0f;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) vd[i][j] = e[j];
                }
            };
            // dO in vd -> dv; the sum t
            auto branch = [&](int i, int cb, bool with_t) __attribute__((always_inline)) {
                if (with_t) {
                    float t[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) t[j] = in ? vd[i][j] * vt[i][j] : 0.0f;
                    if (a.drop.t) {        // a dropped value is 0 times nothing, whatever dO is
#pragma unroll
                        for (int j = 0; j < 32; ++j) t[j] = masked(t[j], bits[i], j);
                    }
                    sum_lanes<LPX>(t, lane);
#pragma unroll
                    for (int e = 0; e < ES; ++e) {
                        if constexpr (R) sacc[i][e] += t[e];
                        else if (unit < a.units && (LPX < 64 || l.px % 2 == 0)) *spart_at(unit, cb, e) += t[e];
                    }
                }
                float f[32];
                load_factor<LPX>(f, a, p, cb * 32);
#pragma unroll
                for (int j = 0; j < 32; ++j) vd[i][j] = dropped(vd[i][j] * f[j], bits[i], j, a.drop);
            };
            float s[2] = {0, 0};
            auto post_moments = [&](int i, int cb) __attribute__((always_inline)) {
                float gm[32];
                load_params<LPX>(gm, a.post.gamma, cb * 32, a.C, 1.0f);
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float g = gm[j] * vd[i][j];
                    s[0] += g;
                    s[1] = fmaf(g, cb * 32 + j < a.C ? vy[i][j] : 0.0f, s[1]);
                }
            };
            if constexpr (R) {
                each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
                    pre_sums(i, cb);
                    through_pre(i, cb);
                    if (in && a.dx.p) store_any<CL>(a.dx, p, cb * 32, a.C, vd[i]);
                    branch(i, cb, want_scale);
                    if (has_post) post_moments(i, cb);
                });
            } else if (has_post) {
                each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
                    load(0, cb);
                    through_pre(0, cb);
                    branch(0, cb, false);
                    post_moments(0, cb);
                });
            }
            float n1 = 0, n2 = 0;
            if (has_post) {
                pixel_sum<LPX>(s, a, l, red[par][1]);
                n1 = a.post.kind == DC_NORM_LAYER ? s[0] * a.invC : 0.0f;
                n2 = s[1] * a.invC;
            }
            each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
                if constexpr (!R) {
                    load(0, cb);
                    pre_sums(0, cb);
                    through_pre(0, cb);
                    if (in && a.dx.p) store_any<CL>(a.dx, p, cb * 32, a.C, vd[0]);
                    branch(0, cb, want_scale);
                }
                if (has_post) {
                    if (want_post) sums(1, i, cb, [&](int j) { return vd[i][j] * vy[i][j]; }, [&](int j) { return vd[i][j]; });
                    float gm[32];
                    load_params<LPX>(gm, a.post.gamma, cb * 32, a.C, 1.0f);
#pragma unroll
                    for (int j = 0; j < 32; ++j) vd[i][j] = r1 * fmaf(-vy[i][j], n2, fmaf(gm[j], vd[i][j], -n1));
                }
                if (in && a.dy.p) store_any<CL>(a.dy, p, cb * 32, a.C, vd[i]);
            });
        }
        if constexpr (R) {
            if (want_scale && unit < a.units)
                each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < ES; ++e)
                        if (LPX < 64 || l.px % 2 == 0) *spart_at(unit, cb, e) = sacc[i][e];
                });
        }
    }
    if constexpr (R) {
        each_block<R>(a, l, [&](int i, int cb) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (want_pre) *part_at(0, cb, e) = acc[0][i][e];
                if (want_post) *part_at(1, cb, e) = acc[1][i][e];
            }
        });
    }
}

// The walkers' sums, added in order: 64 columns and 16 shares of the rows a workgroup.  The
// first workgroups take the norms' parameters ([4][blocks 32] columns), the others t: a
// share adds a sample's units, writes its gate's gradient and goes on to the next sample.
__global__ __launch_bounds__(1024) void join_params_kernel(JoinArgs a) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6, width = a.blocks * 32, four = 2 * a.blocks;
    float s = 0, *out;
    int c;
    if (int(blockIdx.x) < four) {
        const int v = blockIdx.x * 64 + lane, which = v / width;
        c = v - which * width;
        out = which == 0 ? a.dgpre : which == 1 ? a.dbpre : which == 2 ? a.dgpost : a.dbpost;
        const bool there = which < 2 ? a.pre.kind && a.du.p : a.post.kind != DC_NORM_NONE;
        if (out && there) {
            const int rows = a.grid * a.pg;
#pragma unroll 8
            for (int i = share; i < rows; i += 16) s += a.part[int64_t(i) * 4 * width + v];
        }
    } else {
        c = (int(blockIdx.x) - four) * 64 + lane;
        out = a.dscale;
        if ((a.dscale || a.dgate) && c < a.C) {
            const float scale = a.scale ? a.scale[c] : 1.0f;
            if (!a.gate) {
#pragma unroll 8
                for (int i = share; i < a.units; i += 16) s += a.spart[int64_t(i) * width + c];
            } else {
                for (int n = share; n < a.samples; n += 16) {
                    float t = 0;
#pragma unroll 8
                    for (int i = 0; i < a.slices; ++i) t += a.spart[(int64_t(n) * a.slices + i) * width + c];
                    if (a.dgate) {
                        float* d = a.dgate + int64_t(n) * a.C + c;
                        *d = a.accumulate ? fmaf(scale, t, *d) : scale * t;
                    }
                    s = fmaf(a.gate[int64_t(n) * a.C + c], t, s);
                }
            }
        }
    }
    red[share][lane] = s;
    __syncthreads();
    if (share != 0 || !out || c >= a.C) return;
    s = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += red[i][lane];
    out[c] = a.accumulate ? out[c] + s : s;
}

static size_t part_floats(const JoinArgs& a) { return size_t(a.grid) * a.pg * 4 * a.blocks * 32; }

// the larger of the two layouts' (rows of channels or tiles): the workspace does
// not depend on the views' strides
size_t join_bwd_part_bytes(int N, int HW, int C, bool gate) {
    static const float some = 0;
    size_t need = 0;
    for (int cl = 0; cl < 2; ++cl) {
        JoinArgs a{};
        a.px.M = N * HW;
        a.px.HW = HW;
        a.C = C;
        a.cl = cl;
        a.gate = gate ? &some : nullptr;
        join_plan(a, true);
        need = std::max(need, (part_floats(a) + size_t(a.units) * a.blocks * 32) * sizeof(float));
    }
    return need;
}

hipError_t launch_join_bwd(const JoinArgs& a0, hipStream_t s) {
    JoinArgs a = a0;
    a.spart = a.part ? a.part + part_floats(a) : nullptr;
    DC_JOIN_LAUNCH(join_bwd_kernel, 1, a, dim3(unsigned(a.grid)), s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !(a.dscale || a.dgate || a.dgpre || a.dbpre || a.dgpost || a.dbpost)) return e;
    hipLaunchKernelGGL(join_params_kernel, dim3(2 * a.blocks + (a.blocks + 1) / 2), dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace dc
