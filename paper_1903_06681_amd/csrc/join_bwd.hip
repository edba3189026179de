// The join of a branch with its residual stream, backward.
//
//   dO = dr + pre'(du),  dx = dO,  dv = dO scale gate drop,  dy = post'(dv)
//
// with norm'(g) = r (gamma g - mean(gamma g) - xh mean(gamma g xh)) (no first mean for the
// root mean square), and the sums over pixels  dgamma = g xh,  dbeta = g  of both norms and
// t = dO drop(v) a sample, from which dgate = scale t and dscale = sum of gate t.
//
// Bound: memory.  One pass: y, x, du and dr are held in registers, and o is formed from the
// first two as the forward pass formed it, before its rounding (or read, where it is given).  A
// lane keeps to its eight channels, so that the sums over pixels are its own until a workgroup's
// end (40 registers; 32 channels a lane left no room for them, and 160 values a wave's 64 pixels
// to halve across its lanes).  A second launch adds the workgroups' sums in order.  No atomics.  What
// does not fit the registers (R = 0) goes through its channels one eight at a time, three times, with the
// sums in memory: 4096 rows of 8200 bf16 671 us, of 8192 (two eights a lane) 259.
// Two waves a SIMD: 4 x 64 x 256 x 256 with fp32 x 92 us (3.3 TB/s), 8192 rows of 1024 bf16 44 (2.3);
// neither barriers of fewer waves (two a workgroup: 47), nor stores put off until the next
// step's loads are issued (45.5), nor two eights a lane (no barrier, but scratch: 67) change that much.
#include <algorithm>

#include "join.h"

namespace dc {

template <int LPX, int R, bool CL>
__global__ __launch_bounds__(512, 2) void join_bwd_kernel(JoinArgs) {
    constexpr int H = R ? R : 1;
    // The arguments where they lie (constant address space: scalar loads), read again by each part
    // of a step: kept from the start they and what is derived from them do not fit the scalar
    // registers (678 reads of spilled ones; 142 us for 4 x 64 x 256 x 256)
    auto args = __builtin_amdgcn_kernarg_segment_ptr();
    auto fresh = [&]() __attribute__((always_inline)) -> const JoinArgs& {
        auto q = args;
        asm volatile("" : "+s"(q));
        return *(const JoinArgs*)q;
    };
    const JoinArgs& a = *(const JoinArgs*)args;
    __shared__ float red[2][2][2][kJoinWaves * LPX];
    __shared__ float wsum[kJoinWaves][8 * 64];
    const JoinLane l = join_lane<LPX, CL>(a);
    const int lane = threadIdx.x & 63;
    const bool has_pre = a.pre.kind && a.du.p, has_post = a.post.kind != DC_NORM_NONE;
    const bool want_pre = has_pre && (a.dgpre || a.dbpre), want_post = has_post && (a.dgpost || a.dbpost);
    const bool want_scale = a.dscale || a.dgate;
    const uint64_t counter = a.drop.t ? drop_counter(a.drop) : 0;     // read once: in the loop its wait would be the tensors' too
    const int width = a.blocks * 32, wg = CL ? int(blockIdx.x) : xcd_range(blockIdx.x, a.grid);
    // Sums of a lane's eight channels over the workgroup's pixels, from all its lanes and waves,
    // to the eight floats of `to`; every wave comes here.  R = 0: added to what is there.
    auto collect = [&](float (&v)[8], float* to, bool there) __attribute__((always_inline)) {
        if (a.pg > 1) {      // R > 0 only: as many eights in every wave
            if (l.pg > 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) wsum[l.wave][j * 64 + lane] = v[j];
            }
            __syncthreads();
            if (l.pg == 0)
                for (int g = 1; g < a.pg; ++g)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += wsum[g * a.nw + l.wave][j * 64 + lane];
            __syncthreads();
            there = there && l.pg == 0;
        }
        if constexpr (CL) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int d = 64 / LPX; d < 64; d *= 2) v[j] += __shfl_xor(v[j], d);
            if (there && l.px == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (R) to[j] = v[j];
                    else to[j] += v[j];
                }
            }
        } else {
            sum_lanes<LPX>(v, lane);
            constexpr int E = LPX >= 8 ? 1 : 8 / LPX, SAME = LPX >= 8 ? LPX / 8 : 1;   // values a lane, lanes of one value
            const int first = l.px / SAME * E;
            if (there && l.px % SAME == 0) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (R) to[first + e] = v[e];
                    else to[first + e] += v[e];
                }
            }
        }
    };
    float acc[4][H][8], tacc[H][8];       // dgamma, dbeta of pre, of post; t
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[0][i][j] = acc[1][i][j] = acc[2][i][j] = acc[3][i][j] = 0;
    float* const part = a.part + int64_t(wg) * 4 * width;
    if constexpr (!R) {
        each_eight<R>(a, l, [&](int, int e) {
            for (int k = 0; k < 4; ++k)
                if (k < 2 ? want_pre : want_post)
                    for (int j = 0; j < 8; ++j) part[k * width + 8 * e + j] = 0;
        });
        __syncthreads();
    }
    const int per = a.slices * a.pg, steps = (a.groups + per - 1) / per;
    int par = 0;
    // Every wave of a workgroup takes the same units and steps (barriers); a unit's sums are written by
    // the workgroup that takes it and by no other, so one without a unit in the last turn does nothing there.
    for (int unit = wg; unit < a.units; unit += a.grid) {
        const int smp = int(a.dslices.div(uint32_t(unit))), slice = unit - smp * a.slices;
        float* const spart = a.spart + int64_t(unit) * width;
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) tacc[i][j] = 0;
        if constexpr (!R) {
            if (want_scale)
                each_eight<R>(a, l, [&](int, int e) {
                    for (int j = 0; j < 8; ++j) spart[8 * e + j] = 0;
                });
            __syncthreads();
        }
        // A lane's one eight: what does not change within a unit stays in registers, and the next step's
        // tensors are on their way while this one's are worked on: no other load comes after theirs.
        float kg1[8], kb1[8], kg2[8], kf[8];
        if constexpr (R == 1) {
            const int c0 = min(8 * l.unit, a.C - 1);
            Pixel p0{};
            p0.n = a.gate ? smp : 0;
            params8<false>(kg1, a.post.gamma, c0, a.C, 1.0f);
            params8<false>(kb1, a.post.beta, c0, a.C, 0.0f);
            params8<false>(kg2, a.pre.gamma, c0, a.C, 1.0f);
            factor8<false>(kf, a, p0, c0);
        }
        auto kept_or = [&](float (&v)[8], const float (&k)[8], const float* from, int c0, float none) __attribute__((always_inline)) {
            if constexpr (R == 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = k[j];
            } else {
                params8<LPX == 64>(v, from, c0, fresh().C, none);
            }
        };
        auto factor = [&](float (&v)[8], const Pixel& p, int c0) __attribute__((always_inline)) {
            if constexpr (R == 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = kf[j];
            } else {
                factor8<LPX == 64>(v, fresh(), p, c0);
            }
        };
        // where step st's pixel lies (a valid one's place where there is none)
        auto place = [&](int st, bool& in, int& m) __attribute__((always_inline)) {
            const int64_t q = (int64_t(slice + st * a.slices) * a.pg + l.pg) * LPX + l.px;
            in = q < a.span;
            const JoinArgs& b = fresh();
            m = int(smp * int64_t(b.span) + min(q, int64_t(b.span) - 1));
            return pixel_of(b.px, m);
        };
        struct Raw { u32x8 o[H], d[H], y[H], r[H]; };
        struct Moments { float mu1, r1, mu2, r2; };
        // what there is not reads as zeros
        auto fetch = [&](Raw& w, int i, const Pixel& p, int e) __attribute__((always_inline)) {
            const JoinArgs& b = fresh();
            const u32x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
            w.o[i] = b.x.p ? load8<CL>(b.x, b.qm, p, 8 * e, b.C) : zero;
            w.d[i] = b.du.p ? load8<CL>(b.du, b.qm, p, 8 * e, b.C) : zero;
            w.y[i] = b.y.p ? load8<CL>(b.y, b.qm, p, 8 * e, b.C) : zero;
            w.r[i] = b.dr.p ? load8<CL>(b.dr, b.qm, p, 8 * e, b.C) : zero;
        };
        auto fetch_moments = [&](int m) __attribute__((always_inline)) {
            const JoinArgs& b = fresh();
            Moments k{0, 1, 0, 1};
            if (has_post) {
                k.mu1 = b.stat[m];
                k.r1 = b.stat[int64_t(b.px.M) + m];
            }
            if (has_pre) {
                k.mu2 = b.stat[2 * int64_t(b.px.M) + m];
                k.r2 = b.stat[3 * int64_t(b.px.M) + m];
            }
            return k;
        };
        Raw ahead;
        Moments kahead{0, 0, 0, 0};
        auto fetch_ahead = [&](int st) __attribute__((always_inline)) {
            bool in;
            int m;
            const Pixel p = place(st, in, m);
            kahead = fetch_moments(m);
            each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) { fetch(ahead, i, p, e); });
        };
        if constexpr (R == 1) fetch_ahead(0);
        for (int st = 0; st < steps; ++st, par ^= 1) {
            bool in;
            int m;
            const Pixel p = place(st, in, m);
            Raw w;
            Moments k;
            if constexpr (R == 1) {
                w = ahead;
                k = kahead;
                if (st + 1 < steps) fetch_ahead(st + 1);
            } else {
                k = fetch_moments(m);
                if constexpr (R > 1) each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) { fetch(w, i, p, e); });
            }
            // lanes without a pixel have read another one's, maybe after its results were stored over it:
            // zeros instead, which add nothing to the sums
            auto clear = [&](int i) __attribute__((always_inline)) {
                const u32x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
                if (!__all(in)) {
                    w.o[i] = in ? w.o[i] : zero;
                    w.d[i] = in ? w.d[i] : zero;
                    w.y[i] = in ? w.y[i] : zero;
                    w.r[i] = in ? w.r[i] : zero;
                }
            };
            if constexpr (R != 0) {
#pragma unroll
                for (int i = 0; i < H; ++i) clear(i);
            }
            const float mu1 = k.mu1, r1 = k.r1, mu2 = k.mu2, r2 = k.r2;
            DropPixel dp{};
            {
                const JoinArgs& b = fresh();
                if (b.drop.t) dp = DropPixel{drop_position(b.drop, p.n, p.pix), counter};
            }
            // o's normed value; du, then dO, then dv; y's normed value (y without a norm); drop of what the
            // factor multiplies; the mask's factors
            float vo[H][8], vd[H][8], vy[H][8], vt[H][8], keep[H][8];
            auto open = [&](int i, int e) __attribute__((always_inline)) {
                const int c0 = 8 * e;
                if constexpr (!R) {
                    fetch(w, 0, p, e);
                    clear(0);
                }
                {
                    const JoinArgs& b = fresh();
                    keep8(keep[i], b.drop, dp, e);
                    values8<CL>(vy[i], w.y[i], b.y, c0, b.C);
                }
                float g[8], t[8];
                kept_or(g, kg1, a.post.gamma, c0, 1.0f);
                kept_or(t, kb1, a.post.beta, c0, 0.0f);
#pragma unroll
                for (int j = 0; j < 8; ++j) vy[i][j] = (vy[i][j] - mu1) * r1;
                if (has_post) clear8(vy[i], c0, fresh().C);
#pragma unroll
                for (int j = 0; j < 8; ++j) vt[i][j] = dropped(fmaf(g[j], vy[i][j], t[j]), keep[i][j]);    // 1 and 0 without a norm
                if (!has_pre) return;
                const JoinArgs& b = fresh();
                values8<CL>(vo[i], w.o[i], b.x, c0, b.C);
                values8<CL>(vd[i], w.d[i], b.du, c0, b.C);
                if (b.form_o) {      // o as the forward pass formed it
                    float f[8];
                    factor(f, p, c0);
#pragma unroll
                    for (int j = 0; j < 8; ++j) vo[i][j] = fmaf(vt[i][j], f[j], vo[i][j]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) vo[i][j] = (vo[i][j] - mu2) * r2;
                clear8(vo[i], c0, b.C);
            };
            if constexpr (R) {
                each_eight<R>(a, l, open);
            }
            // sums over pixels
            auto add = [&](float (&to)[8], float* mem, auto&& f) __attribute__((always_inline)) {
                if constexpr (R) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) to[j] += f(j);
                } else {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = f(j);
                    collect(v, mem, true);
                }
            };
            auto pre_sums = [&](int i, int e) __attribute__((always_inline)) {
                if (!want_pre) return;
                add(acc[0][i], part + 8 * e, [&](int j) { return vd[i][j] * vo[i][j]; });
                add(acc[1][i], part + width + 8 * e, [&](int j) { return vd[i][j]; });
            };
            float m1 = 0, m2 = 0;
            if (has_pre) {
                float s[2] = {0, 0};
                each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
                    if constexpr (!R) open(0, e);
                    else pre_sums(i, e);
                    float gm[8];
                    kept_or(gm, kg2, a.pre.gamma, 8 * e, 1.0f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float g = gm[j] * vd[i][j];
                        s[0] += g;
                        s[1] = fmaf(g, vo[i][j], s[1]);
                    }
                });
                lane_sum<LPX, CL>(s, a, l, red[par][0]);
                m1 = a.pre.kind == DC_NORM_LAYER ? s[0] * a.invC : 0.0f;
                m2 = s[1] * a.invC;
            }
            // dO in vd
            auto through_pre = [&](int i, int e) __attribute__((always_inline)) {
                const JoinArgs& b = fresh();
                float r[8];
                values8<CL>(r, w.r[i], b.dr, 8 * e, b.C);
                if (has_pre) {
                    float gm[8];
                    kept_or(gm, kg2, a.pre.gamma, 8 * e, 1.0f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) vd[i][j] = fmaf(r2, fmaf(-vo[i][j], m2, fmaf(gm[j], vd[i][j], -m1)), r[j]);
                    clear8(vd[i], 8 * e, b.C);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) vd[i][j] = r[j];
                }
                if constexpr (R) {
                    if (in && b.dx.p) store8<CL>(b.dx, p, 8 * e, b.C, vd[i]);
                }
            };
            // dO in vd -> dv; the sum t
            auto branch = [&](int i, int e, bool with_t) __attribute__((always_inline)) {
                if (with_t) add(tacc[i], spart + 8 * e, [&](int j) { return vd[i][j] * vt[i][j]; });
                float f[8];
                factor(f, p, 8 * e);
#pragma unroll
                for (int j = 0; j < 8; ++j) vd[i][j] = dropped(vd[i][j] * f[j], keep[i][j]);
            };
            float s[2] = {0, 0};
            auto post_moments = [&](int i, int e) __attribute__((always_inline)) {
                float gm[8];
                kept_or(gm, kg1, a.post.gamma, 8 * e, 1.0f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = gm[j] * vd[i][j];
                    s[0] += g;
                    s[1] = fmaf(g, vy[i][j], s[1]);
                }
            };
            if constexpr (R) {
                each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
                    through_pre(i, e);
                    branch(i, e, want_scale);
                    if (has_post) post_moments(i, e);
                });
            } else if (has_post) {
                each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
                    open(0, e);
                    through_pre(0, e);
                    branch(0, e, false);
                    post_moments(0, e);
                });
            }
            float n1 = 0, n2 = 0;
            if (has_post) {
                lane_sum<LPX, CL>(s, a, l, red[par][1]);
                n1 = a.post.kind == DC_NORM_LAYER ? s[0] * a.invC : 0.0f;
                n2 = s[1] * a.invC;
            }
            each_eight<R>(a, l, [&](int i, int e) __attribute__((always_inline)) {
                if constexpr (!R) {
                    open(0, e);
                    pre_sums(0, e);
                    through_pre(0, e);
                    {
                        const JoinArgs& b = fresh();
                        if (in && b.dx.p) store8<CL>(b.dx, p, 8 * e, b.C, vd[0]);
                    }
                    branch(0, e, want_scale);
                }
                if (has_post) {
                    if (want_post) {
                        add(acc[2][i], part + 2 * width + 8 * e, [&](int j) { return vd[i][j] * vy[i][j]; });
                        add(acc[3][i], part + 3 * width + 8 * e, [&](int j) { return vd[i][j]; });
                    }
                    float gm[8];
                    kept_or(gm, kg1, a.post.gamma, 8 * e, 1.0f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) vd[i][j] = r1 * fmaf(-vy[i][j], n2, fmaf(gm[j], vd[i][j], -n1));
                }
                const JoinArgs& b = fresh();
                if (in) store8<CL>(b.dy, p, 8 * e, b.C, vd[i]);
            });
        }
        if constexpr (R) {
            if (want_scale) {
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const int e = l.unit + i * l.ng;
                    collect(tacc[i], spart + 8 * e, 8 * e < a.C);
                }
            }
        }
    }
    if constexpr (R) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (!(k < 2 ? want_pre : want_post)) continue;
                const int e = l.unit + i * l.ng;
                collect(acc[k][i], part + k * width + 8 * e, 8 * e < a.C);
            }
    }
}

// The workgroups' sums, added in order: 64 columns and 16 shares of the rows a workgroup.  The
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
            const int rows = a.grid;
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

static size_t part_floats(const JoinArgs& a) { return size_t(a.grid) * 4 * a.blocks * 32; }

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
    const dim3 g{unsigned(a.grid)}, b(64 * a.nw * a.pg);
    if (a.cl) {
        if (a.lpx == 16) hipLaunchKernelGGL((join_bwd_kernel<16, 1, true>), g, b, 0, s, a);
        else if (a.lpx == 8) hipLaunchKernelGGL((join_bwd_kernel<8, 1, true>), g, b, 0, s, a);
        else if (a.lpx == 4) hipLaunchKernelGGL((join_bwd_kernel<4, 1, true>), g, b, 0, s, a);
        else if (a.lpx == 2) hipLaunchKernelGGL((join_bwd_kernel<2, 1, true>), g, b, 0, s, a);
        else if (a.held == 1) hipLaunchKernelGGL((join_bwd_kernel<1, 1, true>), g, b, 0, s, a);
        else if (a.held == 2) hipLaunchKernelGGL((join_bwd_kernel<1, 2, true>), g, b, 0, s, a);
        else hipLaunchKernelGGL((join_bwd_kernel<1, 0, true>), g, b, 0, s, a);
    } else if (a.lpx == 64) {
        hipLaunchKernelGGL((join_bwd_kernel<64, 1, false>), g, b, 0, s, a);
    } else if (a.lpx == 16) {
        if (a.held == 1) hipLaunchKernelGGL((join_bwd_kernel<16, 1, false>), g, b, 0, s, a);
        else hipLaunchKernelGGL((join_bwd_kernel<16, 0, false>), g, b, 0, s, a);
    } else {
        if (a.held == 1) hipLaunchKernelGGL((join_bwd_kernel<4, 1, false>), g, b, 0, s, a);
        else hipLaunchKernelGGL((join_bwd_kernel<4, 2, false>), g, b, 0, s, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !(a.dscale || a.dgate || a.dgpre || a.dbpre || a.dgpost || a.dbpost)) return e;
    hipLaunchKernelGGL(join_params_kernel, dim3(2 * a.blocks + (a.blocks + 1) / 2), dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace dc
