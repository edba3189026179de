// The gated product over channels, forward, and the gradient at its two sums:
//
//   forward   zg = Wg x + bg, zu = Wu x + bu, h = drop(act(zg) zu)
//   backward  dh = drop(W2^T dy), dzg = dh zu act'(zg), dzu = dh act(zg), and h again
//
// The tile loop of linear.h.  Forward, a workgroup's rows are taken in groups of 32 from Wg
// and Wu in turn, so that a wave holds both sums of a channel in the same place of two
// accumulators: the product of the two is the lane's own work, and x is read once for both.
#pragma once

#include "drop.h"
#include "linear_pass.h"

namespace dc {

struct GateArgs {
    LinearArgs l;      // z: zg; out: h (forward) or dz (backward, of 2 K channels); rows: K
    View zu;           // beside l.z, of its layout
    DropArgs drop;
};
hipError_t launch_gate_fwd(const GateArgs& a, bool f32, hipStream_t s);
hipError_t launch_gate_bwd(const GateArgs& a, bool f32, hipStream_t s);
bool gate_few(const GateArgs& a, bool bwd, bool f32);
hipError_t launch_gate_few(const GateArgs& a, bool bwd, bool f32, hipStream_t s);

// Dropout of the lane's 16 channels of a block (first: o0): 8 g + 4 h .. + 3 for g = 0 .. 3.
// A call of the generator serves eight channels, half of them the partner lane's (32 on):
// each half wave makes two of the four calls, and they trade halves.
__device__ __forceinline__ void drop_half(float (&v)[16], const DropArgs& d, const DropPixel& p, int o0, int h) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int g = k + 2 * h;
        Philox w = philox(p.pos + uint64_t(o0 / 8 + g) * uint64_t(d.plane), p.ctr, d.seed);
        // w[0], w[1]: words 2 h and 2 h + 1 of call k; w[2], w[3]: of call k + 2
        swap_halves(w.w[0], w.w[2]);
        swap_halves(w.w[1], w.w[3]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = 4 * (k + 2 * (j / 4)) + j % 4;
            v[r] = kept(w, j, d.t) ? v[r] * d.scale : 0.0f;
        }
    }
}

__device__ __forceinline__ void clear_past(float (&v)[16], int o0, int h, int rows) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (o0 + 8 * (r / 4) + 4 * h + r % 4 >= rows) v[r] = 0;
}

// f, u: the lane's 16 channels of both sums
__device__ __forceinline__ void gate_epilogue(float (&f)[16], float (&u)[16], const GateArgs& a, const Place& p,
                                              const DropPixel& dp, int o0, int lane) {
    const LinearArgs& l = a.l;
    const int pix = p.c.r * l.s.len + p.w, h = lane >> 5;
    if (l.z.dt == DC_Q8) {
        if (o0 + 32 > l.rows) {
            clear_past(f, o0, h, l.rows);
            clear_past(u, o0, h, l.rows);
        }
        q8_store_half(l.z.p, l.qm, p.c.n, o0 / 32, pix, p.ok, h, f);
        q8_store_half(a.zu.p, l.qm, p.c.n, o0 / 32, pix, p.ok, h, u);
    } else if (l.z.dt >= 0) {
        store_half(f, l.z, p, o0, lane, l.rows);
        store_half(u, a.zu, p, o0, lane, l.rows);
    }
    apply_act(f, l.act);
#pragma unroll
    for (int r = 0; r < 16; ++r) f[r] *= u[r];
    if (a.drop.t) drop_half(f, a.drop, dp, o0, h);
    store_half(f, l.out, p, o0, lane, l.rows);
}

// v: dh before the dropout
__device__ __forceinline__ void gate_slope(float (&v)[16], const GateArgs& a, const Place& p, const DropPixel& dp, int o0, int lane) {
    const LinearArgs& l = a.l;
    const int pix = p.c.r * l.s.len + p.w, h = lane >> 5;
    float f[16], u[16];
    if (l.z.dt == DC_Q8) {
        q8_load_half(f, l.z.p, l.qm, p.c.n, o0 / 32, pix, h);
        q8_load_half(u, a.zu.p, l.qm, p.c.n, o0 / 32, pix, h);
    } else {
        load_half(f, l.z, p, o0, lane, l.rows);
        load_half(u, a.zu, p, o0, lane, l.rows);
    }
    if (a.drop.t) drop_half(v, a.drop, dp, o0, h);
    float g[16];           // dzg
#pragma unroll
    for (int r = 0; r < 16; ++r) g[r] = v[r] * u[r];
    apply_slope(f, g, l.act);
    View out = l.out;
    store_half(g, out, p, o0, lane, l.rows);
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] *= f[r];
    out.p += l.rows * out.sc * (out.dt == DC_F32 ? 4 : 2);
    store_half(v, out, p, o0, lane, l.rows);
    if (l.h.dt >= 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) f[r] *= u[r];
        if (a.drop.t) drop_half(f, a.drop, dp, o0, h);
        store_half(f, l.h, p, o0, lane, l.rows);
    }
}

// BWD: rows are K's channels, weights KR; else rows are Wg's and Wu's, weights RK.
template <typename S, bool BWD, bool CL, bool DIRECT>
__global__ __launch_bounds__(S::TH, S::OCC) void gate_kernel(GateArgs a) {
    typedef typename S::T T;
    constexpr int AK = BWD ? KR : RK, PK = CL ? RK : KR, TM = S::TM, TN = S::TN, PAIRS = BWD ? 1 : 2;
    static_assert(TM % PAIRS == 0);
    // slices while summing, then a wave's blocks (at least one channel group's)
    constexpr int WAVE = S::NST * S::BYTES / (S::TH / 64) > PAIRS * 4096 ? S::NST * S::BYTES / (S::TH / 64) : PAIRS * 4096;
    __shared__ __align__(16) char mem[WAVE * (S::TH / 64)];
    char (*lds)[S::BYTES] = reinterpret_cast<char (*)[S::BYTES]>(mem);
    const LinearArgs& l = a.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // blocks of one column range follow each other on an XCD: they read the same pixels
    const int id = xcd_range(blockIdx.x, l.tr * l.tc);
    const int tc = id / l.tr, tr = id - tc * l.tr;
    const int first = tr * (S::BM / PAIRS);          // of the block's channels
    Stage<T, AK, BWD ? WEIGHT : PAIR, S::BM, S::TH> sa;
    Stage<T, PK, PIXEL, S::BN, S::TH> sb;
    sa.init(l.a, l.s, first);
    sb.init(l.b, l.s, tc * S::BN);
    f32x16_t acc[TM][TN];
    const int row0 = wave / S::WN * (32 * TM), col0 = wave % S::WN * (32 * TN), h = lane >> 5;
    // the sums start from the biases
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float b = 0;
            if constexpr (!BWD) {
                const int o = min(first + (row0 + 32 * i) / 64 * 32 + 8 * (r / 4) + 4 * h + r % 4, l.rows - 1);
                if (l.bias) b = l.bias[o + (i % 2 ? l.rows : 0)];
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j][r] = b;
        }
    tile_loop<S, AK, PK, DIRECT>(acc, sa, sb, l.a, l.b, l.s, 0, l.a.red, lds, row0, col0, lane, [](int, const uint4&) {});

    // as the plain product's: a wave's blocks pass through its share of LDS, both sums of a
    // channel together
    constexpr int Q = TM / PAIRS * TN, ROOM = WAVE / 4096 / PAIRS, PER = Q < ROOM ? Q : ROOM, UP = TM / PAIRS;
    char* mine = mem + wave * (PER * PAIRS * 4096) + lane * 16;
    Place p;
    DropPixel dp{};
    __syncthreads();
    static_for<0, (Q + PER - 1) / PER>([&](auto part) __attribute__((always_inline)) {
        constexpr int q0 = decltype(part)::value * PER, q1 = q0 + PER < Q ? q0 + PER : Q;
        static_for<q0, q1>([&](auto qc) __attribute__((always_inline)) {
            constexpr int q = decltype(qc)::value;
#pragma unroll
            for (int s = 0; s < PAIRS; ++s)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x16_t& t = acc[q % UP * PAIRS + s][q / UP];
                    *reinterpret_cast<f32x4_t*>(mine + ((q - q0) * PAIRS + s) * 4096 + g * 1024) =
                        f32x4_t{t[4 * g], t[4 * g + 1], t[4 * g + 2], t[4 * g + 3]};
                }
        });
#pragma unroll 1
        for (int q = q0; q < q1; ++q) {
            const int o0 = first + row0 / PAIRS + 32 * (q % UP);
            if (q % UP == 0) {
                p = place_of<CL ? 1 : S::E>(l.s, tc * S::BN + col0 + 32 * (q / UP) + (lane & 31));
                if (a.drop.t) dp = drop_pixel(a.drop, p.c.n, p.c.r * l.s.len + p.w);
            }
            if (o0 >= l.rows) continue;
            float v[PAIRS][16];
#pragma unroll
            for (int s = 0; s < PAIRS; ++s)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4_t t = *reinterpret_cast<const f32x4_t*>(mine + ((q - q0) * PAIRS + s) * 4096 + g * 1024);
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[s][4 * g + r] = t[r];
                }
            if constexpr (BWD) gate_slope(v[0], a, p, dp, o0, lane);
            else gate_epilogue(v[0], v[1], a, p, dp, o0, lane);
        }
    });
}

template <typename T> using GateLarge = Shape<T, 256, 256, 2, 4, 2, 2>;
template <typename T> using GateMiddle = Shape<T, 64, 128, 2, 1, 4, 3>;
template <typename T> using GateShort = Shape<T, 64, 128, 1, 1, 4, 4>;     // one slice: half the LDS
template <typename T> using GateSmall = Shape<T, 64, 64, 2, 1, 2, 2>;

template <typename S, bool BWD>
static void launch_gate_shape(GateArgs a, hipStream_t s) {
    const int rows = a.l.rows * (BWD ? 1 : 2);
    a.l.tr = ((rows + (BWD ? 0 : 63)) / (BWD ? 1 : 64) * (BWD ? 1 : 64) + S::BM - 1) / S::BM;
    a.l.tc = int((int64_t(a.l.s.chunks) * a.l.s.per + S::BN - 1) / S::BN);
    const dim3 g(unsigned(a.l.tr) * unsigned(a.l.tc)), t(S::TH);
    if (a.l.cl && a.l.direct) hipLaunchKernelGGL((gate_kernel<S, BWD, true, true>), g, t, 0, s, a);
    else if (a.l.cl) hipLaunchKernelGGL((gate_kernel<S, BWD, true, false>), g, t, 0, s, a);
    else if (a.l.direct) hipLaunchKernelGGL((gate_kernel<S, BWD, false, true>), g, t, 0, s, a);
    else hipLaunchKernelGGL((gate_kernel<S, BWD, false, false>), g, t, 0, s, a);
}

template <typename T, bool BWD>
static hipError_t launch_gate(const GateArgs& a, hipStream_t s) {
    const int64_t slots = int64_t(a.l.s.chunks) * a.l.s.per, rows = int64_t(a.l.rows) * (BWD ? 1 : 2);
    auto blocks = [&](int r, int c) { return (rows + r - 1) / r * ((slots + c - 1) / c); };
    if (a.l.a.red > 128 && blocks(256, 256) >= 256) launch_gate_shape<GateLarge<T>, BWD>(a, s);
    else if (blocks(64, 128) >= 512 && a.l.a.red <= GateShort<T>::BK) launch_gate_shape<GateShort<T>, BWD>(a, s);
    else if (blocks(64, 128) >= 512) launch_gate_shape<GateMiddle<T>, BWD>(a, s);
    else launch_gate_shape<GateSmall<T>, BWD>(a, s);
    return hipGetLastError();
}

}  // namespace dc
