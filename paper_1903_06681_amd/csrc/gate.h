// The gated product over channels, forward, and the gradient at its two sums:
//
//   forward   zg = Wg x + bg, zu = Wu x + bu, h = drop(act(zg) zu)
//   backward  dh = drop(W2^T dy), dzg = dh zu act'(zg), dzu = dh act(zg), and h again
//
// The tile loop of linear.h.  Forward, a workgroup's rows are taken in groups of 32 from Wg
// and Wu in turn, so that a wave holds both sums of a channel in the same place of two
// accumulators: the product of the two is the lane's own work, and x is read once for both.
//
// Bound: short sums (64 to twice 256 on 100352 pixels, bf16, both sums kept in 8 bits) by the
// epilogue's vector operations forward, 52 us of which 47 issue 25 M of them, and by memory
// backward, 55 us for 220 MB; long ones by the tile loop (launch_gate).
#pragma once

#include <algorithm>

#include "eight.h"
#include "linear_pass.h"

namespace dc {

struct GateArgs {
    LinearArgs l;      // z: zg; out: h (forward) or dz (backward, of 2 K channels); rows: K
    View zu;           // beside l.z, of its layout
    int32_t rows_kept; // rows of blocks that an XCD goes through the columns with
    FastDiv dset, drows, drest;   // blocks of such a set; its rows; the last set's rows
    DropArgs drop;
};
hipError_t launch_gate_fwd(const GateArgs& a, bool f32, hipStream_t s);
hipError_t launch_gate_bwd(const GateArgs& a, bool f32, hipStream_t s);
bool gate_few(const GateArgs& a, bool bwd, bool f32);
hipError_t launch_gate_few(const GateArgs& a, bool bwd, bool f32, hipStream_t s);

// The mask of the lane's 16 channels of a block (first: o0), 8 g + 4 h .. + 3 for g = 0 .. 3, a bit
// each.  A call of the generator serves eight channels, half of them the partner lane's (32 on):
// each half wave makes two of the four calls, and they trade halves.
__device__ __forceinline__ uint32_t bits_half(const DropArgs& d, const DropPixel& p, int o0, int h) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        Philox w = philox(p.pos + uint64_t(o0 / 8 + i + 2 * h) * uint64_t(d.plane), p.ctr, d.seed);
        // w[0], w[1]: words 2 h and 2 h + 1 of call i; w[2], w[3]: of call i + 2
        swap_halves(w.w[0], w.w[2]);
        swap_halves(w.w[1], w.w[3]);
#pragma unroll
        for (int j = 0; j < 8; ++j) bits |= kept(w, j, d.t) ? 1u << (4 * (i + 2 * (j / 4)) + j % 4) : 0u;
    }
    return bits;
}
__device__ __forceinline__ void drop_half(float (&v)[16], uint32_t bits, float scale) {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = masked(v[r] * scale, bits, r);
}

__device__ __forceinline__ void clear_past(float (&v)[16], int o0, int h, int rows) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (o0 + 8 * (r / 4) + 4 * h + r % 4 >= rows) v[r] = 0;
}

// The biases are added here, not to begin with: a lane's channels of all its blocks would be 64
// loads ahead of the sums (50 us of 490 for 65536 rows, 512 to twice 2048).
template <int N>
__device__ __forceinline__ void add_bias(float (&v)[N], const float* bias, int c0, int last) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] += bias[min(c0 + j, last)];
}
// f, u: the lane's 16 channels of both sums
__device__ __forceinline__ void gate_epilogue(float (&f)[16], float (&u)[16], const GateArgs& a, const Place& p,
                                              const DropPixel& dp, int o0, int lane) {
    const LinearArgs& l = a.l;
    const int pix = p.c.r * l.s.len + p.w, h = lane >> 5;
    if (l.bias && o0 + 32 <= l.rows) {
        typedef float f32x4_at __attribute__((ext_vector_type(4), aligned(4)));
        const float* from = l.bias + o0 + 4 * h;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4_at bf = *reinterpret_cast<const f32x4_at*>(from + 8 * g);
            const f32x4_at bu = *reinterpret_cast<const f32x4_at*>(from + l.rows + 8 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f[4 * g + r] += bf[r];
                u[4 * g + r] += bu[r];
            }
        }
    } else if (l.bias) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int c = min(o0 + 8 * (r / 4) + 4 * h + r % 4, l.rows - 1);
            f[r] += l.bias[c];
            u[r] += l.bias[c + l.rows];
        }
    }
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
    if (a.drop.t) drop_half(f, bits_half(a.drop, dp, o0, h), a.drop.scale);
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
    float g[16];           // dzg
    const uint32_t bits = a.drop.t ? bits_half(a.drop, dp, o0, h) : 0;
    if (a.drop.t) drop_half(v, bits, a.drop.scale);
#pragma unroll
    for (int r = 0; r < 16; ++r) g[r] = v[r] * u[r];
    apply_slope(f, g, l.act);
    if (l.h.dt >= 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) u[r] *= f[r];
        if (a.drop.t) drop_half(u, bits, a.drop.scale);
        store_half(u, l.h, p, o0, lane, l.rows);
    }
    View out = l.out;
    store_half(g, out, p, o0, lane, l.rows);
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] *= f[r];
    out.p += l.rows * out.sc * (out.dt == DC_F32 ? 4 : 2);
    store_half(v, out, p, o0, lane, l.rows);
}

// The same for eight channels of one pixel a lane (rows of channels; four neighbouring lanes hold a
// block of 32): 16 bytes of bf16 a store and whole lines a pixel, where the above stores 8 bytes a
// lane to 32 rows at once.
__device__ __forceinline__ u32x8 load_z(const View& t, const Q8Map& m, const Pixel& p, int c0, int rows) {
    return t.sc == 1 || t.dt == DC_Q8 ? load8<true>(t, m, p, c0, rows) : load8<false>(t, m, p, c0, rows);
}
__device__ __forceinline__ void z_values(float (&v)[8], const u32x8& w, const View& t, int c0, int rows) {
    if (t.sc == 1 || t.dt == DC_Q8) values8<true>(v, w, t, c0, rows);
    else values8<false>(v, w, t, c0, rows);
}
__device__ __forceinline__ void store_z(const View& t, const Pixel& p, int c0, int rows, const float (&v)[8]) {
    if (t.sc == 1) store8<true>(t, p, c0, rows, v);
    else store8<false>(t, p, c0, rows, v);
}
__device__ __forceinline__ void gate_epilogue8(float (&f)[8], float (&u)[8], const GateArgs& a, const Pixel& p, bool in,
                                               const DropPixel& dp, int c0) {
    const LinearArgs& l = a.l;
    if (l.bias) {
        add_bias(f, l.bias, c0, l.rows - 1);
        add_bias(u, l.bias + l.rows, c0, l.rows - 1);
    }
    if (l.z.dt == DC_Q8) {
        clear8(f, c0, l.rows);
        clear8(u, c0, l.rows);
        q8_store_eight(l.z.p, l.qm, p, c0 / 8, in, l.rows, f);
        q8_store_eight(a.zu.p, l.qm, p, c0 / 8, in, l.rows, u);
    }
    if (!in || c0 >= l.rows) return;
    if (l.z.dt >= 0 && l.z.dt != DC_Q8) {
        store_z(l.z, p, c0, l.rows, f);
        store_z(a.zu, p, c0, l.rows, u);
    }
    apply_act(f, l.act);
    float k[8];
    keep8(k, a.drop, dp, c0 / 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = dropped(f[j] * u[j], k[j]);
    store_z(l.out, p, c0, l.rows, f);
}
__device__ __forceinline__ void gate_slope8(float (&v)[8], const GateArgs& a, const Pixel& p, bool in, const DropPixel& dp, int c0) {
    const LinearArgs& l = a.l;
    if (!in || c0 >= l.rows) return;
    const u32x8 wf = load_z(l.z, l.qm, p, c0, l.rows), wu = load_z(a.zu, l.qm, p, c0, l.rows);
    float f[8], u[8], g[8], k[8];
    keep8(k, a.drop, dp, c0 / 8);
    z_values(f, wf, l.z, c0, l.rows);
    z_values(u, wu, a.zu, c0, l.rows);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = dropped(v[j], k[j]);
        g[j] = v[j] * u[j];
    }
    apply_slope(f, g, l.act);
    store_z(l.out, p, c0, l.rows, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= f[j];
    View out = l.out;
    out.p += l.rows * out.sc * (out.dt == DC_F32 ? 4 : 2);
    store_z(out, p, c0, l.rows, v);
    if (l.h.dt >= 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = dropped(f[j] * u[j], k[j]);
        store_z(l.h, p, c0, l.rows, f);
    }
}

// ---- the same where a wave's pixels are rows of channels of one sample and all of its channels
// are there: a tensor is a uniform address and 32 bits of offset a lane, so that an access
// takes a few vector operations instead of some sixty (of 316 for eight values of both sums:
// 237 us of epilogue for 65536 rows of 2048 in 8 bits, against 110 of memory).
struct RowSpot {
    gchar* p;          // of the wave's first pixel and channel
    uint32_t pitch;    // bytes of a pixel
    int32_t f32, big;
};
__device__ __forceinline__ RowSpot row_spot(const View& t, int n, int r, int64_t c) {
    const int es = t.dt == DC_F32 ? 4 : 2;
    return RowSpot{(gchar*)(t.p) + (n * t.sn + r * t.sh + c) * es, uint32_t(t.sh) * es, t.dt == DC_F32, t.big};
}
__device__ __forceinline__ bool row_fits(const View& t) { return t.dt < 0 || t.dt == DC_Q8 || (t.sc == 1 && t.sh < (1 << 22)); }
__device__ __forceinline__ void put_row(const RowSpot& t, uint32_t px, uint32_t c, const float (&v)[8]) {
    if (t.f32) {
        gchar* a = t.p + (px * t.pitch + c * 4);
        const u32x4_any lo = {__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]),
                              __builtin_bit_cast(uint32_t, v[3])};
        const u32x4_any hi = {__builtin_bit_cast(uint32_t, v[4]), __builtin_bit_cast(uint32_t, v[5]), __builtin_bit_cast(uint32_t, v[6]),
                              __builtin_bit_cast(uint32_t, v[7])};
        if (t.big) stream_as(a, lo), stream_as(a + 16, hi);
        else store_as(a, lo), store_as(a + 16, hi);
    } else {
        auto two = [&](int j) __attribute__((always_inline)) {
            return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{v[j], v[j + 1]}), bf16x2_t));
        };
        gchar* a = t.p + (px * t.pitch + c * 2);
        const u32x4_any w = {two(0), two(2), two(4), two(6)};
        if (t.big) stream_as(a, w);
        else store_as(a, w);
    }
}
__device__ __forceinline__ u32x8 get_row(const RowSpot& t, uint32_t px, uint32_t c) {
    if (t.f32) {
        const gchar* a = t.p + (px * t.pitch + c * 4);
        const u32x4_any u = load_as<u32x4_any>(a), u2 = load_as<u32x4_any>(a + 16);
        return u32x8{u.x, u.y, u.z, u.w, u2.x, u2.y, u2.z, u2.w};
    }
    const u32x4_any u = load_as<u32x4_any>(t.p + (px * t.pitch + c * 2));
    return u32x8{u.x, u.y, u.z, u.w, 0, 0, 0, 0};
}
// the 8-bit form: of the wave's first pixel and block
struct BlockSpot {
    gchar *q, *s;
    uint32_t hw;
    int32_t big;
};
__device__ __forceinline__ BlockSpot block_spot(const View& t, const Q8Map& m, int n, int r, int block) {
    const int64_t at = int64_t(block) * m.HW + r;
    return BlockSpot{(gchar*)(t.p) + n * m.qn + at * 32, (gchar*)(t.p) + m.s0 + n * m.sn + at, uint32_t(m.HW), t.big};
}
typedef uint32_t u32x2_al __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void put_block(const BlockSpot& t, uint32_t px, uint32_t e, bool in, const float (&v)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, abs_bits(v[j]));
    top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0xb1, 0xf, 0xf, true)));      // lane ^ 1
    top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0x4e, 0xf, 0xf, true)));      // lane ^ 2
    const uint32_t s = q8_scale(top), at = px + e / 4 * t.hw;
    const float per = q8_per(s);
    const u32x2_al w = {q8_pack(v[0], v[1], v[2], v[3], per), q8_pack(v[4], v[5], v[6], v[7], per)};
    if (!in) return;
    if (t.big) stream_as(t.q + (at * 32 + e % 4 * 8), w);
    else store_as(t.q + (at * 32 + e % 4 * 8), w);
    if (e % 4 == 0) store_as(t.s + at, uint8_t(s));
}
__device__ __forceinline__ u32x8 get_block(const BlockSpot& t, uint32_t px, uint32_t e) {
    const uint32_t at = px + e / 4 * t.hw;
    const u32x2_al w = load_as<u32x2_al>(t.q + (at * 32 + e % 4 * 8));
    return u32x8{w.x, w.y, load_as<uint8_t>(t.s + at), 0, 0, 0, 0, 0};
}

// BWD: rows are K's channels, weights KR; else rows are Wg's and Wu's, weights RK.
template <typename S, bool BWD, bool CL, bool DIRECT>
__global__ __launch_bounds__(S::TH, S::OCC) void gate_kernel(GateArgs a) {
    typedef typename S::T T;
    constexpr int AK = BWD ? KR : RK, PK = CL ? RK : KR, TM = S::TM, TN = S::TN, PAIRS = BWD ? 1 : 2;
    static_assert(TM % PAIRS == 0);
    // Slices while summing, then a wave's blocks of 32 x 32 sums: both of a channel together, and as
    // many groups of 32 channels next to each other as fit (GR; rows of channels: 36 floats a pixel,
    // and 32 more a group, so that the lanes of an access fall on different banks).
    constexpr int BLOCK = CL ? 36 * 32 * 4 + 128 : 4096, UP = TM / PAIRS, Q = UP * TN;
    constexpr int SHARE = S::NST * S::BYTES / (S::TH / 64), GR = CL && UP % 2 == 0 ? 2 : 1;
    constexpr int ROOM = SHARE / (BLOCK * PAIRS) / GR * GR, PER = ROOM < GR ? GR : ROOM < Q ? ROOM : Q;
    constexpr int WAVE = PER * PAIRS * BLOCK > SHARE ? PER * PAIRS * BLOCK : SHARE;
    __shared__ __align__(16) char mem[WAVE * (S::TH / 64)];
    char (*lds)[S::BYTES] = reinterpret_cast<char (*)[S::BYTES]>(mem);
    const LinearArgs& l = a.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Blocks of as many rows as half an XCD's L2 holds the weights of, column by column, then the
    // next rows: an XCD keeps to its rows' weights while the pixels stream by.
    const int id = xcd_range(blockIdx.x, l.tr * l.tc);
    const int set = int(a.dset.div(uint32_t(id))), in_set = id - set * int(a.dset.d);
    const bool rest = (set + 1) * a.rows_kept > l.tr;
    const int tc = int(rest ? a.drest.div(uint32_t(in_set)) : a.drows.div(uint32_t(in_set)));
    const int tr = set * a.rows_kept + in_set - tc * int(rest ? a.drest.d : a.drows.d);
    const int first = tr * (S::BM / PAIRS);          // of the block's channels
    Stage<T, AK, BWD ? WEIGHT : PAIR, S::BM, S::TH, S::KB> sa;
    Stage<T, PK, PIXEL, S::BN, S::TH, S::KB> sb;
    sa.init(l.a, l.s, first);
    sb.init(l.b, l.s, tc * S::BN);
    f32x16_t acc[TM][TN];
    const int row0 = wave / S::WN * (32 * TM), col0 = wave % S::WN * (32 * TN);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    // Blocks of different channels start at different slices: rows lie a power of two apart, and the same
    // slice of all of them on few of L2's channels (forward, all from the first one and so: 65536 rows of
    // 512 to twice 2048 439 us and 424, 8 x 112 x 112 of 256 to twice 1024 279 and 246, its gradient 344 and
    // 336; 8192 rows of 1024 to twice 4096 169 and 171).  By their channels, not by their pixels too (the
    // same times): the order of a sum, and with it its last bits, does not change with a pixel's place.
    tile_loop<S, AK, PK, DIRECT>(acc, sa, sb, l.a, l.b, l.s, 0, l.a.red, lds, row0, col0, lane, [](int, const uint4&) {},
                                 tr % ((l.a.red + S::BK - 1) / S::BK));

    // As the plain product's: a wave's blocks pass through its share of LDS, both sums of a
    // channel together, and the epilogue is one loop.
    char* mine = mem + wave * WAVE;
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
                    const int at = CL ? (lane & 31) * 144 + g * 32 + (lane >> 5) * 16 : g * 1024 + lane * 16;
                    *reinterpret_cast<f32x4_t*>(mine + ((q - q0) * PAIRS + s) * BLOCK + at) =
                        f32x4_t{t[4 * g], t[4 * g + 1], t[4 * g + 2], t[4 * g + 3]};
                }
        });
        if constexpr (CL) {
            // other lanes' values are read: this wave's writes first
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            constexpr int LP = 4 * GR, TURN = 64 / LP, TURNS = 32 / TURN;     // lanes and turns of a pixel's 32 GR channels
            constexpr int AHEAD = BWD ? 4 : 1;       // turns whose sums' loads are on their way at once
            const uint32_t e = lane % LP;
            auto sums = [&](int t, float (&v)[PAIRS][8]) __attribute__((always_inline)) {
                const int set = t / TURNS, px = t % TURNS * TURN + lane / LP;
#pragma unroll
                for (int s = 0; s < PAIRS; ++s) {
                    const char* from = mine + ((set * GR + e / 4) * PAIRS + s) * BLOCK + px * 144 + e % 4 * 32;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const f32x4_t w = *reinterpret_cast<const f32x4_t*>(from + 16 * k);
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[s][4 * k + r] = w[r];
                    }
                }
            };
            const int pixels = l.s.chunks - (tc * S::BN + col0);     // from the wave's first on
            const int n0 = int(l.s.dsample.div(uint32_t(min(tc * S::BN + col0, l.s.chunks - 1))));
            const int r0 = tc * S::BN + col0 - n0 * int(l.s.dsample.d), c0 = first + row0 / PAIRS;
            const bool fast = min(pixels, 32 * TN) <= int(l.s.dsample.d) - r0 && c0 + 32 * UP <= l.rows && l.qm.HW < (1 << 26) &&
                              row_fits(l.out) && row_fits(l.z) && row_fits(l.h);
            if (pixels <= 0) {
                // nothing of this wave's is there
            } else if (fast) {
                if (q0 == 0 && a.drop.t) dp = drop_pixel(a.drop, n0, r0);
                static_assert(TURNS % AHEAD == 0);
#pragma unroll 1
                for (int t0 = 0; t0 < (q1 - q0) / GR * TURNS; t0 += AHEAD) {
                    const int q = q0 + t0 / TURNS * GR, cu = c0 + 32 * (q % UP);     // the set's first channel
                    const RowSpot out = row_spot(l.out, n0, r0, cu);
                    auto pixel = [&](int t) __attribute__((always_inline)) {
                        return uint32_t(32 * (q / UP) + t % TURNS * TURN + lane / LP);
                    };
                    float keep[8];
                    if constexpr (BWD) {
                        u32x8 wf[AHEAD], wu[AHEAD];
                        if (l.z.dt == DC_Q8) {
                            const BlockSpot zf = block_spot(l.z, l.qm, n0, r0, cu / 32), zu = block_spot(a.zu, l.qm, n0, r0, cu / 32);
#pragma unroll
                            for (int i = 0; i < AHEAD; ++i) {
                                const uint32_t px = min(pixel(t0 + i), uint32_t(pixels - 1));
                                wf[i] = get_block(zf, px, e), wu[i] = get_block(zu, px, e);
                            }
                        } else {
                            const RowSpot zf = row_spot(l.z, n0, r0, cu), zu = row_spot(a.zu, n0, r0, cu);
#pragma unroll
                            for (int i = 0; i < AHEAD; ++i) {
                                const uint32_t px = min(pixel(t0 + i), uint32_t(pixels - 1));
                                wf[i] = get_row(zf, px, 8 * e), wu[i] = get_row(zu, px, 8 * e);
                            }
                        }
                        RowSpot out2 = out;
                        out2.p += int64_t(l.rows) * (out.f32 ? 4 : 2);
                        const RowSpot again = row_spot(l.h, n0, r0, cu);
#pragma unroll
                        for (int i = 0; i < AHEAD; ++i) {
                            const uint32_t px = pixel(t0 + i);
                            float v[PAIRS][8], f[8], u[8], g[8];
                            sums(t0 + i, v);
                            DropPixel dt = dp;
                            dt.pos += uint64_t(px) * uint64_t(a.drop.cols);
                            keep8(keep, a.drop, dt, cu / 8 + e);
                            values8<true>(f, wf[i], l.z, 0, 8);
                            values8<true>(u, wu[i], a.zu, 0, 8);
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                v[0][j] = dropped(v[0][j], keep[j]);
                                g[j] = v[0][j] * u[j];
                            }
                            apply_slope(f, g, l.act);
                            if (int(px) < pixels) {
                                put_row(out, px, 8 * e, g);
#pragma unroll
                                for (int j = 0; j < 8; ++j) g[j] = v[0][j] * f[j];
                                put_row(out2, px, 8 * e, g);
                                if (l.h.dt >= 0) {
#pragma unroll
                                    for (int j = 0; j < 8; ++j) g[j] = dropped(f[j] * u[j], keep[j]);
                                    put_row(again, px, 8 * e, g);
                                }
                            }
                        }
                    } else {
                        const uint32_t px = pixel(t0);
                        const bool in = int(px) < pixels;
                        float v[PAIRS][8];
                        sums(t0, v);
                        if (l.bias) {
                            add_bias(v[0], l.bias + cu, 8 * e, 32 * GR - 1);
                            add_bias(v[1], l.bias + l.rows + cu, 8 * e, 32 * GR - 1);
                        }
                        if (l.z.dt == DC_Q8) {
                            put_block(block_spot(l.z, l.qm, n0, r0, cu / 32), px, e, in, v[0]);
                            put_block(block_spot(a.zu, l.qm, n0, r0, cu / 32), px, e, in, v[1]);
                        } else if (l.z.dt >= 0 && in) {
                            put_row(row_spot(l.z, n0, r0, cu), px, 8 * e, v[0]);
                            put_row(row_spot(a.zu, n0, r0, cu), px, 8 * e, v[1]);
                        }
                        apply_act(v[0], l.act);
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[0][j] *= v[1][j];
                        if (a.drop.t) {
                            DropPixel dt = dp;
                            dt.pos += uint64_t(px) * uint64_t(a.drop.cols);
                            keep8(keep, a.drop, dt, cu / 8 + e);
#pragma unroll
                            for (int j = 0; j < 8; ++j) v[0][j] = dropped(v[0][j], keep[j]);
                        }
                        if (in) put_row(out, px, 8 * e, v[0]);
                    }
                }
            } else {
#pragma unroll 1
                for (int t = 0; t < (q1 - q0) / GR * TURNS; ++t) {
                    const int q = q0 + t / TURNS * GR;
                    const Place at = place_of<1>(l.s, tc * S::BN + col0 + 32 * (q / UP) + t % TURNS * TURN + lane / LP);
                    const Pixel pp{at.c.n, at.c.r, 0, at.c.r};
                    DropPixel dt{};
                    if (a.drop.t) dt = drop_pixel(a.drop, pp.n, pp.pix);
                    float v[PAIRS][8];
                    sums(t, v);
                    if constexpr (BWD) gate_slope8(v[0], a, pp, at.ok, dt, c0 + 32 * (q % UP) + 8 * e);
                    else gate_epilogue8(v[0], v[1], a, pp, at.ok, dt, c0 + 32 * (q % UP) + 8 * e);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        } else {
#pragma unroll 1
            for (int q = q0; q < q1; ++q) {
                const int o0 = first + row0 / PAIRS + 32 * (q % UP);
                if (q % UP == 0) {
                    p = place_of<S::E>(l.s, tc * S::BN + col0 + 32 * (q / UP) + (lane & 31));
                    if (a.drop.t) dp = drop_pixel(a.drop, p.c.n, p.c.r * l.s.len + p.w);
                }
                if (o0 >= l.rows) continue;
                float v[PAIRS][16];
#pragma unroll
                for (int s = 0; s < PAIRS; ++s)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4_t t =
                            *reinterpret_cast<const f32x4_t*>(mine + ((q - q0) * PAIRS + s) * BLOCK + g * 1024 + lane * 16);
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[s][4 * g + r] = t[r];
                    }
                if constexpr (BWD) gate_slope(v[0], a, p, dp, o0, lane);
                else gate_epilogue(v[0], v[1], a, p, dp, o0, lane);
            }
        }
    });
}

// Long sums over many pixels: several workgroups a compute unit, so that one's epilogue goes on
// beside another's products (three slices of 64 bytes leave LDS for two or three).  65536 rows, 512 to
// twice 2048, both sums in 8 bits: forward 256 x 128 in 452 to 540 us (the chip lowers its clock under
// the load), 128 x 128 in 473 to 550, 256 x 256 alone on its compute unit 503 to 550; the gradient,
// bound by what it reads and stores, 393 to 466, 351 to 420 and 412 to 464.  The others as for the
// plain product (linear_pass.h), of which a channel's two sums are rows.
template <typename T, bool BWD> struct GateShapes { typedef Shape<T, 256, 128, 3, 2, 2, 2, 64> Large; };
template <typename T> struct GateShapes<T, true> { typedef Shape<T, 128, 128, 3, 2, 2, 3, 64> Large; };
template <typename T> using GateMiddle = Shape<T, 64, 128, 2, 1, 4, 3>;
template <typename T> using GateShort = Shape<T, 64, 128, 1, 1, 4, 4>;     // one slice: half the LDS
template <typename T> using GateSmall = Shape<T, 64, 64, 2, 1, 2, 2>;

template <typename S, bool BWD>
static void launch_gate_shape(GateArgs a, hipStream_t s) {
    const int rows = a.l.rows * (BWD ? 1 : 2);
    a.l.tr = ((rows + (BWD ? 0 : 63)) / (BWD ? 1 : 64) * (BWD ? 1 : 64) + S::BM - 1) / S::BM;
    a.l.tc = int((int64_t(a.l.s.chunks) * a.l.s.per + S::BN - 1) / S::BN);
    a.rows_kept = int(std::clamp<int64_t>((2 << 20) / (int64_t(S::BM) * a.l.a.red * int64_t(sizeof(typename S::T))), 1, a.l.tr));
    a.dset = fast_div(uint32_t(a.rows_kept) * uint32_t(a.l.tc));
    a.drows = fast_div(uint32_t(a.rows_kept));
    a.drest = fast_div(uint32_t(a.l.tr % a.rows_kept ? a.l.tr % a.rows_kept : a.rows_kept));
    const dim3 g(unsigned(a.l.tr) * unsigned(a.l.tc)), t(S::TH);
    if (a.l.cl && a.l.direct) hipLaunchKernelGGL((gate_kernel<S, BWD, true, true>), g, t, 0, s, a);
    else if (a.l.cl) hipLaunchKernelGGL((gate_kernel<S, BWD, true, false>), g, t, 0, s, a);
    else if (a.l.direct) hipLaunchKernelGGL((gate_kernel<S, BWD, false, true>), g, t, 0, s, a);
    else hipLaunchKernelGGL((gate_kernel<S, BWD, false, false>), g, t, 0, s, a);
}

// The large block takes sums over more than 128 where 256 x 256 results a compute unit are there (two
// workgroups each forward, four backward).  us, large against middle, by sum, channels and pixels:
//   forward  rows, bf16: 256 to 256 on 16384 (128 x 128 blocks of 256: middle) 18.3 and 14.7, on 32768 25 and 27;
//            160 to 1024 on 8192 22 and 24, 192 22.4 and 21.5, 512 33 and 36, 1024 48 and 57, 128 20.4 and 20.2,
//            64 17.4 and 16.3.  fp32: 192 on 8192 69 and 74, 512 145 and 156, 128 54 and 56, 64 39 and 37;
//            1024 on 4096 (middle) 147 and 153.  Planes much as rows (fp32, 512 to 1024 on 4096, middle, 83 and 95).
//   backward rows, bf16: 160 to 1024 on 16384 33.5 and 33.5, 512 47 and 46, 1024 66 and 67, on 32768 137 and 154;
//            128 32 and 32; 1024 to 1024 on 8192 (middle) 35 and 39.  fp32: 192 on 16384 120 and 111, 512 184
//            and 185, 1024 314 and 320.  Planes, bf16: 192 on 16384 63 and 57, 512 70 and 61, 1024 83 and 83, on
//            32768 145 and 149: there the middle one would be the better up to sums over 512.
template <typename T, bool BWD>
static hipError_t launch_gate(const GateArgs& a, hipStream_t s) {
    const int64_t slots = int64_t(a.l.s.chunks) * a.l.s.per, rows = int64_t(a.l.rows) * (BWD ? 1 : 2);
    auto blocks = [&](int r, int c) { return (rows + r - 1) / r * ((slots + c - 1) / c); };
    if (a.l.a.red > 128 && blocks(256, 256) >= 256) launch_gate_shape<typename GateShapes<T, BWD>::Large, BWD>(a, s);
    else if (blocks(64, 128) >= 512 && a.l.a.red <= GateShort<T>::BK) launch_gate_shape<GateShort<T>, BWD>(a, s);
    else if (blocks(64, 128) >= 512) launch_gate_shape<GateMiddle<T>, BWD>(a, s);
    else launch_gate_shape<GateSmall<T>, BWD>(a, s);
    return hipGetLastError();
}

}  // namespace dc
