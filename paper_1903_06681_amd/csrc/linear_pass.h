// Forward pass and input gradient of a product over channels: the tile loop of
// linear.h with rows = output channels and columns = slots (pixels), and the
// epilogue in registers.  Bound: memory for short sums (64 to 256 channels on 100352
// pixels, z in 8 bits, 90 MB: 29 us); for long ones the tile loop, the epilogue's vector
// operations and the stores, one after the other (512 to 2048 on 65536, 137 GFLOP, 474 MB:
// 285 to 310 us, of which 154, 90 and 95 each alone; its gradient 376 to 432).
//
// In the result of the matrix instruction a lane holds one pixel's 16 of a block's
// 32 channels (its partner, 32 lanes on, the others): bias, activation, its slope
// and the residual are the lane's own work, and a block is just the 8-bit form's
// group, whose scale takes one exchange between the two halves.
#pragma once

#include "linear.h"

namespace dc {

// Halves of a wave trade: a's upper lanes against b's lower lanes.
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// The lane's 16 channels of a block: group g holds 8 g + 4 h .. + 3 (h: the half).
// As bytes in memory order the lower half takes dwords 0-3, the upper 4-7.
__device__ __forceinline__ void q8_store_half(char* q, const Q8Map& m, int n, int cb, int pix, bool ok, int h,
                                              const float (&v)[16]) {
    uint32_t top = 0;
#pragma unroll
    for (int r = 0; r < 16; ++r) top = max(top, abs_bits(v[r]));
    uint32_t other = top;
    swap_halves(top, other);            // both halves' largest in the two
    const uint32_t s = q8_scale(max(top, other));
    const float per = q8_per(s);
    uint32_t w[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) w[g] = q8_pack(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3], per);
    swap_halves(w[0], w[2]);
    swap_halves(w[1], w[3]);
    if (!ok) return;
    const int64_t at = int64_t(cb) * m.HW + pix;
    *reinterpret_cast<uint4*>(q + n * m.qn + at * 32 + 16 * h) = make_uint4(w[0], w[2], w[1], w[3]);
    if (h == 0) reinterpret_cast<uint8_t*>(q)[m.s0 + n * m.sn + at] = uint8_t(s);
}

// n, cb, pix are in range on every lane
__device__ __forceinline__ void q8_load_half(float (&v)[16], const char* q, const Q8Map& m, int n, int cb, int pix, int h) {
    const int64_t at = int64_t(cb) * m.HW + pix;
    const uint4 u = *reinterpret_cast<const uint4*>(q + n * m.qn + at * 32 + 16 * h);
    const float step = q8_step(reinterpret_cast<const uint8_t*>(q)[m.s0 + n * m.sn + at]);
    uint32_t w[4] = {u.x, u.z, u.y, u.w};
    swap_halves(w[0], w[2]);
    swap_halves(w[1], w[3]);
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = q8_value(w[r / 4], r % 4, step);
}

// ---- a lane's 16 channels of one pixel in memory, channel by channel: the pixels are
// contiguous over a half wave (64 bytes in bf16, 128 in fp32).  (Four lanes trading values
// for 8 bytes of one channel each changed nothing: the stores are not what bounds.)

// Where a lane's pixel lies: in range on every lane; ok: there is one.
struct Place {
    Chunk c;
    int w, ok;
    __device__ __forceinline__ int64_t at(const View& t) const { return c.n * t.sn + c.r * t.sh + w; }
};
template <int PER>
__device__ __forceinline__ Place place_of(const Slots& s, int slot) {
    Place p;
    p.c = chunk_of(s, slot / PER);
    p.ok = slot % PER < p.c.left;
    p.w = p.ok ? p.c.col + slot % PER : 0;
    return p;
}

template <typename T>
__device__ __forceinline__ void load_half(float (&v)[16], const View& t, const Place& p, int o0, int lane, int rows) {
    // channels past the last one repeat its address, for results that nobody keeps
    const int first = o0 + 4 * (lane >> 5);
    const int64_t step = t.sc * int64_t(sizeof(T));
    char* a = t.p + (p.at(t) + min(first, rows - 1) * t.sc) * int64_t(sizeof(T));
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        v[r] = load1(reinterpret_cast<const T*>(a));
        const int on = r % 4 == 3 ? 5 : 1;
        next(a, first + 8 * (r / 4) + r % 4 + on < rows ? on * step : 0);
    }
}
__device__ __forceinline__ void load_half(float (&v)[16], const View& t, const Place& p, int o0, int lane, int rows) {
    if (t.dt == DC_F32)
        load_half<float>(v, t, p, o0, lane, rows);
    else
        load_half<__bf16>(v, t, p, o0, lane, rows);
}

template <typename T>
__device__ __forceinline__ void store_half(const float (&v)[16], const View& t, const Place& p, int o0, int lane, int rows) {
    const int h = lane >> 5;
    const int64_t step = t.sc * int64_t(sizeof(T));
    auto packed = [&](int r) __attribute__((always_inline)) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{v[r], v[r + 1]}), bf16x2_t));
    };
    if (!p.ok) return;
    char* a = t.p + (p.at(t) + (o0 + 4 * h) * t.sc) * int64_t(sizeof(T));
    if (t.sc == 1 && o0 + 32 <= rows) {      // rows of channels: four lie together
#pragma unroll
        for (int g = 0; g < 4; ++g, a += 8 * sizeof(T)) {
            if constexpr (sizeof(T) == 4)
                *reinterpret_cast<u32x4_any*>(a) =
                    u32x4_any{__builtin_bit_cast(uint32_t, v[4 * g]), __builtin_bit_cast(uint32_t, v[4 * g + 1]),
                              __builtin_bit_cast(uint32_t, v[4 * g + 2]), __builtin_bit_cast(uint32_t, v[4 * g + 3])};
            else
                *reinterpret_cast<u32x2_any*>(a) = u32x2_any{packed(4 * g), packed(4 * g + 2)};
        }
        return;
    }
    const int64_t skip = 5 * step;
    auto all = [&](auto stream) __attribute__((always_inline)) {
        auto put = [&](auto f) __attribute__((always_inline)) {
            if constexpr (decltype(stream)::value) __builtin_nontemporal_store(f, reinterpret_cast<decltype(f)*>(a));
            else *reinterpret_cast<decltype(f)*>(a) = f;
        };
#pragma unroll
        for (int r = 0; r < 16; r += 2, next(a, r % 4 ? step : skip)) {
            if constexpr (sizeof(T) == 4) {
                put(v[r]);
                next(a, step);
                put(v[r + 1]);
            } else {
                const uint32_t two = packed(r);      // one conversion, its halves stored
                put(uint16_t(two));
                next(a, step);
                put(uint16_t(two >> 16));
            }
        }
    };
    if (o0 + 32 <= rows && t.big) {
        all(std::true_type{});
    } else if (o0 + 32 <= rows) {
        all(std::false_type{});
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r, next(a, r % 4 ? step : skip))
            if (o0 + 8 * (r / 4) + 4 * h + r % 4 < rows) store1(reinterpret_cast<T*>(a), v[r]);
    }
}
__device__ __forceinline__ void store_half(const float (&v)[16], const View& t, const Place& p, int o0, int lane, int rows) {
    if (t.dt == DC_F32)
        store_half<float>(v, t, p, o0, lane, rows);
    else
        store_half<__bf16>(v, t, p, o0, lane, rows);
}

template <int N>
__device__ __forceinline__ void apply_act(float (&v)[N], int act) {
    switch (act) {      // the same for the whole launch
        case DC_ACT_RELU:
#pragma unroll
            for (int r = 0; r < N; ++r) v[r] = act_fwd<DC_ACT_RELU>(v[r]);
            break;
        case DC_ACT_GELU:
#pragma unroll
            for (int r = 0; r < N; ++r) v[r] = act_fwd<DC_ACT_GELU>(v[r]);
            break;
        case DC_ACT_SILU:
#pragma unroll
            for (int r = 0; r < N; ++r) v[r] = act_fwd<DC_ACT_SILU>(v[r]);
            break;
        case ACT_GELU_F32:
#pragma unroll
            for (int r = 0; r < N; ++r) v[r] = act_fwd<ACT_GELU_F32>(v[r]);
            break;
        default: break;
    }
}
// z -> act(z), v -> v act'(z)
template <int N>
__device__ __forceinline__ void apply_slope(float (&z)[N], float (&v)[N], int act) {
    auto each = [&](auto tag) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float a, d;
            act_both<decltype(tag)::value>(z[r], a, d);
            z[r] = a;
            v[r] *= d;
            if (r % 8 == 7) __builtin_amdgcn_sched_barrier(0);   // eight at a time: registers
        }
    };
    switch (act) {
        case DC_ACT_RELU: each(std::integral_constant<int, DC_ACT_RELU>{}); break;
        case DC_ACT_GELU: each(std::integral_constant<int, DC_ACT_GELU>{}); break;
        case DC_ACT_SILU: each(std::integral_constant<int, DC_ACT_SILU>{}); break;
        case ACT_GELU_F32: each(std::integral_constant<int, ACT_GELU_F32>{}); break;
        default: break;
    }
}

// A lane's 16 channels (first of the block: o0) of a pixel, summed up: what is left to do
// and to store.
template <bool BWD>
__device__ __forceinline__ void epilogue(float (&v)[16], const LinearArgs& a, const Place& p, int o0, int lane) {
    const int pix = p.c.r * a.s.len + p.w, h = lane >> 5;
    if constexpr (BWD) {
        if (a.act != DC_ACT_NONE) {
            float z[16];
            if (a.z.dt == DC_Q8)
                q8_load_half(z, a.z.p, a.qm, p.c.n, o0 / 32, pix, h);
            else
                load_half(z, a.z, p, o0, lane, a.rows);
            apply_slope(z, v, a.act);
            if (a.h.dt >= 0) store_half(z, a.h, p, o0, lane, a.rows);
        }
    } else {
        if (a.z.dt == DC_Q8) {
            if (o0 + 32 > a.rows) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (o0 + 8 * (r / 4) + 4 * h + r % 4 >= a.rows) v[r] = 0;
            }
            q8_store_half(a.z.p, a.qm, p.c.n, o0 / 32, pix, p.ok, h, v);
        } else if (a.z.dt >= 0) {
            store_half(v, a.z, p, o0, lane, a.rows);
        }
        apply_act(v, a.act);
        if (a.res.dt >= 0) {
            float e[16];
            load_half(e, a.res, p, o0, lane, a.rows);
#pragma unroll
            for (int r = 0; r < 16; ++r) v[r] += e[r];
        }
    }
    store_half(v, a.out, p, o0, lane, a.rows);
}

// BWD: the input gradient (weights KR), else the forward pass (weights RK).
// CL: pixels RK (rows of channels), else KR.  DIRECT: operands on 16-byte boundaries.
template <typename S, bool BWD, bool CL, bool DIRECT>
__global__ __launch_bounds__(S::TH, S::OCC) void linear_kernel(LinearArgs a) {
    typedef typename S::T T;
    constexpr int AK = BWD ? KR : RK, PK = CL ? RK : KR, TM = S::TM, TN = S::TN;
    __shared__ __align__(16) char lds[S::NST][S::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // blocks of one column range follow each other on an XCD: they read the same pixels
    const int id = xcd_range(blockIdx.x, a.tr * a.tc);
    const int tc = id / a.tr, tr = id - tc * a.tr;
    Stage<T, AK, WEIGHT, S::BM, S::TH> sa;
    Stage<T, PK, PIXEL, S::BN, S::TH> sb;
    sa.init(a.a, a.s, tr * S::BM);
    sb.init(a.b, a.s, tc * S::BN);
    f32x16_t acc[TM][TN];
    const int row0 = wave / S::WN * (32 * TM), col0 = wave % S::WN * (32 * TN), h = lane >> 5;
    // the sums start from the bias
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int o = min(tr * S::BM + row0 + 32 * i + 8 * (r / 4) + 4 * h + r % 4, a.rows - 1);
            const float b = !BWD && a.bias ? a.bias[o] : 0.0f;
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j][r] = b;
        }
    tile_loop<S, AK, PK, DIRECT>(acc, sa, sb, a.a, a.b, a.s, 0, a.a.red, lds, row0, col0, lane, [](int, const uint4&) {});

    // The blocks of 32 x 32 pass through the wave's share of LDS, a lane's values back to
    // the lane: a loop at run time instead of one copy of the epilogue per block, which
    // overran the registers and the instruction cache.
    constexpr int Q = TM * TN, ROOM = S::NST * S::BYTES / (S::TH * 64), PER = Q < ROOM ? Q : ROOM;
    char* mine = &lds[0][0] + wave * (PER * 4096) + lane * 16;
    Place p;
    __syncthreads();
    static_for<0, (Q + PER - 1) / PER>([&](auto part) __attribute__((always_inline)) {
        constexpr int q0 = decltype(part)::value * PER, q1 = q0 + PER < Q ? q0 + PER : Q;
        static_for<q0, q1>([&](auto qc) __attribute__((always_inline)) {
            constexpr int q = decltype(qc)::value;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x16_t& t = acc[q % TM][q / TM];
                *reinterpret_cast<f32x4_t*>(mine + (q - q0) * 4096 + g * 1024) =
                    f32x4_t{t[4 * g], t[4 * g + 1], t[4 * g + 2], t[4 * g + 3]};
            }
        });
#pragma unroll 1
        for (int q = q0; q < q1; ++q) {
            const int o0 = tr * S::BM + row0 + 32 * (q % TM);
            if (q % TM == 0) p = place_of<CL ? 1 : S::E>(a.s, tc * S::BN + col0 + 32 * (q / TM) + (lane & 31));
            if (o0 >= a.rows) continue;
            float v[16];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4_t t = *reinterpret_cast<const f32x4_t*>(mine + (q - q0) * 4096 + g * 1024);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[4 * g + r] = t[r];
            }
            epilogue<BWD>(v, a, p, o0, lane);
        }
    });
}

// Long sums over many pixels: the largest block, whose operands are read least often (512
// channels to 2048 on 65536 pixels, forward with gelu and z in 8 bits, 300 us against 338
// with 128 x 256, 357 with 64 x 128).  Short sums are bound by what they store and by the
// epilogue: more and smaller workgroups at a time (64 to 256 on 100352, stored through the
// caches: 33 us against 40 with 128 x 256 and 43 with 256 x 256; 29 past them).  Few
// pixels: blocks small enough for the chip to have some.
template <typename T> using Large = Shape<T, 256, 256, 2, 4, 2, 2>;
template <typename T> using Middle = Shape<T, 64, 128, 2, 1, 4, 3>;
template <typename T> using Short = Shape<T, 64, 128, 1, 1, 4, 4>;     // one slice: half the LDS
template <typename T> using Small = Shape<T, 64, 64, 2, 2, 2, 4>;

template <typename S, bool BWD>
static void launch_shape(LinearArgs a, hipStream_t s) {
    a.tr = (a.rows + S::BM - 1) / S::BM;
    a.tc = int((int64_t(a.s.chunks) * a.s.per + S::BN - 1) / S::BN);
    const dim3 g(unsigned(a.tr) * unsigned(a.tc)), t(S::TH);
    if (a.cl && a.direct) hipLaunchKernelGGL((linear_kernel<S, BWD, true, true>), g, t, 0, s, a);
    else if (a.cl) hipLaunchKernelGGL((linear_kernel<S, BWD, true, false>), g, t, 0, s, a);
    else if (a.direct) hipLaunchKernelGGL((linear_kernel<S, BWD, false, true>), g, t, 0, s, a);
    else hipLaunchKernelGGL((linear_kernel<S, BWD, false, false>), g, t, 0, s, a);
}

template <typename T, bool BWD>
static hipError_t launch_linear(const LinearArgs& a, hipStream_t s) {
    const int64_t slots = int64_t(a.s.chunks) * a.s.per;
    auto blocks = [&](int r, int c) { return (a.rows + r - 1) / r * ((slots + c - 1) / c); };
    if (a.a.red > 128 && blocks(256, 256) >= 256) launch_shape<Large<T>, BWD>(a, s);
    else if (blocks(64, 128) >= 512 && a.a.red <= Short<T>::BK) launch_shape<Short<T>, BWD>(a, s);
    else if (blocks(64, 128) >= 512) launch_shape<Middle<T>, BWD>(a, s);
    else launch_shape<Small<T>, BWD>(a, s);
    return hipGetLastError();
}

}  // namespace dc
