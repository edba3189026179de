// Forward pass and input gradient of a product over channels: the tile loop of
// linear.h with rows = output channels and columns = slots (pixels), and the
// epilogue in registers.
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

// A lane's 16 channels of one pixel in a view; rows: channels of the view.
// `whole`: the block lies inside them.
template <typename T>
__device__ __forceinline__ void load_half(float (&v)[16], const View& t, int64_t at, int o0, int h, int rows) {
    const T* p = reinterpret_cast<const T*>(t.p) + at;
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = load1(p + min(o0 + 8 * (r / 4) + 4 * h + r % 4, rows - 1) * t.sc);
}
__device__ __forceinline__ void load_half(float (&v)[16], const View& t, int64_t at, int o0, int h, int rows) {
    if (t.dt == DC_F32)
        load_half<float>(v, t, at, o0, h, rows);
    else
        load_half<__bf16>(v, t, at, o0, h, rows);
}
template <typename T>
__device__ __forceinline__ void store_half(const float (&v)[16], const View& t, int64_t at, int o0, int h, int rows) {
    T* p = reinterpret_cast<T*>(t.p) + at;
    if (t.sc == 1 && o0 + 32 <= rows) {      // rows of channels: four lie together
        typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            T w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) store1(w + i, v[4 * g + i]);
            if constexpr (sizeof(T) == 4) {
                u32x4_any d;
                __builtin_memcpy(&d, w, 16);
                *reinterpret_cast<u32x4_any*>(p + o0 + 8 * g + 4 * h) = d;
            } else {
                u32x2_any d;
                __builtin_memcpy(&d, w, 8);
                *reinterpret_cast<u32x2_any*>(p + o0 + 8 * g + 4 * h) = d;
            }
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int o = o0 + 8 * (r / 4) + 4 * h + r % 4;
        if (o < rows) store1(p + o * t.sc, v[r]);
    }
}
__device__ __forceinline__ void store_half(const float (&v)[16], const View& t, int64_t at, int o0, int h, int rows) {
    if (t.dt == DC_F32)
        store_half<float>(v, t, at, o0, h, rows);
    else
        store_half<__bf16>(v, t, at, o0, h, rows);
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
        }
    };
    switch (act) {
        case DC_ACT_RELU: each(std::integral_constant<int, DC_ACT_RELU>{}); break;
        case DC_ACT_GELU: each(std::integral_constant<int, DC_ACT_GELU>{}); break;
        case DC_ACT_SILU: each(std::integral_constant<int, DC_ACT_SILU>{}); break;
        default: break;
    }
}

// BWD: the input gradient (weights KR), else the forward pass (weights RK).
// CL: pixels RK (rows of channels), else KR.
template <typename T, bool BWD, bool CL, int BM, int BN>
__global__ __launch_bounds__(kLinThreads) void linear_kernel(LinearArgs a) {
    constexpr int AK = BWD ? KR : RK, PK = CL ? RK : KR;
    typedef Stage<T, AK, WEIGHT, BM> SA;
    typedef Stage<T, PK, PIXEL, BN> SB;
    constexpr int TM = BM / 64, TN = BN / 64, BK = SA::BK;
    __shared__ __align__(16) char lds[2][SA::BYTES + SB::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // blocks of one column range follow each other on an XCD: they read the same pixels
    const int id = xcd_range(blockIdx.x, a.tr * a.tc);
    const int tc = id / a.tr, tr = id - tc * a.tr;
    SA sa;
    SB sb;
    sa.init(a.a, a.s, tr * BM);
    sb.init(a.b, a.s, tc * BN);
    uint4 va[SA::U], vb[SB::U];
    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    const int row0 = (wave >> 1) * (BM / 2), col0 = (wave & 1) * (BN / 2);
    sa.load(va, a.a, 0);
    sb.load(vb, a.b, 0);
    sa.store(va, lds[0]);
    sb.store(vb, lds[0] + SA::BYTES);
    __syncthreads();
    const int red = a.a.red;
    for (int k = 0, buf = 0; k < red; k += BK, buf ^= 1) {
        const bool more = k + BK < red;
        if (more) {
            sa.load(va, a.a, k + BK);
            sb.load(vb, a.b, k + BK);
        }
        slice<T, AK, PK, BM, BN, TM, TN>(acc, lds[buf], lds[buf] + SA::BYTES, row0, col0, lane, [](int, const uint4&) {});
        if (more) {
            sa.store(va, lds[buf ^ 1]);
            sb.store(vb, lds[buf ^ 1] + SA::BYTES);
        }
        __syncthreads();
    }

    const int h = lane >> 5;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int slot = tc * BN + col0 + 32 * j + (lane & 31);
        const int per = CL ? 1 : SB::E, sub = CL ? 0 : slot % SB::E;
        const Chunk c = chunk_of(a.s, slot / per);
        const bool ok = sub < c.left;
        const int w = ok ? c.col + sub : 0, pix = c.r * a.s.len + w;   // in range on every lane
        auto at = [&](const View& t) __attribute__((always_inline)) { return c.n * t.sn + c.r * t.sh + w; };
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int o0 = tr * BM + row0 + 32 * i;
            if (o0 >= a.rows) continue;
            float v[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) v[r] = acc[i][j][r];
            if constexpr (BWD) {
                if (a.act != DC_ACT_NONE) {
                    float z[16];
                    if (a.z.dt == DC_Q8)
                        q8_load_half(z, a.z.p, a.qm, c.n, o0 / 32, pix, h);
                    else
                        load_half(z, a.z, at(a.z), o0, h, a.rows);
                    apply_slope(z, v, a.act);
                    if (a.h.dt >= 0 && ok) store_half(z, a.h, at(a.h), o0, h, a.rows);
                }
            } else {
                if (a.bias) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[r] += a.bias[min(o0 + 8 * (r / 4) + 4 * h + r % 4, a.rows - 1)];
                }
                if (a.z.dt == DC_Q8) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (o0 + 8 * (r / 4) + 4 * h + r % 4 >= a.rows) v[r] = 0;
                    q8_store_half(a.z.p, a.qm, c.n, o0 / 32, pix, ok, h, v);
                } else if (a.z.dt >= 0 && ok) {
                    store_half(v, a.z, at(a.z), o0, h, a.rows);
                }
                apply_act(v, a.act);
                if (a.res.dt >= 0) {
                    float e[16];
                    load_half(e, a.res, at(a.res), o0, h, a.rows);
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[r] += e[r];
                }
            }
            if (ok) store_half(v, a.out, at(a.out), o0, h, a.rows);
        }
    }
}

// Blocks of 128 x 128, or of 64 x 64 where those would not fill the chip.
template <typename T, bool BWD>
static hipError_t launch_linear(LinearArgs a, hipStream_t s) {
    const int64_t slots = int64_t(a.s.chunks) * a.s.per;
    auto blocks = [&](int b) { return ((a.rows + b - 1) / b) * ((slots + b - 1) / b); };
    const int b = blocks(128) >= 512 ? 128 : 64;
    a.tr = (a.rows + b - 1) / b;
    a.tc = int((slots + b - 1) / b);
    const dim3 g(unsigned(a.tr) * unsigned(a.tc)), t(kLinThreads);
    if (a.cl && b == 128) hipLaunchKernelGGL((linear_kernel<T, BWD, true, 128, 128>), g, t, 0, s, a);
    else if (a.cl) hipLaunchKernelGGL((linear_kernel<T, BWD, true, 64, 64>), g, t, 0, s, a);
    else if (b == 128) hipLaunchKernelGGL((linear_kernel<T, BWD, false, 128, 128>), g, t, 0, s, a);
    else hipLaunchKernelGGL((linear_kernel<T, BWD, false, 64, 64>), g, t, 0, s, a);
    return hipGetLastError();
}

}  // namespace dc
