// Eight channels of one pixel a lane: what a call of dropout's generator serves, 16 bytes of
// bf16 in rows of channels, a quarter of the 8-bit form's block.
#pragma once

#include "drop.h"

namespace dc {

// Eight channels as they lie in memory; channels past C repeat the last one.  (A vector, not an
// array: stores to different elements in different branches would be joined to one at a chosen
// address, and the array kept in scratch.)
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));

// Addresses in global memory as such: a pointer whose steps the optimiser may not see through
// (next, act.h) would else count as one to anything, whose accesses also wait for LDS's.
typedef __attribute__((address_space(1))) char gchar;
template <typename T> using global_ptr = __attribute__((address_space(1))) T*;
__device__ __forceinline__ void next(gchar*& p, int64_t step) {
    p += step;
    asm("" : "+v"(p));
}
template <typename T, typename P>
__device__ __forceinline__ T load_as(P p) {
    return *(global_ptr<const T>)(p);
}
template <typename T, typename P>
__device__ __forceinline__ void store_as(P p, T v) {
    *(global_ptr<T>)(p) = v;
}
// past the caches: they are left to what is read
template <typename T, typename P>
__device__ __forceinline__ void stream_as(P p, T v) {
    __builtin_nontemporal_store(v, (global_ptr<T>)(p));
}
__device__ __forceinline__ gchar* spot8(const View& t, const Pixel& p, int64_t c, int es) {
    return (gchar*)(t.p) + (p.n * t.sn + p.h * t.sh + p.w + c) * es;
}

// Channels from c0 on; known only here, so that what follows from it is formed where it is used,
// not ahead of a loop (eight steps or masks for every tensor).
__device__ __forceinline__ int left_of(int c0, int C) {
    int left = C - c0;
    asm volatile("" : "+v"(left));
    return left;
}

template <bool CL>
__device__ __forceinline__ u32x8 load8(const View& t, const Q8Map& qm, const Pixel& p, int c0, int C) {
    if (t.dt == DC_Q8) {
        const int64_t at = int64_t(c0 / 32) * qm.HW + p.pix;
        typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
        const u32x2_t b = load_as<u32x2_t>((gchar*)(t.p) + p.n * qm.qn + at * 32 + c0 % 32);
        return u32x8{b.x, b.y, load_as<uint8_t>((gchar*)(t.p) + qm.s0 + p.n * qm.sn + at), 0, 0, 0, 0, 0};
    }
    const int es = t.dt == DC_F32 ? 4 : 2;
    gchar* a = spot8(t, p, c0 * (CL ? 1 : t.sc), es);
    if (CL && c0 + 8 <= C) {
        const u32x4_any u = load_as<u32x4_any>(a);
        if (es == 2) return u32x8{u.x, u.y, u.z, u.w, 0, 0, 0, 0};
        const u32x4_any u2 = load_as<u32x4_any>(a + 16);
        return u32x8{u.x, u.y, u.z, u.w, u2.x, u2.y, u2.z, u2.w};
    }
    const int64_t step = (CL ? 1 : t.sc) * es;
    u32x8 r;
    auto all = [&](auto type, auto&& on) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 8; ++j, next(a, on(j))) r[j] = load_as<decltype(type)>(a);
    };
    if (!CL && c0 + 8 <= C) {
        auto on = [&](int) __attribute__((always_inline)) { return step; };
        es == 4 ? all(uint32_t(0), on) : all(uint16_t(0), on);
    } else {
        const int left = left_of(c0, C);
        auto on = [&](int j) __attribute__((always_inline)) { return j < left ? step : 0; };
        es == 4 ? all(uint32_t(0), on) : all(uint16_t(0), on);
        if (CL && es == 4) return r;
    }
    if constexpr (!CL) return r;
    return u32x8{r[0] | r[1] << 16, r[2] | r[3] << 16, r[4] | r[5] << 16, r[6] | r[7] << 16, 0, 0, 0, 0};
}

__device__ __forceinline__ void clear8(float (&v)[8], int c0, int C) {
    if (c0 + 8 <= C) return;
    const int left = left_of(c0, C);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? v[j] : 0.0f;
}

// their values; channels past C are zero
template <bool CL>
__device__ __forceinline__ void values8(float (&v)[8], const u32x8& w, const View& t, int c0, int C) {
    if (t.dt == DC_Q8) {
        const float step = q8_step(w[2]);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = q8_value(j < 4 ? w[0] : w[1], j % 4, step);
    } else if (t.dt == DC_F32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(float, uint32_t(w[j]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (CL) v[j] = __builtin_bit_cast(float, uint32_t(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16));
            else v[j] = __builtin_bit_cast(float, uint32_t(w[j] << 16));
        }
    }
    clear8(v, c0, C);
}

template <bool CL>
__device__ __forceinline__ void store8(const View& t, const Pixel& p, int c0, int C, const float (&v)[8]) {
    auto bits = [&](int j) __attribute__((always_inline)) { return __builtin_bit_cast(uint32_t, v[j]); };
    auto two = [&](int j) __attribute__((always_inline)) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{v[j], v[j + 1]}), bf16x2_t));
    };
    const int es = t.dt == DC_F32 ? 4 : 2;
    gchar* a = spot8(t, p, c0 * (CL ? 1 : t.sc), es);
    if (CL && c0 + 8 <= C) {
        if (es == 4) {
            store_as(a, u32x4_any{bits(0), bits(1), bits(2), bits(3)});
            store_as(a + 16, u32x4_any{bits(4), bits(5), bits(6), bits(7)});
        } else {
            store_as(a, u32x4_any{two(0), two(2), two(4), two(6)});
        }
        return;
    }
    const int64_t step = (CL ? 1 : t.sc) * es;
    auto all = [&](int left) __attribute__((always_inline)) {
        if (es == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j, next(a, step))
                if (j < left) store_as(a, v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; j += 2, next(a, step)) {
                const uint32_t w = two(j);      // one conversion, its halves stored
                if (j < left) store_as(a, uint16_t(w));
                next(a, step);
                if (j + 1 < left) store_as(a, uint16_t(w >> 16));
            }
        }
    };
    c0 + 8 <= C ? all(8) : all(left_of(c0, C));
}

// Eight parameters from p on (c0: of channel c0); where there is none, `none`.  UNIFORM: the same
// for the wave, scalar loads.  Else vector loads whose address is formed here (ahead of a loop the
// eight addresses of every parameter would take the registers).
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
template <bool UNIFORM>
__device__ __forceinline__ void params8(float (&v)[8], const float* p, int c0, int C, float none) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = none;
        return;
    }
    if constexpr (UNIFORM) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = p[min(c0 + j, C - 1)];
        return;
    }
    gchar* a = (gchar*)(const_cast<float*>(p + c0));
    next(a, 0);
    if (c0 + 8 <= C) {
        const f32x4_any f = load_as<f32x4_any>(a), g = load_as<f32x4_any>(a + 16);
        v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
        v[4] = g.x, v[5] = g.y, v[6] = g.z, v[7] = g.w;
    } else {
        const int left = left_of(c0, C);
#pragma unroll
        for (int j = 0; j < 8; ++j, next(a, j < left ? 4 : 0)) v[j] = load_as<float>(a);
    }
}
// The mask of eight channels as what they are multiplied by: 0, or what keeps the mean.
__device__ __forceinline__ void keep8(float (&k)[8], const DropArgs& d, const DropPixel& dp, int e) {
    if (!d.t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) k[j] = 1.0f;
        return;
    }
    const Philox w = philox(dp.pos + uint64_t(e) * uint64_t(d.plane), dp.ctr, d.seed);
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] = kept(w, j, d.t) ? d.scale : 0.0f;
}
// 0 times anything is 0 here, NaN and infinities included: what is dropped leaves nothing
__device__ __forceinline__ float dropped(float v, float keep) {
    float r;
    asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(v), "v"(keep));
    return r;
}

// The 8-bit form of eight channels (e: which of the tensor's eights), written; four
// neighbouring lanes of the wave hold a block of 32, and all four come here, those past the
// last channel too (with zeros).
__device__ __forceinline__ void q8_store_eight(char* q, const Q8Map& m, const Pixel& p, int e, bool in, int C, const float (&v)[8]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, abs_bits(v[j]));
    top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0xb1, 0xf, 0xf, true)));      // lane ^ 1
    top = max(top, uint32_t(__builtin_amdgcn_update_dpp(0, int(top), 0x4e, 0xf, 0xf, true)));      // lane ^ 2
    const uint32_t s = q8_scale(top);
    const float per = q8_per(s);
    if (!in || e / 4 * 32 >= C) return;
    typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
    const int64_t at = int64_t(e / 4) * m.HW + p.pix;
    store_as((gchar*)q + p.n * m.qn + at * 32 + e % 4 * 8,
             u32x2_t{q8_pack(v[0], v[1], v[2], v[3], per), q8_pack(v[4], v[5], v[6], v[7], per)});
    if (e % 4 == 0) store_as((gchar*)q + m.s0 + p.n * m.sn + at, uint8_t(s));
}

}  // namespace dc
