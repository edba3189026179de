// What the kernels between two convolutions (norm, pointwise products, 8-bit
// checkpoints) share: views of tiles, pixel numbering, activations, the 8-bit form.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include <cstdint>

#include "dc.h"

namespace dc {

// n / d for n < 2^31 by the host's m = ceil(2^(31+l) / d), l = ceil(log2 d): the
// error of m adds less than n 2^l / (d 2^(31+l)) < 1 / d to the quotient.
// m = 0 stands for d = 1.
struct FastDiv {
    uint32_t m, sh, d;
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return m ? __umulhi(n, m) >> sh : n; }
};

inline FastDiv fast_div(uint32_t d) {
    FastDiv f{0, 0, d};
    if (d > 1) {
        int l = 0;
        while ((uint64_t(1) << l) < d) ++l;
        f.m = uint32_t(((uint64_t(1) << (31 + l)) + d - 1) / d);
        f.sh = uint32_t(l - 1);
    }
    return f;
}

// A view on the device: pointer, element strides, type.
struct View {
    char* p;
    int64_t sn, sc, sh;
    int32_t dt;        // DC_F32, DC_BF16, DC_Q8; -1: absent
    int32_t big;       // large enough to be stored past the caches (products)
};

// The pixels of a set of views, numbered sample by sample in rows of `len`: the
// tile's rows, or all of an image as one row where every view's rows follow each
// other without a gap (then sh is never used).
struct Pixels {
    int32_t M;         // N H W
    int32_t HW, len;
    FastDiv dHW, dlen;
};

// 8-bit form: q at 32 bytes per pixel and block, scales behind (one byte each)
struct Q8Map {
    int64_t qn, s0, sn;   // bytes per sample of q; start and bytes per sample of the scales
    int32_t HW;
};
inline Q8Map q8_map(int64_t N, int C, int64_t HW) {
    const int64_t cb = (C + 31) / 32;
    return Q8Map{cb * HW * 32, N * cb * HW * 32, cb * HW, int32_t(HW)};
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// one element; bf16 widens exactly
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __bf16* p) {
    return __builtin_bit_cast(float, uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(__bf16* p, float v) { *p = static_cast<__bf16>(v); }   // nearest, ties to even

// ---- activations, formed in fp32.
//
// gelu is z Phi(z) with the normal distribution's Phi; its slope Phi(z) + z phi(z).  The
// value is z times Phi(z) as written: +infinity stays (z less |z| times the tail would be
// infinity times 0), and at -infinity it is NaN, as the formula's -infinity times 0.
//
// Results in bf16.  Phi's tail is phi-like, so one exponential serves both: for a = |z| /
// sqrt 2, erfc(a) = t (a1 + t (a2 + ...)) e^(-a^2), t = 1 / (1 + p a), with the
// coefficients of Abramowitz and Stegun, Handbook of Mathematical Functions (1964),
// 7.1.26 (here halved, p over sqrt 2): |error| <= 1.5e-7, far below a rounding to bf16.
// Thirteen vector operations, the exponential and the reciprocal a value: an epilogue's
// vector operations weigh as much as its matrix ones.
struct Normal { float phi, e; };   // Phi(z), e^(-z^2 / 2)
__device__ __forceinline__ Normal normal(float z) {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.23164189f, 1.0f));
    const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    float s = fmaf(0.5307027145f, t, -0.7265760135f);
    s = fmaf(s, t, 0.7107068705f);
    s = fmaf(s, t, -0.142248368f);
    s = fmaf(s, t, 0.127414796f);
    const float tail = s * t * e;      // Phi(-|z|)
    return Normal{z < 0 ? tail : 1.0f - tail, e};
}

// Results in fp32, where the above is three to five roundings off near 0: Phi(-a) =
// 2^(-1 - a R(a)) for a = |z|, R a polynomial of nine degrees fitted here by least squares
// reweighted towards the largest error (5.3e-9 of the tail; relative 7e-8 to a = 3, 1e-6 at
// 4, 5e-4 at 6; a R(a) only grows, so that large a give 0).  Near 0 the exponent vanishes
// and its error with it: over values of scale 0.05 the root mean square error is 5.7e-8 of
// theirs, one rounding 4e-8, the form above 1.8e-7.  The gradient needs phi's exponential
// besides.  32 to 128 channels on 512 x 512 take 47.7 us either way; 64 to 256 on 100352,
// z in 8 bits, 31.7 us and 30.1, the gradient 35.9 and 32.2, so bf16 stays with the above.
__device__ __forceinline__ Normal normal_f32(float z) {
    const float a = fabsf(z);
    float s = fmaf(-3.9319481e-8f, a, 1.07841856e-6f);
    s = fmaf(s, a, -1.28321344e-5f);
    s = fmaf(s, a, 8.47210322e-5f);
    s = fmaf(s, a, -3.00129468e-4f);
    s = fmaf(s, a, 2.80938257e-5f);
    s = fmaf(s, a, 6.92720432e-3f);
    s = fmaf(s, a, -5.24358973e-2f);
    s = fmaf(s, a, -0.459220618f);
    s = fmaf(s, a, -1.15110433f);
    const float t = __builtin_amdgcn_exp2f(s * a);      // twice the tail
    return Normal{z < 0 ? 0.5f * t : fmaf(-0.5f, t, 1.0f), __builtin_amdgcn_exp2f(z * z * -0.72134752f)};
}

// gelu whose result is kept in fp32, beside dc_activation's
enum { ACT_GELU_F32 = DC_ACT_SILU + 1 };
inline int32_t act_code(int32_t act, bool f32) { return f32 && act == DC_ACT_GELU ? int32_t(ACT_GELU_F32) : act; }

__device__ __forceinline__ float logistic(float z) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

template <int ACT>
__device__ __forceinline__ float act_fwd(float z) {
    if constexpr (ACT == DC_ACT_RELU) return z <= 0 ? 0.0f : z;   // NaN stays
    if constexpr (ACT == DC_ACT_GELU) return z * normal(z).phi;
    if constexpr (ACT == ACT_GELU_F32) return z * normal_f32(z).phi;
    if constexpr (ACT == DC_ACT_SILU) return z * logistic(z);
    return z;
}

// value and slope at once
template <int ACT>
__device__ __forceinline__ void act_both(float z, float& v, float& d) {
    if constexpr (ACT == DC_ACT_RELU) {
        v = z <= 0 ? 0.0f : z;
        d = z <= 0 ? 0.0f : z > 0 ? 1.0f : z;
    } else if constexpr (ACT == DC_ACT_GELU || ACT == ACT_GELU_F32) {
        const Normal n = ACT == DC_ACT_GELU ? normal(z) : normal_f32(z);
        v = z * n.phi;
        d = fmaf(z * 0.39894228f, n.e, n.phi);
    } else if constexpr (ACT == DC_ACT_SILU) {
        const float s = logistic(z);
        v = z * s;
        d = fmaf(v, 1.0f - s, s);
    } else {
        v = z;
        d = 1.0f;
    }
}

// ---- the 8-bit form
__device__ __forceinline__ uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
// scale byte of a block whose largest magnitude has these bits (as integers they
// order like the magnitudes, NaN above infinity)
__device__ __forceinline__ uint32_t q8_scale(uint32_t top) { return max(top >> 23, 7u); }
__device__ __forceinline__ float q8_per(uint32_t s) { return __builtin_bit_cast(float, (260u - s) << 23); }
__device__ __forceinline__ float q8_step(uint32_t s) {
    return __builtin_bit_cast(float, s == 255u ? 0x7fc00000u : (s - 6u) << 23);
}
// four values -> four bytes, lowest first.  per is a power of two, so v per is exact
// and 1.5 2^23 + v per rounds to an integer, ties to even, whose low byte is q's.  The
// block of a NaN may hold any q.
__device__ __forceinline__ uint32_t q8_bits(float v, float per) {
    constexpr float kInt = 12582912.0f;
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(fmaf(v, per, kInt), kInt - 127.0f, kInt + 127.0f));
}
__device__ __forceinline__ uint32_t q8_pack(float a, float b, float c, float d, float per) {
    const uint32_t lo = __builtin_amdgcn_perm(q8_bits(b, per), q8_bits(a, per), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(q8_bits(d, per), q8_bits(c, per), 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}
// byte k of w as a value
__device__ __forceinline__ float q8_value(uint32_t w, int k, float step) {
    return float(int32_t(w << (24 - 8 * k)) >> 24) * step;
}

// Where pixel m of the numbering lies; the last one's place for m past it.
struct Pixel { int n, h, w, pix; };
__device__ __forceinline__ Pixel pixel_of(const Pixels& x, int m0) {
    Pixel r;
    const int m = min(m0, x.M - 1);
    r.n = int(x.dHW.div(uint32_t(m)));
    r.pix = m - r.n * x.HW;
    r.h = int(x.dlen.div(uint32_t(r.pix)));
    r.w = r.pix - r.h * x.len;
    return r;
}

// The lane's address of a pixel in a view.
template <typename T>
__device__ __forceinline__ char* spot_of(const View& v, const Pixel& p) {
    return v.p + (p.n * v.sn + p.h * v.sh + p.w) * int64_t(sizeof(T));
}
// The next channel's address.  Kept from the optimiser, which would otherwise form the
// offsets of 32 channels of every tensor ahead of a loop and run out of registers (2.5 KB
// of scratch a lane in the norm's backward pass).
__device__ __forceinline__ void next(char*& p, int64_t step) {
    p += step;
    asm("" : "+v"(p));
}

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element's address

// Values of one pixel's block of 32 channels (first: c0), loaded and stored.  CL: the
// channels are contiguous, so a block is 16-byte vectors (and single elements at C's end);
// else every channel is an access of its own, contiguous over the wave's pixels.  (In bf16
// that is 2 bytes a lane.  Four lanes trading values for 8 bytes of one channel each were
// slower: a save of 4 x 64 x 256 x 256 14.0 us against 10.2.)
template <typename T, bool CL>
__device__ __forceinline__ void load_block(float (&v)[32], const View& t, const Pixel& p, int c0, int C) {
    char* a = spot_of<T>(t, p) + c0 * (CL ? 1 : t.sc) * int64_t(sizeof(T));
    if constexpr (CL) {
        constexpr int VE = 16 / int(sizeof(T));
#pragma unroll
        for (int j = 0; j < 32 / VE; ++j) {
            u32x4_any u{0, 0, 0, 0};
            const int left = C - (c0 + j * VE);
            if (left >= VE) {
                u = *reinterpret_cast<const u32x4_any*>(a + j * 16);
            } else if (left > 0) {
                T e[VE];
#pragma unroll
                for (int i = 0; i < VE; ++i) e[i] = i < left ? reinterpret_cast<const T*>(a + j * 16)[i] : T(0);
                __builtin_memcpy(&u, e, 16);
            }
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                if constexpr (VE == 4)
                    v[j * VE + i] = __builtin_bit_cast(float, w[i]);
                else
                    v[j * VE + i] = __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
            }
        }
    } else {
        const int64_t step = t.sc * int64_t(sizeof(T));
        if (__all(c0 + 32 <= C)) {
#pragma unroll
            for (int j = 0; j < 32; ++j, next(a, step)) v[j] = load1(reinterpret_cast<const T*>(a));
        } else {
            // Channels past C repeat the last one's address and count as zero: a branch for
            // eight of them, not for each (which waits for each load in turn).
            int left = C - c0;
            asm volatile("" : "+v"(left));   // 32 comparisons here, not 32 results ahead of a loop
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0;
#pragma unroll
            for (int g = 0; g < 32; g += 8) {
                if (!__any(g < left)) break;
#pragma unroll
                for (int j = g; j < g + 8; ++j) {
                    const float f = load1(reinterpret_cast<const T*>(a));
                    v[j] = j < left ? f : 0.0f;
                    next(a, j + 1 < left ? step : 0);
                }
            }
        }
    }
}

template <typename T, bool CL>
__device__ __forceinline__ void store_block(const View& t, const Pixel& p, int c0, int C, const float (&v)[32]) {
    char* a = spot_of<T>(t, p) + c0 * (CL ? 1 : t.sc) * int64_t(sizeof(T));
    if constexpr (CL) {
        constexpr int VE = 16 / int(sizeof(T));
#pragma unroll
        for (int j = 0; j < 32 / VE; ++j) {
            const int left = C - (c0 + j * VE);
            if (left < VE) {
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    if (i < left) store1(reinterpret_cast<T*>(a + j * 16) + i, v[j * VE + i]);
                continue;
            }
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (VE == 4)
                    w[i] = __builtin_bit_cast(uint32_t, v[j * VE + i]);
                else
                    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                                                            (f32x2_t{v[j * VE + 2 * i], v[j * VE + 2 * i + 1]}), bf16x2_t));
            }
            *reinterpret_cast<u32x4_any*>(a + j * 16) = u32x4_any{w[0], w[1], w[2], w[3]};
        }
    } else {
        const int64_t step = t.sc * int64_t(sizeof(T));
        if (c0 + 32 <= C) {
#pragma unroll
            for (int j = 0; j < 32; ++j, next(a, step)) store1(reinterpret_cast<T*>(a), v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j, next(a, step))
                if (c0 + j < C) store1(reinterpret_cast<T*>(a), v[j]);
        }
    }
}

// a block's bytes and scale <-> its values
__device__ __forceinline__ void q8_store_block(char* q, const Q8Map& m, const Pixel& p, int cb, const float (&v)[32]) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) top = max(top, abs_bits(v[j]));
    const uint32_t s = q8_scale(top);
    const float per = q8_per(s);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = q8_pack(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3], per);
    const int64_t at = int64_t(cb) * m.HW + p.pix;
    uint4* d = reinterpret_cast<uint4*>(q + p.n * m.qn + at * 32);
    d[0] = make_uint4(w[0], w[1], w[2], w[3]);
    d[1] = make_uint4(w[4], w[5], w[6], w[7]);
    reinterpret_cast<uint8_t*>(q)[m.s0 + p.n * m.sn + at] = uint8_t(s);
}

__device__ __forceinline__ void q8_load_block(float (&v)[32], const char* q, const Q8Map& m, const Pixel& p, int cb) {
    const int64_t at = int64_t(cb) * m.HW + p.pix;
    const uint4* d = reinterpret_cast<const uint4*>(q + p.n * m.qn + at * 32);
    const uint4 a = d[0], b = d[1];
    const float step = q8_step(reinterpret_cast<const uint8_t*>(q)[m.s0 + p.n * m.sn + at]);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = q8_value(w[j / 4], j % 4, step);
}

// Workgroup index with each of the 8 XCDs (round-robin dispatch) on a contiguous
// range, so that neighbours share their XCD's L2; total is the grid.
__device__ __forceinline__ int xcd_range(int b, int total) {
    const int per = total / 8, rest = total % 8, x = b % 8, i = b / 8;
    return x * per + min(x, rest) + i;
}

}  // namespace dc
