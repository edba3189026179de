// What the products over channels on few pixels share (linear_few.hip, gate_few.hip): sixteen
// waves (or eight) share the sum of a 16-row block of the result, fragments straight from memory.
#pragma once

#include "linear_pass.h"

namespace dc {

static constexpr int kFewWaves = 16;
typedef float f32x4_acc __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ void multiply16(f32x4_acc& acc, const uint4& a, const uint4& b) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0,
                                                      0, 0);
    } else {
        const f32x4_t fa = __builtin_bit_cast(f32x4_t, a), fb = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[i], fb[i], acc, 0, 0, 0);
    }
}

// element of channel 0 of pixel m
template <typename V>
__device__ __forceinline__ int64_t few_offset(const Slots& s, int hw, int m, const V& v) {
    const int n = m / hw, pix = m - n * hw, r = pix / s.len;
    return n * v.sn + r * v.sh + (pix - r * s.len);
}

// The waves' sums of a block: 16 rows (row: the lane's, of lane % 16) by NT tiles of 16 pixels
// from m0 on.  BWD: weights [k][row].  DEEP: whole steps of k several at once.
template <typename T, bool BWD, bool CL, int NT, int WAVES, bool DEEP = true>
__device__ __forceinline__ void few_sums(float (&sums)[WAVES][NT * 256], const LinearArgs& a, int row, int m0, int M, int hw,
                                         int lane, int wave) {
    constexpr int E = 16 / int(sizeof(T)), STEP = 4 * E;      // k of a lane's chunk, of a wave's step
    const int red = a.a.red;
    const T* w = reinterpret_cast<const T*>(a.a.p);
    const T* x = reinterpret_cast<const T*>(a.b.p);
    int64_t xo[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) xo[t] = few_offset(a.s, hw, min(m0 + t * 16 + (lane & 15), M - 1), a.b);
    // eight (four) values of k of which n count, `step` elements apart; past the end the last one's address
    auto gather = [&](const T* p, int64_t step, int n) __attribute__((always_inline)) {
        T e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const T f = p[max(min(i, n - 1), 0) * step];
            e[i] = i < n ? f : T(0);
        }
        uint4 r;
        __builtin_memcpy(&r, e, 16);
        return r;
    };
    // this wave's steps of k
    const int steps = (red + STEP - 1) / STEP, per = (steps + WAVES - 1) / WAVES;
    const int s0 = wave * per, s1 = min(s0 + per, steps), whole = min(s1, red / STEP);
    f32x4_acc acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4_acc{0, 0, 0, 0};
    // Steps that lie within k as a whole: D at once on their way, no lane asks what is there (one by
    // one, each with its questions, the gated product of a pixel, 2048 to twice 8192 in bf16, takes 24.8 us,
    // so 14.5; eight at once 15.1).
    auto some = [&](auto depth, int& s) __attribute__((always_inline)) {
        constexpr int D = decltype(depth)::value;
        auto row_of = [&](const T* p) __attribute__((always_inline)) {
            const u32x4_any v = *reinterpret_cast<const u32x4_any*>(p);
            return make_uint4(v.x, v.y, v.z, v.w);
        };
        auto column = [&](const T* p, int64_t step) __attribute__((always_inline)) {
            T e[E];
#pragma unroll
            for (int i = 0; i < E; ++i) e[i] = p[i * step];
            uint4 r;
            __builtin_memcpy(&r, e, 16);
            return r;
        };
        for (; s + D <= whole; s += D) {
            uint4 fa[D], fb[D][NT];
#pragma unroll
            for (int d = 0; d < D; ++d) {
                const int64_t k = (s + d) * STEP + (lane >> 4) * E;
                if constexpr (BWD) fa[d] = column(w + k * a.a.ld + row, a.a.ld);
                else fa[d] = row_of(w + row * a.a.ld + k);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if constexpr (CL) fb[d][t] = row_of(x + xo[t] + k);
                    else fb[d][t] = column(x + xo[t] + k * a.b.sc, a.b.sc);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < D; ++d)
#pragma unroll
                for (int t = 0; t < NT; ++t) multiply16<T>(acc[t], fa[d], fb[d][t]);
        }
    };
    int s = s0;
    if constexpr (DEEP) {
        some(std::integral_constant<int, NT == 4 ? 2 : 4>{}, s);
        if constexpr (NT != 4) some(std::integral_constant<int, 2>{}, s);
    }
#pragma unroll(DEEP ? 1 : 4)
    for (; s < s1; ++s) {
        const int k = s * STEP + (lane >> 4) * E, n = red - k, kk = min(k, red - 1);
        uint4 fa = make_uint4(0, 0, 0, 0), fb[NT];
        if constexpr (BWD) fa = gather(w + int64_t(kk) * a.a.ld + row, a.a.ld, n);
        else if (n > 0) fa = keep16<T>(load16(w, row * a.a.ld + k, a.a.end), n);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            fb[t] = make_uint4(0, 0, 0, 0);
            if constexpr (CL) {
                if (n > 0) fb[t] = keep16<T>(load16(x, xo[t] + k, a.b.end), n);
            } else {
                fb[t] = gather(x + xo[t] + kk * a.b.sc, a.b.sc, n);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) multiply16<T>(acc[t], fa, fb[t]);
    }
    // lane: pixel lane % 16, channels 4 (lane / 16) .. + 3
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][t * 256 + (4 * (lane >> 4) + r) * 16 + (lane & 15)] = acc[t][r];
    __syncthreads();
}

inline int few_pixels(const LinearArgs& a) {
    return a.s.chunks / int(a.s.dsample.d) * (int(a.s.dsample.d) / a.s.cpr * a.s.len);
}

}  // namespace dc
