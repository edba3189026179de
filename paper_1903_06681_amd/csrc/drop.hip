// Dropout of a tensor, and with the same arguments of its gradient.
//
// Bound: memory and the generator's multipliers alike.  A thread takes eight channels, which
// share a call of the generator, and as many pixels as 16 bytes hold; in rows of channels
// eight channels of one pixel, which lie together.
#include <algorithm>

#include "drop.h"

namespace dc {

typedef uint32_t u32x2_at __attribute__((ext_vector_type(2), aligned(2)));

// V values of a type from, to an address on any element
template <typename T, int V>
__device__ __forceinline__ void get(float (&v)[V], const char* p, int left) {
    if (left >= V) {
        uint32_t w[V * sizeof(T) / 4];
        if constexpr (V * sizeof(T) == 16) {
            const u32x4_any u = *reinterpret_cast<const u32x4_any*>(p);
            __builtin_memcpy(w, &u, 16);
        } else if constexpr (V * sizeof(T) == 32) {
            const u32x4_any u = *reinterpret_cast<const u32x4_any*>(p), u2 = *reinterpret_cast<const u32x4_any*>(p + 16);
            __builtin_memcpy(w, &u, 16);
            __builtin_memcpy(w + 4, &u2, 16);
        } else {
            const u32x2_at u = *reinterpret_cast<const u32x2_at*>(p);
            __builtin_memcpy(w, &u, 8);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = __builtin_bit_cast(float, w[i]);
            else v[i] = __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < left ? load1(reinterpret_cast<const T*>(p) + i) : 0.0f;
    }
}

template <typename T, int V>
__device__ __forceinline__ void put(const float (&v)[V], char* p, int left) {
    if (left >= V) {
        uint32_t w[V * sizeof(T) / 4];
#pragma unroll
        for (int i = 0; i < int(V * sizeof(T) / 4); ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __builtin_bit_cast(uint32_t, v[i]);
            else w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{v[2 * i], v[2 * i + 1]}), bf16x2_t));
        }
        if constexpr (V * sizeof(T) >= 16) {
#pragma unroll
            for (int i = 0; i < int(V * sizeof(T) / 4); i += 4)
                *reinterpret_cast<u32x4_any*>(p + 4 * i) = u32x4_any{w[i], w[i + 1], w[i + 2], w[i + 3]};
        } else {
            *reinterpret_cast<u32x2_at*>(p) = u32x2_at{w[0], w[1]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) store1(reinterpret_cast<T*>(p) + i, v[i]);
    }
}

// planes: V pixels of a row, eight channels
template <typename XT, typename YT, int V>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
    const int ci = int(blockIdx.x * 256 + threadIdx.x);
    if (ci >= a.chunks) return;
    const int n = int(a.dsample.div(uint32_t(ci))), rem = ci - n * int(a.dsample.d);
    const int r = int(a.dcpr.div(uint32_t(rem))), col = (rem - r * a.cpr) * V, left = a.len - col;
    uint64_t pos[V];
    uint64_t ctr = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const DropPixel p = drop_pixel(a.d, n, min(r * a.len + col + i, a.HW - 1));
        pos[i] = p.pos;
        ctr = p.ctr;
    }
    const char* x = a.x.p + (n * a.x.sn + r * a.x.sh + col) * int64_t(sizeof(XT));
    char* y = a.y.p + (n * a.y.sn + r * a.y.sh + col) * int64_t(sizeof(YT));
    for (int g = int(blockIdx.y); g < a.d.groups; g += int(gridDim.y)) {
        const int c0 = 8 * g, cn = a.C - c0;
        float v[8][V];
#pragma unroll
        for (int j = 0; j < 8; ++j) get<XT, V>(v[j], x + (c0 + min(j, cn - 1)) * a.x.sc * int64_t(sizeof(XT)), left);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Philox w = philox(pos[i] + uint64_t(g) * uint64_t(a.d.plane), ctr, a.d.seed);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j][i] = kept(w, j, a.d.t) ? v[j][i] * a.d.scale : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < cn) put<YT, V>(v[j], y + (c0 + j) * a.y.sc * int64_t(sizeof(YT)), left);
    }
}

// rows of channels: eight channels of a pixel, neighbouring eights on neighbouring threads
template <typename XT, typename YT>
__global__ __launch_bounds__(256) void dropout_rows_kernel(DropoutArgs a, FastDiv dg) {
    // 256 threads take several pixels, or 256 eights of one
    const int per = a.d.groups < 256 ? 256 / a.d.groups : 1;
    const int i = per > 1 ? int(dg.div(threadIdx.x)) : 0;
    const int g = per > 1 ? int(threadIdx.x) - i * a.d.groups : int(blockIdx.y * 256 + threadIdx.x);
    if (i >= per || g >= a.d.groups) return;
    for (int64_t m = int64_t(blockIdx.x) * per + i; m < a.chunks; m += int64_t(gridDim.x) * per) {
        const int n = int(a.dsample.div(uint32_t(m))), pix = int(m) - n * a.HW;
        const DropPixel p = drop_pixel(a.d, n, pix);
        float v[8];
        get<XT, 8>(v, a.x.p + (n * a.x.sn + pix * a.x.sh + 8 * g) * int64_t(sizeof(XT)), a.C - 8 * g);
        const Philox w = philox(p.pos + uint64_t(g) * uint64_t(a.d.plane), p.ctr, a.d.seed);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = kept(w, j, a.d.t) ? v[j] * a.d.scale : 0.0f;
        put<YT, 8>(v, a.y.p + (n * a.y.sn + pix * a.y.sh + 8 * g) * int64_t(sizeof(YT)), a.C - 8 * g);
    }
}

int dropout_chunk(const View& x, const View& y, bool rows) {
    return rows ? 1 : x.dt == DC_BF16 && y.dt == DC_BF16 ? 8 : 4;
}

template <typename XT, typename YT>
static void launch(const DropoutArgs& a, hipStream_t s) {
    if (a.rows) {
        const int per = a.d.groups < 256 ? 256 / a.d.groups : 1;
        const int64_t sets = (int64_t(a.chunks) + per - 1) / per;
        const dim3 g(unsigned(std::min(sets, int64_t(1) << 22)), unsigned((a.d.groups + 255) / 256));   // threads of a dimension: 32 bits
        hipLaunchKernelGGL((dropout_rows_kernel<XT, YT>), g, dim3(256), 0, s, a, fast_div(uint32_t(a.d.groups)));
        return;
    }
    constexpr int V = sizeof(XT) == 2 && sizeof(YT) == 2 ? 8 : 4;
    const unsigned gx = unsigned((int64_t(a.chunks) + 255) / 256);
    hipLaunchKernelGGL((dropout_kernel<XT, YT, V>), dim3(gx, unsigned(std::min(a.d.groups, 65535))), dim3(256), 0, s, a);
}

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
    if (a.x.dt == DC_F32) a.y.dt == DC_F32 ? launch<float, float>(a, s) : launch<float, __bf16>(a, s);
    else a.y.dt == DC_F32 ? launch<__bf16, float>(a, s) : launch<__bf16, __bf16>(a, s);
    return hipGetLastError();
}

}  // namespace dc
