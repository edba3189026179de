// Dropout of a tensor, and with the same arguments of its gradient.
//
// Bound: memory.  A thread takes eight channels, which share a call of the generator, and as
// many pixels as 16 bytes hold; in rows of channels eight channels of one pixel, which lie
// together.  The masks are made while the loads are on their way: 4 x 64 x 256 x 256 bf16 16.5
// us, 4.1 TB/s; after them (the values widened first) 26.
#include <algorithm>

#include "drop.h"

namespace dc {

// V elements of a row as they lie in memory, from an address on any element: those past the row's
// end (left of them are there) are not touched
template <typename T, int V>
struct Run {
    static constexpr int W = V * int(sizeof(T)) / 4;
    typedef uint32_t Words __attribute__((ext_vector_type(W), aligned(2)));
    uint32_t w[W];
    __device__ __forceinline__ void load(const char* p, int left) {
        if (left >= V) {
            const Words u = *reinterpret_cast<const Words*>(p);
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = u[i];
            return;
        }
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < left ? load1(reinterpret_cast<const T*>(p) + i) : 0.0f;
        set(f);
    }
    __device__ __forceinline__ void set(const float (&f)[V]) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __builtin_bit_cast(uint32_t, f[i]);
            else w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{f[2 * i], f[2 * i + 1]}), bf16x2_t));
        }
    }
    __device__ __forceinline__ float value(int i) const {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
        else return __builtin_bit_cast(float, i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void store(char* p, int left) const {
        if (left >= V) {
            Words u;
#pragma unroll
            for (int i = 0; i < W; ++i) u[i] = w[i];
            *reinterpret_cast<Words*>(p) = u;
            return;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) store1(reinterpret_cast<T*>(p) + i, value(i));
    }
};
// the mask of eight channels, a bit each
__device__ __forceinline__ uint32_t mask8(const DropArgs& d, const DropPixel& p, uint64_t pos) {
    const Philox w = philox(pos, p.ctr, d.seed);
    uint32_t b = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) b |= kept(w, j, d.t) ? 1u << j : 0u;
    return b;
}

// planes: V pixels of a row, eight channels
template <typename XT, typename YT, int V>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
    const int ci = int(blockIdx.x * 256 + threadIdx.x);
    if (ci >= a.chunks) return;
    const int n = int(a.dsample.div(uint32_t(ci))), rem = ci - n * int(a.dsample.d);
    const int r = int(a.dcpr.div(uint32_t(rem))), col = (rem - r * a.cpr) * V, left = a.len - col;
    // the first pixel's position; those after it follow, or where the image's row ends begin the next
    const int pix = r * a.len + col, ends = a.d.W - (pix - int(a.d.dW.div(uint32_t(pix))) * a.d.W);
    const DropPixel p = drop_pixel(a.d, n, pix);
    const char* x = a.x.p + (n * a.x.sn + r * a.x.sh + col) * int64_t(sizeof(XT));
    char* y = a.y.p + (n * a.y.sn + r * a.y.sh + col) * int64_t(sizeof(YT));
    for (int g = int(blockIdx.y); g < a.d.groups; g += int(gridDim.y)) {
        const int c0 = 8 * g, cn = a.C - c0;
        Run<XT, V> v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j].load(x + (c0 + min(j, cn - 1)) * a.x.sc * int64_t(sizeof(XT)), left);
        // the masks while the loads are on their way
        uint32_t bits[V];
        const uint64_t first = p.pos + uint64_t(g) * uint64_t(a.d.plane);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            uint64_t pos = first + i;
            if (i >= ends) pos = drop_pixel(a.d, n, min(pix + i, a.HW - 1)).pos + uint64_t(g) * uint64_t(a.d.plane);
            bits[i] = mask8(a.d, p, pos);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f[V];
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = masked(v[j].value(i) * a.d.scale, bits[i], j);
            Run<YT, V> u;
            u.set(f);
            if (j < cn) u.store(y + (c0 + j) * a.y.sc * int64_t(sizeof(YT)), left);
        }
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
        Run<XT, 8> v;
        v.load(a.x.p + (n * a.x.sn + pix * a.x.sh + 8 * g) * int64_t(sizeof(XT)), a.C - 8 * g);
        const uint32_t bits = mask8(a.d, p, p.pos + uint64_t(g) * uint64_t(a.d.plane));
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = masked(v.value(j) * a.d.scale, bits, j);
        Run<YT, 8> u;
        u.set(f);
        u.store(a.y.p + (n * a.y.sn + pix * a.y.sh + 8 * g) * int64_t(sizeof(YT)), a.C - 8 * g);
    }
}

// 16 bytes a thread, or 8 where that leaves the chip fewer than two waves a SIMD: 3 x 43 x 93 x
// 75 fp32 4.9 us (490 waves otherwise: 5.9), 4 x 64 x 256 x 256 bf16 17.6 (16.5).
int dropout_chunk(const View& x, const View& y, bool rows, int64_t pixels, int groups) {
    if (rows) return 1;
    const int v = x.dt == DC_BF16 && y.dt == DC_BF16 ? 8 : 4;
    return pixels / v * groups < 2048 * 64 ? v / 2 : v;
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
    const dim3 g(unsigned((int64_t(a.chunks) + 255) / 256), unsigned(std::min(a.d.groups, 65535)));
    if (a.per == V) hipLaunchKernelGGL((dropout_kernel<XT, YT, V>), g, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((dropout_kernel<XT, YT, V / 2>), g, dim3(256), 0, s, a);
}

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
    if (a.x.dt == DC_F32) a.y.dt == DC_F32 ? launch<float, float>(a, s) : launch<float, __bf16>(a, s);
    else a.y.dt == DC_F32 ? launch<__bf16, float>(a, s) : launch<__bf16, __bf16>(a, s);
    return hipGetLastError();
}

}  // namespace dc
