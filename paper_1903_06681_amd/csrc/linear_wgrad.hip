// Weight and bias gradient of a product over channels: dw[k][c] = sum over pixels
// of dy[k] x[c], db[k] = sum over pixels of dy[k].
//
// The tile loop of linear.h with k running over the slots (pixels).  The result is
// small and the sum long, so the slices are dealt out in shares, each with its own
// sums in the workspace; a second launch adds the shares in order.  db is the
// row sum of dy: the first column of blocks adds up the fragments that it
// multiplies.
#include <algorithm>

#include "linear.h"

namespace dc {

template <typename T>
__device__ __forceinline__ float sum16(const uint4& f) {
    const uint32_t w[4] = {f.x, f.y, f.z, f.w};
    float s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4)
            s += __builtin_bit_cast(float, w[i]);
        else
            s += __builtin_bit_cast(float, w[i] << 16) + __builtin_bit_cast(float, w[i] & 0xffff0000u);
    }
    return s;
}

template <typename T, bool CL, int BM, int BN>
__global__ __launch_bounds__(kLinThreads) void linear_wgrad_kernel(LinWgradArgs a) {
    constexpr int KIND = CL ? KR : RK;
    typedef StagePix<T, KIND, BM> SA;
    typedef StagePix<T, KIND, BN> SB;
    constexpr int TM = BM / 64, TN = BN / 64, BK = SA::BK;
    __shared__ __align__(16) char lds[2][SA::BYTES + SB::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int blocks = a.tr * a.tc;
    // the blocks of a share follow each other on an XCD: they read the same pixels
    const int id = xcd_range(blockIdx.x, blocks * a.shares);
    const int share = id / blocks, blk = id - share * blocks;
    const int tr = blk / a.tc, tc = blk - tr * a.tc;
    SA sa;
    SB sb;
    sa.init(a.a, tr * BM);
    sb.init(a.b, tc * BN);
    uint4 va[SA::U], vb[SB::U];
    f32x16_t acc[TM][TN];
    float bsum[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        bsum[i] = 0;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    }
    const int row0 = (wave >> 1) * (BM / 2), col0 = (wave & 1) * (BN / 2);
    const bool bias = a.db && tc == 0 && (wave & 1) == 0;
    const int slots = a.s.chunks * a.s.per;
    const int k0 = share * a.per * BK, k1 = min(slots, k0 + a.per * BK);
    sa.load(va, a.a, a.s, k0);
    sb.load(vb, a.b, a.s, k0);
    sa.store(va, lds[0]);
    sb.store(vb, lds[0] + SA::BYTES);
    __syncthreads();
    for (int k = k0, buf = 0; k < k1; k += BK, buf ^= 1) {
        const bool more = k + BK < k1;
        if (more) {
            sa.load(va, a.a, a.s, k + BK);
            sb.load(vb, a.b, a.s, k + BK);
        }
        slice<T, KIND, KIND, BM, BN, TM, TN>(acc, lds[buf], lds[buf] + SA::BYTES, row0, col0, lane,
                                             [&](int i, const uint4& f) __attribute__((always_inline)) {
                                                 if (bias) bsum[i] += sum16<T>(f);
                                             });
        if (more) {
            sa.store(va, lds[buf ^ 1]);
            sb.store(vb, lds[buf ^ 1] + SA::BYTES);
        }
        __syncthreads();
    }

    const int h = lane >> 5;
    const bool last = a.shares == 1;
    float* dw = last ? a.dw : a.part + int64_t(share) * a.K * a.C;
    float* db = last ? a.db : a.part + int64_t(a.shares) * a.K * a.C + int64_t(share) * a.K;
    const bool add = last && a.accumulate;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int o0 = tr * BM + row0 + 32 * i;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int c = tc * BN + col0 + 32 * j + (lane & 31);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int o = o0 + 8 * (r / 4) + 4 * h + r % 4;
                if (o < a.K && c < a.C) {
                    float* d = dw + int64_t(o) * a.C + c;
                    *d = add ? *d + acc[i][j][r] : acc[i][j][r];
                }
            }
        }
        if (bias) {
            const float s = bsum[i] + __shfl_xor(bsum[i], 32);
            const int o = o0 + (lane & 31);
            if (h == 0 && o < a.K) db[o] = add ? db[o] + s : s;
        }
    }
}

// sums of the shares in order; the last row of the result is db
__global__ __launch_bounds__(256) void linear_wgrad_sum_kernel(LinWgradArgs a) {
    const int64_t n = int64_t(a.K) * a.C, all = n + (a.db ? a.K : 0);
    const int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (e >= all) return;
    const bool bias = e >= n;
    const float* p = bias ? a.part + a.shares * n + (e - n) : a.part + e;
    const int64_t step = bias ? a.K : n;
    float s = 0;
    for (int i = 0; i < a.shares; ++i) s += p[i * step];
    float* d = bias ? a.db + (e - n) : a.dw + e;
    *d = a.accumulate ? *d + s : s;
}

// Blocks of 128 x 128, or of 64 x 64 for small results; shares so that about 512
// workgroups run, none with fewer than four slices.
static int block_of(const LinWgradArgs& a) { return a.K > 64 && a.C > 64 ? 128 : 64; }

void linear_wgrad_plan(LinWgradArgs& a, bool f32) {
    const int b = block_of(a), bk = f32 ? 32 : 64;
    a.tr = (a.K + b - 1) / b;
    a.tc = (a.C + b - 1) / b;
    const int64_t slots = int64_t(a.s.chunks) * a.s.per;
    const int slices = int((slots + bk - 1) / bk), blocks = a.tr * a.tc;
    const int want = std::max(1, std::min(512 / std::max(1, blocks), (slices + 3) / 4));
    a.per = (slices + want - 1) / want;
    a.shares = (slices + a.per - 1) / a.per;
}

size_t linear_wgrad_part_bytes(const LinWgradArgs& a) {
    return a.shares == 1 ? 0 : (size_t(a.shares) * a.K * (size_t(a.C) + 1) * sizeof(float) + 15) / 16 * 16;
}

template <typename T>
static void launch(const LinWgradArgs& a, hipStream_t s) {
    const dim3 g(unsigned(a.tr) * a.tc * a.shares), t(kLinThreads);
    const bool big = block_of(a) == 128;
    if (a.cl && big) hipLaunchKernelGGL((linear_wgrad_kernel<T, true, 128, 128>), g, t, 0, s, a);
    else if (a.cl) hipLaunchKernelGGL((linear_wgrad_kernel<T, true, 64, 64>), g, t, 0, s, a);
    else if (big) hipLaunchKernelGGL((linear_wgrad_kernel<T, false, 128, 128>), g, t, 0, s, a);
    else hipLaunchKernelGGL((linear_wgrad_kernel<T, false, 64, 64>), g, t, 0, s, a);
}

hipError_t launch_linear_wgrad(const LinWgradArgs& a, bool f32, hipStream_t s) {
    if (f32) launch<float>(a, s);
    else launch<__bf16>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.shares == 1) return e;
    const int64_t all = int64_t(a.K) * a.C + (a.db ? a.K : 0);
    hipLaunchKernelGGL(linear_wgrad_sum_kernel, dim3(unsigned((all + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace dc
