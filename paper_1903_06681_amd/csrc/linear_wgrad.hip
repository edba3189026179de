// Weight and bias gradient of a product over channels: dw[k][c] = sum over pixels
// of dy[k] x[c], db[k] = sum over pixels of dy[k].
//
// The tile loop of linear.h with k running over the slots (pixels).  The result is
// small and the sum long, so the slices are dealt out in shares, each with its own
// sums in the workspace; a second launch adds the shares in order.  db is the
// row sum of dy: the first column of blocks adds up the fragments that it
// multiplies.  2048 x 512 over 65536 pixels (bf16, 137 GFLOP): 154 us, 890 TFLOP/s, and 13
// for the 16 shares; the loads from L2 bound the loop (1,150 TFLOP/s without them).
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

template <typename S, bool CL, bool DIRECT>
__global__ __launch_bounds__(S::TH, S::OCC) void linear_wgrad_kernel(LinWgradArgs a) {
    typedef typename S::T T;
    constexpr int KIND = CL ? KR : RK, TM = S::TM, TN = S::TN;
    __shared__ __align__(16) char lds[S::NST][S::BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int blocks = a.tr * a.tc;
    // the blocks of a share follow each other on an XCD: they read the same pixels
    const int id = xcd_range(blockIdx.x, blocks * a.shares);
    const int share = id / blocks, blk = id - share * blocks;
    const int tr = blk / a.tc, tc = blk - tr * a.tc;
    Stage<T, KIND, LONG, S::BM, S::TH> sa;
    Stage<T, KIND, LONG, S::BN, S::TH> sb;
    sa.init(a.a, a.s, tr * S::BM);
    sb.init(a.b, a.s, tc * S::BN);
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
    const int row0 = wave / S::WN * (32 * TM), col0 = wave % S::WN * (32 * TN);
    const bool bias = a.db && tc == 0 && wave % S::WN == 0;
    const int k0 = share * a.per * S::BK, k1 = min(a.s.chunks * a.s.per, k0 + a.per * S::BK);
    tile_loop<S, KIND, KIND, DIRECT>(acc, sa, sb, a.a, a.b, a.s, k0, k1, lds, row0, col0, lane,
                                     [&](int i, const uint4& f) __attribute__((always_inline)) {
                                         if (bias) bsum[i] += sum16<T>(f);
                                     });

    const int h = lane >> 5;
    const bool last = a.shares == 1;
    float* dw = last ? a.dw : a.part + int64_t(share) * a.K * a.C;
    float* db = last ? a.db : a.part + int64_t(a.shares) * a.K * a.C + int64_t(share) * a.K;
    const bool add = last && a.accumulate;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int o0 = tr * S::BM + row0 + 32 * i;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int c = tc * S::BN + col0 + 32 * j + (lane & 31);
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

// The sums of the shares, in a fixed order: 64 lanes of V results a workgroup, its four
// waves a quarter of the shares each.  The last K results are db.  V: 4 where n and K are
// multiples of it (16 shares of 2048 x 512: 17.0 us with V = 1).
template <int V>
__global__ __launch_bounds__(256) void linear_wgrad_sum_kernel(LinWgradArgs a) {
    typedef float fv __attribute__((ext_vector_type(V)));
    __shared__ fv red[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n = int64_t(a.K) * a.C, all = n + (a.db ? a.K : 0);
    const int64_t e = (int64_t(blockIdx.x) * 64 + lane) * V;
    const bool in = e < all, bias = e >= n;
    const float* p = bias ? a.part + a.shares * n + (e - n) : a.part + e;
    const int64_t step = bias ? a.K : n;
    const int per = (a.shares + 3) / 4, i1 = min((wave + 1) * per, a.shares);
    fv s = 0;
    if (in) {
#pragma unroll 8
        for (int i = wave * per; i < i1; ++i) s += *reinterpret_cast<const fv*>(p + i * step);
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || !in) return;
    s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
    fv* d = reinterpret_cast<fv*>(bias ? a.db + (e - n) : a.dw + e);
    *d = a.accumulate ? *d + s : s;
}

// Blocks of 256 x 256 where the result has them and each compute unit gets eight slices of
// one, or of 64 x 64 (95 rows of channels, 160 x 320, fp32: 35 us in two large blocks);
// shares so that one (two) workgroups a compute unit run, none with fewer than four slices.
template <typename T> using Large = Shape<T, 256, 256, 2, 4, 2, 2>;
template <typename T> using Small = Shape<T, 64, 64, 2, 2, 2, 4>;
static bool large(const LinWgradArgs& a, bool f32) {
    const int64_t slices = int64_t(a.s.chunks) * a.s.per / (f32 ? 32 : 64);
    return a.K > 128 && a.C > 128 && int64_t((a.K + 255) / 256) * ((a.C + 255) / 256) * slices >= 8 * 256;
}

template <typename S>
static void plan(LinWgradArgs& a) {
    a.tr = (a.K + S::BM - 1) / S::BM;
    a.tc = (a.C + S::BN - 1) / S::BN;
    const int slices = int((int64_t(a.s.chunks) * a.s.per + S::BK - 1) / S::BK), blocks = a.tr * a.tc, groups = S::BM == 256 ? 256 : 512;
    int want = std::max(1, std::min(groups / blocks, (slices + 3) / 4));
    // 257 to 511 small blocks leave the chip uneven: long sums in two shares all the same (3556
    // rows of channels, 1984 x 736, bf16: 43 us, 57 in one; 1000 rows, 16 slices: 22 and 20)
    if (S::BM < 256 && want == 1 && blocks < groups && slices >= 32) want = 2;
    a.per = (slices + want - 1) / want;
    a.shares = (slices + a.per - 1) / a.per;
}

void linear_wgrad_plan(LinWgradArgs& a, bool f32) {
    if (large(a, f32)) f32 ? plan<Large<float>>(a) : plan<Large<__bf16>>(a);
    else f32 ? plan<Small<float>>(a) : plan<Small<__bf16>>(a);
}

size_t linear_wgrad_part_bytes(const LinWgradArgs& a) {
    return a.shares == 1 ? 0 : (size_t(a.shares) * a.K * (size_t(a.C) + 1) * sizeof(float) + 15) / 16 * 16;
}

template <typename S>
static void launch(const LinWgradArgs& a, hipStream_t s) {
    const dim3 g(unsigned(a.tr) * a.tc * a.shares), t(S::TH);
    if (a.cl && a.direct) hipLaunchKernelGGL((linear_wgrad_kernel<S, true, true>), g, t, 0, s, a);
    else if (a.cl) hipLaunchKernelGGL((linear_wgrad_kernel<S, true, false>), g, t, 0, s, a);
    else if (a.direct) hipLaunchKernelGGL((linear_wgrad_kernel<S, false, true>), g, t, 0, s, a);
    else hipLaunchKernelGGL((linear_wgrad_kernel<S, false, false>), g, t, 0, s, a);
}

hipError_t launch_linear_wgrad(const LinWgradArgs& a, bool f32, hipStream_t s) {
    if (large(a, f32)) f32 ? launch<Large<float>>(a, s) : launch<Large<__bf16>>(a, s);
    else f32 ? launch<Small<float>>(a, s) : launch<Small<__bf16>>(a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.shares == 1) return e;
    const int64_t all = int64_t(a.K) * a.C + (a.db ? a.K : 0);
    if (a.K % 4 == 0)
        hipLaunchKernelGGL(linear_wgrad_sum_kernel<4>, dim3(unsigned((all + 255) / 256)), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL(linear_wgrad_sum_kernel<1>, dim3(unsigned((all + 63) / 64)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace dc
