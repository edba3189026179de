// Dropout whose mask is never stored: it is formed again from counters wherever it is read.
//
// The counters' generator is Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011).  One call serves eight channels
// of a pixel, 16 bits each: a call is ten rounds of two 32 x 32 -> 64 bit products, which
// quarter-rate multipliers make as dear as the memory traffic of eight bf16 values; with
// 32 bits a value it would be twice that.  What that costs is the share's grain of 2^-16.
#pragma once

#include "act.h"

namespace dc {

// The position of a pixel in the whole image, and the draw.  t = 0: no dropout.
struct DropArgs {
    uint64_t seed, offset;
    const uint64_t* step;      // null: 0
    int64_t plane, cols;       // pixels and columns of the whole image
    int32_t groups, t;         // eights of channels; threshold of 16 bits
    float scale;               // of what is kept
    int32_t n0, h0, w0, H, W, Q;
    FastDiv per, dW, dQ;       // samples of a tile, columns of the view, tiles of a row
};

struct DropPixel {
    uint64_t pos, ctr;         // counter of the first eight channels, its upper half
};

__device__ __forceinline__ uint64_t drop_counter(const DropArgs& d) { return d.offset + (d.step ? *d.step : 0); }
__device__ __forceinline__ uint64_t drop_position(const DropArgs& d, int n, int pix) {
    const int tile = int(d.per.div(uint32_t(n))), tp = int(d.dQ.div(uint32_t(tile)));
    const int r = int(d.dW.div(uint32_t(pix)));
    const int64_t s = d.n0 + int64_t(n - tile * int(d.per.d));
    const int64_t h = d.h0 + int64_t(tp) * d.H + r, w = d.w0 + int64_t(tile - tp * d.Q) * d.W + (pix - r * d.W);
    return uint64_t(s * d.groups * d.plane + h * d.cols + w);
}
__device__ __forceinline__ DropPixel drop_pixel(const DropArgs& d, int n, int pix) {
    return DropPixel{drop_position(d, n, pix), drop_counter(d)};
}

// four words for eight channels
struct Philox { uint32_t w[4]; };
__device__ __forceinline__ Philox philox(uint64_t pos, uint64_t ctr, uint64_t seed) {
    uint32_t a = uint32_t(pos), b = uint32_t(pos >> 32), c = uint32_t(ctr), d = uint32_t(ctr >> 32);
    uint32_t k0 = uint32_t(seed), k1 = uint32_t(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i, k0 += 0x9E3779B9u, k1 += 0xBB67AE85u) {
        const uint64_t x = uint64_t(a) * 0xD2511F53u, y = uint64_t(c) * 0xCD9E8D57u;
        a = uint32_t(y >> 32) ^ b ^ k0;
        b = uint32_t(y);
        c = uint32_t(x >> 32) ^ d ^ k1;
        d = uint32_t(x);
    }
    return Philox{{a, b, c, d}};
}

// whether channel j of the eight stays
__device__ __forceinline__ bool kept(const Philox& p, int j, int t) {
    return j & 1 ? p.w[j / 2] >= uint32_t(t) << 16 : uint16_t(p.w[j / 2]) >= uint16_t(t);
}

// v where bit j is set, else 0, whatever v is
__device__ __forceinline__ float masked(float v, uint32_t bits, int j) {
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) & uint32_t(int32_t(bits << (31 - j)) >> 31));
}

struct DropoutArgs {
    View x, y;
    DropArgs d;
    int32_t C, HW, len;        // pixels of a sample, of a row of the numbering
    int32_t per;               // pixels of a chunk
    int32_t chunks, cpr;       // chunks in all, of a row
    FastDiv dsample, dcpr;     // chunks of a sample, of a row
    int32_t rows;              // rows of channels
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);
int dropout_chunk(const View& x, const View& y, bool rows, int64_t pixels, int groups);    // pixels a thread takes

}  // namespace dc
