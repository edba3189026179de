// Products over the channels of every pixel on the matrix cores: the tile loop
// that the forward pass, the input gradient and the weight gradient share.
//
//   out[row][col] = sum over k of A[row][k] B[col][k]
//
// A workgroup of four waves (two by two) holds a BM x BN block of the result in
// accumulators and walks along k in slices of 128 bytes an operand row, staged in
// LDS while the slice before is multiplied.  An operand lies in memory in one of
// two ways, and in LDS as in memory:
//
//   RK  k contiguous:     [row][k], fragments are 16-byte reads; the row's eight
//                         16-byte chunks are permuted by the row (chunk ^ row & 7),
//                         so that the lanes of a read fall on different banks
//   KR  rows contiguous:  [k][row] (a tile's channels are planes: the pixels are
//                         contiguous, not the channels).  bf16 fragments are
//                         transposing reads of 4 x 16 elements, chunks permuted by k;
//                         fp32 ones are 4-byte reads, contiguous over the lanes
//
// so no operand is ever transposed by instructions.  fp32 runs on the fp32 matrix
// instruction: products and sums are fp32, infinities and NaN are taken whole.
#pragma once

#include "act.h"
#include "act_kernels.h"

namespace dc {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element's address

enum { RK = 0, KR = 1 };
static constexpr int kLinThreads = 256;

// 16 bytes from element `off` of p; what lies past element `end` reads as zero.
// Elements between two rows of a view are read with them and never used.
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p, int64_t off, int64_t end) {
    constexpr int E = 16 / int(sizeof(T));
    if (off + E <= end) {
        const u32x4_any v = *reinterpret_cast<const u32x4_any*>(p + off);
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    uint4 r = make_uint4(0, 0, 0, 0);
    T t[E];
#pragma unroll
    for (int i = 0; i < E; ++i) t[i] = off + i < end ? p[off + i] : T(0);
    __builtin_memcpy(&r, t, 16);
    return r;
}

// keep the first n elements (n < 1: none), zero the rest
template <typename T>
__device__ __forceinline__ uint4 keep16(uint4 v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4)
            w[i] = i < n ? w[i] : 0;
        else
            w[i] &= (2 * i < n ? 0x0000ffffu : 0u) | (2 * i + 1 < n ? 0xffff0000u : 0u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- slots: the pixels as the kernels number them.  A tile's rows are cut in
// chunks of 16 bytes, and a chunk's slots past the row's end are no pixels;
// where a sample's row is a single pixel (rows of channels) a slot is a pixel.
struct Chunk { int n, r, col, left; };   // left: pixels from col on (< 1: none)
__device__ __forceinline__ Chunk chunk_of(const Slots& s, int ci) {
    Chunk c;
    const int cc = min(ci, s.chunks - 1);
    c.n = int(s.dsample.div(uint32_t(cc)));
    const int rem = cc - c.n * int(s.dsample.d);
    c.r = int(s.dcpr.div(uint32_t(rem)));
    c.col = (rem - c.r * s.cpr) * s.per;
    c.left = ci < s.chunks ? s.len - c.col : 0;
    return c;
}

// How chunk (row or col, k) of an operand is found.
enum { WEIGHT, PIXEL };

// ---- staging of one operand's slice: R rows (or columns) of 128 bytes
template <typename T, int KIND, int SRC, int R>
struct Stage {
    static constexpr int E = 16 / int(sizeof(T));
    static constexpr int BK = 128 / int(sizeof(T));
    static constexpr int CPR = KIND == RK ? 8 : R / E;          // chunks of an LDS row
    static constexpr int U = R * 8 / kLinThreads;               // chunks a thread
    static constexpr int STEP = kLinThreads / CPR;              // LDS rows between them
    static constexpr int BYTES = R * 128;

    const T* p;
    int r0, c;             // this thread's first LDS row, its chunk
    int64_t off[KIND == RK ? U : 1];
    int left;              // KR pixels: slots of the chunk that are pixels

    __device__ __forceinline__ static uint32_t at(int row, int chunk) {
        if constexpr (KIND == RK) return row * 128 + ((chunk ^ (row & 7)) << 4);
        else if constexpr (sizeof(T) == 2)
            return row * (R * 2) + ((chunk ^ (R == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1))) << 4);
        else return row * (R * 4) + (chunk << 4);
    }

    // first: the block's first row (weights), channel or slot
    __device__ __forceinline__ void init(const Operand& o, const Slots& s, int first) {
        p = reinterpret_cast<const T*>(o.p);
        r0 = threadIdx.x / CPR;
        c = threadIdx.x % CPR;
        left = E;
        if constexpr (KIND == RK) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int row = first + r0 + i * STEP;
                if constexpr (SRC == WEIGHT) {
                    off[i] = row < o.rows ? row * o.ld : -1;
                } else {                       // rows of channels: a slot is a pixel
                    const Chunk k = chunk_of(s, row);
                    off[i] = k.left > 0 ? k.n * o.sn + k.r * o.sh : -1;
                }
            }
        } else {
            if constexpr (SRC == WEIGHT) {
                off[0] = first + c * E;
                left = o.rows - int(off[0]);
            } else {
                const Chunk k = chunk_of(s, first / E + c);
                off[0] = k.n * o.sn + k.r * o.sh + k.col;
                left = k.left;
            }
        }
    }

    // slice from k0 on
    __device__ __forceinline__ void load(uint4 (&v)[U], const Operand& o, int k0) const {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            v[i] = make_uint4(0, 0, 0, 0);
            if constexpr (KIND == RK) {
                const int k = k0 + c * E;
                if (off[i] >= 0 && k < o.red) {
                    v[i] = load16(p, off[i] + k, o.end);
                    if (k + E > o.red) v[i] = keep16<T>(v[i], o.red - k);
                }
            } else {
                const int k = k0 + r0 + i * STEP;
                if (left > 0 && k < o.red) v[i] = load16(p, off[0] + k * (SRC == WEIGHT ? o.ld : o.sc), o.end);
            }
        }
    }
    __device__ __forceinline__ void store(const uint4 (&v)[U], char* lds) const {
#pragma unroll
        for (int i = 0; i < U; ++i) *reinterpret_cast<uint4*>(lds + at(r0 + i * STEP, c)) = v[i];
    }
};

// ---- the weight gradient's operands: k runs over the pixels
template <typename T, int KIND, int R>
struct StagePix {
    static constexpr int E = 16 / int(sizeof(T));
    static constexpr int BK = 128 / int(sizeof(T));
    typedef Stage<T, KIND, PIXEL, R> S;
    static constexpr int CPR = S::CPR, U = S::U, STEP = S::STEP, BYTES = S::BYTES;

    const T* p;
    int r0, c, first;

    __device__ __forceinline__ void init(const Operand& o, int first_) {
        p = reinterpret_cast<const T*>(o.p);
        r0 = threadIdx.x / CPR;
        c = threadIdx.x % CPR;
        first = first_;
    }
    // slice k0 (slots); RK: planes of pixels, KR: rows of channels
    __device__ __forceinline__ void load(uint4 (&v)[U], const Operand& o, const Slots& s, int k0) const {
        if constexpr (KIND == RK) {
            const Chunk k = chunk_of(s, k0 / E + c);
            const int64_t at = k.n * o.sn + k.r * o.sh + k.col;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int row = first + r0 + i * STEP;
                v[i] = make_uint4(0, 0, 0, 0);
                if (k.left > 0 && row < o.rows) {
                    v[i] = load16(p, at + row * o.sc, o.end);
                    if (k.left < E) v[i] = keep16<T>(v[i], k.left);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const Chunk k = chunk_of(s, k0 + r0 + i * STEP);
                v[i] = make_uint4(0, 0, 0, 0);
                if (k.left > 0 && first + c * E < o.rows) v[i] = load16(p, k.n * o.sn + k.r * o.sh + first + c * E, o.end);
            }
        }
    }
    __device__ __forceinline__ void store(const uint4 (&v)[U], char* lds) const {
#pragma unroll
        for (int i = 0; i < U; ++i) *reinterpret_cast<uint4*>(lds + S::at(r0 + i * STEP, c)) = v[i];
    }
};

// ---- fragments.  k-group g: 16 (bf16) or 8 (fp32) values of k.  bf16: lane l
// holds row l % 32, k 8 (l / 32) .. + 7.  fp32: k 4 (l / 32) + i for i = 0 .. 3,
// one matrix instruction each.
template <typename T, int KIND, int R>
__device__ __forceinline__ void fragment(uint4& f, const char* lds, int row0, int g, int lane) {
    typedef Stage<T, KIND, WEIGHT, R> S;
    const int h = lane >> 5, r = lane & 31;
    if constexpr (KIND == RK) {
        f = *reinterpret_cast<const uint4*>(lds + S::at(row0 + r, 2 * g + h));
    } else if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) s16x4_t* lds4;
        const int k = 16 * g + 8 * h + ((lane & 15) >> 2);
        const int chunk = row0 / 8 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        auto* base = (__attribute__((address_space(3))) const char*)lds;
        const uint32_t b = uint32_t(uintptr_t(base));
        const uint32_t a0 = b + S::at(k, chunk) + (lane & 1) * 8, a1 = b + S::at(k + 4, chunk) + (lane & 1) * 8;
        const s16x4_t f0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)a0);
        const s16x4_t f1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(uintptr_t)a1);
        f = __builtin_bit_cast(uint4, __builtin_shufflevector(f0, f1, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = *reinterpret_cast<const uint32_t*>(lds + (8 * g + 4 * h + i) * (R * 4) + (row0 + r) * 4);
        f = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <typename T>
__device__ __forceinline__ void multiply(f32x16_t& acc, const uint4& a, const uint4& b) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                      acc, 0, 0, 0);
    } else {
        const f32x4_t fa = __builtin_bit_cast(f32x4_t, a), fb = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[i], fb[i], acc, 0, 0, 0);
    }
}

// One slice: the wave's TM x TN blocks of 32 x 32.  seen(i, fragment) for every A
// fragment (the weight gradient's row sums).
template <typename T, int AK, int BK_, int BM, int BN, int TM, int TN, typename F>
__device__ __forceinline__ void slice(f32x16_t (&acc)[TM][TN], const char* a, const char* b, int row0, int col0, int lane,
                                      F&& seen) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint4 fa[TM], fb[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) fragment<T, AK, BM>(fa[i], a, row0 + 32 * i, g, lane);
#pragma unroll
        for (int j = 0; j < TN; ++j) fragment<T, BK_, BN>(fb[j], b, col0 + 32 * j, g, lane);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            seen(i, fa[i]);
#pragma unroll
            for (int j = 0; j < TN; ++j) multiply<T>(acc[i][j], fa[i], fb[j]);
        }
    }
}

}  // namespace dc
