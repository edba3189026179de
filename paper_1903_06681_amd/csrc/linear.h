// Products over the channels of every pixel on the matrix cores: the tile loop
// that the forward pass, the input gradient and the weight gradient share.
//
//   out[row][col] = sum over k of A[row][k] B[col][k]
//
// A workgroup of WM x WN waves holds a BM x BN block of the result in
// accumulators and walks along k in slices of 128 bytes an operand row, staged in
// LDS while the slice before is multiplied.  An operand lies in memory in one of
// two ways, and in LDS as in memory:
//
//   RK  k contiguous:     [row][k], fragments are 16-byte reads; the row's eight
//                         16-byte chunks are permuted by the row,
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
#include "bf16util.h"

namespace dc {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

enum { RK = 0, KR = 1 };

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

// 16 bytes a lane from memory to LDS, the lanes' one after the other from `to` (the
// wave's).  Written out: the compiler would wait for it before any LDS read.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"     // m0 is a reserved register; the compiler does write it
__device__ __forceinline__ void direct16(const void* p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(__builtin_amdgcn_readfirstlane(to)), "v"(p) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void wait_direct() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const char* p) {
    return uint32_t(uintptr_t((__attribute__((address_space(3))) const char*)p));
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

enum { WEIGHT, PIXEL, LONG, PAIR };   // which way an operand is found: see Stage

static constexpr int kRow = 128;   // bytes of k a slice

// The shape of a workgroup's block: BM x BN of the result, NST slices in LDS (2 or 3, or 1 where
// there is only one) of KB bytes of k, WM x WN waves; OCC waves a SIMD that the registers leave
// room for.
template <typename T_, int BM_, int BN_, int NST_, int WM_, int WN_, int OCC_, int KB_ = kRow>
struct Shape {
    typedef T_ T;
    static constexpr int BM = BM_, BN = BN_, NST = NST_, WM = WM_, WN = WN_, OCC = OCC_, KB = KB_;
    static constexpr int E = 16 / int(sizeof(T)), BK = KB / int(sizeof(T));
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32, GROUPS = KB / 32;
    static constexpr int ABYTES = BM * KB, BYTES = (BM + BN) * KB;
    static constexpr int TH = 64 * WM * WN;
};

// ---- staging of one operand's slice: R rows by KB bytes of k.
//   WEIGHT  a matrix, rows [row][k] (RK) or [k][row] (KR)
//   PIXEL   rows are slots: k the channels' planes (KR), or contiguous (RK: rows of channels)
//   LONG    k runs over the slots, rows are channels: planes (RK), or rows of channels (KR)
//   PAIR    two matrices of o.rows rows, one below the other (RK): of the block's rows,
//           groups of 32 are taken from the one and the other in turn
// A thread's chunks of 16 bytes follow each other in LDS at a distance of the
// workgroup; which chunk of memory they hold is permuted, so that LDS is written in
// order (as direct loads must) and read without bank conflicts.
template <typename T, int KIND, int SRC, int R, int TH, int KB = kRow>
struct Stage {
    static constexpr int E = 16 / int(sizeof(T));
    static constexpr int CPR = KIND == RK ? KB / 16 : R / E;    // chunks of an LDS row
    static constexpr int U = R * KB / 16 / TH;         // chunks a thread
    static constexpr int STEP = TH / CPR;              // LDS rows between them
    // pointers a thread keeps: one for all chunks where they lie at equal distances
    static constexpr int P = SRC == PIXEL && KIND == RK ? U : 1;

    int64_t at[P];         // element of chunk 0 in slice 0 (LONG: of row or channel 0), -1: nothing there
    int32_t r0, c, left;   // first LDS row; chunk; rows or slots of the chunk that there are
    bool whole;            // all of the wave's chunks lie inside the rows

    // the permutation of an LDS row's chunks; the same for all rows of a thread
    __device__ __forceinline__ static int mix(int row) {
        if constexpr (KIND == RK) return KB == 128 ? (row >> 1) & 7 : (row >> 2) & 3;   // 16 lanes, 256 bytes a cycle
        else if constexpr (sizeof(T) == 2) return R >= 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
        else return 0;
    }
    __device__ __forceinline__ static uint32_t lds_at(int row, int chunk) { return (row * CPR + (chunk ^ mix(row))) << 4; }

    // first: the block's first row, slot or channel
    __device__ __forceinline__ void init(const Operand& o, const Slots& s, int first) {
        static_assert(CPR <= TH && U >= 1 && (KIND == RK || STEP % 4 == 0 || sizeof(T) == 4));
        r0 = threadIdx.x / CPR;
        c = (threadIdx.x % CPR) ^ mix(r0);
        left = E;
        bool in = true;
        if constexpr (SRC == PAIR) {               // first: of the pair
            static_assert(KIND == RK && (STEP <= 32 || STEP % 64 == 0));
            const int row = first + r0 / 64 * 32 + r0 % 32;
            at[0] = (int64_t(row) + (r0 / 32 % 2 ? o.rows : 0)) * o.ld + c * E;
            left = o.rows - row;
        } else if constexpr (SRC == WEIGHT && KIND == RK) {
            at[0] = int64_t(first + r0) * o.ld + c * E;
            left = o.rows - (first + r0);          // rows from this one on
        } else if constexpr (SRC == WEIGHT) {
            at[0] = first + c * E + r0 * o.ld;
            left = o.rows - (first + c * E);
        } else if constexpr (SRC == PIXEL && KIND == RK) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const Chunk k = chunk_of(s, first + r0 + i * STEP);
                at[i] = k.left > 0 ? k.n * o.sn + k.r * o.sh + c * E : -1;
                in = in && k.left > 0;
            }
        } else if constexpr (SRC == PIXEL) {
            const Chunk k = chunk_of(s, first / E + c);
            at[0] = k.n * o.sn + k.r * o.sh + k.col + r0 * o.sc;
            left = k.left;
        } else if constexpr (KIND == RK) {
            at[0] = (first + r0) * o.sc;
            left = o.rows - (first + r0);          // channels from this one on
        } else {
            at[0] = first + c * E;
            left = o.rows - (first + c * E);
        }
        whole = __all(in && left > (SRC == PAIR ? pair_row(U - 1) : KIND == RK && SRC != PIXEL ? (U - 1) * STEP : 0));
    }

    // PAIR: row of chunk i after chunk 0's; whether it is one of the second matrix (of the other, where
    // a thread's chunks lie whole pairs of groups apart)
    __device__ __forceinline__ static constexpr int pair_row(int i) {
        return STEP >= 64 ? i * STEP / 2 : (i * STEP / 32) / 2 * 32 + i * STEP % 32;
    }
    __device__ __forceinline__ static constexpr bool pair_second(int i) { return STEP < 64 && (i * STEP / 32) % 2; }

    // f(i, element, elements of the chunk that count) for the chunks of the slice at k0
    template <typename F>
    __device__ __forceinline__ void each(const Operand& o, const Slots& s, int k0, F&& f) const {
        if constexpr (SRC == LONG && KIND == RK) {
            const Chunk k = chunk_of(s, k0 / E + c);
            int64_t e = k.n * o.sn + k.r * o.sh + k.col + at[0];
#pragma unroll
            for (int i = 0; i < U; ++i, e += STEP * o.sc) f(i, e, left - i * STEP > 0 ? k.left : 0);
        } else if constexpr (SRC == LONG) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const Chunk k = chunk_of(s, k0 + r0 + i * STEP);
                f(i, k.n * o.sn + k.r * o.sh + at[0], k.left > 0 ? left : 0);
            }
        } else if constexpr (KIND == RK) {
            const int n = o.red - (k0 + c * E);
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if constexpr (SRC == PIXEL) f(i, at[i] + k0, at[i] >= 0 ? n : 0);
                else if constexpr (SRC == PAIR)
                    f(i, at[0] + k0 + (pair_row(i) + (pair_second(i) ? int64_t(o.rows) : 0)) * o.ld, left - pair_row(i) > 0 ? n : 0);
                else f(i, at[0] + k0 + i * STEP * o.ld, left - i * STEP > 0 ? n : 0);
            }
        } else {
            const int64_t ld = SRC == WEIGHT ? o.ld : o.sc;
            int64_t e = at[0] + k0 * ld;
#pragma unroll
            for (int i = 0; i < U; ++i, e += STEP * ld) f(i, e, k0 + r0 + i * STEP < o.red ? left : 0);
        }
    }

    // chunks past an end are zero, and so are elements past k's end; elements past a
    // row's end (KR) are whatever lies there, for results that nobody keeps
    __device__ __forceinline__ void load(uint4 (&v)[U], const Operand& o, const Slots& s, int k0) const {
        const T* p = reinterpret_cast<const T*>(o.p);
        each(o, s, k0, [&](int i, int64_t e, int n) __attribute__((always_inline)) {
            v[i] = make_uint4(0, 0, 0, 0);
            if (n > 0) {
                v[i] = load16(p, e, o.end);
                if (KIND == RK && n < E) v[i] = keep16<T>(v[i], n);
            }
        });
    }
    __device__ __forceinline__ void store(const uint4 (&v)[U], char* lds) const {
#pragma unroll
        for (int i = 0; i < U; ++i) *reinterpret_cast<uint4*>(lds + (threadIdx.x + i * TH) * 16) = v[i];
    }

    // the same without registers, for aligned operands (their chunks are whole); all:
    // every lane's chunk is there
    template <bool ALL>
    __device__ __forceinline__ void fetch(const Operand& o, const Slots& s, int k0, char* lds, uint32_t to) const {
        const T* p = reinterpret_cast<const T*>(o.p);
        each(o, s, k0, [&](int i, int64_t e, int n) __attribute__((always_inline)) {
            if (ALL || n > 0)
                direct16(p + e, to + (i * TH + (threadIdx.x & ~63)) * 16);
            else
                *reinterpret_cast<uint4*>(lds + (threadIdx.x + i * TH) * 16) = make_uint4(0, 0, 0, 0);
        });
    }
};

// ---- fragments.  k-group g: 16 (bf16) or 8 (fp32) values of k.  bf16: lane l
// holds row l % 32, k 8 (l / 32) .. + 7.  fp32: k 4 (l / 32) + i for i = 0 .. 3,
// one matrix instruction each.
template <typename T, int KIND, int R, int TH, int KB = kRow>
__device__ __forceinline__ void fragment(uint4& f, const char* lds, int row0, int g, int lane) {
    typedef Stage<T, KIND, WEIGHT, R, TH, KB> S;
    const int h = lane >> 5, r = lane & 31;
    if constexpr (KIND == RK) {
        f = *reinterpret_cast<const uint4*>(lds + S::lds_at(row0 + r, 2 * g + h));
    } else if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) s16x4_t* lds4;
        const int k = 16 * g + 8 * h + ((lane & 15) >> 2);
        const int chunk = row0 / 8 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        const uint32_t b = lds_address(lds);
        const uint32_t a0 = b + S::lds_at(k, chunk) + (lane & 1) * 8, a1 = b + S::lds_at(k + 4, chunk) + (lane & 1) * 8;
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

// The tile loop: the slices of k0 .. k1 - 1 (elements of k) of the operands that sa and sb
// stage, summed into acc.  seen(i, fragment) for every A fragment.
//
// A wave reads the next k-group's fragments while it multiplies the last read one's, also
// from one slice to the next: before a slice's last group every wave has read all of it
// (one barrier a slice), so its buffer is free and the next one's is in place.  DIRECT:
// slices come straight into LDS; else through registers.  rot: the slice that comes first.
template <typename S, int AK, int BK_, bool DIRECT, typename SA, typename SB, typename F>
__device__ __forceinline__ void tile_loop(f32x16_t (&acc)[S::TM][S::TN], const SA& sa, const SB& sb, const Operand& oa,
                                          const Operand& ob, const Slots& s, int k0, int k1, char (*lds)[S::BYTES], int row0,
                                          int col0, int lane, F&& seen, int rot = 0) {
    typedef typename S::T T;
    constexpr int NST = S::NST;
    uint4 fa[2][S::TM], fb[2][S::TN];
    auto read = [&](int to, const char* a, int g) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::TM; ++i) fragment<T, AK, S::BM, S::TH, S::KB>(fa[to][i], a, row0 + 32 * i, g, lane);
#pragma unroll
        for (int j = 0; j < S::TN; ++j) fragment<T, BK_, S::BN, S::TH, S::KB>(fb[to][j], a + S::ABYTES, col0 + 32 * j, g, lane);
    };
    auto multiply_group = [&](int from) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::TM; ++i) {
            seen(i, fa[from][i]);
#pragma unroll
            for (int j = 0; j < S::TN; ++j) multiply<T>(acc[i][j], fa[from][i], fb[from][j]);
        }
    };
    const uint32_t base = lds_address(lds[0]);
    const bool whole = sa.whole && sb.whole;
    const int n = (k1 - k0 + S::BK - 1) / S::BK;       // steps
    // slice by slice from the rot-th on, then the first ones
    auto slice_k = [&](int step) __attribute__((always_inline)) {
        const int t = step + rot;
        return k0 + (t >= n ? t - n : t) * S::BK;
    };
    auto all_there = [&](int step) __attribute__((always_inline)) { return whole && slice_k(step) + S::BK <= k1; };
    auto fetch = [&](int step, int buf) __attribute__((always_inline)) {
        const uint32_t to = base + buf * S::BYTES;
        const int k = slice_k(step);
        if (all_there(step)) {
            sa.template fetch<true>(oa, s, k, lds[buf], to);
            sb.template fetch<true>(ob, s, k, lds[buf] + S::ABYTES, to + S::ABYTES);
        } else {
            sa.template fetch<false>(oa, s, k, lds[buf], to);
            sb.template fetch<false>(ob, s, k, lds[buf] + S::ABYTES, to + S::ABYTES);
        }
    };
    uint4 va[SA::U], vb[SB::U];
    auto load = [&](int step) __attribute__((always_inline)) {
        const int k = slice_k(step);
        sa.load(va, oa, s, k);
        sb.load(vb, ob, s, k);
    };
    auto store = [&](int buf) __attribute__((always_inline)) {
        sa.store(va, lds[buf]);
        sb.store(vb, lds[buf] + S::ABYTES);
    };
    // Slice `step` is there: of the direct loads only those of the slice after it may be on
    // their way (as many as chunks, where all of its are there; three slices).
    auto wait_for = [&](int step) __attribute__((always_inline)) {
        if constexpr (NST == 3) {
            if (step + 1 < n && all_there(step + 1)) {
                asm volatile("s_waitcnt vmcnt(%0)" :: "n"(SA::U + SB::U) : "memory");
                return;
            }
        }
        wait_direct();
    };
    if constexpr (DIRECT) {
        fetch(0, 0);
        if (NST == 3 && 1 < n) fetch(1, 1);
        wait_for(0);
    } else {
        load(0);
        store(0);
        if (1 < n) load(1);
    }
    __syncthreads();
    if (DIRECT && NST > 1 && NST - 1 < n) fetch(NST - 1, NST - 1);
    read(0, lds[0], 0);
    for (int step = 0, buf = 0; step < n; ++step) {
        const int next = NST == 1 ? 0 : buf + 1 == NST ? 0 : buf + 1;
        const bool more = step + 1 < n;
        // The slice's first fragments were read before the last products and are there: said so here,
        // else the compiler, which does not follow them round the loop, waits for the next ones too
        __builtin_amdgcn_s_waitcnt(0xc07f);     // lgkmcnt(0)
        if (!DIRECT && NST > 1 && more) {
            store(next);
            if (step + 2 < n) load(step + 2);
        }
        static_for<0, S::GROUPS>([&](auto gc) __attribute__((always_inline)) {
            constexpr int g = decltype(gc)::value;
            if constexpr (g + 1 < S::GROUPS) {
                read((g + 1) & 1, lds[buf], g + 1);
            } else if (NST > 1 && more) {
                if (DIRECT) wait_for(step + 1);
                __syncthreads();
                if (DIRECT && step + NST < n) fetch(step + NST, buf);
                read(0, lds[next], 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply_group(g & 1);
            __builtin_amdgcn_sched_barrier(0);
        });
        buf = next;
    }
}

}  // namespace dc
