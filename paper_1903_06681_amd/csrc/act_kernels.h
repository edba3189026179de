// Arguments and launchers of the kernels between two convolutions.
#pragma once

#include "act.h"

namespace dc {

struct CkptArgs {
    View x;            // saved from, or loaded to
    char* q;
    Q8Map qm;
    Pixels px;
    int32_t C, act, cl;
};
hipError_t launch_ckpt(const CkptArgs& a, bool save, hipStream_t s);

struct NormArgs {
    View x, u;                 // forward: in and out; backward: x or its checkpoint, and u again (or absent)
    View du, res, dx;          // backward
    char* q;                   // checkpoint written (forward) or read (backward); null: none
    Q8Map qm;
    Pixels px;
    const float *gamma, *beta; // null: 1 and 0
    float* stat;               // null (forward only): not kept
    float *dgamma, *dbeta;     // null: not wanted
    float* part;               // workspace: [workgroup][2][32 blocks]
    float eps, invC;
    int32_t C, blocks;         // channels, blocks of 32
    int32_t lpx;               // pixels a wave spans (64, 16 or 4): 64 / lpx blocks side by side
    int32_t nw, pg;            // waves along the channels, pixel groups of a workgroup
    int32_t held;              // blocks a lane holds; 0: any number, read again for every pass
    int32_t groups, grid;      // pixel groups, workgroups
    int32_t accumulate, cl;
};
void norm_plan(NormArgs& a, bool backward);
size_t norm_bwd_part_bytes(int M, int C);
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s);

struct Slots {             // the pixels as the products number them (linear.h)
    int32_t chunks;        // chunks in all
    int32_t per;           // slots of a chunk: 16 / element size, or 1
    int32_t len, cpr;      // pixels and chunks of a row
    FastDiv dsample, dcpr; // chunks of a sample, of a row
};
struct Operand {
    const char* p;
    int64_t ld;            // weights: elements of a row
    int64_t sn, sc, sh;    // pixels: strides
    int64_t end;           // elements up to the last one, included
    int32_t rows, red;     // extents: rows (channels, pixels), k
};

struct LinearArgs {
    Operand a, b;          // weights, pixels
    Slots s;
    const float* bias;     // null: none
    View res, z, h, out;   // dt -1: absent
    Q8Map qm;
    int32_t rows;          // channels of the result
    int32_t act, cl;       // cl: rows of channels
    int32_t direct;        // operands on 16-byte boundaries
    int32_t tr, tc;        // blocks along rows and columns
};
hipError_t launch_linear_fwd(const LinearArgs& a, bool f32, hipStream_t s);
bool linear_few(const LinearArgs& a, bool bwd, bool f32);    // too few blocks of pixels: a kernel of its own
hipError_t launch_linear_few(const LinearArgs& a, bool bwd, bool f32, hipStream_t s);
hipError_t launch_linear_bwd(const LinearArgs& a, bool f32, hipStream_t s);

struct LinWgradArgs {
    Operand a, b;          // dy, x
    Slots s;
    float *dw, *db;        // db null: not wanted
    float* part;           // workspace: [share][K][C], then [share][K]
    int32_t K, C;
    int32_t tr, tc;        // blocks of the result
    int32_t shares, per;   // shares of the slices, slices of a share
    int32_t accumulate, cl;
    int32_t direct;        // operands on 16-byte boundaries, rows of whole chunks
};
void linear_wgrad_plan(LinWgradArgs& a, bool f32);
size_t linear_wgrad_part_bytes(const LinWgradArgs& a);
hipError_t launch_linear_wgrad(const LinWgradArgs& a, bool f32, hipStream_t s);

}  // namespace dc
