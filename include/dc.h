/*
 * dc.h -- one GPU's share of a spatially decomposed 2-D convolution layer on
 * AMD MI355X (gfx950): forward, backward-data and backward-filter on an NCHW
 * sub-domain tile, and the halo pack/unpack that borders the tile.
 *
 * Method: Dryden et al., "Improving Strong-Scaling of CNN Training by
 * Exploiting Finer-Grained Parallelism" (IPDPS 2019, arXiv 1903.06681).
 *   - the layer and its six tensors: Sec. II-A; Eqs. (1) forward, (2) weight
 *     gradient, (3) input gradient;
 *   - blocked spatial (+ sample) distribution, the halo set and the local
 *     passes on a tile: Sec. III-A;
 *   - halo message terms (north/south, east/west, four corners): Sec. V-A.
 *
 * Notation map (paper -> this interface): N -> N (this GPU's samples),
 * C -> C, F (filters) -> K, filter K x K -> R x S, stride S -> stride,
 * padding P -> pad, O = floor(K/2) (halo width) -> halo.  The paper's blocked
 * distributions of H and W are the P x Q grid below; C and F are replicated.
 *
 * Everything is C ABI, never throws, allocates and frees nothing, keeps no
 * state and is reentrant.  All device pointers are caller-owned.  Work is
 * enqueued on `stream` (a hipStream_t; NULL = the null stream) and the calls
 * return without synchronising.
 */
#ifndef DC_H
#define DC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DC_OK              =  0,
    DC_ERR_NULL        = -1,  /* a required pointer is NULL */
    DC_ERR_SHAPE       = -2,  /* a size is non-positive, or sizes are inconsistent */
    DC_ERR_DTYPE       = -3,  /* dtype is not DC_F32 / DC_BF16 */
    DC_ERR_HALO        = -4,  /* halo narrower than the pass needs, or wider than a tile */
    DC_ERR_UNSUPPORTED = -5,  /* uneven tiles, or a decomposed output grid not aligned with the input grid */
    DC_ERR_WORKSPACE   = -6,  /* workspace NULL or smaller than dc_bwd_filter_workspace_bytes() */
    DC_ERR_ALIGN       = -7,  /* a device pointer is not 16-byte aligned */
    DC_ERR_HIP         = -8,  /* the HIP runtime reported an error at launch */
    DC_ERR_TILE        = -9,  /* tile index out of range */
    DC_ERR_ARG         = -10, /* other invalid argument (which, accumulate) */
    DC_ERR_TOO_LARGE   = -11  /* a tensor exceeds the 32-bit element indexing of the kernels */
} dc_status;

typedef enum { DC_F32 = 0, DC_BF16 = 1 } dc_dtype;   /* dtype of x, w and dy; y, dx, dw are fp32 */
typedef enum { DC_X = 0, DC_DY = 1 } dc_which;       /* which tensor a tile/halo call refers to */

#define DC_ALL_TILES (-1)   /* every tile of the grid in one launch (single-device emulation) */

/*
 * The layer and its decomposition (Sec. II-A, Sec. III-A).
 *
 * H, W are the GLOBAL input extents.  The grid splits them into P x Q
 * blocked tiles of Ht = H/P by Wt = W/Q input pixels (the paper's blocked
 * distributions of H and W).  The global output is Ho x Wo with
 * Ho = (H + 2*pad - R)/stride + 1; a tile owns Hot = Ho/P by Wot = Wo/Q of it.
 * With P = Q = 1 any geometry with Ho, Wo >= 1 is accepted; with more than one
 * tile the output grid must line up with the input grid, Ho * stride = H and
 * Wo * stride = W (stride 1: "same" output), and Ho % P = Wo % Q = 0, so that
 * a tile owns exactly the outputs whose taps start in its input block.  At
 * stride > 1 a tile may need no halo on one side (e.g. 3x3 stride 2 pad 1: x
 * 1 below, 0 above): the layout keeps the margin h on every side, and the
 * halo calls move only the band each side needs (dc_halo_bands).
 *
 * halo is the margin width h kept on every side of every tile (for both the x
 * and the dy tile).  It must be at least what each pass reads beyond the tile
 * (see dc_required_halo) and, with more than one tile along an axis, at most
 * the input and the output tile extent along it (halos come from the
 * adjacent tile only).
 */
typedef struct {
    int32_t N, C, K;       /* samples on this GPU, input channels, filters */
    int32_t H, W;          /* global input height, width */
    int32_t R, S;          /* filter height, width */
    int32_t stride, pad;   /* same in both spatial dimensions */
    int32_t P, Q;          /* spatial grid: P tiles along H, Q along W */
    int32_t halo;          /* margin width h on every side of a tile */
    int32_t dtype;         /* dc_dtype */
} dc_problem;

/*
 * Tile layouts (all dense, row-major, element type = dtype unless stated):
 *   x_pad  [N][C][Ht+2h][pitch_x]     interior (owned block) at row h, col h
 *   dy_pad [N][K][Hot+2h][pitch_dy]   interior at row h, col h
 *   w      [K][C][R][S]               replicated on every tile (Sec. III-A)
 *   y      [N][K][Hot][Wot]   fp32
 *   dx     [N][C][Ht][Wt]     fp32
 *   dw     [K][C][R][S]       fp32
 * pitch = dc_tile_pitch(): at least width+2h, rounded up to 16 bytes.  Pitch
 * columns beyond width+2h are never written; kernels may read them (as part
 * of an aligned 16-byte access), and their values never reach a result.
 *
 * Tiles are numbered tile = ti*Q + tj, ti = 0..P-1 top to bottom, tj = 0..Q-1
 * left to right.  With tile = DC_ALL_TILES every per-tile buffer argument
 * (tile, send/recv, y, dx) is an array of P*Q consecutive per-tile buffers in
 * tile order, and one launch serves the whole grid.
 *
 * Halo bands (Sec. III-A).  A tile's margin ring is supplied by its eight
 * neighbours; the band from each side is as wide as the passes read on that
 * side (dc_halo_bands: rows above bN, below bS, columns left bW, right bE;
 * all equal to h for the usual stride-1 "same" layers).  Margin cells outside
 * the bands, and bands whose neighbour does not exist, hold zeros after
 * unpack: the convolution's zero padding.
 *
 * Packed halo buffers (send/recv) hold eight regions, in the order
 * N, S, W, E, NW, NE, SW, SE, each laid out [N][channels][rows][cols].
 * Region d of a RECV buffer holds the band of margin d: N bN x Wt, S bS x Wt,
 * W Ht x bW, E Ht x bE, NW bN x bW, NE bN x bE, SW bS x bW, SE bS x bE
 * (output-tile extents Hot, Wot for dy).  Region d of a SEND buffer holds the
 * band of the owned block that the neighbour in direction d receives, i.e.
 * the shape of that neighbour's margin opposite to d (S for d = N, ...).
 * Regions follow each other without gaps; the two layouts have the same
 * total.  dc_halo_elems() is that total rounded up to a multiple of 16 bytes
 * (the padding at the end is never written), so the consecutive buffers of an
 * all-tiles call each start 16-byte aligned.
 */

/* band classes of the margin ring, for dc_halo_pack_bands / dc_halo_unpack_bands */
#define DC_BAND_NS      1   /* rows above and below the owned block (regions N, S) */
#define DC_BAND_WE      2   /* columns left and right of it (regions W, E) */
#define DC_BAND_CORNERS 4   /* the four corner blocks (regions NW, NE, SW, SE) */
#define DC_BAND_ALL     7

/* ---- the five operations ---- */

/*
 * Arithmetic.  Products of bf16 inputs are exact, those of fp32 inputs exact or,
 * in layers that run on the bf16 matrix instruction with each value split in
 * three bf16 parts, within 2^-24 of a product; sums are fp32 in a fixed order.
 * Infinities, NaN and values at the ends of fp32's range are taken whole: outputs
 * that read them are formed with the fp32 instruction, no others are.
 */

/*
 * Forward propagation on one tile, Eq. (1) (Sec. II-A) restricted to the
 * tile's samples and output pixels (Sec. III-A):
 *   y[n,k,p,q] = sum_{c,r,s} x[n,c, p*stride-pad+r, q*stride-pad+s] * w[k,c,r,s]
 * reading x from x_pad, halo included.  Cross-correlation, no bias, fp32
 * accumulation.  Writes all of y; reads only what the sum touches.
 */
dc_status dc_conv_fwd(const dc_problem* prob, int32_t tile, const void* x_pad,
                      const void* w, float* y, void* stream);

/*
 * Input gradient on one tile, Eq. (3) (Sec. II-A; Sec. III-A):
 *   dx[n,c,i,j] = sum_{k,r,s} dy[n,k,(i+pad-r)/stride,(j+pad-s)/stride] * w[k,c,r,s]
 * (terms exist where both divisions are exact), reading dy from dy_pad, halo
 * included.  Writes all of dx.
 */
dc_status dc_conv_bwd_data(const dc_problem* prob, int32_t tile, const void* dy_pad,
                           const void* w, float* dx, void* stream);

/*
 * Local weight gradient of one tile, Eq. (2) restricted to the tile's samples
 * and output pixels (Sec. III-A):
 *   dw[k,c,r,s] (=|+=) sum_{n,p,q in tile} dy[n,k,p,q] * x[n,c,p*stride-pad+r,q*stride-pad+s]
 * reading x from x_pad (halo included) and only the interior of dy_pad: the
 * dy halo is not needed (Sec. III-A), so this pass may overlap the dy halo
 * exchange.  accumulate = 0 overwrites dw, 1 adds the partial to dw.
 * With tile = DC_ALL_TILES, dw receives the sum over all tiles in row-major
 * tile order: the single-device stand-in for the allreduce that completes dw.
 * workspace: device scratch of at least dc_bwd_filter_workspace_bytes(prob,
 * tile) bytes, contents undefined on entry and exit.  Results are
 * deterministic: a fixed summation order, no atomics.
 */
dc_status dc_conv_bwd_filter(const dc_problem* prob, int32_t tile, const void* x_pad,
                             const void* dy_pad, float* dw, int32_t accumulate,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * Allocation-free weight gradient, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid allocation).  Same operation, arguments, kernels and results as
 * dc_conv_bwd_filter, without a workspace argument: the chunk partials live
 * in a fixed device array of DC_BWD_FILTER_NOALLOC_MAX_BYTES that the library
 * holds on every GPU it runs on until the process ends (its address is looked
 * up on the first call on a device).  Returns DC_ERR_WORKSPACE, launching
 * nothing, when dc_bwd_filter_workspace_bytes(prob, tile) exceeds that size.
 * Calls no hipMalloc, hipFree or allocating routine.  Every call on one GPU
 * shares that GPU's array: calls that overlap on one GPU (two streams, two
 * host threads) race and must be serialised by the caller.
 */
#define DC_BWD_FILTER_NOALLOC_MAX_BYTES ((size_t)64 << 20)
dc_status dc_conv_bwd_filter_noalloc(const dc_problem* prob, int32_t tile, const void* x_pad,
                                     const void* dy_pad, float* dw, int32_t accumulate,
                                     void* stream);

/*
 * Halo pack (Sec. III-A; message terms of Sec. V-A): copy the bands of the
 * owned block of t_pad (which = DC_X: an x tile; DC_DY: a dy tile) that each
 * existing neighbour needs into the send buffer.  Reads only the owned block
 * (and pitch columns, see above); writes only regions whose neighbour
 * exists.  Bitwise copy.  When dc_halo_elems is 0 (every band empty: a
 * margin no pass reads, e.g. a 1x1 filter) send may be NULL and nothing is
 * launched; for dc_halo_unpack recv may then be NULL, and the call only
 * zero-fills the margin ring.
 */
dc_status dc_halo_pack(const dc_problem* prob, int32_t tile, int32_t which,
                       const void* t_pad, void* send, void* stream);

/*
 * Halo unpack (Sec. III-A): write the whole h-wide margin ring of t_pad.  The
 * band of margin d receives region d of recv when the neighbour in direction
 * d exists; every other margin cell becomes zero (the convolution's zero
 * padding, Sec. II-A, and margin beyond the band widths).  Writes only
 * margins, never the owned block.  With tile = DC_ALL_TILES, recv is the
 * array of all tiles' SEND buffers and each margin is read directly from the
 * neighbour's opposite region: that read is the emulated exchange.
 */
dc_status dc_halo_unpack(const dc_problem* prob, int32_t tile, int32_t which,
                         const void* recv, void* t_pad, void* stream);

/*
 * dc_halo_pack / dc_halo_unpack restricted to some band classes (bands: an OR
 * of DC_BAND_*; DC_BAND_ALL is the full call): pack writes only the regions of
 * those classes, unpack writes only the margin cells of those classes.  Lets
 * a caller move the contiguous N/S rows and the strided W/E columns at
 * different times (or time them apart).  DC_ERR_ARG for an empty or unknown
 * mask.
 */
dc_status dc_halo_pack_bands(const dc_problem* prob, int32_t tile, int32_t which, int32_t bands,
                             const void* t_pad, void* send, void* stream);
dc_status dc_halo_unpack_bands(const dc_problem* prob, int32_t tile, int32_t which, int32_t bands,
                               const void* recv, void* t_pad, void* stream);

/*
 * Interior / boundary split of the forward and input-gradient passes, so that
 * the halo exchange can overlap computation (Sec. IV-A; stride 1 only, else
 * DC_ERR_UNSUPPORTED).  The boundary of the output tile is the frame of
 * outputs whose sum reads a margin: for dc_conv_fwd_region the rows above /
 * below and columns left / right of widths dc_halo_bands(DC_X); for
 * dc_conv_bwd_data_region those of dc_halo_bands(DC_DY).
 *   DC_REGION_ALL:      the plain call.
 *   DC_REGION_INTERIOR: every output outside the frame is final; the frame is
 *                       left unspecified.  It may run while the margins are
 *                       being written (e.g. by dc_halo_unpack on another
 *                       stream): margin values reach frame outputs only.
 *   DC_REGION_BOUNDARY: computes the frame only (the margins must be in
 *                       place); every other output is left untouched.
 * INTERIOR followed by BOUNDARY gives the plain call's result.
 */
typedef enum { DC_REGION_ALL = 0, DC_REGION_INTERIOR = 1, DC_REGION_BOUNDARY = 2 } dc_region;
dc_status dc_conv_fwd_region(const dc_problem* prob, int32_t tile, int32_t region, const void* x_pad,
                             const void* w, float* y, void* stream);
dc_status dc_conv_bwd_data_region(const dc_problem* prob, int32_t tile, int32_t region,
                                  const void* dy_pad, const void* w, float* dx, void* stream);

/* ---- host-only helpers (no GPU needed) ---- */

/* Check a problem and tile index (DC_ALL_TILES allowed); no launch. */
dc_status dc_validate(const dc_problem* prob, int32_t tile);

/* Row pitch (elements) of the padded x or dy tile; -1 on an invalid problem. */
int64_t dc_tile_pitch(const dc_problem* prob, int32_t which);

/* Elements of one padded x or dy tile ([N][ch][rows+2h][pitch]); -1 if invalid. */
int64_t dc_tile_elems(const dc_problem* prob, int32_t which);

/* Elements of one tile's packed halo buffer for x or dy (16-byte multiple); -1 if invalid. */
int64_t dc_halo_elems(const dc_problem* prob, int32_t which);

/* Workspace bytes dc_conv_bwd_filter needs for this tile argument (0 if none). */
size_t dc_bwd_filter_workspace_bytes(const dc_problem* prob, int32_t tile);

/*
 * Margins each pass reads beyond a tile, independent of the halo field:
 * which = DC_X: rows/cols of x the forward pass (and weight gradient) reads
 * before (lohi[0]) and after (lohi[1]) the tile; which = DC_DY: the same for
 * the dy rows the input gradient reads.  Same in both spatial dimensions.
 */
dc_status dc_required_halo(const dc_problem* prob, int32_t which, int32_t lohi[2]);

/*
 * Band widths the halo calls move for x (which = DC_X) or dy (DC_DY):
 * bw = {rows above, rows below, columns left, columns right} of a tile, the
 * margins the passes read (x: forward and weight gradient, Eq. (1)/(2);
 * dy: input gradient, Eq. (3)).  Each is at most the problem's halo.
 */
dc_status dc_halo_bands(const dc_problem* prob, int32_t which, int32_t bw[4]);

/* Tile extents: dims = {Ht, Wt, Hot, Wot}. */
dc_status dc_tile_dims(const dc_problem* prob, int32_t dims[4]);

/* Static string for a status code. */
const char* dc_status_string(int32_t status);

/* ---- between two convolutions: norm, pointwise products, 8-bit checkpoints ---- */

/*
 * What a network applies between two convolutions of a decomposed layer
 * (Sec. III-A: these operations need no halo and no other tile): layer norm over
 * the channels of each pixel, products over the channels (1x1 layers, the
 * matrices of a feed-forward block) with bias, activation and residual in the
 * epilogue, and activations kept for the backward pass in 8 bits.  They read and
 * write tiles where they lie: the fp32 output of a convolution, the interior of
 * a padded tile, rows of channels.
 *
 * A view describes a tensor [N][C][H][W] in memory: element strides of samples,
 * channels and rows; columns are contiguous.  H = W = 1 with sc = 1 is a matrix
 * of N rows of C channels, W = 1 with sc = 1 and sh = C one of N H rows.  A
 * pointer goes with every view: 16-byte aligned for fp32 gamma, beta, bias,
 * weights, gradients, statistics, checkpoints and workspaces; aligned to its
 * element for a view (an interior starts anywhere).  What lies in memory between
 * the first and the last element of a view (margins, the gap after a row) may be
 * read with it; those values never reach a result.  Strides of tensors that are read may be 0
 * (broadcast); those of tensors that are written must not make elements overlap
 * (DC_ERR_SHAPE).  Outputs must not overlap inputs, except where said.
 * Offsets are 64-bit.  Sizes (DC_ERR_TOO_LARGE past them): N H W up to 2^31 - 2^16, for
 * products with every row of a tile that is not contiguous rounded up to 16 bytes; C up
 * to 2^20; for products K C below 2^31 and at most 2^22 blocks of 128 channels (of the
 * wider side) by 128 pixels.
 */
#define DC_Q8 2   /* view dtype: a checkpoint in 8 bits (layout below, strides ignored) */
typedef struct {
    int32_t N, C, H, W;
    int64_t sn, sc, sh;    /* element strides: sample, channel, row */
    int32_t dtype;         /* DC_F32, DC_BF16 or DC_Q8 */
} dc_view;

/*
 * max(z, 0), z Phi(z) with the normal distribution's Phi, z / (1 + e^-z).  +infinity
 * stays and NaN stays; at -infinity relu is 0, the other two NaN (-infinity times 0).
 * Formed in fp32: gelu within 1.6e-7 |z| for results in fp32, 3e-7 |z| before the
 * rounding for results in bf16; silu within 4e-7 + 8e-8 |z| of its value.
 */
typedef enum { DC_ACT_NONE = 0, DC_ACT_RELU = 1, DC_ACT_GELU = 2, DC_ACT_SILU = 3 } dc_activation;

/*
 * The 8-bit form of a tensor: the 32 channels 32k .. 32k+31 of a pixel are a
 * block and share a scale byte s, the biased fp32 exponent of their largest
 * magnitude, at least 7.  A value is q * 2^(s-133), q the nearest integer (ties
 * to even) within -127 .. 127: the error is at most 2^-7 of the block's power of
 * two (2^-6 at its very top), and every value is exact in bf16.  A block with an
 * infinity or NaN has s = 255 and stands for NaN throughout.
 * Layout: q [N][ceil(C/32)][H W][32] int8, then s [N][ceil(C/32)][H W]; channels
 * past C hold q = 0.  dc_ckpt_bytes() is the total, a multiple of 16; -1 for an
 * invalid view.
 */
int64_t dc_ckpt_bytes(const dc_view* vq);

/* x (fp32 or bf16) -> its 8-bit form q (dc_ckpt_bytes of the same N, C, H, W). */
dc_status dc_ckpt_save(const dc_view* vx, const void* x, void* q, void* stream);

/* y = act(what q stands for), y fp32 or bf16. */
dc_status dc_ckpt_load(const dc_view* vq, const void* q, int32_t act, const dc_view* vy, void* y,
                       void* stream);

/*
 * Layer norm of each pixel over its C channels, in fp32 with the variance from
 * centred values:  u = gamma (x - mu) r + beta,  mu = mean x,  r = (var x +
 * eps)^-1/2.  gamma and beta are fp32 [C]; either may be NULL (1 and 0).
 * stat [2][N][H][W] (mu, then r) and ckpt (x in 8 bits) are written unless NULL;
 * the backward pass reads stat, and x or its checkpoint.  u may be x itself
 * (same view and type).
 */
dc_status dc_norm_fwd(const dc_view* vx, const void* x, const float* gamma, const float* beta, float eps,
                      const dc_view* vu, void* u, float* stat, void* ckpt, void* stream);

/*
 * Its backward pass: with xh = (x - mu) r and g = gamma du,
 *   dx = r (g - mean g - xh mean(g xh)) [+ res],
 *   dgamma (=|+=) sum over pixels of du xh,  dbeta (=|+=) sum over pixels of du.
 * x is the forward's input, or its checkpoint where vx->dtype is DC_Q8; stat is
 * what the forward wrote.  res (a skip path's gradient), u (gamma xh + beta once
 * more, for a weight gradient that reads it), dgamma and dbeta may be NULL; beta
 * is read for u only.  dx may be du or res (same view and type).  accumulate = 0
 * overwrites dgamma and dbeta, 1 adds to them.  workspace: device scratch of at
 * least dc_norm_bwd_workspace_bytes(vdu) bytes.  The summation order is fixed.
 */
dc_status dc_norm_bwd(const dc_view* vdu, const void* du, const dc_view* vx, const void* x, const float* stat,
                      const float* gamma, const float* beta, const dc_view* vres, const void* res,
                      const dc_view* vu, void* u, const dc_view* vdx, void* dx, float* dgamma, float* dbeta,
                      int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream);
size_t dc_norm_bwd_workspace_bytes(const dc_view* vdu);

/*
 * Product over the channels of every pixel:  z = W x + bias,  y = act(z) + res.
 * w is [K][C] with K = vy->C and C = vx->C, of x's type; bias fp32 [K] or NULL;
 * res (fp32 or bf16) or NULL; z is written too unless NULL, whole (fp32, bf16) or
 * in 8 bits (vz->dtype DC_Q8), for dc_linear_bwd_data.  y is fp32 or bf16 and may
 * be res (same view and type).  bf16 products are exact, fp32 ones fp32; sums are
 * fp32 in a fixed order.
 */
dc_status dc_linear_fwd(const dc_view* vx, const void* x, const void* w, const float* bias, int32_t act,
                        const dc_view* vres, const void* res, const dc_view* vz, void* z,
                        const dc_view* vy, void* y, void* stream);

/*
 * Gradient at what an activation read, from the gradient dy of the product after
 * it:  dx = (W^T dy) act'(z),  w [K][C] of dy's type, K = vdy->C, C = vdx->C.  z
 * (whole or DC_Q8) is read unless act is DC_ACT_NONE, where dx is the plain input
 * gradient and vz, z, vh and h are NULL.  h = act(z) is written unless NULL: the
 * product's input again, for its weight gradient.
 */
dc_status dc_linear_bwd_data(const dc_view* vdy, const void* dy, const void* w, int32_t act,
                             const dc_view* vz, const void* z, const dc_view* vh, void* h,
                             const dc_view* vdx, void* dx, void* stream);

/*
 * Weight and bias gradient of a product:  dw[k][c] (=|+=) sum over pixels of
 * dy[k] x[c],  db[k] (=|+=) sum over pixels of dy[k];  db may be NULL.  x and dy
 * are of one type.  workspace: at least dc_linear_bwd_filter_workspace_bytes()
 * bytes (0: none).  The summation order is fixed.
 */
dc_status dc_linear_bwd_filter(const dc_view* vx, const void* x, const dc_view* vdy, const void* dy,
                               float* dw, float* db, int32_t accumulate, void* workspace,
                               size_t workspace_bytes, void* stream);
size_t dc_linear_bwd_filter_workspace_bytes(const dc_view* vx, const dc_view* vdy);

/* ---- a gated residual block: the gated product, the join, dropout ---- */

/*
 * What such a block adds to the calls above:
 *
 *   u -> dc_gate_fwd -> h -> dc_linear_fwd -> y,   dc_join_fwd(y, x) -> o, and the next block's u
 *
 * and back: dc_join_bwd, then dc_gate_bwd_data through the second product, whose result is
 * what dc_linear_bwd_data (act DC_ACT_NONE) and dc_linear_bwd_filter take for the first.
 * Views, alignment, sizes and numbers as above; a view with H tokens of N sequences in rows
 * of channels is W = 1, sc = 1, sh = C, sn = H C.
 */

/*
 * Dropout whose mask is never stored: forward and backward passes form it again from these
 * arguments, and the tiles of a decomposed image draw the mask of the whole one.
 *
 * A value is dropped with a chance of t / 65536, t the integer nearest 65536 p (ties to
 * even, 65535 at most), and multiplied by 65536 / (65536 - t) if it stays; what is dropped is
 * 0, whatever stood there.  0 <= p < 1.  Channels 8k .. 8k+7 of a pixel share the four words
 * w0 .. w3 of Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, SC 2011) for the key
 * `seed` and the counter whose lower 64 bits are the position
 *   ((n ceil(C/8) + k) H + h) W + w       (sample n, row h, column w of the whole tensor)
 * and whose upper 64 bits are offset + *step modulo 2^64: of the 16 bits that channel j of
 * the eight takes, w[j/2]'s lower half for even j, its upper half for odd j, those below t
 * drop it.  An offset of its own for each use (layer and training step) gives each a mask of
 * its own.  step, in device memory (8-byte aligned) and read when the kernel runs, may be
 * NULL (0): a captured graph's replays draw new masks as the program counts it up.
 *
 * The tensor lies in the whole one with its first sample, row and column at n0, h0, w0; H and
 * W are the whole one's rows and columns, 0: as far as the tensor reaches.  P x Q (0: 1): the
 * tensor holds the tiles of such a grid as consecutive samples, tile by tile, N / (P Q) of
 * each, as DC_ALL_TILES tensors do; tile (p, q) starts at row h0 + p (view's H), column w0 +
 * q (view's W).  Positions stay below 2^63 (DC_ERR_TOO_LARGE).
 */
typedef struct {
    double p;
    uint64_t seed, offset;
    const uint64_t* step;
    int32_t n0, h0, w0, H, W, P, Q;
} dc_drop;

/* y = x dropped out; with dy for x, its gradient.  y may be x (same view and type). */
dc_status dc_dropout(const dc_drop* drop, const dc_view* vx, const void* x, const dc_view* vy, void* y, void* stream);

/*
 * Gated product over the channels of every pixel:
 *   zg = Wg x + bg,  zu = Wu x + bu,  h = drop(act(zg) zu).
 * w is [2K][C], Wg then Wu, of x's type; bias fp32 [2K], bg then bu, or NULL; drop NULL: none.
 * zg and zu are written too unless both are NULL, for dc_gate_bwd_data: two tensors of one
 * view (K channels), whole (fp32, bf16) or in 8 bits (DC_Q8).  K = vh->C; h is fp32 or bf16.
 * Numbers are dc_linear_fwd's: the act DC_ACT_NONE takes zg itself.  As there, the order of a sum is the
 * same for every pixel of a call.
 */
dc_status dc_gate_fwd(const dc_view* vx, const void* x, const void* w, const float* bias, int32_t act, const dc_drop* drop,
                      const dc_view* vz, void* zg, void* zu, const dc_view* vh, void* h, void* stream);

/*
 * Gradient at its two sums from the gradient dy of the product after it:
 *   dh = drop(W2^T dy),  dz = (dh zu act'(zg), then dh act(zg)),
 * w is W2, [vdy->C][K] of dy's type, K = vz->C; dz has 2K channels, so that the first
 * product's gradients are dc_linear_bwd_data's and dc_linear_bwd_filter's of w as a [2K][C]
 * matrix.  h, drop(act(zg) zu) once more from what was kept, is written unless NULL.  As 2K channels
 * are a view's, K is up to 2^19 here (forward 2^20, with 2 K C below 2^31).
 */
dc_status dc_gate_bwd_data(const dc_view* vdy, const void* dy, const void* w, int32_t act, const dc_drop* drop,
                           const dc_view* vz, const void* zg, const void* zu, const dc_view* vh, void* h,
                           const dc_view* vdz, void* dz, void* stream);

/*
 * A norm of a pixel x over its channels, in fp32: layer, (x - mean) r with r = (mean (x -
 * mean)^2 + eps)^-1/2, or root mean square, x r with r = (mean x^2 + eps)^-1/2; times gamma,
 * plus beta (fp32 [C] or NULL: 1 and 0).
 */
typedef enum { DC_NORM_NONE = 0, DC_NORM_LAYER = 1, DC_NORM_RMS = 2 } dc_norm_kind;
typedef struct {
    int32_t kind;
    float eps;
    const float *gamma, *beta;
} dc_norm;

/*
 * Join of a block's branch y with the residual stream x:
 *   o = x + scale gate drop(post(y)),  u = pre(o).
 * post is the norm after the block, pre the one before the next block; NULL or DC_NORM_NONE:
 * none (then u is NULL).  scale is fp32 [C], gate fp32 [N][C], one factor a sample and channel;
 * either may be NULL (1).  x may be NULL (0).  u is formed from o before o's rounding.  stat
 * [4][N][H][W] (mean and r of y, then of o; a mean of 0 for root mean square; untouched where
 * there is no norm) is written unless NULL, and so is ckpt, o in 8 bits.  o may be x, u may
 * be y (same view and type).
 */
dc_status dc_join_fwd(const dc_view* vy, const void* y, const dc_norm* post, const float* scale, const float* gate,
                      const dc_drop* drop, const dc_view* vx, const void* x, const dc_norm* pre, const dc_view* vo, void* o,
                      const dc_view* vu, void* u, float* stat, void* ckpt, void* stream);

/*
 * Its backward pass from du and d_o, the gradients at u and at o from elsewhere (either may be
 * NULL, not both; without du the call goes as far as o, and pre, vx, x, vo, o are not looked at):
 *   dO = d_o + (gradient of pre at o),  dx = dO,  dy = (gradient of post at y) of dO scale gate drop.
 * With du, o is formed once more from y and x (NULL: 0), as the forward pass formed it; or, unless
 * o is NULL, read as it was stored, in its type's precision, and x is not looked at.  y is needed
 * where o is formed, where there is a post norm and where a gradient of scale or gate is wanted, else
 * it may be NULL.  y, x and o may be in 8 bits (DC_Q8).  stat is what the forward pass wrote.  dx
 * may be NULL.  grads (NULL: none): fp32, [C] each and [N][C] for gate; NULL where not wanted, and for
 * a gate, a pre or a post norm that the call does not have (DC_ERR_ARG); scale, gamma and beta that
 * are NULL, 1 or 0, have a gradient all the same.  accumulate = 0 overwrites them, 1 adds to them.
 * dx may be d_o, dy may be y or du (same view and type); nothing else overlaps.  workspace: at least
 * dc_join_bwd_workspace_bytes(vdy, whether there is a gate) bytes, if there are grads.  The
 * summation order is fixed.
 */
typedef struct {
    float *scale, *gate, *gamma_post, *beta_post, *gamma_pre, *beta_pre;
} dc_join_grads;
dc_status dc_join_bwd(const dc_view* vdu, const void* du, const dc_view* vdo, const void* d_o, const dc_view* vy, const void* y,
                      const dc_view* vx, const void* x, const dc_view* vo, const void* o, const float* stat,
                      const dc_norm* post, const float* scale,
                      const float* gate, const dc_drop* drop, const dc_norm* pre, const dc_view* vdx, void* dx,
                      const dc_view* vdy, void* dy, const dc_join_grads* grads, int32_t accumulate, void* workspace,
                      size_t workspace_bytes, void* stream);
size_t dc_join_bwd_workspace_bytes(const dc_view* vdy, int32_t gate);

#ifdef __cplusplus
}
#endif

#endif /* DC_H */
