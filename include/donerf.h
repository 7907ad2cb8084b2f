/*
 * donerf.h - C ABI of the DONeRF per-ray inference library for MI355X (gfx950).
 *
 * The library renders camera images with DONeRF (Neff et al., "DONeRF: Towards
 * Real-Time Rendering of Compact Neural Radiance Fields using Depth Oracle
 * Networks", EGSR 2021).  For every pixel ray (Sec. 4, Eq. 1) it
 *   1. moves the ray origin onto the sphere around the view cell (Sec. 5.2),
 *   2. evaluates the depth-oracle network once on the encoded unified origin
 *      and direction (or on the paper's unencoded input: unified origin,
 *      direction and one position per class centre, Sec. 5.2), giving one
 *      score per logarithmic depth class (Sec. 5.1, Eq. 3 discretisation),
 *   3. keeps the N best-scoring classes and places one sample at the centre
 *      of each (Eq. 1 with the class centre as depth),
 *   4. warps each sample towards the view cell (Eq. 4-5) and encodes it,
 *   5. evaluates the shading network at the N samples, with the encoded ray
 *      direction fed again into its last layer (App. D), and
 *   6. alpha-composites the N samples front to back over a black background.
 * Both networks have 8 linear layers of 256 units with ReLU (App. D).
 *
 * Conventions
 *   - All functions return a donerf_status; 0 is success.
 *   - Every argument is validated before any HIP call, so invalid arguments
 *     are reported without touching the GPU.
 *   - Pointers documented as "host" are read during the call only; pointers
 *     documented as "device" must be device memory of the current HIP device
 *     and are accessed asynchronously on the handle's stream.
 *   - A handle is not reentrant: one render in flight per handle at a time.
 *   - The message of the most recent failure in the calling thread is kept in
 *     donerf_last_error().
 */
#ifndef DONERF_H
#define DONERF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct donerf_handle donerf_t;

typedef enum donerf_status {
    DONERF_OK = 0,
    DONERF_E_INVALID_ARG = -1, /* NULL pointer, size or enum out of range    */
    DONERF_E_SIZE = -2,        /* weight count does not match the config     */
    DONERF_E_NONFINITE = -3,   /* NaN or Inf in weights, poses or config     */
    DONERF_E_DEVICE = -4,      /* no HIP device, or the device is not gfx950 */
    DONERF_E_NOMEM = -5,       /* device or host allocation failed           */
    DONERF_E_HIP = -6,         /* a HIP call failed; see donerf_last_error() */
    DONERF_E_UNSUPPORTED = -7  /* valid request the library does not handle */
} donerf_status;

typedef enum donerf_precision {
    DONERF_FP32 = 0, /* fp32 weights, features and activations: each the sum
                        of three bf16 values, exact from 2^-110 on (below, to
                        2^-134), products from six bf16 MFMA products with fp32
                        accumulation.  Infinite activations act as in fp32; one
                        of 0x1.ffp127 or more (3.396e38) counts as infinite   */
    DONERF_BF16 = 1, /* bf16 weights, features and hidden activations (RNE),
                        fp32 accumulation, fp32 scores, heads, compositing;
                        sine, cosine, exp and reciprocal of the encoding and
                        compositing from the hardware instructions           */
    DONERF_FP8 = 2   /* the lower bit width Sec. 6.1 leaves as headroom: the
                        six hidden layers of each network in OCP E4M3 (weights
                        W 2^s rounded to nearest even with the largest s that
                        keeps max|W| 2^s <= 448, one s per layer; their inputs
                        clamped to [0, 448] after ReLU and rounded to E4M3);
                        the first layers and heads as in DONERF_BF16, fp32
                        accumulation throughout                               */
} donerf_precision;

typedef enum donerf_select {
    DONERF_SELECT_TOPN = 0,         /* one sample at the centre of each of the N
                                       highest-scoring classes; its width is
                                       the class width                          */
    DONERF_SELECT_TOPN_SOFTMAX = 1, /* the scores filtered by a softmax: the
                                       selection ranks the raw scores exactly
                                       as DONERF_SELECT_TOPN (the softmax is
                                       monotone; in fp32 it can also map
                                       distinct scores to equal values, so it
                                       is not ranked itself); the softmax only
                                       transforms the scores a debug render
                                       dumps                                   */
    DONERF_SELECT_CDF = 2           /* Sec. 5.1, Fig. 7: the class values
                                       sigmoid(score) as a piecewise-constant
                                       PDF over the classes (uniform in the
                                       coordinate of Eq. 3), its CDF inverted at
                                       u_i = (i + 0.5)/N; sample i's width is the
                                       depth extent of the slice [i/N, (i+1)/N].
                                       fp32 arithmetic                        */
} donerf_select;

typedef enum donerf_depth_input {
    DONERF_DEPTH_ENCODED = 0,  /* encode(unified origin / d_max, 10) and encode(r, 4):
                                  90 inputs (layout below)                      */
    DONERF_DEPTH_POSITIONS = 1 /* Sec. 5.2, App. D: unified origin / d_max, r and
                                  one position (x_k - c) / d_max per class
                                  centre, x_k = o + c_k r from the camera origin,
                                  unencoded: 6 + 3 n_bins inputs in the order
                                  [origin xyz, r xyz, x_0 xyz, ..., x_{B-1} xyz].
                                  The first layer's weights are folded at create
                                  into 9 columns (the positions are affine in the
                                  ray) and evaluated in fp32 in both precisions;
                                  its inputs are not rounded to bf16           */
} donerf_depth_input;

/* Maximum number of samples per ray a handle can be created for. */
#define DONERF_MAX_SAMPLES 16

typedef struct donerf_cfg {
    float near_dist;   /* d_min > 0: nearest sample depth along the ray (Eq. 1) */
    float far_dist;    /* d_max > d_min: farthest depth; also the normalisation
                          of Eq. 2 and the warp scale of Eq. 5                 */
    int32_t n_bins;    /* B: number of logarithmic depth classes (Eq. 3);
                          the library supports 64, 128, 192 and 256          */
    int32_t n_max;     /* largest N a render may request, 1..16, n_max <= B   */
    float fov_x_deg;   /* horizontal field of view of the pinhole camera, in
                          degrees, 0 < fov < 180                               */
    float centre[3];   /* view-cell centre c (Eq. 2, Eq. 4)                    */
    float radius;      /* radius > 0 of the unification sphere (Sec. 5.2)      */
    int32_t precision; /* donerf_precision                                     */
    int32_t select;    /* donerf_select                                        */
    int32_t depth_input; /* donerf_depth_input                                 */
} donerf_cfg;

/*
 * Number of fp32 values in the weight blob for B depth classes and the given
 * donerf_depth_input, or 0 if B is not positive or depth_input is unknown.
 *
 * Blob layout (host, fp32): depth network layers 0..7, then shading network
 * layers 0..7; each layer is W[out][in] row-major followed by b[out].
 *   depth  : 90 (or 6 + 3 B) -> 256, 6 x (256 -> 256), 256 -> B
 *   shading: 63 -> 256, 6 x (256 -> 256), (256 + 27) -> 4
 * Depth layer 0 reads the encoding of the unified origin divided by d_max
 * (63 values) followed by the encoding of the direction (27 values).  The
 * encoding of v with L frequencies is [v, sin(2^0 pi v), cos(2^0 pi v), ...,
 * sin(2^(L-1) pi v), cos(2^(L-1) pi v)], each block over x, y, z; L = 10 for
 * positions, 4 for directions.  Shading layer 0 reads the encoding of the
 * warped sample (63); shading layer 7 reads the 256 hidden values followed by
 * the direction encoding (27) and outputs (r, g, b, sigma) before activation.
 */
size_t donerf_weight_count(int32_t n_bins, int32_t depth_input);

/*
 * Create a renderer on the current HIP device.
 *   cfg       host, read during the call
 *   weights   host fp32 blob of n_weights values (layout above); the library
 *             converts and copies it to the device, so the caller may free it
 *             on return
 *   out       receives the handle; set to NULL on failure
 * Errors: E_INVALID_ARG (NULL, cfg ranges), E_UNSUPPORTED (n_bins not in the
 * supported set), E_SIZE (n_weights !=
 * donerf_weight_count(cfg->n_bins, cfg->depth_input)),
 * E_NONFINITE (NaN/Inf in cfg or weights), E_DEVICE (no device or not
 * gfx950), E_NOMEM, E_HIP.
 */
int donerf_create(const donerf_cfg* cfg, const float* weights, size_t n_weights,
                  donerf_t** out);

/* Release the handle and its device memory.  NULL is allowed. */
void donerf_destroy(donerf_t* h);

/*
 * Bind the HIP stream (a hipStream_t passed as void*) on which the handle's
 * work is enqueued.  NULL selects the null stream (the default).
 */
int donerf_set_stream(donerf_t* h, void* stream);

/*
 * Render P camera images of H x W pixels with N samples per ray.
 *   cam_poses  host, P x 12 fp32: camera-to-world 3x4 row-major [R | o] per
 *              image; the camera looks down its -z axis, +y is up; pixel
 *              (i, j), i along the width and j downwards, is the ray through
 *              the pixel centre
 *   N          samples per ray, 1 <= N <= cfg.n_max (and <= B)
 *   out_rgb    device, P x H x W x 3 fp32, row-major, caller-owned
 *   out_depth  device, P x H x W fp32 (sum of sample weight x sample depth),
 *              or NULL to skip
 * The work is enqueued on the handle's stream; results are valid once the
 * stream has been synchronised.  No allocation, no host synchronisation.
 * The call issues kernel launches only (the poses travel in the launch
 * arguments; no memset or copy), so it can be captured into a HIP graph on
 * the handle's stream and replayed; a replay renders the poses, sizes and
 * buffers of the captured call.  Calls on one handle share its scratch
 * buffer for the split tail: do not let two of them overlap on different
 * streams.
 * Errors: E_INVALID_ARG (NULL handle/poses/out_rgb, P, H, W < 1, N out of
 * range, P*H*W >= 2^31, H*W > 2^24), E_NONFINITE (pose), E_HIP (launch
 * failed).
 */
int donerf_render(donerf_t* h, const float* cam_poses, int32_t P, int32_t H, int32_t W,
                  int32_t N, float* out_rgb, float* out_depth);

/*
 * donerf_render for callers that cannot allocate device memory at all (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same kernels and results, with the split tail's partial
 * results kept in a static device array of the library instead of the
 * handle's buffer.  The array holds 5 x 256 x 256 floats (1.25 MiB) on every
 * device the library runs on, until the process ends; its address is looked
 * up when a handle is created, so this call makes no HIP call other than its
 * kernel launches and allocates nothing.  Every call on one device shares that
 * device's array (no contents need clearing: each launch writes every part it
 * reads back), so calls that overlap on one device, on any handles or
 * streams, race and must not be issued.
 * Arguments and errors as donerf_render, plus E_UNSUPPORTED when a launch's
 * split tail needs more than the array holds (only on devices with more than
 * 256 compute units) and E_HIP when the array's address could not be looked
 * up at create.
 */
int donerf_render_static_scratch(donerf_t* h, const float* cam_poses, int32_t P, int32_t H, int32_t W,
                                 int32_t N, float* out_rgb, float* out_depth);

/*
 * donerf_render with optional per-ray intermediate outputs, for testing.
 *   out_bins     device, P x H x W x N int32: the class of each sample in sample
 *                (= depth) order, or NULL
 *   out_scores   device, P x H x W x B fp32: depth-network scores, or NULL;
 *                with DONERF_SELECT_TOPN_SOFTMAX the softmax probabilities
 *   out_samples  device, P x H x W x N x 2 fp32: depth and width of each
 *                sample, or NULL
 * Same errors as donerf_render.
 */
int donerf_render_debug(donerf_t* h, const float* cam_poses, int32_t P, int32_t H,
                        int32_t W, int32_t N, float* out_rgb, float* out_depth,
                        int32_t* out_bins, float* out_scores, float* out_samples);

/*
 * How donerf_render cuts a call, for testing; needs no device.  On a device of
 * n_cu compute units (1..2^16), launch `launch` (0, 1, ...) of the call takes
 *   out[0]  poses (0 past the last launch, and the rest then 0)
 *   out[1]  rays per tile
 *   out[2]  tiles rendered whole, by one workgroup each
 *   out[3]  tiles split by samples
 *   out[4]  workgroups per split tile
 *   out[5]  threads per workgroup
 * Errors: E_INVALID_ARG, E_NONFINITE and E_UNSUPPORTED for a cfg that
 * donerf_create refuses; E_INVALID_ARG (NULL out, n_cu or launch out of range,
 * sizes that donerf_render refuses).
 */
int donerf_debug_plan(const donerf_cfg* cfg, int32_t n_cu, int32_t P, int32_t H, int32_t W, int32_t N,
                      int32_t launch, int32_t* out);

/*
 * Run the device top-N selection on given scores, for testing: the code that a
 * render of that many rays on this handle would select with (kernels of
 * different tile sizes split a ray's classes over 2, 8 or 16 lanes).
 *   scores   device, rays x B fp32
 *   out_idx  device, rays x N int32: the N classes with the highest scores,
 *            ties broken towards the lower class index, +0 and -0 equal,
 *            NaN below every number, written in ascending class order
 * Errors: E_INVALID_ARG (NULL, rays < 1, N out of range), E_HIP.
 */
int donerf_debug_topn(donerf_t* h, const float* scores, int32_t rays, int32_t N,
                      int32_t* out_idx);

/*
 * Measured ceiling of the matrix cores, for the roofline of donerf_render:
 * a register-fed MFMA loop in the handle's precision (BF16: 32 x 32 x 16
 * bf16; FP8: 32 x 32 x 64 E4M3; FP32: 32 x 32 x 2 fp32), on the handle's
 * stream.  workgroups x 4 waves each run four independent accumulator chains
 * of `iters` steps on seeded random register operands drawn like the
 * render's: A uniform in [-1, 1) like weights, B the positive part of such
 * values like ReLU activations (no memory traffic, no dependence stalls).
 *   workgroups  1..2^20 (a few per compute unit fill the device)
 *   iters       1..2^24 steps per chain
 *   sink        device, workgroups x 256 fp32, caller-owned: one sum of
 *               accumulators per thread, written so the work is kept
 *   flop        host, may be NULL: the launch's FLOP (2 per multiply-add)
 * Time the launch with events on the handle's stream.
 * Errors: E_INVALID_ARG (NULL handle or sink, sizes out of range), E_HIP.
 */
int donerf_debug_mfma_peak(donerf_t* h, int32_t workgroups, int32_t iters, float* sink, double* flop);

/*
 * Training targets of the depth oracle (Sec. 5.1) for P depth maps, on the
 * handle's depth classes and stream:
 *   Eq. 6  C(z) = 1 for the class z with b_z <= d < b_{z+1} of the pixel's
 *          first-surface depth d (no class where d is outside [d_min, d_max)
 *          or not finite),
 *   Eq. 7  C^(z) = max over the offsets |i|, |j| <= floor(K/2) of
 *          C_{x+i,y+j}(z) minus sqrt(i^2 + j^2) / (sqrt(2) floor(K/2))
 *          (neighbours outside the image left out; K = 1 keeps C; an even
 *          K spans K + 1 pixels and gives the targets of K + 1),
 *   Eq. 8  C`(z) = min(sum_{|i| <= floor(Z/2)} C^(z + i) (floor(Z/2) + 1 - |i|)
 *          / (floor(Z/2) + 1), 1) (classes outside [0, B) left out).
 *   depth  device, P x H x W fp32: the distance from the camera to the first
 *          surface along each pixel's ray (Eq. 1's d), row-major
 *   K, Z   window sizes, 1..15 (the paper evaluates 1, 5 and 9 and uses
 *          K = Z = 5)
 *   out    device, P x H x W x B fp32, caller-owned; B = cfg.n_bins
 * Enqueued on the handle's stream; no allocation.
 * Errors: E_INVALID_ARG (NULL, P, H, W < 1, K or Z out of range, too many
 * pixels), E_HIP.
 */
int donerf_targets(donerf_t* h, const float* depth, int32_t P, int32_t H, int32_t W, int32_t K, int32_t Z,
                   float* out);

/* ------------------------------------------------------------------------
 * Layers of the networks as operators of their own: products with 4-bit weights
 * for serving, and a layer's forward and backward pass for training, with its
 * activations kept in 8 bits in between.
 *
 * They take matrices in device memory, row by row, and work on any sizes: in and
 * out of a layer need not be those of the handle's networks, whose weights they
 * do not touch.  The handle gives them its device and its stream.  They allocate
 * nothing, launch kernels only and keep nothing between calls, so they can be
 * captured into a HIP graph; calls that overlap on different streams are safe as
 * far as their buffers (the workspace among them) are different ones.
 * ------------------------------------------------------------------------ */

typedef enum donerf_type {
    DONERF_TYPE_FP32 = 0,
    DONERF_TYPE_BF16 = 1,
    DONERF_TYPE_MXFP4 = 2, /* microscaled E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and
                              their negatives)                                */
    DONERF_TYPE_MXFP8 = 3  /* microscaled E4M3 (largest value 448)            */
} donerf_type;

/*
 * A matrix in device memory.  fp32 and bf16: rows of values, at least `cols`
 * apart.  Microscaled: a row's columns form blocks of 32, the last one filled
 * up with zeros, and the values of a block are its elements times its scale
 * 2^(c - 127), c one byte, 255 for NaN (OCP Microscaling Formats v1.0).
 *   data    fp32, bf16: aligned to the type's size.  Microscaled: the elements'
 *           codes, aligned to 16 bytes; 16 bytes a block in MXFP4 (the even
 *           column in a byte's low half), 32 bytes a block in MXFP8
 *   ld      from row to row: values (fp32, bf16) or bytes, a multiple of 16
 *           (microscaled); at least a row's length.  What lies between the rows
 *           of an input may be read, but is not used; that between the rows of
 *           an output is left as it is
 *   scales  microscaled: one byte per block, aligned to 8 bytes; else NULL
 *   ld_scales  bytes from one row's scales to the next's, a multiple of 8 and at
 *           least a row's blocks.  Bytes behind the last block's are neither
 *           used nor written
 * What a call writes (an output's data and scales, db, the workspace as far as it
 * is needed) may share memory with nothing else that the call is given; a call in
 * which it does is refused (E_INVALID_ARG).  Columns of one buffer side by
 * side share none if their rows are equally far apart; with different strides the
 * whole range from first to last row counts.
 * Both directions of every conversion treat a block the same way: its scale is
 * the smallest power of two, 2^-127 or more, that holds its largest value as an
 * element (6 or 448 times the scale), and elements are rounded to the nearest,
 * ties to even.  In MXFP8 a value other than zero never becomes zero but at
 * least the smallest element, and NaN and infinities become NaN.  In MXFP4 a block
 * that holds a NaN or an infinity gets the scale NaN, and all of it reads as NaN.
 */
typedef struct donerf_mat {
    void* data;
    int64_t ld;
    uint8_t* scales;
    int64_t ld_scales;
    int32_t type; /* donerf_type */
} donerf_mat;

/* Largest number of columns, and of a layer's inputs and outputs. */
#define DONERF_MAX_COLS 65536

/*
 * Convert x (FP32 or BF16) to q (MXFP4 or MXFP8), and back (MXFP4 or MXFP8 to
 * FP32 or BF16; the values are exact but for the rounding of the smallest and the
 * overflow of the largest scales, and of MXFP8 below BF16's smallest numbers).
 *   rows  0..2^31 - 1; with 0 the call does nothing
 *   cols  1..DONERF_MAX_COLS
 * x, q and y must not overlap.
 * Errors: E_INVALID_ARG (NULL handle or matrix, a size, type, alignment or ld
 * that the above rules out), E_DEVICE (the current device is not the handle's),
 * E_HIP.
 */
int donerf_mx_quantize(donerf_t* h, const donerf_mat* x, const donerf_mat* q, int64_t rows, int32_t cols);
int donerf_mx_dequantize(donerf_t* h, const donerf_mat* q, const donerf_mat* y, int64_t rows, int32_t cols);

/*
 * y = act(x w^T + bias) with both factors in MXFP4.
 *   x     rows x in: MXFP4, or FP32 or BF16, converted on the way as
 *         donerf_mx_quantize does
 *   w     out x in, MXFP4
 *   bias  device, out fp32, or NULL
 *   relu  0: act is the identity; 1: max(z, 0), NaN kept
 *   y     rows x out: FP32, BF16 or MXFP4 (converted from the fp32 results)
 *   workspace  device, 16-byte aligned, at least donerf_mx_linear_workspace(...)
 *         bytes, the call's own until it is done (for some sizes unused: the query
 *         does not know `out`); may be NULL if that is 0
 * Products are exact, sums fp32.  y must not overlap the inputs.
 * rows 0..2^31 - 1 (0: nothing is done), in and out 1..DONERF_MAX_COLS.
 * Errors: as above, and E_SIZE (workspace too small), E_UNSUPPORTED (rows x out
 * of 2^38 or more, or more results than a launch's grid counts).
 */
int donerf_mx_linear(donerf_t* h, const donerf_mat* x, const donerf_mat* w, const float* bias, int32_t relu,
                     const donerf_mat* y, int64_t rows, int32_t in, int32_t out, void* workspace,
                     size_t workspace_bytes);

/* Bytes of workspace for x of this donerf_type: 0 where none is needed (MXFP4, a
   few rows), and for sizes that are refused. */
size_t donerf_mx_linear_workspace(int32_t x_type, int64_t rows, int32_t in);

/*
 * A layer's forward pass for training: y = act(x w^T + bias) in BF16, and kept,
 * the same values (before their rounding to BF16) in MXFP8 for the backward pass
 * of the layer that reads them.
 *   x     rows x in, BF16
 *   w     out x in, BF16
 *   bias, relu  as above
 *   y     rows x out, BF16, or NULL
 *   kept  rows x out, MXFP8, or NULL; one of the two at least
 * fp32 accumulation.  The outputs overlap neither each other nor the inputs.
 * Sizes and errors: as for donerf_mx_linear.
 */
int donerf_train_linear(donerf_t* h, const donerf_mat* x, const donerf_mat* w, const float* bias, int32_t relu,
                        const donerf_mat* y, const donerf_mat* kept, int64_t rows, int32_t in, int32_t out);

/*
 * The layer's backward pass, from the gradient dz of its z = x w^T + bias:
 *   dx = dz w (rounded to BF16), dw = dz^T x, db = the sum of dz's rows.
 *   dz    rows x out, BF16
 *   x     rows x in: what the forward pass of the layer before kept (MXFP8), or
 *         BF16 (a network's input)
 *   relu  1: x is a ReLU's output, and dx is the gradient of that ReLU's input:
 *         0 where x is zero, in MXFP8 where its element is, whatever the block's
 *         scale (a zero of a block whose scale is NaN stops the gradient, too,
 *         though x reads as NaN there).  0: dx is the gradient of x
 *   w     out x in, BF16; may be NULL without dx
 *   dx    rows x in, BF16, or NULL
 *   dw    out x in, FP32, or NULL
 *   db    device, out fp32, or NULL
 *   accumulate  0: dw and db are written; 1: they are added to
 *   workspace  device, 16-byte aligned, donerf_train_linear_backward_workspace(...)
 *         bytes at least, the call's own until it is done
 * fp32 accumulation; the same call gives the same bits.  With rows = 0, dw and
 * db are zero (or stay, with accumulate).  Outputs overlap nothing.
 * Sizes and errors: as for donerf_mx_linear.
 */
int donerf_train_linear_backward(donerf_t* h, const donerf_mat* dz, const donerf_mat* x, int32_t relu,
                                 const donerf_mat* w, const donerf_mat* dx, const donerf_mat* dw, float* db,
                                 int32_t accumulate, int64_t rows, int32_t in, int32_t out, void* workspace,
                                 size_t workspace_bytes);

/* Bytes of workspace on the handle's device: 0 where none is needed (a few rows),
   and for sizes that are refused. */
size_t donerf_train_linear_backward_workspace(const donerf_t* h, int64_t rows, int32_t in, int32_t out);

/* The device and the stream that a handle's work goes to; each may be NULL. */
int donerf_get_stream(const donerf_t* h, int32_t* device, void** stream);

/*
 * Copy the handle's depth-class table to host memory: bounds (B + 1 values,
 * may be NULL), centres (B), widths (B).  Bounds b_k = d_min + (d_max - d_min
 * + 1)^(k/B) - 1 (the inverse of Eq. 3 on a uniform grid), centres at
 * (k + 0.5)/B, widths b_{k+1} - b_k; computed in fp64, stored as fp32.
 */
int donerf_debug_bins(const donerf_t* h, float* bounds, float* centres, float* widths);

/* Static description of a status code. */
const char* donerf_status_str(int status);

/* Message of the most recent failure in the calling thread ("" if none). */
const char* donerf_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* DONERF_H */
