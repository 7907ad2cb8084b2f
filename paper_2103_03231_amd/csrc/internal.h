// internal.h - interface between the host planner (host.cpp) and the kernels
// (kernels.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "layout.h"

namespace donerf {

constexpr int kMaxSamples = 16;   // samples per ray (include/donerf.h DONERF_MAX_SAMPLES)

// Everything one render launch needs, passed by value as the kernel argument.
struct RenderArgs {
    const uint4* d_frags;   // depth network fragments (bf16 and fp8 networks: chunk-padded per layer)
    const uint4* s_frags;   // shading network fragments
    const float* bias;      // all biases (layout.h bias_len); the depth head's last
    const float* bins;      // centres[B] then widths[B]
    float* out_rgb;         // rays x 3
    float* out_depth;       // rays, or null
    int32_t* out_bins;      // rays x N, or null
    float* out_scores;      // rays x B, or null
    float* out_samples;     // rays x N x (depth, width), or null
    int32_t n_d_chunks;     // chunks of the two streams, for the kernel that copies them (bf16)
    int32_t n_s_chunks;
    int32_t bias_len;       // floats in bias
    int32_t H, W, n_poses, N, B;
    uint32_t total_rays;    // n_poses * H * W
    // Workgroups b < n_full render tile b whole.  Workgroups b >= n_full
    // split the remaining tiles by samples: with c = b - n_full, tile
    // n_full + c / split, samples [j N / split, (j + 1) N / split) for
    // j = c % split.  With split > 1 such a part writes its composite (C rgb,
    // depth, transmittance) to partial[(local_ray * split + j) * 5], local_ray
    // counted from the first ray of tile n_full, instead of the outputs.
    uint32_t n_full;
    int32_t split;
    float* partial;
    int32_t tile_rays;      // rays of a tile
    float focal, half_w, half_h;
    float cx, cy, cz;
    float radius;
    float near;             // d_min
    float dmax;             // d_max
    float log2_span1;       // log2(d_max - d_min + 1), for the inverse of Eq. 3
    // inverse-CDF targets (Sec. 5.1): cdf_u[i] = (i + 1/2) / N, the centre of
    // probability slice i < N, and cdf_u[kMaxSamples + i] = (i + 1) / N, the
    // inner end of slice i < N - 1; 2 elsewhere.  Each is the correctly
    // rounded fp32 quotient, as the kernel's own division would give.
    float cdf_u[2 * kMaxSamples];
    int32_t wscale[16];     // per streamed layer (depth 0-7, shading 8-15): E8M0 scale of
                            // its fp8 weights, 127 - s for weights stored as W 2^s
    float poses[kMaxPosesPerLaunch][12];
};

// Launch shape of the bf16 render kernel: 32-ray column blocks per wave and
// waves per workgroup, and waves per SIMD the register budget is sized for.
#ifndef DONERF_BF16_CB
#define DONERF_BF16_CB 1
#endif
#ifndef DONERF_BF16_NW
#define DONERF_BF16_NW 8
#endif
#ifndef DONERF_BF16_OCC
#define DONERF_BF16_OCC 2
#endif
constexpr int kBf16CB = DONERF_BF16_CB;
constexpr int kBf16NW = DONERF_BF16_NW;
constexpr int kBf16Occ = DONERF_BF16_OCC;

// 32-ray column blocks of the main kernels of fp32 and fp8 networks, and the
// rays of a tile of each precision's main kernel (prec: layout.h Precision of
// the network).
constexpr int kF32CB = 2;
constexpr int kF8CB = 4;
// Waves per workgroup of the fp8 main kernel and of rows_kernel.h's.
constexpr int kF8Waves = 4;
constexpr int kRowWaves = 8;
inline int rays_per_block(int prec) {
    return prec == kF32 ? 32 * kF32CB : prec == kFP8 ? 32 * kF8CB : kBf16NW * 32 * kBf16CB;
}
// Threads of the workgroup that renders a tile of tile_rays rays.
inline int tile_threads(int prec, int tile_rays) {
    return 64 * (prec == kF32 || tile_rays != rays_per_block(prec) ? kRowWaves : prec == kFP8 ? kF8Waves : kBf16NW);
}

// Launches a.n_full whole tiles plus n_split_tiles tiles split a.split ways.
// place: layout.h Placement; din: layout.h DepthInput; a.tile_rays: the main
// kernel's, or rows_kernel.h's smaller tiles'.
hipError_t launch_render(int prec, int ncap, int place, int din, const RenderArgs& a, uint32_t n_split_tiles,
                         hipStream_t stream);
// The main kernels of bf16 and fp8 networks by placement (render_*.hip).
hipError_t launch_render_bf16_topn(int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
hipError_t launch_render_bf16_cdf(int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
hipError_t launch_render_bf16_cdf_wide(int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
hipError_t launch_render_fp8_topn(int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
hipError_t launch_render_fp8_cdf(int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
hipError_t launch_render_fp8_cdf_wide(int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
// rows_kernel.h's tiles of 32 and 64 rays, for fp32 networks all there are
// (render_rows_*.hip); any other tile is hipErrorInvalidValue.
hipError_t launch_rows_bf16(int cdf, int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
hipError_t launch_rows_fp8(int cdf, int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
hipError_t launch_rows_fp32(int cdf, int ncap, int din, const RenderArgs& a, dim3 grid, hipStream_t stream);
// Composites the split parts of rays [n_full * tile_rays, total_rays) into
// out_rgb / out_depth.
hipError_t launch_combine(const RenderArgs& a, hipStream_t stream);
// Floats of the static device scratch behind donerf_render_static_scratch:
// the split tail's parts (5 floats per ray and part) of up to 256 compute
// units x 256 rays, 1.25 MiB per device.
constexpr size_t kStaticScratchFloats = (size_t)5 * 256 * 256;
constexpr int kMaxDevices = 64;
// Device address of that scratch on `device`, which must be the current
// device; looked up once per device, then cached.
hipError_t static_scratch_address(int device, float** out);
hipError_t launch_softmax_rows(float* scores, uint32_t rows, int B, hipStream_t stream);
// The selection that the kernel of a tile runs, on given scores.
hipError_t launch_topn(int prec, int tile_rays, int ncap, const float* scores, int32_t rays, int32_t N, int32_t B,
                       int32_t* out_idx, hipStream_t stream);

// Register-fed MFMA loop (kernels.hip): workgroups x 4 waves, four
// independent 32 x 32 chains of `iters` steps per wave in precision prec;
// sink holds workgroups x 256 floats.
hipError_t launch_mfma_peak(int prec, int workgroups, int iters, uint32_t seed, float* sink, hipStream_t stream);
// FLOP of one chain step: a 32 x 32 x 16 bf16, 32 x 32 x 64 E4M3 or four
// 32 x 32 x 2 fp32 MFMAs.
constexpr double mfma_step_flop(int prec) {
    return prec == kFP8 ? 2.0 * 32 * 32 * 64 : prec == kBF16 ? 2.0 * 32 * 32 * 16 : 2.0 * 32 * 32 * 8;
}

// Training targets (targets.hip): P depth maps of H x W, class bounds
// bounds[0..B], window sizes K and Z (1..kTgtMaxK), out P x H x W x B.
constexpr int kMaxBins = 256;
constexpr int kTgtMaxK = 15;
hipError_t launch_targets(const float* depth, int P, int H, int W, const float* bounds, int B, int K, int Z,
                          float inv_l2span, float* out, hipStream_t stream);

// ---- layer operators (include/donerf.h): microscaled formats (mx_convert.hip),
// products with 4-bit weights (mx_linear.hip), layers whose activations are kept
// in 8 bits (train_linear.hip).

// A matrix's rows as bytes: codes of a microscaled one, or the values of a bf16
// one.  ld: bytes from row to row.
struct MxIn {
    const uint8_t* codes;
    int64_t ld;
    const uint8_t* scales;   // microscaled only
    int64_t ld_scales;
};
struct MxOut {
    uint8_t* codes;
    int64_t ld;
    uint8_t* scales;
    int64_t ld_scales;
};

// A product y[m][n] = sum_k a[n][k] b[m][k] and what follows it (layer_gemm.h).
struct GemmArgs {
    MxIn a, b;               // N and M rows of K columns
    const float* bias;       // N, or null
    uint8_t* y;              // bf16 or fp32 rows, or null
    int64_t ldy;             // values from row to row
    MxOut q;                 // microscaled outputs
    const uint8_t* mask;     // E4M3 codes or bf16 rows of masked epilogues
    int64_t ld_mask;         // bytes (E4M3) or values (bf16)
    int32_t M, N, K;
    int32_t relu;
    uint32_t tiles_n, tiles_m;
};

// Outputs of mx_linear.
constexpr int kOutBf16 = 0, kOutF32 = 1, kOutMx4 = 2;

hipError_t launch_mx_quantize(const void* x, int64_t ldx, bool x_bf16, const MxOut& q, bool fp8, int64_t rows, int cols,
                              int n_cu, hipStream_t stream);
hipError_t launch_mx_dequantize(const MxIn& q, bool fp8, void* y, int64_t ldy, bool y_bf16, int64_t rows, int cols,
                                int n_cu, hipStream_t stream);
// g.a, g.b E2M1.
hipError_t launch_mx_linear(const GemmArgs& g, int out, int n_cu, hipStream_t stream);
// g.b fp32 or bf16 rows (ld in bytes), converted where they are multiplied: for sizes
// that mx_linear_converts takes.
bool mx_linear_converts(const GemmArgs& g, int n_cu);
hipError_t launch_mx_linear_convert(const GemmArgs& g, bool x_bf16, int out, int n_cu, hipStream_t stream);
// The same for up to kFewRows rows, x fp32 (0), bf16 (1) or E2M1 (2).
constexpr int kFewRows = 32;
struct FewRowsArgs {
    const uint8_t* x;
    int64_t ldx;             // values, or bytes of E2M1 rows
    const uint8_t* x_scales;
    int64_t ldx_scales;
    const uint8_t* w;
    int64_t ldw;             // bytes
    const uint8_t* w_scales;
    int64_t ldw_scales;
    const float* bias;
    uint8_t* y;              // fp32 or bf16 rows
    int64_t ldy;
    MxOut q;                 // or E2M1 ones
    int32_t M, N, K, relu, out;
};
hipError_t launch_mx_few_rows(const FewRowsArgs& g, int x_kind, hipStream_t stream);
// g.a, g.b bf16; y and q may each be null.
hipError_t launch_train_linear(const GemmArgs& g, int n_cu, hipStream_t stream);

// The backward pass of a layer: dz (M x N bf16), x (M x K, E4M3 or bf16), w
// (N x K bf16).  dx, dw and db may each be null.
struct BackwardArgs {
    const uint16_t* dz;
    int64_t lddz;
    MxIn x;                  // E4M3, or bf16 rows (x_bf16), ld in bytes
    int32_t x_bf16;
    int32_t relu;            // x is a ReLU's output
    const uint16_t* w;
    int64_t ldw;
    uint16_t* dx;
    int64_t lddx;
    float* dw;
    int64_t lddw;
    float* db;
    int32_t accumulate;      // dw and db are added to
    int32_t M, N, K;
    uint8_t* workspace;
};
// Bytes of workspace for these sizes.
size_t backward_workspace(int64_t M, int N, int K, int n_cu);
hipError_t launch_train_linear_backward(const BackwardArgs& a, int n_cu, hipStream_t stream);

// ---- operators around the layers: layer norm (train_norm.hip), lookup
// (train_embedding.hip), distillation loss (train_distill.hip).

// Rows of whole numbers, 32 or 64 bits (wide) each.
struct IntRows {
    const void* p;
    int64_t ld;
    int32_t wide;
    __device__ __forceinline__ int64_t at(int64_t row, int col) const {
        const int64_t i = row * ld + col;
        return wide ? ((const int64_t*)p)[i] : (int64_t)((const int32_t*)p)[i];
    }
};
// Rows of fp32 or bf16 numbers, read one at a time.
struct FloatRows {
    const void* p;
    int64_t ld;
    int32_t bf16;
    __device__ __forceinline__ float at(int64_t row, int col) const {
        const int64_t i = row * ld + col;
        return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16) : ((const float*)p)[i];
    }
};

// Rows of fp32 or bf16 results; rows.h stores them.
struct RowsOut {
    void* base;
    int64_t ld;
    int32_t bf16;
};

// Types of rows that kernels are built for.
constexpr int kRowsF32 = 0, kRowsBf16 = 1, kRowsMx8 = 2;

struct NormArgs {
    const void* x;           // fp32 or bf16
    int64_t ldx;
    const float* w;          // cols, or null
    const float* b;          // cols, or null
    float eps;
    int32_t relu;
    RowsOut y;               // base null without it
    MxOut q;                 // E4M3, or codes null
    float* stats;            // rows x (mean, 1 / standard deviation)
    uint32_t rows;
    int32_t cols;
    float inv_cols;
};
hipError_t launch_train_norm(const NormArgs& a, bool x_bf16, int n_cu, hipStream_t stream);

struct NormBackwardArgs {
    const void* dz;          // fp32 or bf16
    int64_t lddz;
    MxIn x;                  // ld in values (fp32, bf16) or bytes (E4M3)
    int32_t relu;            // x is a ReLU's output
    const float* w;          // cols, or null
    const float* stats;
    RowsOut dx;              // base null without it
    float* dw;               // cols, or null
    float* db;               // cols, or null
    int32_t accumulate;
    uint32_t rows;
    int32_t cols;
    float inv_cols;
    float* parts;            // set by the launch: each workgroup's dw and db, or null
    uint32_t row_groups;     // and the workgroups of the rows, where others sum the columns
};
size_t norm_backward_workspace(int64_t rows, int cols, int n_cu);
hipError_t launch_train_norm_backward(const NormBackwardArgs& a, int x_type, bool dz_bf16, void* workspace, int n_cu,
                                      hipStream_t stream);

struct EmbeddingArgs {
    const void* table;       // n x cols, fp32 or bf16
    int64_t ldt;
    IntRows ids;
    float scale;
    RowsOut y;
    int64_t rows, n;
    int32_t cols;
};
hipError_t launch_train_embedding(const EmbeddingArgs& a, bool table_bf16, int n_cu, hipStream_t stream);

// Rows [begin, end) of a table of zeros.
struct ZeroFill {
    float* table;
    int64_t ld;
    int32_t cols;
    int32_t past;            // by stores that pass the caches
    int64_t begin, end;
};
// One pass of the sort of rows by their ids.
constexpr int kSortBits = 10;   // most bits of a pass
struct SortPass {
    IntRows ids;             // what the first pass makes its keys of
    const uint32_t* keys_in; // null in the first pass
    const uint32_t* rows_in; // null in the first pass
    uint32_t* keys_out;
    uint32_t* rows_out;
    uint32_t* counts;        // tiles x bins
    uint32_t* totals;        // bins
    uint32_t rows, tile, tiles;   // keys, those of a workgroup, workgroups
    int64_t n;
    int32_t shift, bits;
    int32_t scanned;         // counts are those of the tiles before, totals theirs
};
struct EmbeddingGradArgs {
    const void* dy;          // rows x cols, fp32 or bf16
    int64_t lddy;
    float scale;
    float* dtable;           // n x cols
    int64_t lddt;
    int32_t accumulate;
    int64_t rows, n;
    int32_t cols;
    const uint32_t* keys;    // set by the launch, as the rest: sorted ids, and their rows
    const uint32_t* order;
    float* ends;             // sums of runs that cross the parts' ends
    uint32_t part;           // sorted rows of a part
    int32_t block_bits;      // parts that one workgroup sums, as a power of two
    uint32_t slabs;          // workgroups that sum, where one launch does all
};
size_t embedding_backward_workspace(int64_t rows, int64_t n, int cols);
hipError_t launch_train_embedding_backward(EmbeddingGradArgs a, const IntRows& ids, bool dy_bf16, void* workspace, int n_cu,
                                           hipStream_t stream);

constexpr int kMostEntries = 128;   // of a teacher's row (include/donerf.h DONERF_MAX_TOP)
struct DistillArgs {
    const void* x;           // fp32 or bf16
    int64_t ldx;
    IntRows classes;
    FloatRows teacher;
    const float* weight;     // rows, or null
    float temp, inv_temp, log2e_over_t;
    float* loss;             // rows, or null
    RowsOut dx;              // base null without it
    uint32_t rows;
    int32_t cols, k;
};
hipError_t launch_train_distill(const DistillArgs& a, bool x_bf16, int n_cu, hipStream_t stream);

}  // namespace donerf
