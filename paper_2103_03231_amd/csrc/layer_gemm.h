// layer_gemm.h - the products of the layer operators on gfx950: for batch rows b
// (M of them) and weight rows a (N), y[m][n] = sum_k a[n][k] b[m][k], on bf16
// MFMAs or block-scaled E2M1 ones, with what follows the product in its epilogue.
//
// A workgroup computes a tile of BN weight rows by BM batch rows in stages of
// 128 bytes of every row (64 bf16 or 256 E2M1 columns).  In LDS a row's eight
// 16-byte chunks are permuted, chunk c at position c ^ (row & 7), so that the
// eight lanes which an LDS cycle serves, eight rows of one chunk, meet eight
// different bank groups.  Two such stages alternate in two arrays: the copy of
// one runs while the other is multiplied.
//
// The weights are the MFMA's A operand and the batch its B operand, so a lane's
// accumulators are 16 of a block's 32 outputs of one batch row, and a swap of
// registers with the lane 32 further makes them 16 consecutive ones: bias, ReLU,
// the block scales of microscaled outputs and wide stores need nothing else.
#pragma once

#include "internal.h"
#include "mx.h"

namespace donerf {
namespace {

constexpr int kOpBf16 = 0, kOpMx4 = 1;
constexpr int kStageBytes = 128;   // of each row
constexpr int kStageChunks = kStageBytes / 16;

// What follows the product.
constexpr int kEpiBf16 = 0;    // y bf16
constexpr int kEpiF32 = 1;     // y fp32
constexpr int kEpiMx4 = 2;     // y E2M1
constexpr int kEpiKept = 3;    // y bf16 and its E4M3 checkpoint, either may be absent
constexpr int kEpiMasked = 4;  // y bf16, zero where the ReLU's output (E4M3 or bf16) is

// 16 zero bytes: what a lane copies in place of chunks behind the last column.
__device__ const uint32_t kZeroChunk[4] = {0, 0, 0, 0};

// 16 bytes of a row: 8 bf16 or a block of 32 E2M1.  Zeros behind the last column.
template <int OP>
__device__ __forceinline__ u32x4 load_chunk(const uint8_t* row, int chunk, int K) {
    if (OP == kOpBf16) {
        if (chunk * 8 >= K) return u32x4{0, 0, 0, 0};
        return Row8<uint16_t>::load_raw((const uint16_t*)row, chunk * 8, K);
    }
    return chunk * kMxBlock < K ? *(const u32x4*)(row + (size_t)chunk * 16) : u32x4{0, 0, 0, 0};
}

// Copies of one operand's rows [row0, row0 + ROWS) into a stage in LDS.
template <int OP, int ROWS, int NW, bool DIRECT>
struct StageCopy {
    static constexpr int PER = ROWS / 8 / NW;   // copies per wave, 8 rows each
    static_assert(ROWS % (8 * NW) == 0, "rows split evenly over the waves");
    const uint8_t* row[PER];   // of this lane, in each copy
    u32x4 held[DIRECT ? 1 : PER];
    int chunk;                 // of this lane, in every row
    __device__ __forceinline__ void init(const MxIn& src, int64_t row0, int64_t rows, int wave, int lane) {
        chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            // rows behind the last one repeat it: their results are not stored
            int64_t r = row0 + (i * NW + wave) * 8 + (lane >> 3);
            r = r < rows ? r : rows - 1;
            row[i] = src.codes + r * src.ld;
        }
    }
    // Straight into LDS (rows of 16-byte alignment), or into registers, to be
    // stored after the products that run meanwhile.
    __device__ __forceinline__ void issue(u32x4* lds, int stage, int K, int wave) {
        const int c = stage * kStageChunks + chunk;
        constexpr int per_chunk = OP == kOpBf16 ? 8 : kMxBlock;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if constexpr (DIRECT) {
                const uint8_t* p = c * per_chunk < K ? row[i] + (size_t)c * 16 : (const uint8_t*)kZeroChunk;
                __builtin_amdgcn_global_load_lds((const u32x4*)p, lds + (i * NW + wave) * 64, 16, 0, 0);
            } else {
                held[i] = load_chunk<OP>(row[i], c, K);
            }
        }
    }
    __device__ __forceinline__ void store(u32x4* lds, int wave, int lane) {
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < PER; ++i) lds[(i * NW + wave) * 64 + lane] = held[i];
    }
};

// One row's scales of a stage as the four steps' MFMAs take them: byte s the
// scale of block 2 s + half.  Blocks behind the last column get 2^-127.
__device__ __forceinline__ uint32_t stage_scales(const uint8_t* scales, int stage, int K, int half) {
    const int left = (K + kMxBlock - 1) / kMxBlock - stage * 8;
    uint64_t w = *(const uint64_t*)(scales + (size_t)stage * 8);
    if (left < 8) w &= ((uint64_t)1 << (8 * left)) - 1;
    return __builtin_amdgcn_perm((uint32_t)(w >> 32), (uint32_t)w, half ? 0x07050301u : 0x06040200u);
}

template <int OP, int S>
__device__ __forceinline__ f32x16 mma_step(u32x4 a, u32x4 b, f32x16 c, uint32_t sa, uint32_t sb) {
    if constexpr (OP == kOpBf16) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    } else {
        const i32x8 av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
        const i32x8 bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bv, c, 4, 4, S, (int)sa, S, (int)sb);
    }
}

// A 32 x 32 accumulator (lane: column lane & 31, row (i & 3) + 8 (i >> 2) +
// 4 (lane >> 5)) as the 16 consecutive rows from 16 (lane >> 5) on.
__device__ __forceinline__ void consecutive_rows(const f32x16& acc, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i]), __float_as_uint(acc[8 + i]), false, false);
        auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[4 + i]), __float_as_uint(acc[12 + i]), false, false);
        v[i] = __uint_as_float(p[0]);
        v[4 + i] = __uint_as_float(p[1]);
        v[8 + i] = __uint_as_float(q[0]);
        v[12 + i] = __uint_as_float(q[1]);
    }
}

// The larger of this lane's and the lane's 32 further.
__device__ __forceinline__ uint32_t pair_max(uint32_t v) {
    auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(p[0], p[1]);
}

// 16 consecutive outputs from column n on of batch row m, in a block of 32 that
// this lane shares with the one 32 further; every lane of the wave calls it.
template <int EPI>
__device__ __forceinline__ void epilogue16(const GemmArgs& g, float* v, int64_t m, int n) {
    const bool live = m < g.M;
    if (EPI != kEpiMasked) {
        if (g.bias) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += n + i < g.N ? g.bias[n + i] : 0.0f;
        }
        if (g.relu) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = v[i] <= 0.0f ? 0.0f : v[i];   // NaN stays
        }
    }
    if constexpr (EPI == kEpiMx4 || EPI == kEpiKept) {
        // values behind the last column are zero in the block
        if (n + 16 > g.N) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = n + i < g.N ? v[i] : 0.0f;
        }
    }
    const int block = n / kMxBlock;
    const bool in_block = live && block * kMxBlock < g.N;
    if constexpr (EPI == kEpiMx4) {
        const int code = mx4_code(pair_max(top_bits<16>(v)));
        const u32x2 p = {to_e2m1x8(v, code), to_e2m1x8(v + 8, code)};
        if (in_block) {
            *(u32x2*)(g.q.codes + m * g.q.ld + n / 2) = p;
            if (!(n & 16)) g.q.scales[m * g.q.ld_scales + block] = (uint8_t)code;
        }
        return;
    }
    if constexpr (EPI == kEpiKept) {
        if (g.q.codes) {
            uint32_t top = pair_max(top_bits<16>(v));
            if (__any(top >= 0x7f800000u)) {
                const uint32_t fin = pair_max(finite_top_bits<16>(v));
                top = top >= 0x7f800000u ? fin : top;
            }
            const int code = mx8_code(top);
            const u32x4 p = {to_e4m3x4(v, code), to_e4m3x4(v + 4, code), to_e4m3x4(v + 8, code), to_e4m3x4(v + 12, code)};
            if (in_block) {
                *(u32x4*)(g.q.codes + m * g.q.ld + n) = p;
                if (!(n & 16)) g.q.scales[m * g.q.ld_scales + block] = (uint8_t)code;
            }
        }
        if (!g.y) return;
    }
    if (!live || n >= g.N) return;
    if constexpr (EPI == kEpiMasked) {
        if (g.mask_type == kMaskMx8) {   // a whole half block is there to be read
            const u32x4 c = *(const u32x4*)(g.mask + m * g.ld_mask + n);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = (c[i / 4] >> (8 * (i % 4))) & 0x7fu ? v[i] : 0.0f;
        } else if (g.mask_type == kMaskBf16) {
            const uint16_t* row = (const uint16_t*)g.mask + m * g.ld_mask;
            const u32x4 c0 = Row8<uint16_t>::load_raw(row, n, g.N), c1 = Row8<uint16_t>::load_raw(row, n + 8, g.N);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t w = i < 8 ? c0[(i / 2) & 3] : c1[(i / 2) & 3];
                v[i] = (w >> (16 * (i & 1))) & 0x7fffu ? v[i] : 0.0f;
            }
        }
    }
    if constexpr (EPI == kEpiF32) {
        float* row = (float*)g.y + m * g.ldy;
        Row8<float>::store(row, n, g.N, v);
        Row8<float>::store(row, n + 8, g.N, v + 8);
    } else {
        uint16_t* row = (uint16_t*)g.y + m * g.ldy;
        Row8<uint16_t>::store(row, n, g.N, v);
        Row8<uint16_t>::store(row, n + 8, g.N, v + 8);
    }
}

template <int OP, int BN, int BM, int WN, int WM, bool DA, bool DB, int EPI>
__global__ void __launch_bounds__(64 * WN * WM) layer_gemm_kernel(GemmArgs g) {
    constexpr int NW = WN * WM, TN = BN / (32 * WN), TM = BM / (32 * WM);
    __shared__ u32x4 ring0[(BN + BM) * kStageChunks];
    __shared__ u32x4 ring1[(BN + BM) * kStageChunks];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int wn = wave % WN, wm = wave / WN;

    // Tiles of the same batch rows go to the same XCD (workgroups are dealt to
    // the eight XCDs in turn), so that its L2 reads those rows once.
    const uint32_t tiles = g.tiles_n * g.tiles_m, per_xcd = (tiles + 7) / 8;
    const uint32_t t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (t >= tiles) return;
    const int n0 = (int)(t % g.tiles_n) * BN;
    const int64_t m0 = (int64_t)(t / g.tiles_n) * BM;

    StageCopy<OP, BN, NW, DA> ca;
    StageCopy<OP, BM, NW, DB> cb;
    ca.init(g.a, n0, g.N, wave, lane);
    cb.init(g.b, m0, g.M, wave, lane);
    const uint8_t *sa[TN], *sb[TM];
    if constexpr (OP == kOpMx4) {
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int r = n0 + (wn * TN + i) * 32 + col;
            sa[i] = g.a.scales + (int64_t)(r < g.N ? r : g.N - 1) * g.a.ld_scales;
        }
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            const int64_t r = m0 + (wm * TM + j) * 32 + col;
            sb[j] = g.b.scales + (r < g.M ? r : g.M - 1) * g.b.ld_scales;
        }
    }
    f32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    constexpr int stage_cols = OP == kOpBf16 ? 64 : 256;
    const int stages = (g.K + stage_cols - 1) / stage_cols;
    auto compute = [&](const u32x4* lds, int stage) {
        uint32_t va[TN], vb[TM];
        if constexpr (OP == kOpMx4) {
#pragma unroll
            for (int i = 0; i < TN; ++i) va[i] = stage_scales(sa[i], stage, g.K, half);
#pragma unroll
            for (int j = 0; j < TM; ++j) vb[j] = stage_scales(sb[j], stage, g.K, half);
        }
        sfor<4>([&](auto S) {
            const int c = (2 * CV(S) + half) ^ (col & 7);
            u32x4 fa[TN], fb[TM];
#pragma unroll
            for (int i = 0; i < TN; ++i) fa[i] = lds[((wn * TN + i) * 32 + col) * kStageChunks + c];
#pragma unroll
            for (int j = 0; j < TM; ++j) fb[j] = lds[(BN + (wm * TM + j) * 32 + col) * kStageChunks + c];
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    acc[i][j] = mma_step<OP, CV(S)>(fa[i], fb[j], acc[i][j], OP == kOpMx4 ? va[i] : 0u, OP == kOpMx4 ? vb[j] : 0u);
        });
    };
    auto step = [&](u32x4* now, u32x4* next, int stage) {
        const bool more = stage + 1 < stages;
        if (more) {
            ca.issue(next, stage + 1, g.K, wave);
            cb.issue(next + BN * kStageChunks, stage + 1, g.K, wave);
        }
        compute(now, stage);
        if (more) {
            ca.store(next, wave, lane);
            cb.store(next + BN * kStageChunks, wave, lane);
            wait_vmcnt<0>();
            lds_barrier();
        }
    };
    ca.issue(ring0, 0, g.K, wave);
    cb.issue(ring0 + BN * kStageChunks, 0, g.K, wave);
    ca.store(ring0, wave, lane);
    cb.store(ring0 + BN * kStageChunks, wave, lane);
    wait_vmcnt<0>();
    lds_barrier();
    for (int s = 0; s < stages; s += 2) {
        step(ring0, ring1, s);
        if (s + 1 < stages) step(ring1, ring0, s + 1);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            float v[16];
            consecutive_rows(acc[i][j], v);
            epilogue16<EPI>(g, v, m0 + (wm * TM + j) * 32 + col, n0 + (wn * TN + i) * 32 + 16 * half);
        }
}

template <int OP, bool DA, bool DB, int EPI>
hipError_t launch_layer_gemm(GemmArgs g, int n_cu, hipStream_t stream) {
    auto tiles = [&](int b) { return (uint64_t)((g.N + b - 1) / b) * (uint64_t)((g.M + b - 1) / b); };
    const int b = tiles(128) >= (uint64_t)n_cu ? 128 : 64;
    g.tiles_n = (uint32_t)((g.N + b - 1) / b);
    g.tiles_m = (uint32_t)((g.M + b - 1) / b);
    const dim3 grid((g.tiles_n * g.tiles_m + 7) / 8 * 8);
    if (b == 128) hipLaunchKernelGGL((layer_gemm_kernel<OP, 128, 128, 2, 2, DA, DB, EPI>), grid, dim3(256), 0, stream, g);
    else hipLaunchKernelGGL((layer_gemm_kernel<OP, 64, 64, 2, 2, DA, DB, EPI>), grid, dim3(256), 0, stream, g);
    return hipGetLastError();
}

}  // namespace
}  // namespace donerf
