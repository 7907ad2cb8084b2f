// layer_gemm.h - the products of the layer operators on gfx950: for batch rows b
// (M of them) and weight rows a (N), y[m][n] = sum_k a[n][k] b[m][k], on bf16
// MFMAs or block-scaled E2M1 ones, with what follows the product in its epilogue.
//
// A workgroup computes a tile of BN weight rows by BM batch rows in stages of
// 128 bytes of every row (64 bf16 or 256 E2M1 columns).  In LDS a row's eight
// 16-byte chunks are permuted (row_key), so that reads of one chunk of sixteen rows
// meet all 64 banks.  Two such stages alternate in two arrays: the copy of one runs
// while the other is multiplied, but not within an E2M1 workgroup, where a stage's
// scales are loaded behind the next stage's copies and arrive after them: there only
// the other workgroup of the compute unit multiplies meanwhile.
//
// The weights are the MFMA's A operand and the batch its B operand, so a lane's
// accumulators are 16 of a block's 32 outputs of one batch row, which it shares
// with the lane 32 further: bias, ReLU, the scales of microscaled outputs and wide
// stores need no more than exchanges of registers between the two.
#pragma once

#include "internal.h"
#include "mx.h"

namespace donerf {
namespace {

constexpr int kOpBf16 = 0, kOpMx4 = 1;
constexpr int kStageBytes = 128;   // of each row
constexpr int kStageChunks = kStageBytes / 16;

// What follows the product.
constexpr int kEpiBf16 = 0;      // y bf16
constexpr int kEpiF32 = 1;       // y fp32
constexpr int kEpiMx4 = 2;       // y E2M1
constexpr int kEpiKept = 3;      // y bf16 and its E4M3 checkpoint, either may be absent
constexpr int kEpiMaskMx8 = 4;   // y bf16, zero where the ReLU's output (E4M3) is
constexpr int kEpiMaskBf16 = 5;  // the same, the ReLU's output in bf16
constexpr bool masked(int epi) { return epi == kEpiMaskMx8 || epi == kEpiMaskBf16; }

// In LDS, chunk c of a row of CHUNKS 16-byte chunks lies at c ^ row_key(row): sixteen
// consecutive rows' chunks c then cover the banks' 256 bytes, to which the row's own
// place adds what CHUNKS leaves of it.
template <int CHUNKS>
__device__ __forceinline__ int row_key(int row) {
    if constexpr (CHUNKS >= 16) return row & 15;
    else return (row / (16 / CHUNKS)) & (CHUNKS - 1);
}

// 16 zero bytes: what a lane copies in place of chunks behind the last column.
__device__ const uint32_t kZeroChunk[4] = {0, 0, 0, 0};

// Copies of one operand's rows [row0, row0 + ROWS) into a stage in LDS: straight
// into it (DIRECT: rows of whole, 16-byte aligned chunks), or, for bf16 rows of
// any other kind, by way of registers that are stored after the products which
// run meanwhile.
template <int OP, int ROWS, int NW, bool DIRECT>
struct StageCopy {
    static constexpr int PER = ROWS / 8 / NW;   // copies per wave, 8 rows each
    static_assert(ROWS % (8 * NW) == 0, "rows split evenly over the waves");
    static_assert(DIRECT || OP == kOpBf16, "microscaled rows are aligned");
    const uint8_t* row[DIRECT ? PER : 1];   // of this lane, in each copy
    int64_t off[DIRECT ? 1 : PER];          // the same in values
    u32x4 held[DIRECT ? 1 : PER];
    Bf16Rows any;
    int64_t first;             // row of this lane in the wave's first copy
    int chunk;                 // of this lane, in every row
    __device__ __forceinline__ void init(const MxIn& src, int64_t row0, int64_t rows, int K, int wave, int lane) {
        // copies of a wave are 8 NW rows apart, which the key does not see
        static_assert(NW % 2 == 0, "row_key");
        chunk = (lane & 7) ^ row_key<kStageChunks>(wave * 8 + (lane >> 3));
        first = row0 + wave * 8 + (lane >> 3);
        if constexpr (DIRECT) {
#pragma unroll
            for (int i = 0; i < PER; ++i) row[i] = src.codes + row_of(i, rows) * src.ld;
        } else {
            any = Bf16Rows((const uint16_t*)src.codes, src.ld / 2, rows, K);
#pragma unroll
            for (int i = 0; i < PER; ++i) off[i] = row_of(i, rows) * any.ld;
        }
    }
    // rows behind the last one repeat it: their results are not stored
    __device__ __forceinline__ int64_t row_of(int i, int64_t rows) const {
        const int64_t r = first + i * NW * 8;
        return r < rows ? r : rows - 1;
    }
    __device__ __forceinline__ void issue(u32x4* lds, int stage, int K, int wave) {
        const int c = stage * kStageChunks + chunk;
        constexpr int per_chunk = OP == kOpBf16 ? 8 : kMxBlock;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if constexpr (DIRECT) {
                const uint8_t* p = row[i] + (size_t)c * 16;
                p = c * per_chunk < K ? p : (const uint8_t*)kZeroChunk;
                __builtin_amdgcn_global_load_lds((const u32x4*)p, lds + (i * NW + wave) * 64, 16, 0, 0);
            } else {
                held[i] = any.load_at(off[i] + c * 8, c * 8);
            }
        }
    }
    __device__ __forceinline__ void store(u32x4* lds, int stage, int wave, int lane) {
        if constexpr (!DIRECT) {
            const int c = stage * kStageChunks + chunk;
            if ((stage + 1) * kStageChunks * 8 > any.cols)   // the stage that holds the rows' ends
#pragma unroll
                for (int i = 0; i < PER; ++i) held[i] = any.fix(held[i], row_of(i, any.rows), c * 8);
#pragma unroll
            for (int i = 0; i < PER; ++i) lds[(i * NW + wave) * 64 + lane] = held[i];
        }
    }
};

// Where chunk c (8 columns) of row m of a stage with CHUNKS chunks a row lies, if
// the stage is read by columns: a transposing read takes 64 bytes of eight rows at
// once, and rows that follow each other start 64 bytes apart in the banks.
template <int CHUNKS>
__device__ __forceinline__ int column_slot(int m, int c) {
    return m * CHUNKS + (c ^ ((m & (CHUNKS >= 16 ? 3 : CHUNKS >= 8 ? 1 : 0)) << 2));
}

// The MFMA operand of 32 columns from column n on and 16 rows from row m on of
// such a stage: lane l has column n + (l & 31), rows m + 8 (l >> 5) + (0..7).
// Sixteen lanes read four rows of 16 columns, 8 bytes each, and get a column each.
template <int CHUNKS>
__device__ __forceinline__ bf16x8 read_columns(const u32x4* lds, int m, int n, int lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int col = n + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int row = m + 8 * (lane >> 5) + ((lane >> 2) & 3);
    struct { s16x4 lo, hi; } v;
    const char* base = (const char*)lds;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + column_slot<CHUNKS>(row, col >> 3) * 16 + (col & 7) * 2));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + column_slot<CHUNKS>(row + 4, col >> 3) * 16 + (col & 7) * 2));
    return __builtin_bit_cast(bf16x8, v);
}

// Copies of a bf16 operand that is transposed in memory: a stage is ROWS of its
// rows (the products' terms) by COLS of its columns.  Rows behind `rows` are zeros.
template <int ROWS, int COLS, int NW, bool DIRECT>
struct ColumnCopy {
    static constexpr int CHUNKS = COLS / 8, EACH = 64 / CHUNKS;   // rows per copy of 64 chunks
    static constexpr int PER = ROWS / EACH / NW;
    static_assert(ROWS % (EACH * NW) == 0 && CHUNKS <= 64, "rows split evenly over the waves");
    Bf16Rows any;
    u32x4 held[DIRECT ? 1 : PER];
    int64_t begin, end;   // rows
    int64_t off;          // of this lane's chunk in the first stage, in values
    int row, col, col0;   // of this lane in the wave's first copy; first column of the stage
    __device__ __forceinline__ void init(const uint16_t* p, int64_t ld, int64_t rows, int cols, int64_t begin_, int64_t end_,
                                         int col0_, int wave, int lane) {
        any = Bf16Rows(p, ld, rows, cols);
        begin = begin_;
        end = end_;
        row = wave * EACH + lane / CHUNKS;
        // the chunk whose slot is the lane's; the swizzle goes by the row's low
        // bits, which further copies of a wave, multiples of four rows away, keep
        static_assert((EACH * NW) % 4 == 0, "swizzle");
        col0 = col0_;
        col = col0_ + ((lane % CHUNKS) ^ (column_slot<CHUNKS>(row, 0) - row * CHUNKS)) * 8;
        off = (begin + row) * ld + col;
    }
    __device__ __forceinline__ void issue(u32x4* lds, int stage, int wave) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int64_t first = (int64_t)stage * ROWS + i * EACH * NW, at = off + first * any.ld;
            if constexpr (DIRECT) {
                const uint8_t* p = (const uint8_t*)(any.base + at);
                p = begin + first + row < end && col < any.cols ? p : (const uint8_t*)kZeroChunk;
                __builtin_amdgcn_global_load_lds((const u32x4*)p, lds + (i * NW + wave) * 64, 16, 0, 0);
            } else {
                held[i] = any.load_at(at, col);   // rows from `end` on are cleared afterwards
            }
        }
    }
    __device__ __forceinline__ void store(u32x4* lds, int stage, int wave, int lane) {
        if constexpr (!DIRECT) {
            if (col0 + COLS > any.cols || begin + (int64_t)(stage + 1) * ROWS > end)
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int64_t m = begin + (int64_t)stage * ROWS + row + i * EACH * NW;
                    held[i] = m < end ? any.fix(held[i], m, col) : u32x4{0, 0, 0, 0};
                }
#pragma unroll
            for (int i = 0; i < PER; ++i) lds[(i * NW + wave) * 64 + lane] = held[i];
        }
    }
};

// The eight scales of one row's stage as the four steps' MFMAs take them: byte s
// the scale of block 2 s + half.  Blocks behind the last column get 2^-127.
__device__ __forceinline__ uint32_t pack_scales(uint64_t w, int stage, int K, int half) {
    const int left = (K + kMxBlock - 1) / kMxBlock - stage * 8;
    if (left < 8) w = left <= 0 ? 0 : w & (((uint64_t)1 << (8 * left)) - 1);
    return __builtin_amdgcn_perm((uint32_t)(w >> 32), (uint32_t)w, half ? 0x07050301u : 0x06040200u);
}
__device__ __forceinline__ uint32_t stage_scales(const uint8_t* scales, int stage, int K, int half) {
    const int at = stage * 8 * kMxBlock < K ? stage * 8 : 0;
    return pack_scales(*(const uint64_t*)(scales + at), stage, K, half);
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

// A 32 x 32 accumulator holds, in a lane, 16 rows of column lane & 31: four
// consecutive ones, from 4 (lane >> 5) on, of every eight.  Where they are stored, a
// lane shall hold the 16 consecutive ones from 16 (lane >> 5) on instead: with four
// registers a (b) for the first (third) or the second (fourth) eight rows, whatever
// their type, this exchange makes a the first half of eight consecutive rows and b
// the second.  It is its own inverse.
__device__ __forceinline__ void exchange(uint32_t& a, uint32_t& b) {
    const auto p = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = p[0];
    b = p[1];
}

// The larger of this lane's and the lane's 32 further.
__device__ __forceinline__ uint32_t pair_max(uint32_t v) {
    auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(p[0], p[1]);
}

// The bias of the 32 outputs from column n on where a lane's accumulators start
// from it; zeros without one.
__device__ __forceinline__ f32x16 bias_rows(const GemmArgs& g, int n, int half) {
    f32x16 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int at = n + 8 * q + 4 * half;
        float b[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (g.bias && at + 4 <= g.N) {
            __builtin_memcpy(b, g.bias + at, sizeof b);
        } else if (g.bias) {
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = g.bias[at + i < g.N ? at + i : g.N - 1];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * q + i] = b[i];
    }
    return v;
}

// What a masked epilogue reads for the 32 outputs from n0 on of 32 batch rows from
// m0 on: loaded early, used late.
struct Mask16 {
    u32x4 lo, hi;
};
template <int EPI>
__device__ __forceinline__ Mask16 load_mask(const GemmArgs& g, int64_t m0, int n0, int lane) {
    Mask16 k;
    const int n = n0 + 16 * (lane >> 5);
    int64_t r = m0 + (lane & 31);
    r = r < g.M ? r : g.M - 1;
    if constexpr (EPI == kEpiMaskMx8) {
        // a half block is whole in memory; behind the last block any will do
        const int last = (g.N - 1) / kMxBlock * kMxBlock + 16;
        k.lo = *(const u32x4*)(g.mask + r * g.ld_mask + (n < last ? n : last));
    } else if constexpr (EPI == kEpiMaskBf16) {
        const Bf16Rows x((const uint16_t*)g.mask, g.ld_mask, g.M, g.N);
        k.lo = x.load(r, n);
        k.hi = x.load(r, n + 8);
        if (n0 + 32 > g.N) {
            k.lo = x.fix(k.lo, r, n);
            k.hi = x.fix(k.hi, r, n + 8);
        }
    }
    return k;
}

// A tile's results on their way out, ROWS batch rows by COLS outputs: waves put
// theirs into LDS, then all threads store whole rows.  A wave's own 32 outputs of 32
// rows would be that many pieces of 16 to 64 bytes (stored like that, six 4-bit hidden
// layers of 640000 rows took 412 us, and 186 us without their stores).  In LDS, a row's
// 16-byte chunks are permuted (row_key).
template <int EPI, int ROWS, int COLS>
struct Outgoing {
    static constexpr bool kY = EPI != kEpiMx4, kQ = EPI == kEpiMx4 || EPI == kEpiKept;
    static constexpr int kYChunks = kY ? COLS * (EPI == kEpiF32 ? 4 : 2) / 16 : 0;    // per row
    static constexpr int kQChunks = !kQ ? 0 : EPI == kEpiMx4 ? COLS / 32 : COLS / 16;
    static constexpr int kBlocks = COLS / kMxBlock;                                     // scales per row
    static constexpr int kAt = ROWS * kYChunks, kScaleAt = kAt + ROWS * kQChunks;
    static constexpr int kSize = kScaleAt + (kQ ? ROWS * kBlocks / 16 : 0);             // chunks
    static_assert(ROWS * kBlocks % 16 == 0, "whole chunks");

    template <int CHUNKS>
    __device__ static __forceinline__ int slot(int row, int c) { return row * CHUNKS + (c ^ row_key<CHUNKS>(row)); }

    // What follows the product for the accumulator of rows [r0, r0 + 32) and
    // outputs [c0, c0 + 32) of the tile, which starts at output n_tile.
    __device__ static __forceinline__ void put(u32x4* lds, const GemmArgs& g, const f32x16& acc, const Mask16& mask, int r0,
                                               int c0, int n_tile, int lane) {
        const int half = lane >> 5, row = r0 + (lane & 31), n0 = n_tile + c0;
        const float floor = g.relu ? 0.0f : -__builtin_inff();
        float v[16];   // outputs n0 + 8 (i / 4) + 4 half + i % 4
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            v[i] = acc[i];
            // NaN stays.  E2M1 codes have their ReLU afterwards
            if constexpr (!masked(EPI) && EPI != kEpiMx4) v[i] = __builtin_elementwise_maximum(v[i], floor);
        }
        if constexpr (EPI == kEpiMaskMx8) {
            uint32_t d[4] = {mask.lo.x, mask.lo.z, mask.lo.y, mask.lo.w};
            exchange(d[0], d[2]);
            exchange(d[1], d[3]);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = d[i / 4] & (0x7fu << (8 * (i % 4))) ? v[i] : 0.0f;
        } else if constexpr (EPI == kEpiMaskBf16) {
            uint32_t d[8] = {mask.lo.x, mask.lo.y, mask.hi.x, mask.hi.y, mask.lo.z, mask.lo.w, mask.hi.z, mask.hi.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) exchange(d[i], d[4 + i]);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = d[i / 2] & (0x7fffu << (16 * (i % 2))) ? v[i] : 0.0f;
        }
        if constexpr (kQ)
            if (n0 + 32 > g.N)   // values behind the last column are zero in the block
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = n0 + 8 * (i / 4) + 4 * half + i % 4 < g.N ? v[i] : 0.0f;
        if constexpr (EPI == kEpiMx4) {
            float t = g.relu ? 0.0f : __builtin_fabsf(v[0]);
            if (g.relu) {
#pragma unroll
                for (int i = 0; i < 16; ++i) t = __builtin_elementwise_maximum(t, v[i]);
            } else {
#pragma unroll
                for (int i = 1; i < 16; ++i) t = __builtin_elementwise_maximum(t, __builtin_fabsf(v[i]));
            }
            const int code = mx4_code(pair_max(abs_bits(t)));
            // four outputs are two bytes; this lane's of the first and second eight
            // rows, of the third and fourth
            uint32_t a = to_e2m1x8(v, code), b = to_e2m1x8(v + 8, code);
            exchange(a, b);
            u32x2 p = {__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(b, a, 0x07060302u)};
            if (g.relu) p = u32x2{relu_e2m1x8(p.x), relu_e2m1x8(p.y)};
            ((u32x2*)(lds + kAt))[slot<kQChunks>(row, c0 / 32) * 2 + half] = p;
            if (lane < 32) ((uint8_t*)(lds + kScaleAt))[row * kBlocks + c0 / kMxBlock] = (uint8_t)code;
        }
        if constexpr (EPI == kEpiKept) {
            if (g.q.codes) {
                uint32_t top = pair_max(top_bits<16>(v));
                const bool bad = __any(top >= kInfBits);
                if (bad) {
                    const uint32_t fin = pair_max(finite_top_bits<16>(v));
                    top = top >= kInfBits ? fin : top;
                }
                const int code = mx8_code(top);
                // values other than zero that would round to it: few tiles have any
                uint32_t low = 0xffffffffu;
#pragma unroll
                for (int i = 0; i < 16; ++i) low = min(low, (g.relu ? __float_as_uint(v[i]) : abs_bits(v[i])) - 1u);
                const bool tiny = __any(low < __float_as_uint(least_e4m3(code)));
                uint32_t p[4];
                if (tiny) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = to_e4m3x4(v + 4 * i, code);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = round_e4m3x4(v + 4 * i, code);
                }
                if (bad)
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = e4m3_not_finite(p[i], v + 4 * i);
                exchange(p[0], p[2]);
                exchange(p[1], p[3]);
                lds[kAt + slot<kQChunks>(row, c0 / 16 + half)] = u32x4{p[0], p[2], p[1], p[3]};
                if (lane < 32) ((uint8_t*)(lds + kScaleAt))[row * kBlocks + c0 / kMxBlock] = (uint8_t)code;
            }
        }
        if constexpr (EPI == kEpiF32) {
            // four outputs are a chunk
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                u32x4 p;
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = __float_as_uint(v[4 * q + i]);
                lds[slot<kYChunks>(row, c0 / 4 + 2 * q + half)] = p;
            }
        } else if constexpr (kY) {
            uint32_t p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) exchange(p[i], p[4 + i]);
            lds[slot<kYChunks>(row, c0 / 8 + 2 * half)] = u32x4{p[0], p[1], p[4], p[5]};
            lds[slot<kYChunks>(row, c0 / 8 + 2 * half + 1)] = u32x4{p[2], p[3], p[6], p[7]};
        }
    }

    // Store instructions of a wave of THREADS / 64 for a tile whose rows all exist,
    // at the least: every instruction has some row's first chunk.
    static constexpr int stores_y(int threads) { return ROWS * kYChunks / threads; }
    static constexpr int stores_q(int threads) { return ROWS * kQChunks / threads; }

    // The tile at batch row m0 and output n_tile goes to memory.
    template <int THREADS>
    __device__ static __forceinline__ void store(const u32x4* lds, const GemmArgs& g, int64_t m0, int n_tile, int tid) {
        const int rows = g.M - m0 < ROWS ? (int)(g.M - m0) : ROWS;
        const bool whole = n_tile + COLS <= g.N;
        if constexpr (kY) {
            if (EPI != kEpiKept || g.y) {
                constexpr int E = EPI == kEpiF32 ? 4 : 8;   // outputs of a chunk
#pragma unroll
                for (int q = 0; q < (ROWS * kYChunks + THREADS - 1) / THREADS; ++q) {
                    if (ROWS * kYChunks % THREADS && q * THREADS + tid >= ROWS * kYChunks) break;
                    const int at = q * THREADS + tid, row = at / kYChunks, c = at % kYChunks, n = n_tile + c * E;
                    const u32x4 v = lds[slot<kYChunks>(row, c)];
                    uint8_t* y = g.y + ((m0 + row) * g.ldy + n) * (16 / E);
                    if (row < rows && (whole || n + E <= g.N)) {
                        __builtin_memcpy(y, &v, 16);
                    } else if (row < rows) {
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            if (n + i >= g.N) continue;
                            if constexpr (E == 4) ((float*)y)[i] = __uint_as_float(v[i]);
                            else ((uint16_t*)y)[i] = (uint16_t)(v[i / 2] >> (16 * (i & 1)));
                        }
                    }
                }
            }
        }
        if constexpr (kQ) {
            if (EPI == kEpiKept && !g.q.codes) return;
            constexpr int E = COLS / kQChunks;              // outputs of a chunk: a block, or half of one
#pragma unroll
            for (int q = 0; q < (ROWS * kQChunks + THREADS - 1) / THREADS; ++q) {
                if (ROWS * kQChunks % THREADS && q * THREADS + tid >= ROWS * kQChunks) break;
                const int at = q * THREADS + tid, row = at / kQChunks, c = at % kQChunks, n = n_tile + c * E;
                const u32x4 v = lds[kAt + slot<kQChunks>(row, c)];
                if (row < rows && n / kMxBlock * kMxBlock < g.N)
                    *(u32x4*)(g.q.codes + (m0 + row) * g.q.ld + (EPI == kEpiMx4 ? n / 2 : n)) = v;
            }
            if (tid < rows) {
                const uint8_t* from = (const uint8_t*)(lds + kScaleAt) + tid * kBlocks;
                uint8_t* to = g.q.scales + (m0 + tid) * g.q.ld_scales + n_tile / kMxBlock;
                const int left = (g.N - n_tile + kMxBlock - 1) / kMxBlock;
                if (left >= kBlocks) {
                    __builtin_memcpy(to, from, kBlocks);
                } else {
#pragma unroll
                    for (int i = 0; i < kBlocks; ++i)
                        if (i < left) to[i] = from[i];
                }
            }
        }
    }
};

// TA: the weights are transposed in memory, a[k][n] (bf16 only).
// Measured, a call's results at the rate of their products: bf16 16,384 x 2048 x 2048
// on 256 x 256 tiles 150 us forward (920 TFLOP/s) and 158 us dx (870 TFLOP/s; matrix
// pipes 35 % busy, half of the waves' time waits for the next stage and the barrier
// that publishes it), dx 190 us on 128 x 128; E2M1 8192 x 4096 x 4096 on 128 x 128 129
// us (2.1 PFLOP/s; a stage's scales wait for the next one's copies, see above).
template <int OP, int BN, int BM, int WN, int WM, bool TA, bool DA, bool DB, int EPI>
__global__ void __launch_bounds__(64 * WN * WM, 2) layer_gemm_kernel(GemmArgs g) {
    constexpr int NW = WN * WM, TN = BN / (32 * WN), TM = BM / (32 * WM);
    static_assert(!TA || OP == kOpBf16, "transposed weights are bf16");
    using Out = Outgoing<EPI, 32 * WM, BN>;   // of the results, a block of each wave at a time
    __shared__ u32x4 ring0[(BN + BM) * kStageChunks];
    __shared__ u32x4 ring1[(BN + BM) * kStageChunks];
    static_assert(Out::kSize <= (BN + BM) * kStageChunks, "results pass through the stages' memory");
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

    constexpr int stage_cols = OP == kOpBf16 ? 64 : 256;
    const int stages = (g.K + stage_cols - 1) / stage_cols;
    StageCopy<OP, BN, NW, DA || OP != kOpBf16> ca;
    ColumnCopy<64, BN, NW, DA> ct;
    StageCopy<OP, BM, NW, DB> cb;
    if constexpr (TA) ct.init((const uint16_t*)g.a.codes, g.a.ld / 2, g.K, g.N, 0, g.K, n0, wave, lane);
    else ca.init(g.a, n0, g.N, g.K, wave, lane);
    cb.init(g.b, m0, g.M, g.K, wave, lane);
    const uint8_t *sa[TN], *sb[TM];
    if constexpr (OP == kOpMx4) {
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const int r = n0 + (wn * TN + i) * 32 + col;
            sa[i] = g.a.scales + (int64_t)(r < g.N ? r : g.N - 1) * g.a.ld_scales;
        }
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            const int64_t r = m0 + (j * WM + wm) * 32 + col;
            sb[j] = g.b.scales + (r < g.M ? r : g.M - 1) * g.b.ld_scales;
        }
    }
    f32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        const f32x16 bias = bias_rows(g, n0 + (wn * TN + i) * 32, half);
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = bias;
    }

    auto issue = [&](u32x4* lds, int stage) {
        if constexpr (TA) ct.issue(lds, stage, wave);
        else ca.issue(lds, stage, g.K, wave);
        cb.issue(lds + BN * kStageChunks, stage, g.K, wave);
    };
    auto arrive = [&](u32x4* lds, int stage) {
        if constexpr (TA) ct.store(lds, stage, wave, lane);
        else ca.store(lds, stage, wave, lane);
        cb.store(lds + BN * kStageChunks, stage, wave, lane);
        wait_vmcnt<0>();
        lds_barrier();
    };
    auto compute = [&](const u32x4* lds, int stage) {
        uint32_t va[TN], vb[TM];
        if constexpr (OP == kOpMx4) {
#pragma unroll
            for (int i = 0; i < TN; ++i) va[i] = stage_scales(sa[i], stage, g.K, half);
#pragma unroll
            for (int j = 0; j < TM; ++j) vb[j] = stage_scales(sb[j], stage, g.K, half);
        }
        sfor<4>([&](auto S) {
            const int c = (2 * CV(S) + half) ^ row_key<kStageChunks>(col);
            u32x4 fa[TN], fb[TM];
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                if constexpr (TA) fa[i] = __builtin_bit_cast(u32x4, read_columns<BN / 8>(lds, CV(S) * 16, (wn * TN + i) * 32, lane));
                else fa[i] = lds[((wn * TN + i) * 32 + col) * kStageChunks + c];
            }
#pragma unroll
            for (int j = 0; j < TM; ++j) fb[j] = lds[(BN + (j * WM + wm) * 32 + col) * kStageChunks + c];
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    acc[i][j] = mma_step<OP, CV(S)>(fa[i], fb[j], acc[i][j], OP == kOpMx4 ? va[i] : 0u, OP == kOpMx4 ? vb[j] : 0u);
        });
    };
    auto step = [&](u32x4* now, u32x4* next, int stage) {
        const bool more = stage + 1 < stages;
        if (more) issue(next, stage + 1);
        compute(now, stage);
        if (more) arrive(next, stage + 1);
    };
    issue(ring0, 0);
    arrive(ring0, 0);
    for (int s = 0; s < stages; s += 2) {
        step(ring0, ring1, s);
        if (s + 1 < stages) step(ring1, ring0, s + 1);
    }
    lds_barrier();
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        u32x4* const out = j & 1 ? ring1 : ring0;
        Mask16 mask[TN];
#pragma unroll
        for (int i = 0; i < TN; ++i) mask[i] = load_mask<EPI>(g, m0 + (j * WM + wm) * 32, n0 + (wn * TN + i) * 32, lane);
        // (a place is written again after a barrier that follows its last readers)
#pragma unroll
        for (int i = 0; i < TN; ++i) Out::put(out, g, acc[i][j], mask[i], wm * 32, (wn * TN + i) * 32, n0, lane);
        lds_barrier();
        if (m0 + j * 32 * WM < g.M) Out::template store<64 * NW>(out, g, m0 + j * 32 * WM, n0, threadIdx.x);
    }
}

// A layer whose weights fit into one workgroup's registers: up to 256 outputs
// (32 per wave) of KS stages of 128 bytes.  They are read once per workgroup, and
// tiles of 64 batch rows stream past them through a ring of three, two ahead, so
// that the batch is read once and nothing else moves but the results.  WN waves
// along the outputs, 8 / WN along the rows.  SRC: how the batch gets there.
// Measured at 256 x 256: 160,000 rows forward with both outputs 55 us (207 MB, 3.8
// TB/s), dx 50 us, E2M1 from bf16 32 us (164 MB, 5.1 TB/s); 640,000 rows from E2M1 to
// E2M1 51 us (174 MB, 3.4 TB/s), to bf16 70 us (415 MB, 5.9 TB/s).  What bounds E2M1 to
// E2M1 is in part that one of the three unrolled steps waits for all copies under way
// before it reads its tile (the compiler's wait: it does not tell the ring's slots
// apart there), so that the ring drains on every third tile; the epilogue's
// instructions and the two barriers of a tile are the rest.
constexpr int kSrcCopies = 0;     // rows of whole, 16-byte aligned chunks: straight into LDS
constexpr int kSrcBf16Rows = 1;   // any bf16 rows: through registers, a tile ahead
constexpr int kSrcF32 = 2;        // fp32 or bf16 rows that become E2M1, likewise
constexpr int kSrcBf16 = 3;
constexpr int kRowsTile = 64;
// LDS: a tile's stages, then its rows' scales, KS words of eight each, or a stage of
// transposed weights, three times; and the results.
constexpr int kLdsPerCu = 160 * 1024;
template <int OP, int KS, int WN, bool TA, int EPI>
struct RowsLds {
    static constexpr int kChunks = kRowsTile * KS * kStageChunks, kScaleWords = OP == kOpMx4 ? kRowsTile * KS * 2 : 0;
    static constexpr int kTile = kChunks + kScaleWords / 4, kRing = TA ? 64 * 32 : 0;
    static constexpr int kSlot = kTile > kRing ? kTile : kRing;
    static constexpr int kBytes = (3 * kSlot + Outgoing<EPI, kRowsTile, 32 * WN>::kSize) * 16;
};
// Workgroups that share a compute unit: two where a tile's batch is small and copied,
// if LDS holds them.  fp32 results of more than 128 outputs take 64 KiB of it: a grid
// of two workgroups per unit there, half of which waited for the other half, took 11.1
// us for 20,000 x 256 x 256 and 17.3 for 50,000; a grid of one takes 9.1 and 15.0.
template <int OP, int KS, int WN, bool TA, int SRC, int EPI>
constexpr int rows_workgroups() {
    return OP == kOpMx4 && KS == 1 && SRC == kSrcCopies && 2 * RowsLds<OP, KS, WN, TA, EPI>::kBytes <= kLdsPerCu ? 2 : 1;
}
template <int OP, int KS, int WN, bool TA, int SRC, int EPI, int WGS = rows_workgroups<OP, KS, WN, TA, SRC, EPI>()>
__global__ void __launch_bounds__(512, WGS * 2) layer_rows_kernel(GemmArgs g) {
    constexpr bool DB = SRC == kSrcCopies, kConvert = SRC == kSrcF32 || SRC == kSrcBf16;
    static_assert(!kConvert || (OP == kOpMx4 && KS == 1), "conversion is to E2M1, of one stage");
    constexpr int NW = 8, WM = NW / WN, RT = kRowsTile, RB = RT / 32 / WM, CP = RT * KS / 8 / NW;
    using Out = Outgoing<EPI, RT, 32 * WN>;
    using Lds = RowsLds<OP, KS, WN, TA, EPI>;
    constexpr int kChunks = Lds::kChunks, kScaleWords = Lds::kScaleWords, kSlot = Lds::kSlot;
    static_assert(WGS * Lds::kBytes <= kLdsPerCu, "workgroups that share a compute unit share its LDS");
    __shared__ u32x4 ring0[kSlot], ring1[kSlot], ring2[kSlot];
    __shared__ u32x4 out[Out::kSize];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int wn = wave % WN, wm = wave / WN;
    const uint32_t tiles = g.tiles_m;

    // ---- the weights
    u32x4 fa[KS][4];
    uint32_t va[KS];
    if constexpr (TA) {
        // stages of 64 rows by all outputs, through the ring, two at a time
        u32x4* const rings[2] = {ring0, ring1};
        sfor<(KS + 1) / 2>([&](auto P) {
            constexpr int S0 = 2 * CV(P), PAIR = KS - S0 < 2 ? 1 : 2;
            ColumnCopy<64, 256, NW, false> ct[PAIR];
            sfor<PAIR>([&](auto S) {
                ct[CV(S)].init((const uint16_t*)g.a.codes, g.a.ld / 2, g.K, g.N, 0, g.K, 0, wave, lane);
                ct[CV(S)].issue(rings[CV(S)], S0 + CV(S), wave);
            });
            sfor<PAIR>([&](auto S) { ct[CV(S)].store(rings[CV(S)], S0 + CV(S), wave, lane); });
            lds_barrier();
            sfor<PAIR>([&](auto S) {
                sfor<4>([&](auto I) {
                    fa[S0 + CV(S)][CV(I)] = __builtin_bit_cast(u32x4, read_columns<32>(rings[CV(S)], CV(I) * 16, wn * 32, lane));
                });
            });
            lds_barrier();
        });
    } else {
        const int64_t r = wn * 32 + col < g.N ? wn * 32 + col : g.N - 1;
        const Bf16Rows rows((const uint16_t*)g.a.codes, g.a.ld / 2, g.N, g.K);
        sfor<KS>([&](auto S) {
            sfor<4>([&](auto I) {
                const int c = CV(S) * kStageChunks + 2 * CV(I) + half;
                if constexpr (OP == kOpBf16) {
                    fa[CV(S)][CV(I)] = rows.fix(rows.load(r, c * 8), r, c * 8);
                } else {
                    const uint8_t* p = c * kMxBlock < g.K ? g.a.codes + r * g.a.ld + c * 16 : (const uint8_t*)kZeroChunk;
                    fa[CV(S)][CV(I)] = *(const u32x4*)p;
                }
            });
            if constexpr (OP == kOpMx4) va[CV(S)] = stage_scales(g.a.scales + r * g.a.ld_scales, CV(S), g.K, half);
        });
    }
    const f32x16 bias = bias_rows(g, wn * 32, half);

    // ---- the batch
    static_assert(RT == 8 * NW, "a wave's copies are the same rows of each stage");
    const int chunk = (lane & 7) ^ row_key<kStageChunks>(wave * 8 + (lane >> 3));
    const Bf16Rows rows((const uint16_t*)g.b.codes, g.b.ld / 2, g.M, g.K);
    u32x4 held[SRC == kSrcBf16Rows ? CP : 1];
    // converted rows: 8 columns a lane, four lanes a block, 16 rows of the tile a turn
    constexpr int kTurns = RT / 16;
    u32x4 raw[kConvert ? kTurns : 1][SRC == kSrcF32 ? 2 : 1];
    const int crow = threadIdx.x / 32, ccol = threadIdx.x % 32 * 8;
    const Bf16Rows xrows((const uint16_t*)g.b.codes, g.b.ld / 2, g.M, g.K);
    const bool ragged = ccol + 8 > g.K;
    // copy i of a wave: eight rows of one stage
    auto place = [&](uint32_t tile, int i, int64_t& r, int& c) {
        const int q = i * NW + wave;
        r = (int64_t)tile * RT + (q % (RT / 8)) * 8 + (lane >> 3);
        r = r < g.M ? r : g.M - 1;
        c = q / (RT / 8) * kStageChunks + chunk;
    };
    auto issue = [&](u32x4* lds, uint32_t tile) {
        if constexpr (kConvert) {
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                int64_t r = (int64_t)tile * RT + i * 16 + crow;
                r = r < g.M ? r : g.M - 1;
                if constexpr (SRC == kSrcBf16) {
                    raw[i][0] = xrows.load(r, ccol);
                } else {
                    const float* p = (const float*)(g.b.codes + r * g.b.ld);
                    if (g.K % 8 == 0) {   // chunks are whole, or not there
                        __builtin_memcpy(raw[i], p + (ragged ? 0 : ccol), 32);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) raw[i][e / 4][e % 4] = __float_as_uint(p[ccol + e < g.K ? ccol + e : g.K - 1]);
                    }
                }
            }
            return;
        }
        if constexpr (OP == kOpMx4) {
            const int word = wave * 64 + lane, w = word % (2 * KS);   // of the tile, of its row
            if (wave * 64 < kScaleWords) {
                int64_t r = (int64_t)tile * RT + word / (2 * KS);
                r = r < g.M ? r : g.M - 1;
                const uint8_t* p = g.b.scales + r * g.b.ld_scales + w * 4;
                p = w / 2 * 8 * kMxBlock < g.K ? p : (const uint8_t*)kZeroChunk;
                __builtin_amdgcn_global_load_lds((const uint32_t*)p, (uint32_t*)(lds + kChunks) + wave * 64, 4, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < CP; ++i) {
            int64_t r;
            int c;
            place(tile, i, r, c);
            if constexpr (DB) {
                const uint8_t* p = g.b.codes + r * g.b.ld + c * 16;
                p = c * (OP == kOpBf16 ? 8 : kMxBlock) < g.K ? p : (const uint8_t*)kZeroChunk;
                __builtin_amdgcn_global_load_lds((const u32x4*)p, lds + (i * NW + wave) * 64, 16, 0, 0);
            } else {
                held[i] = rows.load(r, c * 8);
            }
        }
    };
    auto store = [&](u32x4* lds, uint32_t tile) {
        if constexpr (kConvert) {
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                float v[8];
                if constexpr (SRC == kSrcBf16) {
                    int64_t r = (int64_t)tile * RT + i * 16 + crow;
                    r = r < g.M ? r : g.M - 1;
                    const u32x4 p = ragged ? xrows.fix(raw[i][0], r, ccol) : raw[i][0];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? p[e / 2] & 0xffff0000u : p[e / 2] << 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = !ragged || ccol + e < g.K ? __uint_as_float(raw[i][e / 4][e % 4]) : 0.0f;
                }
                const int code = mx4_code(quad_max(top_bits<8>(v))), row = i * 16 + crow, block = ccol / kMxBlock;
                ((uint32_t*)(lds + row * kStageChunks + (block ^ row_key<kStageChunks>(row))))[ccol / 8 % 4] = to_e2m1x8(v, code);
                if (ccol % kMxBlock == 0) ((uint8_t*)(lds + kChunks))[row * 8 + block] = (uint8_t)code;
            }
        } else if constexpr (!DB)
#pragma unroll
            for (int i = 0; i < CP; ++i) {
                int64_t r;
                int c;
                place(tile, i, r, c);
                lds[(i * NW + wave) * 64 + lane] = rows.fix(held[i], r, c * 8);
            }
    };
    auto product = [&](const u32x4* lds, int j) {
        f32x16 acc = bias;
        const int row = (wm * RB + j) * 32 + col;
        sfor<KS>([&](auto S) {
            uint32_t vb = 0;
            if constexpr (OP == kOpMx4) vb = pack_scales(((const uint64_t*)(lds + kChunks))[row * KS + CV(S)], CV(S), g.K, half);
            sfor<4>([&](auto I) {
                const u32x4 fb = lds[(CV(S) * RT + row) * kStageChunks + ((2 * CV(I) + half) ^ row_key<kStageChunks>(col))];
                acc = mma_step<OP, CV(I)>(fa[CV(S)][CV(I)], fb, acc, OP == kOpMx4 ? va[CV(S)] : 0u, vb);
            });
        });
        return acc;
    };
    // A tile: the next block's products run while a block's results are finished,
    // where registers for both are left.
    constexpr bool kTwo = DB || KS < 4;
    const uint32_t G = gridDim.x;
    // Store instructions of a wave in a tile whose rows all exist, at the least.
    constexpr int kStoresY = Out::stores_y(512), kStoresQ = Out::stores_q(512);
    const bool has_y = EPI != kEpiKept || g.y, has_q = EPI != kEpiKept || g.q.codes;
    // Waits until this wave's copies of `tile` are done.  Copies and stores leave
    // the counter in the order of their issue; those of the tile after it, and the
    // stores of the two tiles that were finished since, came later.
    auto wait_copies = [&](uint32_t tile, auto stores) {
        constexpr int S = 2 * CV(stores);
        if (tile + G < tiles) wait_vmcnt<CP + S>();
        else wait_vmcnt<S>();
    };
    auto step = [&](u32x4* now, u32x4* next, u32x4* into, uint32_t tile) {
        if constexpr (DB) {
            if (tile < 2 * G) wait_copies(tile, std::integral_constant<int, 0>{});
            else if (EPI != kEpiKept || (has_y && has_q)) wait_copies(tile, std::integral_constant<int, kStoresY + kStoresQ>{});
            else if (has_y) wait_copies(tile, std::integral_constant<int, kStoresY>{});
            else wait_copies(tile, std::integral_constant<int, kStoresQ>{});
            bare_barrier();
        } else {
            lds_barrier();
        }
        const int64_t m0 = (int64_t)tile * RT;
        Mask16 mask[RB];
#pragma unroll
        for (int j = 0; j < RB; ++j) mask[j] = load_mask<EPI>(g, m0 + (wm * RB + j) * 32, wn * 32, lane);
        const uint32_t ahead = tile + (DB ? 2 : 1) * G;
        u32x4* const to = DB ? into : next;
        if (ahead < tiles) issue(to, ahead);
        f32x16 acc;
        if (kTwo) acc = product(now, 0);
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            f32x16 after;
            if (!kTwo) acc = product(now, j);
            if (kTwo && j + 1 < RB) after = product(now, j + 1);
            Out::put(out, g, acc, mask[j], (wm * RB + j) * 32, wn * 32, 0, lane);
            if (kTwo) acc = after;
        }
        if (!DB && ahead < tiles) store(to, ahead);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        bare_barrier();
        Out::template store<512>(out, g, m0, 0, threadIdx.x);
    };
    uint32_t tile = blockIdx.x;
    issue(ring0, tile);
    store(ring0, tile);
    if constexpr (DB)
        if (tile + G < tiles) issue(ring1, tile + G);
    while (true) {
        step(ring0, ring1, ring2, tile);
        if ((tile += G) >= tiles) break;
        step(ring1, ring2, ring0, tile);
        if ((tile += G) >= tiles) break;
        step(ring2, ring0, ring1, tile);
        if ((tile += G) >= tiles) break;
    }
}

// Products with so few results that tiles would leave most compute units without
// work: a workgroup takes 32 outputs of 32 batch rows, and its eight waves split the
// terms, a stage each in turn, and add up their parts in LDS, in the waves' order.
// A stage passes through a part of LDS that is the wave's own, so that its loads
// cover eight rows' 128 bytes at once (whole cache lines) and no wave waits for
// another.  Measured: 14 x 3001 x 352 13 us, 37 us on tiles of 64 x 64 (six workgroups,
// 47 stages one after the other).
template <int OP, bool TA, int EPI>
__global__ void __launch_bounds__(512, 2) layer_split_kernel(GemmArgs g) {
    constexpr int NW = 8, stage_cols = OP == kOpBf16 ? 64 : 256, kChunk = OP == kOpBf16 ? 8 : kMxBlock;
    using Out = Outgoing<EPI, 32, 32>;
    __shared__ f32x4 part[NW][4][64];
    __shared__ u32x4 out[Out::kSize];
    __shared__ u32x4 stage_lds[NW][2][32 * kStageChunks];   // transposed weights: 64 terms of 4 chunks
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int n0 = (int)(blockIdx.x % g.tiles_n) * 32;
    const int64_t m0 = (int64_t)(blockIdx.x / g.tiles_n) * 32;
    const int stages = (g.K + stage_cols - 1) / stage_cols;
    const Bf16Rows a((const uint16_t*)g.a.codes, g.a.ld / 2, TA ? g.K : g.N, TA ? g.N : g.K);
    const Bf16Rows b((const uint16_t*)g.b.codes, g.b.ld / 2, g.M, g.K);
    u32x4 *const la = stage_lds[wave][0], *const lb = stage_lds[wave][1];

    // copy i of a stage: rows 8 i + lane / 8, chunk lane % 8; of transposed weights
    // terms 16 i + lane / 4, chunk lane % 4
    auto row_a = [&](int i) { const int64_t r = n0 + 8 * i + lane / 8; return r < g.N ? r : g.N - 1; };
    auto row_b = [&](int i) { const int64_t r = m0 + 8 * i + lane / 8; return r < g.M ? r : g.M - 1; };
    const int n_ta = n0 + lane % 4 * 8;
    const uint8_t *sa = nullptr, *sb = nullptr;
    if constexpr (OP == kOpMx4) {
        sa = g.a.scales + (int64_t)(n0 + col < g.N ? n0 + col : g.N - 1) * g.a.ld_scales;
        sb = g.b.scales + (m0 + col < g.M ? m0 + col : g.M - 1) * g.b.ld_scales;
    }
    struct Held {
        u32x4 a[4], b[4];
        uint64_t sa, sb;
    };
    auto load = [&](Held& h, int stage) {
        const int c = stage * kStageChunks + lane % 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (OP == kOpBf16) {
                h.b[i] = b.load(row_b(i), c * 8);
                if constexpr (TA) h.a[i] = a.load_at((int64_t)(stage * 64 + 16 * i + lane / 4) * a.ld + n_ta, n_ta);
                else h.a[i] = a.load(row_a(i), c * 8);
            } else {
                const uint8_t *pa = g.a.codes + row_a(i) * g.a.ld + c * 16, *pb = g.b.codes + row_b(i) * g.b.ld + c * 16;
                h.a[i] = *(const u32x4*)(c * kChunk < g.K ? pa : (const uint8_t*)kZeroChunk);
                h.b[i] = *(const u32x4*)(c * kChunk < g.K ? pb : (const uint8_t*)kZeroChunk);
            }
        }
        if constexpr (OP == kOpMx4) {
            const int at = stage * 8 * kMxBlock < g.K ? stage * 8 : 0;
            h.sa = *(const uint64_t*)(sa + at);
            h.sb = *(const uint64_t*)(sb + at);
        }
    };
    f32x16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
    auto multiply = [&](Held& h, int stage) {
        const bool last = (stage + 1) * stage_cols > g.K;
        if constexpr (OP == kOpBf16) {
            const int k = (stage * kStageChunks + lane % 8) * 8;
            if (last)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h.b[i] = b.fix(h.b[i], row_b(i), k);
                    if constexpr (!TA) h.a[i] = a.fix(h.a[i], row_a(i), k);
                }
            if constexpr (TA)
                if (last || n0 + 32 > g.N)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t term = stage * 64 + 16 * i + lane / 4;
                        h.a[i] = term < g.K ? a.fix(h.a[i], term, n_ta) : u32x4{0, 0, 0, 0};
                    }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * i + lane / 8, at = row * kStageChunks + (lane % 8 ^ row_key<kStageChunks>(row));
            lb[at] = h.b[i];
            la[TA ? i * 64 + lane : at] = h.a[i];
        }
        wave_lds_fence();
        uint32_t va = 0, vb = 0;
        if constexpr (OP == kOpMx4) {
            va = pack_scales(h.sa, stage, g.K, half);
            vb = pack_scales(h.sb, stage, g.K, half);
        }
        sfor<4>([&](auto S) {
            const int at = col * kStageChunks + ((2 * CV(S) + half) ^ row_key<kStageChunks>(col));
            u32x4 fa;
            if constexpr (TA) fa = __builtin_bit_cast(u32x4, read_columns<4>(la, CV(S) * 16, 0, lane));
            else fa = la[at];
            acc = mma_step<OP, CV(S)>(fa, lb[at], acc, va, vb);
        });
        wave_lds_fence();
    };
    Held h0, h1;
    if (wave < stages) load(h0, wave);
    for (int s = wave; s < stages; s += 2 * NW) {
        if (s + NW < stages) load(h1, s + NW);
        multiply(h0, s);
        if (s + 2 * NW < stages) load(h0, s + 2 * NW);
        if (s + NW < stages) multiply(h1, s + NW);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) part[wave][q][lane] = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    lds_barrier();
    if (wave > 0) return;
    acc = bias_rows(g, n0, half);
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[4 * q + i] += part[w][q][lane][i];
    Out::put(out, g, acc, load_mask<EPI>(g, m0, n0, lane), 0, 0, n0, lane);
    wave_lds_fence();
    Out::template store<64>(out, g, m0, n0, threadIdx.x);
}

template <int OP, int KS, int WN, bool TA, int SRC, int EPI>
void launch_rows_of(GemmArgs g, int n_cu, hipStream_t stream) {
    g.tiles_m = (uint32_t)(((int64_t)g.M + kRowsTile - 1) / kRowsTile);
    const uint32_t most = rows_workgroups<OP, KS, WN, TA, SRC, EPI>() * (uint32_t)n_cu;
    const dim3 grid(g.tiles_m < most ? g.tiles_m : most);
    hipLaunchKernelGGL((layer_rows_kernel<OP, KS, WN, TA, SRC, EPI>), grid, dim3(512), 0, stream, g);
}
template <int OP, int KS, bool TA, int SRC, int EPI>
hipError_t launch_layer_rows(const GemmArgs& g, int n_cu, hipStream_t stream) {
    if (g.N > 128) launch_rows_of<OP, KS, 8, TA, SRC, EPI>(g, n_cu, stream);
    else launch_rows_of<OP, KS, 4, TA, SRC, EPI>(g, n_cu, stream);
    return hipGetLastError();
}

// Layers for layer_rows_kernel: weights for a workgroup, and a tile of rows for every
// compute unit.
inline bool fits_rows(const GemmArgs& g, int most_k, int n_cu) {
    return g.N <= 256 && g.K <= most_k && (int64_t)g.M >= (int64_t)kRowsTile * n_cu;
}

template <int OP, bool TA, bool DA, bool DB, int EPI>
hipError_t launch_layer_gemm(GemmArgs g, int n_cu, hipStream_t stream) {
    constexpr int stage_cols = OP == kOpBf16 ? 64 : 256;
    const int stages = (g.K + stage_cols - 1) / stage_cols;
    if (fits_rows(g, OP == kOpMx4 ? 512 : 256, n_cu)) {
        constexpr int SRC = DB ? kSrcCopies : kSrcBf16Rows;
        if (stages == 1) return launch_layer_rows<OP, 1, TA, SRC, EPI>(g, n_cu, stream);
        if (stages == 2) return launch_layer_rows<OP, 2, TA, SRC, EPI>(g, n_cu, stream);
        if constexpr (OP == kOpBf16) return launch_layer_rows<OP, 4, TA, SRC, EPI>(g, n_cu, stream);
    }
    auto tiles = [&](int b) { return (uint64_t)((g.N + b - 1) / b) * (uint64_t)((g.M + b - 1) / b); };
    // the largest tiles that leave every compute unit one
    constexpr bool kBig = OP == kOpBf16 && DA && DB;
    const bool big = kBig && tiles(256) >= (uint64_t)n_cu;
    const bool split = 2 * tiles(64) <= (uint64_t)n_cu && stages >= 4;
    const int b = big ? 256 : split ? 32 : tiles(128) >= (uint64_t)n_cu ? 128 : 64;
    g.tiles_n = (uint32_t)((g.N + b - 1) / b);
    g.tiles_m = (uint32_t)((g.M + b - 1) / b);
    const dim3 grid((g.tiles_n * g.tiles_m + 7) / 8 * 8);
    if constexpr (kBig) {   // E2M1 runs slower on 256 x 256 (165 us for 8192 x 4096 x 4096, 129 us on 128 x 128)
        if (b == 256) {
            hipLaunchKernelGGL((layer_gemm_kernel<OP, 256, 256, 4, 2, TA, DA, DB, EPI>), grid, dim3(512), 0, stream, g);
            return hipGetLastError();
        }
    }
    if (b == 32) hipLaunchKernelGGL((layer_split_kernel<OP, TA, EPI>), dim3(g.tiles_n * g.tiles_m), dim3(512), 0, stream, g);
    else if (b == 128) hipLaunchKernelGGL((layer_gemm_kernel<OP, 128, 128, 2, 2, TA, DA, DB, EPI>), grid, dim3(256), 0, stream, g);
    else hipLaunchKernelGGL((layer_gemm_kernel<OP, 64, 64, 2, 2, TA, DA, DB, EPI>), grid, dim3(256), 0, stream, g);
    return hipGetLastError();
}

}  // namespace
}  // namespace donerf
