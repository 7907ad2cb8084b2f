// mx_few_rows.hip - y = act(x W^T + b) for a few batch rows, W in E2M1: the form
// for single tokens and handfuls of rays, bound by reading W once.
//
// A workgroup takes 16 outputs (32 for E2M1 results, whose blocks have 32) and all
// rows; its eight waves split the columns, 128 at a time in turn, and add up their
// parts in LDS.  A lane of a 16 x 16 x 128 MFMA holds whole blocks of 32 columns,
// one of W and one of x, so x is converted in the lane that multiplies it, with no
// exchange and no pass of its own: one launch, with the loads of several steps under
// way before the first product.  Measured: one bf16 row through 4096 x 4096 6.7 us
// (8.9 MB; 1.3 TB/s, bound by the latency of a cold read and the launch); 13 fp32 rows
// through 256 x 256 3.8 us.
//
// The rule that takes it is on rows alone, so that up to 32 of them need no workspace.
// Against a conversion and a product (in a graph of calls, on four weights in turn, bf16
// rows / fp32 rows, us; these two launches come to the same for both):
//                    1 row          8 rows         16 rows        32 rows
//     256 x 256       3.4/3.1  4.9   3.4/3.2  5.0   3.5/3.5  5.3   4.3/3.9  5.4
//    1024 x 1024      4.7/4.2  5.6   5.8/5.5  5.9   7.2/6.7  6.0   7.2/6.8  6.0
//    4096 x 4096      6.7/7.6  7.7   7.6/9.6  7.9   8.9/12.4 8.1  13.2/19.3 8.4
//    4096 -> 16,384  20.2/23.8 18.2 24.0/32.1 18.5 29.2/43.0 18.7 46.5/70.5 19.0
// Every workgroup reads and converts all of x again, which costs more than a second
// launch from about 16 rows of 1024 columns, 8 of 4096, or 16,384 outputs on.
#include "internal.h"
#include "mx.h"

namespace donerf {
namespace {

constexpr int kWaves = 8;   // of a workgroup
constexpr int kXF32 = 0, kXBf16 = 1, kXMx4 = 2;
// Steps whose loads are issued together, as many as the registers hold: a step
// takes 32, 16 or 4 of them for each group of rows.
constexpr int steps_ahead(int xt, int tm) { return xt == kXMx4 ? 4 : xt == kXBf16 ? 4 / tm : 2 / tm; }

// The batch: fp32, bf16, or E2M1 already.  ld: values, or bytes of E2M1 rows.
struct XRows {
    const uint8_t* p;
    int64_t ld;
    const uint8_t* scales;
    int64_t ld_scales;
    int64_t M;
    int K;
};
struct Block {   // 32 columns of a row in E2M1
    u32x4 codes;
    int scale;
};
template <int XT>
struct XBlock {   // as loaded
    u32x4 raw[XT == kXF32 ? 8 : XT == kXBf16 ? 4 : 1];
    int scale;
};
// A block that exists.  ragged: the rows' last block is not whole.
template <int XT>
__device__ __forceinline__ void load_block(XBlock<XT>& b, const XRows& x, int64_t row, int block, bool ragged) {
    if constexpr (XT == kXMx4) {
        b.raw[0] = *(const u32x4*)(x.p + row * x.ld + block * 16);
        b.scale = x.scales[row * x.ld_scales + block];
    } else if constexpr (XT == kXBf16) {
        const Bf16Rows rows((const uint16_t*)x.p, x.ld, x.M, x.K);
#pragma unroll
        for (int i = 0; i < 4; ++i) b.raw[i] = rows.load(row, block * kMxBlock + 8 * i);
    } else {
        const float* p = (const float*)x.p + row * x.ld;
        if (!ragged) {
            __builtin_memcpy(b.raw, p + block * kMxBlock, 128);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int k = block * kMxBlock + i;
                b.raw[i / 4][i % 4] = __float_as_uint(p[k < x.K ? k : x.K - 1]);
            }
        }
    }
}
template <int XT>
__device__ __forceinline__ Block to_block(const XBlock<XT>& b, const XRows& x, int64_t row, int block, bool ragged) {
    if constexpr (XT == kXMx4) return Block{b.raw[0], b.scale};
    float v[32];
    if constexpr (XT == kXBf16) {
        const Bf16Rows rows((const uint16_t*)x.p, x.ld, x.M, x.K);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x4 p = b.raw[i];
            if (ragged) p = rows.fix(p, row, block * kMxBlock + 8 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * i + 2 * j] = __uint_as_float(p[j] << 16);
                v[8 * i + 2 * j + 1] = __uint_as_float(p[j] & 0xffff0000u);
            }
        }
    } else if constexpr (XT == kXF32) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            v[i] = __uint_as_float(b.raw[i / 4][i % 4]);
            if (ragged) v[i] = block * kMxBlock + i < x.K ? v[i] : 0.0f;
        }
    }
    const int code = mx4_code(top_bits<32>(v));
    return Block{u32x4{to_e2m1x8(v, code), to_e2m1x8(v + 8, code), to_e2m1x8(v + 16, code), to_e2m1x8(v + 24, code)}, code};
}

// NB: groups of 16 outputs, TM: groups of 16 rows.
template <int XT, int NB, int TM>
__global__ void __launch_bounds__(64 * kWaves) mx_few_rows_kernel(FewRowsArgs g) {
    __shared__ f32x4 part[kWaves][NB][TM][64];
    __shared__ float result[TM * 16][NB * 16 + 1];
    constexpr int kSteps = steps_ahead(XT, TM);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int at = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * NB * 16;
    const int blocks = (g.K + kMxBlock - 1) / kMxBlock, steps = (blocks + 3) / 4;
    const bool ragged = g.K % kMxBlock != 0;
    const XRows rows{g.x, g.ldx, g.x_scales, g.ldx_scales, g.M, g.K};
    f32x4 acc[NB][TM];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = wave; s0 < steps; s0 += kWaves * kSteps) {
        Block w[kSteps][NB];
        XBlock<XT> x[kSteps][TM];
        // rows, outputs and blocks that do not exist are replaced by ones that do:
        // their results are not stored, their scales (2^-127 for both factors) leave
        // no product that fp32 can hold
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int b = (s0 + s * kWaves) * 4 + quarter, block = b < blocks ? b : blocks - 1;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int n = n0 + i * 16 + at, r = n < g.N ? n : g.N - 1;
                w[s][i].codes = *(const u32x4*)(g.w + (int64_t)r * g.ldw + block * 16);
                w[s][i].scale = g.w_scales[(int64_t)r * g.ldw_scales + block];
            }
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const int m = j * 16 + at;
                load_block<XT>(x[s][j], rows, m < g.M ? m : g.M - 1, block, ragged);
            }
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int b = (s0 + s * kWaves) * 4 + quarter, block = b < blocks ? b : blocks - 1;
            if (s0 + s * kWaves >= steps) break;
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const int m = j * 16 + at;
                const Block xb = to_block<XT>(x[s][j], rows, m < g.M ? m : g.M - 1, block, ragged);
                const i32x8 bv = {(int)xb.codes.x, (int)xb.codes.y, (int)xb.codes.z, (int)xb.codes.w, 0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const u32x4 c = w[s][i].codes;
                    const i32x8 av = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        av, bv, acc[i][j], 4, 4, 0, b < blocks ? w[s][i].scale : 0, 0, b < blocks ? xb.scale : 0);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) part[wave][i][j][lane] = acc[i][j];
    __syncthreads();
    // outputs fastest: neighbouring threads store neighbouring values
    for (int t = threadIdx.x; t < NB * TM * 256; t += 64 * kWaves) {
        const int c = t % (NB * 16), m = t / (NB * 16), n = n0 + c;
        const float* p = (const float*)&part[0][c / 16][m / 16][(c % 16) / 4 * 16 + m % 16] + c % 4;
        float v = g.bias ? g.bias[n < g.N ? n : g.N - 1] : 0.0f;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) v += p[k * NB * TM * 256];
        if (g.relu) v = __builtin_elementwise_maximum(v, 0.0f);
        if (g.out == kOutMx4) result[m][c] = n < g.N ? v : 0.0f;
        else if (m < g.M && n < g.N) {
            if (g.out == kOutF32) ((float*)g.y)[m * g.ldy + n] = v;
            else ((uint16_t*)g.y)[m * g.ldy + n] = (uint16_t)pack_bf16x2(v, v);
        }
    }
    if constexpr (NB == 2) {
        if (g.out != kOutMx4) return;
        __syncthreads();
        const int m = threadIdx.x;
        if (m < TM * 16 && m < g.M) {
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = result[m][i];
            const int code = mx4_code(top_bits<32>(v));
            *(u32x4*)(g.q.codes + m * g.q.ld + n0 / 2) = u32x4{to_e2m1x8(v, code), to_e2m1x8(v + 8, code), to_e2m1x8(v + 16, code), to_e2m1x8(v + 24, code)};
            g.q.scales[m * g.q.ld_scales + n0 / kMxBlock] = (uint8_t)code;
        }
    }
}

template <int XT, int NB>
void launch_groups(const FewRowsArgs& g, hipStream_t stream) {
    const dim3 grid((uint32_t)((g.N + NB * 16 - 1) / (NB * 16)));
    if (g.M <= 16) hipLaunchKernelGGL((mx_few_rows_kernel<XT, NB, 1>), grid, dim3(64 * kWaves), 0, stream, g);
    else hipLaunchKernelGGL((mx_few_rows_kernel<XT, NB, 2>), grid, dim3(64 * kWaves), 0, stream, g);
}

}  // namespace

hipError_t launch_mx_few_rows(const FewRowsArgs& g, int x_kind, hipStream_t stream) {
    const bool two = g.out == kOutMx4;
    if (x_kind == kXF32) two ? launch_groups<kXF32, 2>(g, stream) : launch_groups<kXF32, 1>(g, stream);
    else if (x_kind == kXBf16) two ? launch_groups<kXBf16, 2>(g, stream) : launch_groups<kXBf16, 1>(g, stream);
    else two ? launch_groups<kXMx4, 2>(g, stream) : launch_groups<kXMx4, 1>(g, stream);
    return hipGetLastError();
}

}  // namespace donerf
