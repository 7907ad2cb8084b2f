// train_linear.hip - a layer's forward pass with its activations kept in E4M3,
// and its backward pass from them, on bf16 MFMAs with fp32 accumulation.
//
//   forward   z = x W^T + b, y = act(z): layer_gemm.h with W as its weights.
//   backward  dx = (dz W) where x is not zero (x a ReLU's output), the same
//             product with weights that are transposed in memory;
//             dW = dz^T x and db = sum of dz over the rows, weight_grad_kernel.
#include "layer_gemm.h"

namespace donerf {
namespace {

// Rows of bf16 that 16-byte copies can take chunk by chunk.
bool whole_chunks(const MxIn& x, int cols) {
    return ((uintptr_t)x.codes & 15) == 0 && (x.ld & 15) == 0 && cols % 8 == 0;
}

// ---------------------------------------------------------------- dW, db

constexpr int kGradTileN = 128;   // weight rows of a workgroup

struct GradArgs {
    const uint16_t* dz;
    int64_t lddz;
    MxIn x;
    int32_t x_bf16;
    int32_t M, N, K;
    int32_t rows_per_split;  // a multiple of the kernel's stage
    uint32_t tiles_n, tiles_k, splits;
    float* dw;               // splits x N x K, or the result, or null
    int64_t split_stride;    // values from one split's dw to the next's
    int64_t lddw;
    float* db;               // splits x N, or the result, or null
    int32_t accumulate;      // only where dw is the result
};

// One split's part of dW[n][k] = sum_m dz[m][n] x[m][k] for 128 weight rows and
// 64 TK columns, in stages of R batch rows.  dz goes straight into LDS (DIRECT:
// rows of 16-byte alignment, N a multiple of 8), x through registers, where E4M3
// becomes bf16.  x is loaded a stage before it is stored, but with a lead of one stage's
// products only: the wait for dz's copies, which ends a stage, waits for it too.  Both
// operands' terms are rows in memory and are read from LDS by columns.  db comes from
// the fragments that are there anyway.
// Measured: 160,000 x 256 x 256 44 us (124 MB read, 32 MB of parts written),
// 16,384 x 2048 x 2048 199 us (690 TFLOP/s).  128 x 128 with two workgroups per CU: one
// gave 455 us instead of 341 for the whole backward call, 128 x 256 330 (but 39 instead of
// 32 us at 4000 x 512 x 512, 107 instead of 104 at 160,000 x 256 x 256).
template <bool DIRECT, bool X_BF16, int TK, int R>
__global__ void __launch_bounds__(256, 2) weight_grad_kernel(GradArgs g) {
    constexpr int kTileK = 64 * TK, kChunksK = kTileK / 8;
    constexpr int kPerX = R * kChunksK / 256;               // chunks of x per thread
    constexpr int kRowsX = 256 / kChunksK;                  // rows between them
    __shared__ u32x4 z0[R * kGradTileN / 8], z1[R * kGradTileN / 8];
    __shared__ u32x4 x0[R * kChunksK], x1[R * kChunksK];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave & 1, wk = wave >> 1;
    // A split's tiles go to one XCD, or few: its L2 reads the split's rows once.
    const uint32_t tiles = g.tiles_n * g.tiles_k, all = tiles * g.splits, per_xcd = (all + 7) / 8;
    const uint32_t t = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (t >= all) return;
    const uint32_t tile = t % tiles;
    const int split = (int)(t / tiles);
    const int n0 = (int)(tile % g.tiles_n) * kGradTileN, k0 = (int)(tile / g.tiles_n) * kTileK;
    const int64_t m_begin = (int64_t)split * g.rows_per_split;
    const int64_t m_end = m_begin + g.rows_per_split < g.M ? m_begin + g.rows_per_split : (int64_t)g.M;
    const int stages = (int)((m_end - m_begin + R - 1) / R);
    const bool sums = g.db && k0 == 0 && wk == 0;

    ColumnCopy<R, kGradTileN, 4, DIRECT> z;
    z.init(g.dz, g.lddz, g.M, g.N, m_begin, m_end, n0, wave, lane);
    // x: chunks of 8 columns
    struct Held {
        u32x4 v[kPerX];
        int code[kPerX];
    } ha, hb;
    const int xrow = threadIdx.x / kChunksK, xcol = k0 + (threadIdx.x % kChunksK) * 8;
    const Bf16Rows xrows((const uint16_t*)g.x.codes, g.x.ld / 2, g.M, g.K);
    // codes behind the last block: the last block's, whose products are not stored
    const int k_codes = (g.K + kMxBlock - 1) / kMxBlock * kMxBlock, xcode = xcol < k_codes ? xcol : k_codes - 8;
    auto row_x = [&](int stage, int i) {
        const int64_t m = m_begin + (int64_t)stage * R + xrow + i * kRowsX;
        return m < m_end ? m : m_end - 1;
    };
    auto load_x = [&](Held& h, int stage) {
#pragma unroll
        for (int i = 0; i < kPerX; ++i) {
            const int64_t m = row_x(stage, i);
            if constexpr (X_BF16) {
                h.v[i] = xrows.load(m, xcol);
            } else {
                const u32x2 p = *(const u32x2*)(g.x.codes + m * g.x.ld + xcode);
                h.v[i][0] = p[0];
                h.v[i][1] = p[1];
                h.code[i] = g.x.scales[m * g.x.ld_scales + xcode / kMxBlock];
            }
        }
    };
    auto store_x = [&](u32x4* lds, Held& h, int stage) {
        const bool last = m_begin + (int64_t)(stage + 1) * R > m_end;
#pragma unroll
        for (int i = 0; i < kPerX; ++i) {
            u32x4 v;
            if constexpr (X_BF16) {
                v = h.v[i];
                if (k0 + kTileK > g.K) v = xrows.fix(v, row_x(stage, i), xcol);
            } else {
                v = e4m3x8_as_bf16(u32x2{h.v[i][0], h.v[i][1]}, h.code[i]);
            }
            // a repeated row may hold NaN, which zeros of dz would not cancel
            if (last && m_begin + (int64_t)stage * R + xrow + i * kRowsX >= m_end) v = u32x4{0, 0, 0, 0};
            lds[column_slot<kChunksK>(xrow + i * kRowsX, threadIdx.x % kChunksK)] = v;
        }
    };
    f32x16 acc[2][TK];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < TK; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    float db[2] = {0.0f, 0.0f};   // of this lane's column and half of the rows
    auto compute = [&](const u32x4* zs, const u32x4* xs) {
        sfor<R / 16>([&](auto S) {
            bf16x8 a[2], b[TK];
#pragma unroll
            for (int i = 0; i < 2; ++i) a[i] = read_columns<kGradTileN / 8>(zs, CV(S) * 16, (wn * 2 + i) * 32, lane);
#pragma unroll
            for (int j = 0; j < TK; ++j) b[j] = read_columns<kChunksK>(xs, CV(S) * 16, (wk * TK + j) * 32, lane);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < TK; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
            if (sums)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) db[i] += (float)a[i][e];
        });
    };
    // Stage s is multiplied while dz of s + 1 is copied, x of s + 1 stands in
    // `now` and x of s + 2 is loaded into `later` (all of it has arrived at the end).
    auto step = [&](u32x4* zs, u32x4* zn, u32x4* xs, u32x4* xn, Held& now, Held& later, int s) {
        const bool more = s + 1 < stages;
        if (more) z.issue(zn, s + 1, wave);
        if (s + 2 < stages) load_x(later, s + 2);
        compute(zs, xs);
        if (more) {
            z.store(zn, s + 1, wave, lane);
            store_x(xn, now, s + 1);
            if constexpr (DIRECT) wait_vmcnt<0>();
            lds_barrier();
        }
    };
    z.issue(z0, 0, wave);
    load_x(hb, 0);
    if (stages > 1) load_x(ha, 1);
    z.store(z0, 0, wave, lane);
    store_x(x0, hb, 0);
    if constexpr (DIRECT) wait_vmcnt<0>();
    lds_barrier();
    for (int s = 0; s < stages; s += 2) {
        step(z0, z1, x0, x1, ha, hb, s);
        if (s + 1 < stages) step(z1, z0, x1, x0, hb, ha, s + 1);
    }

    if (g.dw) {
        float* out = g.dw + (int64_t)split * g.split_stride;
        const bool whole = n0 + kGradTileN <= g.N && k0 + kTileK <= g.K;
        auto each = [&](auto f) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < TK; ++j) {
                    const int k = k0 + (wk * TK + j) * 32 + (lane & 31);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int n = n0 + (wn * 2 + i) * 32 + (e & 3) + 8 * (e >> 2) + 4 * (lane >> 5);
                        if (whole || (n < g.N && k < g.K)) f(out + (int64_t)n * g.lddw + k, acc[i][j][e]);
                    }
                }
        };
        if (g.accumulate) each([](float* p, float v) { *p += v; });
        else each([](float* p, float v) { *p = v; });
    }
    if (sums) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = n0 + (wn * 2 + i) * 32 + (lane & 31);
            const float s = db[i] + __shfl_xor(db[i], 32);
            if (lane < 32 && n < g.N) {
                float* p = g.db + (int64_t)split * g.N + n;
                *p = g.accumulate ? *p + s : s;
            }
        }
    }
}

// dW and db from the splits' parts: GROUPS threads a value, each its share of the
// splits in their order, and then the shares.
template <int GROUPS>
__global__ void __launch_bounds__(256) grad_sum_kernel(const float* dw_parts, const float* db_parts, int splits, int N,
                                                       int K, float* dw, int64_t lddw, float* db, int accumulate) {
    constexpr int kValues = 256 / GROUPS;   // of a workgroup
    __shared__ float part[GROUPS][kValues];
    const int c = threadIdx.x % kValues, group = threadIdx.x / kValues;
    const int64_t nk = (int64_t)N * K, total = (dw ? nk : 0) + (db ? N : 0);
    const int from = splits * group / GROUPS, to = splits * (group + 1) / GROUPS;
    for (int64_t i0 = (int64_t)blockIdx.x * kValues; i0 < total; i0 += (int64_t)gridDim.x * kValues) {
        const int64_t i = i0 + c < total ? i0 + c : total - 1;
        const bool is_w = dw && i < nk;
        const int64_t at = is_w ? i : i - (dw ? nk : 0), stride = is_w ? nk : N;
        const float* p = (is_w ? dw_parts : db_parts) + at;
        float s = 0.0f;
#pragma unroll 8
        for (int k = from; k < to; ++k) s += p[k * stride];
        if constexpr (GROUPS > 1) {
            part[group][c] = s;
            __syncthreads();
#pragma unroll
            for (int e = 1; e < GROUPS; ++e) s += group == 0 ? part[e][c] : 0.0f;
            __syncthreads();
        }
        if (group == 0 && i0 + c < total) {
            float* o = is_w ? dw + at / K * lddw + at % K : db + at;
            *o = accumulate ? *o + s : s;
        }
    }
}

struct GradPlan {
    int tiles_n, tiles_k, splits, rows_per_split;
    size_t parts;   // bytes
};

// Columns of a tile, in blocks per wave, and the batch rows of a stage; half of them
// where dz, too, passes through registers.
constexpr int kGradBlocks = 2, kGradRows = 64, kGradRowsAny = 32;

// The batch is split until two workgroups per compute unit have work; the parts, 64
// KiB a workgroup, are what that costs.
GradPlan grad_plan(int64_t M, int N, int K, int n_cu) {
    GradPlan p;
    p.tiles_n = (N + kGradTileN - 1) / kGradTileN;
    p.tiles_k = (K + 64 * kGradBlocks - 1) / (64 * kGradBlocks);
    const int64_t stages = (M + kGradRows - 1) / kGradRows;
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_k;
    int64_t want = 2 * (int64_t)n_cu / tiles;
    want = want < 1 ? 1 : want > stages ? (stages < 1 ? 1 : stages) : want;
    const int64_t per = (stages + want - 1) / want;
    p.rows_per_split = (int)(per < 1 ? kGradRows : per * kGradRows);
    p.splits = M == 0 ? 0 : (int)((M + p.rows_per_split - 1) / p.rows_per_split);
    p.parts = p.splits > 1 ? (size_t)p.splits * ((size_t)N * K + N) * sizeof(float) : 0;
    return p;
}

// dx: the weights as they lie in memory, a row of them per term.
template <int EPI>
hipError_t launch_input_grad(const GemmArgs& g, int n_cu, hipStream_t stream) {
    const bool da = whole_chunks(g.a, g.N), db = whole_chunks(g.b, g.K);
    if (da && db) return launch_layer_gemm<kOpBf16, true, true, true, EPI>(g, n_cu, stream);
    return launch_layer_gemm<kOpBf16, true, false, false, EPI>(g, n_cu, stream);
}

}  // namespace

hipError_t launch_train_linear(const GemmArgs& g, int n_cu, hipStream_t stream) {
    const bool da = whole_chunks(g.a, g.K), db = whole_chunks(g.b, g.K);
    if (da && db) return launch_layer_gemm<kOpBf16, false, true, true, kEpiKept>(g, n_cu, stream);
    return launch_layer_gemm<kOpBf16, false, false, false, kEpiKept>(g, n_cu, stream);
}

size_t backward_workspace(int64_t M, int N, int K, int n_cu) {
    const GradPlan p = grad_plan(M, N, K, n_cu);
    return p.parts;
}

hipError_t launch_train_linear_backward(const BackwardArgs& a, int n_cu, hipStream_t stream) {
    const GradPlan p = grad_plan(a.M, a.N, a.K, n_cu);
    hipError_t e = hipSuccess;
    if (a.dx && a.M > 0) {
        GemmArgs g{};
        g.a = MxIn{(const uint8_t*)a.w, a.ldw * 2, nullptr, 0};
        g.b = MxIn{(const uint8_t*)a.dz, a.lddz * 2, nullptr, 0};
        g.y = (uint8_t*)a.dx;
        g.ldy = a.lddx;
        g.mask = a.x.codes;
        g.ld_mask = a.x_bf16 ? a.x.ld / 2 : a.x.ld;
        g.M = a.M;
        g.N = a.K;
        g.K = a.N;
        e = !a.relu ? launch_input_grad<kEpiBf16>(g, n_cu, stream)
            : a.x_bf16 ? launch_input_grad<kEpiMaskBf16>(g, n_cu, stream) : launch_input_grad<kEpiMaskMx8>(g, n_cu, stream);
        if (e != hipSuccess) return e;
    }
    if (!a.dw && !a.db) return e;
    float* dw_parts = (float*)a.workspace;
    float* db_parts = dw_parts + (size_t)p.splits * a.N * a.K;
    if (p.splits >= 1) {
        const bool direct = p.splits == 1;
        GradArgs g{};
        g.dz = a.dz;
        g.lddz = a.lddz;
        g.x = a.x;
        g.x_bf16 = a.x_bf16;
        g.M = a.M;
        g.N = a.N;
        g.K = a.K;
        g.rows_per_split = p.rows_per_split;
        g.tiles_n = (uint32_t)p.tiles_n;
        g.tiles_k = (uint32_t)p.tiles_k;
        g.splits = (uint32_t)p.splits;
        g.dw = !a.dw ? nullptr : direct ? a.dw : dw_parts;
        g.split_stride = direct ? 0 : (int64_t)a.N * a.K;
        g.lddw = direct ? a.lddw : a.K;
        g.db = !a.db ? nullptr : direct ? a.db : db_parts;
        g.accumulate = direct ? a.accumulate : 0;
        const dim3 grid(((uint32_t)p.tiles_n * p.tiles_k * p.splits + 7) / 8 * 8);
        const bool copies = whole_chunks(MxIn{(const uint8_t*)a.dz, a.lddz * 2, nullptr, 0}, a.N);
        if (copies && !a.x_bf16) hipLaunchKernelGGL((weight_grad_kernel<true, false, kGradBlocks, kGradRows>), grid, dim3(256), 0, stream, g);
        else if (copies) hipLaunchKernelGGL((weight_grad_kernel<true, true, kGradBlocks, kGradRows>), grid, dim3(256), 0, stream, g);
        else if (!a.x_bf16) hipLaunchKernelGGL((weight_grad_kernel<false, false, kGradBlocks, kGradRowsAny>), grid, dim3(256), 0, stream, g);
        else hipLaunchKernelGGL((weight_grad_kernel<false, true, kGradBlocks, kGradRowsAny>), grid, dim3(256), 0, stream, g);
        if ((e = hipGetLastError()) != hipSuccess || direct) return e;
    }
    const int64_t total = (int64_t)a.N * a.K + a.N;
    // few values do not fill the device with a thread each (64 x 48 of 196 splits:
    // 20 us, 16 us by eight threads); many lose by short rows (256 x 256 of 125
    // splits: 9 us, 15 us)
    const bool few = total <= 64 * (int64_t)n_cu;
    const uint64_t values = few ? 32 : 256, wg = ((uint64_t)total + values - 1) / values, most = (uint64_t)n_cu * 32;
    const dim3 grid((uint32_t)(wg < most ? wg : most));
    if (few) hipLaunchKernelGGL(grad_sum_kernel<8>, grid, dim3(256), 0, stream, dw_parts, db_parts, p.splits, a.N, a.K, a.dw, a.lddw, a.db, a.accumulate);
    else hipLaunchKernelGGL(grad_sum_kernel<1>, grid, dim3(256), 0, stream, dw_parts, db_parts, p.splits, a.N, a.K, a.dw, a.lddw, a.db, a.accumulate);
    return hipGetLastError();
}

}  // namespace donerf
