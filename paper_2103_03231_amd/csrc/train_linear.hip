// train_linear.hip - a layer's forward pass with its activations kept in E4M3,
// and its backward pass from them, on bf16 MFMAs with fp32 accumulation.
//
//   forward   z = x W^T + b, y = act(z): layer_gemm.h with W as its weights.
//   backward  dx = (dz W) where x is not zero (x a ReLU's output), the same
//             product with W transposed once into the workspace;
//             dW = dz^T x and db = sum of dz over the rows, weight_grad_kernel.
#include "layer_gemm.h"

namespace donerf {
namespace {

// Rows of bf16 that 16-byte copies can take chunk by chunk.
bool whole_chunks(const MxIn& x, int cols) {
    return ((uintptr_t)x.codes & 15) == 0 && (x.ld & 15) == 0 && cols % 8 == 0;
}

// ---------------------------------------------------------------- W transposed

constexpr int kTrTile = 64;

// out[k][n] = w[n][k], columns from N to ldo zero.
__global__ void __launch_bounds__(256) transpose_kernel(const uint16_t* w, int64_t ldw, int N, int K, uint16_t* out,
                                                        int64_t ldo) {
    __shared__ uint16_t tile[kTrTile][kTrTile + 2];
    const int n0 = blockIdx.x * kTrTile, k0 = blockIdx.y * kTrTile;
    const int c = threadIdx.x & 63, r0 = threadIdx.x >> 6;
    for (int r = r0; r < kTrTile; r += 4)
        tile[r][c] = n0 + r < N && k0 + c < K ? w[(int64_t)(n0 + r) * ldw + k0 + c] : (uint16_t)0;
    __syncthreads();
    for (int r = r0; r < kTrTile; r += 4)
        if (k0 + r < K && n0 + c < ldo) out[(int64_t)(k0 + r) * ldo + n0 + c] = tile[c][r];
}

// ---------------------------------------------------------------- dW, db

constexpr int kGradTile = 128;    // weight rows and columns of a workgroup
constexpr int kGradRows = 64;     // batch rows of a stage
constexpr int kGradChunks = kGradTile / 8;

struct GradArgs {
    const uint16_t* dz;
    int64_t lddz;
    MxIn x;
    int32_t x_bf16;
    int32_t M, N, K;
    int32_t rows_per_split;  // a multiple of kGradRows
    uint32_t tiles_n, tiles_k;
    float* dw;               // splits x N x K, or the result, or null
    int64_t split_stride;    // values from one split's dw to the next's
    int64_t lddw;
    float* db;               // splits x N, or the result, or null
    int32_t accumulate;      // only where dw is the result
};

// Where chunk c (8 columns) of row m of a stage lies.  A transposing read takes
// 64 bytes of eight rows at once; rows that follow each other start 64 bytes
// apart in the banks.
__device__ __forceinline__ int grad_slot(int m, int c) { return m * kGradChunks + (c ^ ((m & 3) << 2)); }

// The MFMA operand of 32 columns from column n on and 16 rows from row m on of a
// stage: lane l has column n + (l & 31), rows m + 8 (l >> 5) + (0..7).  Sixteen
// lanes read four rows of 16 columns, 8 bytes each, and get a column each.
__device__ __forceinline__ bf16x8 read_columns(const u32x4* lds, int m, int n, int lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int col = n + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const int row = m + 8 * (lane >> 5) + ((lane >> 2) & 3);
    struct { s16x4 lo, hi; } v;
    const char* base = (const char*)lds;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + grad_slot(row, col >> 3) * 16 + (col & 7) * 2));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(base + grad_slot(row + 4, col >> 3) * 16 + (col & 7) * 2));
    return __builtin_bit_cast(bf16x8, v);
}

// 8 E4M3 elements as bf16: exact, but for results below bf16's smallest numbers.
__device__ __forceinline__ u32x4 e4m3x8_as_bf16(u32x2 p, int code) {
    float v[8];
    from_e4m3x4(p[0], code, v);
    from_e4m3x4(p[1], code, v + 4);
    return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

__global__ void __launch_bounds__(256) weight_grad_kernel(GradArgs g) {
    constexpr int kPer = kGradRows * kGradChunks / 256;   // chunks per thread, of dz and of x
    __shared__ u32x4 ring0[2 * kGradRows * kGradChunks];
    __shared__ u32x4 ring1[2 * kGradRows * kGradChunks];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave & 1, wk = wave >> 1;
    const uint32_t tile = blockIdx.x % (g.tiles_n * g.tiles_k);
    const int split = (int)(blockIdx.x / (g.tiles_n * g.tiles_k));
    const int n0 = (int)(tile % g.tiles_n) * kGradTile, k0 = (int)(tile / g.tiles_n) * kGradTile;
    const int64_t m_begin = (int64_t)split * g.rows_per_split;
    const int64_t m_end = m_begin + g.rows_per_split < g.M ? m_begin + g.rows_per_split : (int64_t)g.M;
    const int chunk = threadIdx.x % kGradChunks, row0 = threadIdx.x / kGradChunks;
    const int nc = n0 + chunk * 8, kc = k0 + chunk * 8;
    const bool sums = g.db && k0 == 0;
    const int k_whole = (g.K + kMxBlock - 1) / kMxBlock * kMxBlock;   // codes of a row

    float db[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) db[i] = 0.0f;
    u32x4 hz[kPer], hx[kPer];
    uint32_t hs[kPer];
    auto load = [&](int64_t m0) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int64_t m = m0 + row0 + i * (256 / kGradChunks);
            hz[i] = hx[i] = u32x4{0, 0, 0, 0};
            hs[i] = 0;
            if (m < m_end) {
                if (nc < g.N) hz[i] = Row8<uint16_t>::load_raw(g.dz + m * g.lddz, nc, g.N);
                if (g.x_bf16) {
                    if (kc < g.K) hx[i] = Row8<uint16_t>::load_raw((const uint16_t*)(g.x.codes + m * g.x.ld), kc, g.K);
                } else if (kc < k_whole) {
                    const u32x2 p = *(const u32x2*)(g.x.codes + m * g.x.ld + kc);
                    hx[i][0] = p[0];
                    hx[i][1] = p[1];
                    hs[i] = g.x.scales[m * g.x.ld_scales + kc / kMxBlock];
                }
            }
        }
    };
    auto store = [&](u32x4* lds) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int slot = grad_slot(row0 + i * (256 / kGradChunks), chunk);
            lds[slot] = hz[i];
            lds[kGradRows * kGradChunks + slot] = g.x_bf16 ? hx[i] : e4m3x8_as_bf16(u32x2{hx[i][0], hx[i][1]}, (int)hs[i]);
            if (sums)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    db[e] += __uint_as_float(e & 1 ? hz[i][e / 2] & 0xffff0000u : hz[i][e / 2] << 16);
        }
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    auto compute = [&](const u32x4* lds) {
        sfor<kGradRows / 16>([&](auto S) {
            bf16x8 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) a[i] = read_columns(lds, CV(S) * 16, (wn * 2 + i) * 32, lane);
#pragma unroll
            for (int j = 0; j < 2; ++j) b[j] = read_columns(lds + kGradRows * kGradChunks, CV(S) * 16, (wk * 2 + j) * 32, lane);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
        });
    };
    auto step = [&](u32x4* now, u32x4* next, int64_t m0) {
        const bool more = m0 + kGradRows < m_end;
        if (more) load(m0 + kGradRows);
        compute(now);
        if (more) {
            store(next);
            lds_barrier();
        }
    };
    load(m_begin);
    store(ring0);
    lds_barrier();
    for (int64_t m0 = m_begin; m0 < m_end; m0 += 2 * kGradRows) {
        step(ring0, ring1, m0);
        if (m0 + kGradRows < m_end) step(ring1, ring0, m0 + kGradRows);
    }

    float* out = g.dw + (int64_t)split * g.split_stride;
    if (g.dw)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int k = k0 + (wk * 2 + j) * 32 + (lane & 31);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int n = n0 + (wn * 2 + i) * 32 + (e & 3) + 8 * (e >> 2) + 4 * (lane >> 5);
                if (n < g.N && k < g.K) {
                    float* p = out + (int64_t)n * g.lddw + k;
                    *p = g.accumulate ? *p + acc[i][j][e] : acc[i][j][e];
                }
            }
        }
    if (sums) {   // the threads of a chunk's sixteen rows, summed in their order
        lds_barrier();
        float* part = (float*)ring0;
#pragma unroll
        for (int e = 0; e < 8; ++e) part[row0 * kGradTile + chunk * 8 + e] = db[e];
        lds_barrier();
        const int c = threadIdx.x;
        if (c < kGradTile && n0 + c < g.N) {
            float s = 0.0f;
            for (int r = 0; r < 256 / kGradChunks; ++r) s += part[r * kGradTile + c];
            float* p = g.db + (int64_t)split * g.N + n0 + c;
            *p = g.accumulate ? *p + s : s;
        }
    }
}

// dW and db from the splits' parts, added in their order.
__global__ void __launch_bounds__(256) grad_sum_kernel(const float* dw_parts, const float* db_parts, int splits, int N,
                                                       int K, float* dw, int64_t lddw, float* db, int accumulate) {
    const int64_t nk = (int64_t)N * K, total = (dw ? nk : 0) + (db ? N : 0);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const bool is_w = dw && i < nk;
        const int64_t at = is_w ? i : i - (dw ? nk : 0);
        const float* p = is_w ? dw_parts + at : db_parts + at;
        const int64_t stride = is_w ? nk : N;
        float s = 0.0f;
#pragma unroll 8
        for (int k = 0; k < splits; ++k) s += p[k * stride];
        float* o = is_w ? dw + at / K * lddw + at % K : db + at;
        *o = accumulate ? *o + s : s;
    }
}

struct GradPlan {
    int tiles_n, tiles_k, splits, rows_per_split;
    size_t transposed, parts;   // bytes
};

// The batch is split until two workgroups per compute unit have work.
GradPlan grad_plan(int64_t M, int N, int K, int n_cu) {
    GradPlan p;
    p.tiles_n = (N + kGradTile - 1) / kGradTile;
    p.tiles_k = (K + kGradTile - 1) / kGradTile;
    const int64_t stages = (M + kGradRows - 1) / kGradRows;
    const int64_t tiles = (int64_t)p.tiles_n * p.tiles_k;
    int64_t want = 2 * (int64_t)n_cu / tiles;
    want = want < 1 ? 1 : want > stages ? (stages < 1 ? 1 : stages) : want;
    const int64_t per = (stages + want - 1) / want;
    p.rows_per_split = (int)(per < 1 ? kGradRows : per * kGradRows);
    p.splits = M == 0 ? 0 : (int)((M + p.rows_per_split - 1) / p.rows_per_split);
    p.transposed = ((size_t)K * ((size_t)(N + 7) / 8 * 8) * 2 + 255) / 256 * 256;
    p.parts = p.splits > 1 ? (size_t)p.splits * ((size_t)N * K + N) * sizeof(float) : 0;
    return p;
}

}  // namespace

hipError_t launch_train_linear(const GemmArgs& g, int n_cu, hipStream_t stream) {
    const bool da = whole_chunks(g.a, g.K), db = whole_chunks(g.b, g.K);
    if (da && db) return launch_layer_gemm<kOpBf16, true, true, kEpiKept>(g, n_cu, stream);
    return launch_layer_gemm<kOpBf16, false, false, kEpiKept>(g, n_cu, stream);
}

size_t backward_workspace(int64_t M, int N, int K, int n_cu) {
    const GradPlan p = grad_plan(M, N, K, n_cu);
    return p.transposed + p.parts;
}

hipError_t launch_train_linear_backward(const BackwardArgs& a, int n_cu, hipStream_t stream) {
    const GradPlan p = grad_plan(a.M, a.N, a.K, n_cu);
    hipError_t e = hipSuccess;
    if (a.dx && a.M > 0) {
        uint16_t* wt = (uint16_t*)a.workspace;
        const int64_t ldt = (a.N + 7) / 8 * 8;
        const dim3 grid((uint32_t)((ldt + kTrTile - 1) / kTrTile), (uint32_t)((a.K + kTrTile - 1) / kTrTile));
        hipLaunchKernelGGL(transpose_kernel, grid, dim3(256), 0, stream, a.w, a.ldw, a.N, a.K, wt, ldt);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        GemmArgs g{};
        g.a = MxIn{(const uint8_t*)wt, ldt * 2, nullptr, 0};
        g.b = MxIn{(const uint8_t*)a.dz, a.lddz * 2, nullptr, 0};
        g.y = (uint8_t*)a.dx;
        g.ldy = a.lddx;
        g.mask = a.x.codes;
        g.ld_mask = a.x_bf16 ? a.x.ld / 2 : a.x.ld;
        g.mask_type = !a.relu ? kMaskNone : a.x_bf16 ? kMaskBf16 : kMaskMx8;
        g.M = a.M;
        g.N = a.K;
        g.K = a.N;
        e = whole_chunks(g.b, g.K) ? launch_layer_gemm<kOpBf16, true, true, kEpiMasked>(g, n_cu, stream)
                                   : launch_layer_gemm<kOpBf16, true, false, kEpiMasked>(g, n_cu, stream);
        if (e != hipSuccess) return e;
    }
    if (!a.dw && !a.db) return e;
    float* dw_parts = (float*)(a.workspace + p.transposed);
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
        g.dw = !a.dw ? nullptr : direct ? a.dw : dw_parts;
        g.split_stride = direct ? 0 : (int64_t)a.N * a.K;
        g.lddw = direct ? a.lddw : a.K;
        g.db = !a.db ? nullptr : direct ? a.db : db_parts;
        g.accumulate = direct ? a.accumulate : 0;
        const dim3 grid((uint32_t)((size_t)p.tiles_n * p.tiles_k * p.splits));
        hipLaunchKernelGGL(weight_grad_kernel, grid, dim3(256), 0, stream, g);
        if ((e = hipGetLastError()) != hipSuccess || direct) return e;
    }
    const int64_t total = (int64_t)a.N * a.K + a.N;
    const uint64_t wg = (uint64_t)((total + 255) / 256), most = (uint64_t)n_cu * 32;
    hipLaunchKernelGGL(grad_sum_kernel, dim3((uint32_t)(wg < most ? wg : most)), dim3(256), 0, stream, dw_parts, db_parts,
                       p.splits, a.N, a.K, a.dw, a.lddw, a.db, a.accumulate);
    return hipGetLastError();
}

}  // namespace donerf
