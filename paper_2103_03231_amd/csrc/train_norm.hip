// train_norm.hip - layer norm over a row's columns, forward and backward.
//
//   forward   m = mean(x), r = 1/sqrt(mean((x - m)^2) + eps), z = (x - m) r w + b,
//             y = act(z): one pass, the row in registers between its sums.  The
//             first sum's mean is off by its roundings; the differences to it give
//             what it lacks, so that rows far from zero, or of one value, are exact.
//             It is of the values times 2^-17: 65,536 of them do not overflow.  Where
//             their squares do, r = 0, and m is one that x - m is finite with: xh is 0.
//   backward  with xh = (x - m) r and g = dz w:
//             dx = r (g - mean(g) - xh mean(g xh)), dw = sum over rows of dz xh,
//             db = that of dz.  Each workgroup adds up dw and db of its rows in
//             registers, and a second launch adds the workgroups' parts; where values
//             are few, workgroups of the one launch sum them by columns.
//
// Both are bound by memory where rows are many, by the launch where they are few (13 x 256
// 2.2 us forward, 3.1 backward).
#include "rows.h"

namespace donerf {
namespace {

constexpr float kLargest = 0x1.fffffep127f;   // finite
// A row's mean as xh takes it: 0 where r is 0 and a finite value less the mean might not be
// finite (2^102 is a quarter of the largest value's last place).
__device__ __forceinline__ float centre_of(float mean, float r) { return r == 0.0f && __builtin_fabsf(mean) >= 0x1p102f ? 0.0f : mean; }

// ---------------------------------------------------------------- forward

// w and b at a chunk's columns, or at a lane's single one.
__device__ __forceinline__ void affine_at(const NormArgs& a, const Columns& c, int k, float* w, float* b) {
    const RowsIn<float> ws(a.w, 0, a.cols), bs(a.b, 0, a.cols);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.0f, b[i] = 0.0f;
    if (a.w) ws.load(0, k).values(w);
    if (a.b) bs.load(0, k).values(b);
}

// 160,000 x 256 bf16 with y and kept: 40 us, 207 MB, 5.2 TB/s, the rate of a copy.  The
// next row is on its way while a row's three sums wait for each other: fp32 38.8 -> 37.5 us
// at 32,768 x 1024, bf16 level; rows of more than four waves lose by it (16,384 fp32
// columns 46 -> 53 us).
template <class T, int L, int C, bool KEEP>
__global__ void __launch_bounds__(row_threads(L)) norm_kernel(NormArgs a) {
    constexpr int kGroups = row_threads(L) / L;
    constexpr bool kHeld = C <= 2;   // w and b in registers, too
    constexpr bool kAhead = L <= 256;
    __shared__ typename RowReduce<L, 1>::Lds lds;
    RowReduce<L, 1> reduce(&lds);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const RowsIn<T> x((const T*)a.x, a.ldx, a.cols);
    const Columns& c = x.c;
    float w[kHeld ? C : 1][8], b[kHeld ? C : 1][8];
    if constexpr (kHeld)
#pragma unroll
        for (int j = 0; j < C; ++j) affine_at(a, c, 8 * (lane + L * j), w[j], b[j]);
    auto act = [&](float z) { return a.relu ? __builtin_elementwise_maximum(z, 0.0f) : z; };
    Raw<T> next[C];   // the row to come
    float one_next = 0.0f;
    auto load = [&](uint32_t r0) {
        const int64_t row = r0 + group < a.rows ? r0 + group : a.rows - 1;
#pragma unroll
        for (int j = 0; j < C; ++j) next[j] = x.load(row, 8 * (lane + L * j));
        if (c.any_single()) one_next = x.load_single(row, lane);
    };
    if (kAhead) load(blockIdx.x * kGroups);
    // the same number of rows for every wave: sums over a workgroup's waves need them all
    const uint32_t step = gridDim.x * kGroups;
    for (uint32_t r0 = blockIdx.x * kGroups; r0 < a.rows; r0 += step) {
        const bool live = r0 + group < a.rows;
        const int64_t row = live ? r0 + group : a.rows - 1;
        if (!kAhead) load(r0);
        Raw<T> raw[C];
#pragma unroll
        for (int j = 0; j < C; ++j) raw[j] = next[j];
        const float one = one_next;
        if (kAhead && r0 + step < a.rows) load(r0 + step);
        auto total = [&](auto add) {   // over the row's values; add: a sum and a value
            float sum = c.has_single(lane) ? add(0.0f, one) : 0.0f;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                if (c.has(8 * (lane + L * j))) {
                    float v[8];
                    raw[j].values(v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = add(sum, v[i]);
                }
                raw[j].hold();
            }
            return reduce.template one<Add>(sum);
        };
        // (times a power of two: the bits of the plain sum, where that is finite)
        const float sum = total([](float s, float v) { return __builtin_fmaf(v, 0x1p-17f, s); });
        const float first = __builtin_amdgcn_fmed3f(sum * (a.inv_cols * 0x1p17f), -kLargest, kLargest);
        const float rest = total([&](float s, float v) { return s + (v - first); }) * a.inv_cols;
        // where only the differences overflow, the first mean is as good as fp32 has it; where a
        // value is not finite the mean is NaN
        const float mean = first + (__builtin_fabsf(rest) <= kLargest ? rest : sum - sum);
        const float var = total([&](float s, float v) { return s + (v - mean) * (v - mean); }) * a.inv_cols;
        const float r = __builtin_amdgcn_rsqf(var + a.eps), centre = centre_of(mean, r);
        if (!live) continue;   // behind the last sum of this row
        if (lane == 0) *(f32x2*)(a.stats + 2 * row) = f32x2{centre, r};
        float tail[8];   // kept values: the chunk that is not whole, by the lane whose turn it is
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < 8; ++i) tail[i] = 0.0f;
            if (c.any_single() && lane == c.whole / 8 % L)
#pragma unroll
                for (int i = 0; i < 7; ++i) {
                    const int k = c.whole + i < a.cols ? c.whole + i : a.cols - 1;
                    const float xh = (value_of(x.base[row * x.ld + k]) - centre) * r;
                    const float z = act(__builtin_fmaf(xh, a.w ? a.w[k] : 1.0f, a.b ? a.b[k] : 0.0f));
                    tail[i] = c.whole + i < a.cols ? z : 0.0f;
                }
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int k = 8 * (lane + L * j);
            float v[8];
            raw[j].values(v);
            float wj[8], bj[8];
            if constexpr (!kHeld) affine_at(a, c, k, wj, bj);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = act(__builtin_fmaf((v[i] - centre) * r, kHeld ? w[kHeld ? j : 0][i] : wj[i], kHeld ? b[kHeld ? j : 0][i] : bj[i]));
            if (a.y.base && c.has(k)) store8(a.y, row, k, v);
            if constexpr (KEEP) {
                if (!c.has(k))
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = k == c.whole ? tail[i] : 0.0f;
                store_mx8(a.q, row, k, a.cols, v);
            }
        }
        if (c.has_single(lane) && a.y.base) {
            const int k = c.single(lane);
            store1(a.y, row, k, act(__builtin_fmaf((one - centre) * r, a.w ? a.w[k] : 1.0f, a.b ? a.b[k] : 0.0f)));
        }
    }
}

// ---------------------------------------------------------------- backward

// x of type X: float, uint16_t (bf16) or uint8_t (E4M3).
template <class X>
struct NormInput : RowsIn<X> {
    __device__ __forceinline__ explicit NormInput(const NormBackwardArgs& a) : RowsIn<X>((const X*)a.x.codes, a.x.ld, a.cols) {}
};
template <>
struct NormInput<uint8_t> : Mx8In {
    __device__ __forceinline__ explicit NormInput(const NormBackwardArgs& a) : Mx8In(a.x, a.cols) {}
};

// A workgroup's part of dw and db.
struct NormSums {
    float* w;
    float* b;
    __device__ __forceinline__ explicit NormSums(const NormBackwardArgs& a) : w(a.parts + (int64_t)blockIdx.x * 2 * a.cols), b(w + a.cols) {}
};
// Threads of a workgroup of the backward pass.
constexpr int backward_threads(int L) { return L > 512 ? L : 512; }

// The sum of v over the lanes of a wave with the same number modulo 4, in its first four.
__device__ __forceinline__ float fourths_all(float v) {
    v += dpp<0x124>(v);   // rotated by 4 and by 8 among 16
    v += dpp<0x128>(v);
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// dw and db of 32 columns, all rows, by a workgroup: four lanes a row, 128 rows at a time,
// a fourth of each row's cache line or a whole one.  The last slab is that of the single
// columns.
__host__ __device__ inline uint32_t column_slabs(int cols) { return (uint32_t)((cols & ~7) + 31) / 32 + (cols % 8 ? 1 : 0); }
template <class X, class Z, int THREADS>
__device__ __forceinline__ void sum_columns(const NormBackwardArgs& a, uint32_t slab, float (*lds)[64]) {
    const NormInput<X> x(a);
    const RowsIn<Z> dz((const Z*)a.dz, a.lddz, a.cols);
    const Columns& c = dz.c;
    const int lane = threadIdx.x % 4, wave = threadIdx.x / 64, k = 32 * (int)slab + 8 * lane;
    float dw[8] = {0, 0, 0, 0, 0, 0, 0, 0}, db[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const bool singles = 32 * (int)slab >= c.whole;
    if (singles) {   // lanes 0 to 3 have two each
        for (uint32_t row = threadIdx.x / 4; row < a.rows; row += THREADS / 4) {
            const f32x2 st = *(const f32x2*)(a.stats + 2 * (int64_t)row);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float z = dz.load_single(row, lane + 4 * i);
                dw[i] = __builtin_fmaf(z, (x.load_single(row, lane + 4 * i) - st[0]) * st[1], dw[i]);
                db[i] += z;
            }
        }
    } else if (c.has(k)) {
#pragma unroll 4
        for (uint32_t row = threadIdx.x / 4; row < a.rows; row += THREADS / 4) {
            const f32x2 st = *(const f32x2*)(a.stats + 2 * (int64_t)row);
            float v[8], z[8];
            x.load(row, k).values(v);
            dz.load(row, k).values(z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[i] = __builtin_fmaf(z[i], (v[i] - st[0]) * st[1], dw[i]);
                db[i] += z[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        dw[i] = fourths_all(dw[i]);
        db[i] = fourths_all(db[i]);
        if (threadIdx.x % 64 < 4) lds[wave][8 * lane + i] = dw[i], lds[wave][32 + 8 * lane + i] = db[i];
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    float sum = lds[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) sum += lds[w][threadIdx.x];
    const int t = threadIdx.x % 32;
    const int col = singles ? (t % 8 < 2 ? c.whole + t / 8 + 4 * (t % 8) : a.cols) : 32 * (int)slab + t < c.whole ? 32 * (int)slab + t : a.cols;
    float* const out = threadIdx.x < 32 ? a.dw : a.db;
    if (out && col < a.cols) out[col] = a.accumulate ? out[col] + sum : sum;
}
template <class X, class Z>
__global__ void __launch_bounds__(512) norm_few_columns_kernel(NormBackwardArgs a) {
    __shared__ float lds[8][64];
    sum_columns<X, Z, 512>(a, blockIdx.x, lds);
}

// SUMS: each workgroup adds up dw and db of its rows on the way.  Without: the workgroups
// behind those of the rows (a.row_groups of them) do, each for its columns.
// x and dz are read once and dx is written: 160,000 x 256 from 8 bits 43.8 us, 207 MB, 4.7 TB/s;
// 8192 x 4096 from fp32 53 us, 269 MB, 5.1 TB/s.  Loading the next row ahead costs registers that
// the sums need: 39 -> 45 and 50 -> 57 us.
template <class X, class Z, int L, int C, bool SUMS>
__global__ void __launch_bounds__(backward_threads(L), 4) norm_backward_kernel(NormBackwardArgs a) {
    constexpr int kThreads = backward_threads(L), kGroups = kThreads / L;
    typedef RowReduce<L, 2, kThreads> Reduce;
    __shared__ typename Reduce::Lds lds;
    __shared__ float parts[!SUMS ? kThreads : kGroups > 1 ? 8 * kThreads : 1];
    if constexpr (!SUMS)
        if (blockIdx.x >= a.row_groups) return sum_columns<X, Z, kThreads>(a, blockIdx.x - a.row_groups, (float (*)[64])parts);
    const uint32_t workgroups = SUMS ? gridDim.x : a.row_groups;
    Reduce reduce(&lds);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const NormInput<X> x(a);
    const RowsIn<Z> dz((const Z*)a.dz, a.lddz, a.cols);
    const Columns& c = dz.c;
    const RowsIn<float> ws(a.w, 0, a.cols);
    float dw[C][8], db[C][8], w[C][8];
    float dw1 = 0.0f, db1 = 0.0f, w1 = 1.0f;   // of the single column
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = 0.0f, db[j][i] = 0.0f, w[j][i] = 1.0f;
        if (a.w) ws.load(0, 8 * (lane + L * j)).values(w[j]);
    }
    if (a.w) w1 = ws.load_single(0, lane);
    for (uint32_t r0 = blockIdx.x * kGroups; r0 < a.rows; r0 += workgroups * kGroups) {
        const bool live = r0 + group < a.rows;
        const int64_t row = live ? r0 + group : a.rows - 1;
        typename NormInput<X>::Held xr[C];
        Raw<Z> zr[C];
#pragma unroll
        for (int j = 0; j < C; ++j) {
            xr[j] = x.load(row, 8 * (lane + L * j));
            zr[j] = dz.load(row, 8 * (lane + L * j));
        }
        const f32x2 st = *(const f32x2*)(a.stats + 2 * row);
        const float mean = st[0], r = st[1];
        float v1 = 0.0f, z1 = 0.0f;
        if (c.any_single()) {
            v1 = x.load_single(row, lane);
            z1 = dz.load_single(row, lane);
        }
        float s[2] = {0.0f, 0.0f};
        if (live && c.has_single(lane)) {
            const float xh = (v1 - mean) * r, g = z1 * w1;
            s[0] = g;
            s[1] = g * xh;
            if (SUMS) {
                dw1 = __builtin_fmaf(z1, xh, dw1);
                db1 += z1;
            }
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (live && c.has(8 * (lane + L * j))) {
                float v[8], z[8];
                xr[j].values(v);
                zr[j].values(z);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xh = (v[i] - mean) * r, g = z[i] * w[j][i];
                    s[0] += g;
                    s[1] = __builtin_fmaf(g, xh, s[1]);
                    if (SUMS) {
                        dw[j][i] = __builtin_fmaf(z[i], xh, dw[j][i]);
                        db[j][i] += z[i];
                    }
                }
            }
            xr[j].hold();
            zr[j].hold();
        }
        reduce.template all<Add>(s);
        if (!a.dx.base || !live) continue;
        const float one = s[0] * a.inv_cols, two = s[1] * a.inv_cols;
        auto grad = [&](float v, float z, float wk) {
            const float xh = (v - mean) * r;
            return r * __builtin_fmaf(-xh, two, __builtin_fmaf(z, wk, -one));
        };
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int k = 8 * (lane + L * j);
            if (!c.has(k)) continue;
            float v[8], z[8];
            xr[j].values(v);
            zr[j].values(z);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = a.relu && is_zero(xr[j], v, i) ? 0.0f : grad(v[i], z[i], w[j][i]);
            store8(a.dx, row, k, z);
        }
        if (c.has_single(lane))
            store1(a.dx, row, c.single(lane), a.relu && x.single_is_zero(v1, row, lane) ? 0.0f : grad(v1, z1, w1));
    }
    if (!SUMS) return;
    const NormSums out(a);
    if constexpr (kGroups > 1) {
        // the row groups' sums in their order, 8 columns of each lane at a time
        auto join = [&](const float (&v)[8], float* to, int k0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) parts[group * 8 * L + 8 * lane + i] = v[i];
            __syncthreads();
            for (int t = threadIdx.x; t < 8 * L; t += kThreads) {
                float sum = parts[t];
                for (int g = 1; g < kGroups; ++g) sum += parts[g * 8 * L + t];
                if (c.has(k0 + t)) to[k0 + t] = sum;
            }
            __syncthreads();
        };
#pragma unroll
        for (int j = 0; j < C; ++j) {
            join(dw[j], out.w, 8 * L * j);
            join(db[j], out.b, 8 * L * j);
        }
        if (c.any_single()) {
            parts[2 * threadIdx.x] = dw1;
            parts[2 * threadIdx.x + 1] = db1;
            __syncthreads();
            if (group == 0 && c.has_single(lane)) {
                for (int g = 1; g < kGroups; ++g) {
                    dw1 += parts[2 * (g * L + lane)];
                    db1 += parts[2 * (g * L + lane) + 1];
                }
                out.w[c.single(lane)] = dw1;
                out.b[c.single(lane)] = db1;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int k = 8 * (lane + L * j);
            if (!c.has(k)) continue;
            __builtin_memcpy(out.w + k, dw[j], 32);
            __builtin_memcpy(out.b + k, db[j], 32);
        }
        if (c.has_single(lane)) {
            out.w[c.single(lane)] = dw1;
            out.b[c.single(lane)] = db1;
        }
    }
}

// Rows that registers do not hold: dx, read once for their sums and once, from the caches,
// for itself.  200 x 40,000 with dw and db 33 us.
template <class X, class Z>
__global__ void __launch_bounds__(1024) norm_backward_wide_kernel(NormBackwardArgs a) {
    constexpr int L = 1024;
    __shared__ typename RowReduce<L, 2>::Lds lds;
    RowReduce<L, 2> reduce(&lds);
    const NormInput<X> x(a);
    const RowsIn<Z> dz((const Z*)a.dz, a.lddz, a.cols);
    const Columns& c = dz.c;
    const RowsIn<float> ws(a.w, 0, a.cols);
    const int lane = threadIdx.x;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const f32x2 st = *(const f32x2*)(a.stats + 2 * (int64_t)row);
        const float mean = st[0], r = st[1];
        float s[2] = {0.0f, 0.0f}, v[8], z[8], w[8] = {1, 1, 1, 1, 1, 1, 1, 1}, v1 = 0.0f, z1 = 0.0f, w1 = 1.0f;
        if (c.has_single(lane)) {
            v1 = x.load_single(row, lane);
            z1 = dz.load_single(row, lane);
            if (a.w) w1 = ws.load_single(0, lane);
            s[0] = z1 * w1;
            s[1] = z1 * w1 * ((v1 - mean) * r);
        }
        for (int k = 8 * lane; c.has(k); k += 8 * L) {
            x.load(row, k).values(v);
            dz.load(row, k).values(z);
            if (a.w) ws.load(0, k).values(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = z[i] * w[i];
                s[0] += g;
                s[1] = __builtin_fmaf(g, (v[i] - mean) * r, s[1]);
            }
        }
        reduce.template all<Add>(s);
        const float one = s[0] * a.inv_cols, two = s[1] * a.inv_cols;
        auto grad = [&](float vk, float zk, float wk) {
            const float xh = (vk - mean) * r;
            return r * __builtin_fmaf(-xh, two, __builtin_fmaf(zk, wk, -one));
        };
        for (int k = 8 * lane; c.has(k); k += 8 * L) {
            const auto xr = x.load(row, k);
            xr.values(v);
            dz.load(row, k).values(z);
            if (a.w) ws.load(0, k).values(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = a.relu && is_zero(xr, v, i) ? 0.0f : grad(v[i], z[i], w[i]);
            store8(a.dx, row, k, z);
        }
        if (c.has_single(lane))
            store1(a.dx, row, c.single(lane), a.relu && x.single_is_zero(v1, row, lane) ? 0.0f : grad(v1, z1, w1));
    }
}

// Their dw and db: 2048 columns (blockIdx.y) over a share of the rows.
template <class X, class Z>
__global__ void __launch_bounds__(256) norm_columns_kernel(NormBackwardArgs a) {
    const NormInput<X> x(a);
    const RowsIn<Z> dz((const Z*)a.dz, a.lddz, a.cols);
    const Columns& c = dz.c;
    const NormSums out(a);
    const int t = (int)(blockIdx.y * 256 + threadIdx.x), k = 8 * t;
    if (c.has(k)) {
        float dw[8], db[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[i] = 0.0f, db[i] = 0.0f;
#pragma unroll 4
        for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
            const f32x2 st = *(const f32x2*)(a.stats + 2 * (int64_t)row);
            float v[8], z[8];
            x.load(row, k).values(v);
            dz.load(row, k).values(z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[i] = __builtin_fmaf(z[i], (v[i] - st[0]) * st[1], dw[i]);
                db[i] += z[i];
            }
        }
        __builtin_memcpy(out.w + k, dw, 32);
        __builtin_memcpy(out.b + k, db, 32);
    }
    if (c.has_single(t)) {
        float dw = 0.0f, db = 0.0f;
        for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
            const f32x2 st = *(const f32x2*)(a.stats + 2 * (int64_t)row);
            const float z = dz.load_single(row, t);
            dw = __builtin_fmaf(z, (x.load_single(row, t) - st[0]) * st[1], dw);
            db += z;
        }
        out.w[c.single(t)] = dw;
        out.b[c.single(t)] = db;
    }
}

// Sums of n parts of 2 cols values (dw, then db), 32 columns a workgroup (whole cache
// lines), 32 threads each: 4.7 us for 512 parts of 256 and of 4096 columns, two round trips to
// memory and the launch.
__global__ void __launch_bounds__(1024) norm_parts_kernel(const float* parts, uint32_t n, int cols, float* dw, float* db,
                                                          int accumulate) {
    __shared__ float lds[16][32];
    const int c = threadIdx.x % 32, slice = threadIdx.x / 32;
    const int64_t at = (int64_t)blockIdx.x * 32 + c;
    float sum = 0.0f;
    if (at < 2 * cols)
#pragma unroll 16
        for (uint32_t p = slice; p < n; p += 32) sum += parts[p * (int64_t)(2 * cols) + at];
    // a wave's two slices, then the waves
    sum += __shfl_xor(sum, 32, 64);
    if (threadIdx.x % 64 < 32) lds[slice / 2][c] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || at >= 2 * cols) return;
    sum = lds[0][c];
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += lds[w][c];
    float* const out = at < cols ? dw : db;
    const int64_t k = at < cols ? at : at - cols;
    if (out) out[k] = accumulate ? out[k] + sum : sum;
}

__global__ void __launch_bounds__(256) norm_zero_kernel(float* dw, float* db, int cols) {
    const int k = blockIdx.x * 256 + threadIdx.x;
    if (k >= cols) return;
    if (dw) dw[k] = 0.0f;
    if (db) db[k] = 0.0f;
}

// ---------------------------------------------------------------- launches

template <class T, int L, int C>
hipError_t forward_launch(const NormArgs& a, int n_cu, hipStream_t stream) {
    constexpr uint32_t groups = row_threads(L) / L;
    const uint32_t need = (a.rows + groups - 1) / groups, full = (uint32_t)n_cu * (2048 / row_threads(L));
    const dim3 grid(need < full ? need : full), threads(row_threads(L));
    if (a.q.codes) hipLaunchKernelGGL((norm_kernel<T, L, C, true>), grid, threads, 0, stream, a);
    else hipLaunchKernelGGL((norm_kernel<T, L, C, false>), grid, threads, 0, stream, a);
    return hipGetLastError();
}
// 16 columns a lane (33.5 million bf16 values: 256 columns 23.6 us, with 8 a lane 25.6;
// 1024 columns 24.1, with 32 26.9; 2048 24.7, with 32 27.2; 8192 26.8, with 32 28.8), and up
// to 64 where a row would need more than 512 lanes: 16,384 columns 31 us with 512, 33 with
// 256 and with 1024.  Beyond 16,384 one row of a compute unit's has nothing to overlap its three
// sums: 1048 x 32,000 bf16 41.6 us on 26 of memory; and beyond 32,768 a lane's 64 values
// leave 36 to 248 bytes of it in scratch: 1024 x 65,536 bf16 77 us on 52, and more than twice
// that where it is read three times instead.
template <class T>
hipError_t forward_by_width(const NormArgs& a, int n_cu, hipStream_t s) {
    const int c = a.cols;
    return c <= 64 ? forward_launch<T, 8, 1>(a, n_cu, s) : c <= 128 ? forward_launch<T, 8, 2>(a, n_cu, s)
         : c <= 256 ? forward_launch<T, 16, 2>(a, n_cu, s) : c <= 512 ? forward_launch<T, 32, 2>(a, n_cu, s)
         : c <= 1024 ? forward_launch<T, 64, 2>(a, n_cu, s) : c <= 2048 ? forward_launch<T, 128, 2>(a, n_cu, s)
         : c <= 4096 ? forward_launch<T, 256, 2>(a, n_cu, s) : c <= 8192 ? forward_launch<T, 512, 2>(a, n_cu, s)
         : c <= 16384 ? forward_launch<T, 512, 4>(a, n_cu, s) : c <= 32768 ? forward_launch<T, 1024, 4>(a, n_cu, s)
         : forward_launch<T, 1024, 8>(a, n_cu, s);
}

// Lanes of a row in the backward pass, of 16 columns each (8 columns: 160,000 x 256 48 us for
// 46.7, 8192 x 4096 65.5 for 60), 0 for rows that registers do not hold.
int backward_lanes(int cols) {
    int lanes = 8;
    while (lanes < 1024 && 16 * lanes < cols) lanes *= 2;
    return cols <= 16 * 1024 ? lanes : 0;
}
// So few values that dw and db are summed by columns, from the caches, in the launch that
// makes dx: 4 million of rows up to 4096 columns, 8 million of wider ones, whose workgroups
// leave more parts.  Calls with it and in two launches, x in fp32 and in bf16: 1021 x 283
// 11.6 and 15.8 us, 12.0 and 15.5; 2048 x 2048 15.6 and 16.1, 15.5 and 15.2; 1024 x 4096 13.6 and
// 17.5, 13.0 and 19.0; 1170 x 5934 27.3 and 25.6, 23.0 and 23.3; 1024 x 8192 23.6 and 26.0, 22.5
// and 24.1; 512 x 16,384 24.3 and 33.1, 23.0 and 31.6.  Left to two: 1500 x 4096 21.4 and 18.6,
// 21.9 and 17.8; 2048 x 4096 23.4 and 21.2, 22.9 and 19.6; 1024 x 16,384 42.5 and 48.1, 39.1 and
// 38.8 (from 8 bits 42.3 and 37.6); 4096 x 512 18.6 and 15.2.
bool few_values(int64_t rows, int cols) { return rows <= 2048 && rows * cols <= (int64_t)1 << (cols <= 4096 ? 22 : 23); }
// Workgroups of the backward pass that each leave a part of dw and db.
uint32_t backward_groups(int64_t rows, int cols, int n_cu) {
    const int lanes = backward_lanes(cols);
    const int64_t per = lanes ? backward_threads(lanes) / lanes : 16;
    const int64_t need = (rows + per - 1) / per;
    // two workgroups of 512 threads a compute unit, eight of 256 where they share columns (more
    // would leave more parts to add up)
    const int64_t most = lanes ? (int64_t)n_cu * 1024 / backward_threads(lanes) : (int64_t)n_cu * 8 / ((cols + 2047) / 2048) + 1;
    return (uint32_t)(need < most ? need : most);
}

template <class X, class Z, int L, int C>
void backward_kernel(NormBackwardArgs a, uint32_t wg, hipStream_t s) {
    const dim3 threads(backward_threads(L));
    if (a.parts) {
        hipLaunchKernelGGL((norm_backward_kernel<X, Z, L, C, true>), dim3(wg), threads, 0, s, a);
    } else {
        a.row_groups = a.dx.base ? wg : 0;
        const uint32_t columns = a.dw || a.db ? column_slabs(a.cols) : 0;
        hipLaunchKernelGGL((norm_backward_kernel<X, Z, L, C, false>), dim3(a.row_groups + columns), threads, 0, s, a);
    }
}
template <class X, class Z>
hipError_t backward_by_width(NormBackwardArgs a, float* workspace, int n_cu, hipStream_t s) {
    const bool few = few_values(a.rows, a.cols), sums = a.dw || a.db;
    a.parts = sums && !few ? workspace : nullptr;
    uint32_t wg = backward_groups(a.rows, a.cols, n_cu);
    switch (backward_lanes(a.cols)) {
        case 8: backward_kernel<X, Z, 8, 2>(a, wg, s); break;
        case 16: backward_kernel<X, Z, 16, 2>(a, wg, s); break;
        case 32: backward_kernel<X, Z, 32, 2>(a, wg, s); break;
        case 64: backward_kernel<X, Z, 64, 2>(a, wg, s); break;
        case 128: backward_kernel<X, Z, 128, 2>(a, wg, s); break;
        case 256: backward_kernel<X, Z, 256, 2>(a, wg, s); break;
        case 512: backward_kernel<X, Z, 512, 2>(a, wg, s); break;
        case 1024: backward_kernel<X, Z, 1024, 2>(a, wg, s); break;
        default:
            if (a.dx.base) {
                const uint32_t full = (uint32_t)n_cu * 2;
                hipLaunchKernelGGL((norm_backward_wide_kernel<X, Z>), dim3(a.rows < full ? a.rows : full), dim3(1024), 0, s, a);
            }
            if (sums && few) hipLaunchKernelGGL((norm_few_columns_kernel<X, Z>), dim3(column_slabs(a.cols)), dim3(512), 0, s, a);
            else if (sums) hipLaunchKernelGGL((norm_columns_kernel<X, Z>), dim3(wg, (a.cols + 2047) / 2048), dim3(256), 0, s, a);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.parts) return e;
    hipLaunchKernelGGL(norm_parts_kernel, dim3((2 * a.cols + 31) / 32), dim3(1024), 0, s, a.parts, wg, a.cols, a.dw, a.db, a.accumulate);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_train_norm(const NormArgs& a, bool x_bf16, int n_cu, hipStream_t stream) {
    return x_bf16 ? forward_by_width<uint16_t>(a, n_cu, stream) : forward_by_width<float>(a, n_cu, stream);
}

size_t norm_backward_workspace(int64_t rows, int cols, int n_cu) {
    return few_values(rows, cols) ? 0 : (size_t)backward_groups(rows, cols, n_cu) * 2 * (size_t)cols * sizeof(float);
}

hipError_t launch_train_norm_backward(const NormBackwardArgs& a, int x_type, bool dz_bf16, void* workspace, int n_cu,
                                      hipStream_t stream) {
    if (a.rows == 0) {
        if (a.accumulate || (!a.dw && !a.db)) return hipSuccess;
        hipLaunchKernelGGL(norm_zero_kernel, dim3((a.cols + 255) / 256), dim3(256), 0, stream, a.dw, a.db, a.cols);
        return hipGetLastError();
    }
    float* const ws = (float*)workspace;
    if (x_type == kRowsF32)
        return dz_bf16 ? backward_by_width<float, uint16_t>(a, ws, n_cu, stream) : backward_by_width<float, float>(a, ws, n_cu, stream);
    if (x_type == kRowsBf16)
        return dz_bf16 ? backward_by_width<uint16_t, uint16_t>(a, ws, n_cu, stream)
                       : backward_by_width<uint16_t, float>(a, ws, n_cu, stream);
    return dz_bf16 ? backward_by_width<uint8_t, uint16_t>(a, ws, n_cu, stream) : backward_by_width<uint8_t, float>(a, ws, n_cu, stream);
}

}  // namespace donerf
