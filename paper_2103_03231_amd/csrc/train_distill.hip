// train_distill.hip - distillation from a teacher's top logits, loss and gradient.
//
//   p = softmax of t / T over a row's given entries, q = softmax of x / T over its
//   classes, loss = w T^2 sum_e p_e (log p_e - log q_{c_e}),
//   dx_j = w T (q_j - sum of p_e over the e with c_e = j).
//
// One pass over x: a row's exponentials stay in registers between their sum and the
// gradient, and the next row is loaded over the logits that they were made of.  The
// entries' few columns are written a second time, behind the rest of their row and by
// the wave that wrote that: a wave's stores to one address keep their order.
//
// Bound by memory where rows are many: 160,000 x 128 bf16 18.6 us, 88 MB, 4.7 TB/s; 4096 x 32,000
// 102 us, 527 MB, 5.2 TB/s, the rate of a copy.  1021 x 192 4.4 us, round trips: entries, their
// classes' logits, four sums.
#include "../../include/donerf.h"
#include "rows.h"

namespace donerf {
namespace {

constexpr uint32_t kNegInfBits = 0xff800000u;
constexpr float kLn2 = 0.693147180559945f;

// A row's entries in LDS, k each: classes (-1: not given), logits, which become
// powers 2^((t - max) / (T ln 2)), and the powers of their classes' own logits.
struct Entries {
    int32_t* cls;
    float* power;
    float* own;
};

template <class T, int L, int C>
__global__ void __launch_bounds__(row_threads(L)) distill_kernel(DistillArgs a) {
    constexpr int kGroups = row_threads(L) / L;
    constexpr int kTurns = L > 64 ? 2 : 1;
    __shared__ typename RowReduce<L, 2>::Lds lds;
    __shared__ uint8_t owners[kGroups * 8 * L * C];   // a byte a column: one of the entries of that class
    extern __shared__ uint32_t room[];
    RowReduce<L, 2> reduce(&lds);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    // In two places by turns, where a row's waves are several: one that is a row ahead
    // writes to the other.
    int turn = 0;
    uint8_t* const owner = owners + group * 8 * L * C;
    const RowsIn<T> x((const T*)a.x, a.ldx, a.cols);
    const Columns& c = x.c;
    const float neg_inf = __uint_as_float(kNegInfBits);
    // what a row begins with: its chunks, its single column, its lane's first entry and its weight
    Raw<T> raw[C];
    float one, t0, weight;
    int64_t c0;
    auto load = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < C; ++j) raw[j] = x.load(row, 8 * (lane + L * j));
        one = c.any_single() ? x.load_single(row, lane) : 0.0f;
        const int e = lane < a.k ? lane : a.k - 1;
        c0 = a.classes.at(row, e);
        t0 = a.teacher.at(row, e);
        weight = a.weight ? a.weight[row] : 1.0f;
    };
    auto row_of = [&](uint32_t r0) { return (int64_t)(r0 + group < a.rows ? r0 + group : a.rows - 1); };
    const uint32_t step = gridDim.x * kGroups;
    uint32_t r0 = blockIdx.x * kGroups;
    load(row_of(r0));
    // the same number of rows for every wave: sums over a workgroup's waves need them all
    for (; r0 < a.rows; r0 += step) {
        const bool live = r0 + group < a.rows;
        const int64_t row = row_of(r0);
        uint32_t* const place = room + (group * kTurns + turn) * 3 * a.k;
        const Entries en{(int32_t*)place, (float*)place + a.k, (float*)place + 2 * a.k};
        turn ^= kTurns - 1;
        // maxima of the logits and of the entries
        float m[2] = {c.has_single(lane) ? one : neg_inf, neg_inf};
        one = m[0];
        for (int e = lane; e < a.k; e += L) {
            const int64_t at = e == lane ? c0 : a.classes.at(row, e);
            const bool given = at >= 0 && at < a.cols;
            const float t = e == lane ? t0 : a.teacher.at(row, e);
            en.cls[e] = given ? (int32_t)at : -1;
            en.power[e] = given ? t : neg_inf;
            m[1] = Max::of(m[1], en.power[e]);
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (!c.has(8 * (lane + L * j))) raw[j].fill(kNegInfBits);
            float v[8];
            raw[j].values(v);
#pragma unroll
            for (int i = 0; i < 8; i += 2) m[0] = Max::of(Max::of(m[0], v[i]), v[i + 1]);
            raw[j].hold();
        }
        reduce.template all<Max>(m);
        const float top = m[0], top_t = m[1], w = weight;
        // nothing to learn: no weight, no entry, no class
        const bool empty = w == 0.0f || top_t == neg_inf || top == neg_inf;
        // v / (T ln 2) less the maximum's, in one rounding; the maximum's own is the same in
        // every power of the row and in the loss.  Far from zero, where it is a part of 1 and
        // more, differences first.
        const float base = top * a.log2e_over_t;
        const bool far = !(__builtin_fabsf(base) < 1048576.0f);
        auto exponent = [&](float v) { return far ? (v - top) * a.log2e_over_t : __builtin_fmaf(v, a.log2e_over_t, -base); };
        float e1 = __builtin_amdgcn_exp2f(exponent(one));
        float p[C][8], s[2] = {e1, 0.0f};
        if (far) {   // rare, and then for all lanes of a row
#pragma unroll
            for (int j = 0; j < C; ++j) {
                raw[j].values(p[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[j][i] = __builtin_amdgcn_exp2f((p[j][i] - top) * a.log2e_over_t);
            }
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                raw[j].values(p[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[j][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[j][i], a.log2e_over_t, -base));
            }
        }
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += p[j][i];
        float logit = 0.0f;   // the sum of p (t - x) / (T ln 2), each less its maximum
        float from = 0.0f;    // of the first entry's class
        if (lane < a.k) from = value_of(x.base[row * x.ld + (en.cls[lane] < 0 ? 0 : en.cls[lane])]);
        if (r0 + step < a.rows) load(row_of(r0 + step));
        bool twice = false;
        for (int e = lane; e < a.k; e += L) {
            const float t = en.power[e];
            const int at = en.cls[e];
            const float d = (t - top_t) * a.log2e_over_t;
            const float pe = t == neg_inf ? 0.0f : __builtin_amdgcn_exp2f(d);
            s[1] += pe;
            const float xe = e == lane ? from : value_of(x.base[row * x.ld + (at < 0 ? 0 : at)]);
            const float ex = exponent(xe);
            if (at >= 0 && pe != 0.0f) logit += pe * (d - ex);
            en.power[e] = pe;
            en.own[e] = __builtin_amdgcn_exp2f(ex);
            if (at >= 0) owner[at] = (uint8_t)e;
        }
        reduce.template all<Add>(s);
        const float inv = 1.0f / s[0], inv_t = 1.0f / s[1], scale = w * a.temp;
        wave_lds_fence();   // the entries' powers and owners are there (behind the sums' barrier, too)
        // classes that come twice: all but one of their entries find another in their place
        for (int e = lane; e < a.k; e += L) twice |= en.cls[e] >= 0 && owner[en.cls[e]] != (uint8_t)e;
        float l[2] = {logit, twice ? 1.0f : 0.0f};
        reduce.template all<Add>(l);
        twice = l[1] > 0.0f;   // the same for a row's lanes
        if (lane == 0 && live && a.loss) {
            const float loss = l[0] * inv_t * kLn2 + (logf(s[0]) - logf(s[1]));
            a.loss[row] = empty ? 0.0f : loss * w * a.temp * a.temp;
        }
        if (!a.dx.base || !live) continue;
        const float factor = inv * scale;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int k = 8 * (lane + L * j);
            if (!c.has(k)) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) p[j][i] = empty ? 0.0f : p[j][i] * factor;
            store8(a.dx, row, k, p[j]);
        }
        if (c.has_single(lane)) store1(a.dx, row, c.single(lane), empty ? 0.0f : e1 * factor);
        if (empty) continue;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        constexpr int kLanes = L < 64 ? L : 64;
        for (int e = lane % kLanes; e < a.k; e += kLanes) {
            const int at = en.cls[e];
            if (at < 0) continue;
            // the lane that stored this column
            const int by = at < c.whole ? at / 8 % L : at - c.whole;
            if (L > 64 && by / 64 != lane / 64) continue;
            float pe = en.power[e];
            if (twice) {
                pe = 0.0f;
                for (int f = 0; f < a.k; ++f) pe += en.cls[f] == at ? en.power[f] : 0.0f;
            }
            store1(a.dx, row, at, (en.own[e] * inv - pe * inv_t) * scale);
        }
    }
}

// Rows that registers do not hold, by a workgroup each: read three times, from the
// caches but for the first.  107 x 48,791 classes: 15 us a call.
template <class T>
__global__ void __launch_bounds__(1024) distill_wide_kernel(DistillArgs a) {
    constexpr int L = 1024;
    __shared__ typename RowReduce<L, 2>::Lds lds;
    __shared__ uint8_t owner[DONERF_MAX_COLS];   // a byte a column: one of the entries of that class
    __shared__ int32_t cls[kMostEntries];
    __shared__ float power[kMostEntries], own[kMostEntries];
    RowReduce<L, 2> reduce(&lds);
    const int lane = threadIdx.x;
    const RowsIn<T> x((const T*)a.x, a.ldx, a.cols);
    const Columns& c = x.c;
    const float neg_inf = __uint_as_float(kNegInfBits);
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float w = a.weight ? a.weight[row] : 1.0f;
        float one = c.has_single(lane) ? x.load_single(row, lane) : neg_inf, t = neg_inf;
        int64_t at = -1;
        if (lane < a.k) {
            at = a.classes.at(row, lane);
            if (at < 0 || at >= a.cols) at = -1;
            else t = a.teacher.at(row, lane);
        }
        auto chunks = [&](auto f) {
            int k = 8 * lane;
            for (; c.has(k + 24 * L); k += 32 * L) {   // four at a time
                Raw<T> r[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = x.load(row, k + 8 * L * j);
#pragma unroll
                for (int j = 0; j < 4; ++j) f(k + 8 * L * j, r[j]);
            }
            for (; c.has(k); k += 8 * L) f(k, x.load(row, k));
        };
        float m[2] = {one, t};
        chunks([&](int, const Raw<T>& r) {
            float v[8];
            r.values(v);
#pragma unroll
            for (int i = 0; i < 8; i += 2) m[0] = Max::of(Max::of(m[0], v[i]), v[i + 1]);
        });
        reduce.template all<Max>(m);
        const float top = m[0], top_t = m[1];
        const bool empty = w == 0.0f || top_t == neg_inf || top == neg_inf;
        auto exponent = [&](float v) { return (v - top) * a.log2e_over_t; };
        const float e1 = __builtin_amdgcn_exp2f(exponent(one));
        float s[2] = {e1, 0.0f};
        chunks([&](int, const Raw<T>& r) {
            float v[8];
            r.values(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += __builtin_amdgcn_exp2f(exponent(v[i]));
        });
        float logit = 0.0f;
        if (lane < a.k) {
            const float d = (t - top_t) * a.log2e_over_t, p = t == neg_inf ? 0.0f : __builtin_amdgcn_exp2f(d);
            const float ex = exponent(value_of(x.base[row * x.ld + (at < 0 ? 0 : at)]));
            s[1] = p;
            if (at >= 0 && p != 0.0f) logit = p * (d - ex);
            cls[lane] = (int32_t)at;
            power[lane] = p;
            own[lane] = __builtin_amdgcn_exp2f(ex);
            if (at >= 0) owner[at] = (uint8_t)lane;
        }
        reduce.template all<Add>(s);
        const float inv = 1.0f / s[0], inv_t = 1.0f / s[1], scale = w * a.temp;
        // whether a class comes twice: all but one of its entries find another in their place
        float l[2] = {logit, lane < a.k && at >= 0 && owner[at] != (uint8_t)lane ? 1.0f : 0.0f};
        reduce.template all<Add>(l);
        if (lane == 0 && a.loss) {
            const float loss = l[0] * inv_t * kLn2 + (logf(s[0]) - logf(s[1]));
            a.loss[row] = empty ? 0.0f : loss * w * a.temp * a.temp;
        }
        if (a.dx.base) {
            const float factor = inv * scale;
            chunks([&](int k, const Raw<T>& r) {
                float v[8];
                r.values(v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = empty ? 0.0f : __builtin_amdgcn_exp2f(exponent(v[i])) * factor;
                store8(a.dx, row, k, v);
            });
            if (c.has_single(lane)) store1(a.dx, row, c.single(lane), empty ? 0.0f : e1 * factor);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            for (int e = lane % 64; e < a.k && !empty; e += 64) {
                const int to = cls[e], by = to < c.whole ? to / 8 % L : to - c.whole;   // the lane that stored this column
                if (to < 0 || by / 64 != lane / 64) continue;
                float p = power[e];
                if (l[1] > 0.0f) {
                    p = 0.0f;
                    for (int f = 0; f < a.k; ++f) p += cls[f] == to ? power[f] : 0.0f;
                }
                store1(a.dx, row, to, (own[e] * inv - p * inv_t) * scale);
            }
        }
        lds_barrier();   // the next row's entries come into the same place
    }
}

template <class T, int L, int C>
hipError_t distill_launch(const DistillArgs& a, int n_cu, hipStream_t s) {
    constexpr uint32_t groups = row_threads(L) / L;
    const uint32_t need = (a.rows + groups - 1) / groups, full = (uint32_t)n_cu * (2048 / row_threads(L));
    hipLaunchKernelGGL((distill_kernel<T, L, C>), dim3(need < full ? need : full), dim3(row_threads(L)), groups * (L > 64 ? 24 : 12) * a.k, s, a);
    return hipGetLastError();
}
template <class T>
hipError_t distill_wide(const DistillArgs& a, int n_cu, hipStream_t s) {
    const uint32_t full = (uint32_t)n_cu * 2;
    hipLaunchKernelGGL((distill_wide_kernel<T>), dim3(a.rows < full ? a.rows : full), dim3(1024), 0, s, a);
    return hipGetLastError();
}
template <class T>
hipError_t distill_by_width(const DistillArgs& a, int n_cu, hipStream_t s) {
    const int c = a.cols;
    // Few lanes a row: what they share, the sums and the entries, is then done for more rows at
    // once, and LDS holds their entries (48 KB of it).  33.5 million values, 4 entries a row, in
    // bf16: 64 classes 40 us with 4 lanes, 54 with 8; 512 29 with 16, 34 with 32 and 30 with 8;
    // 4096 26.9 with 64, 30.2 with 128; 16,384 28 with 256, 38 with 512.  Rows of single columns,
    // up to 7, have 8 lanes at least.  From 16,385 classes on fp32 rows have 512 lanes (32,000: 67
    // us, 74 with 1024) and bf16 ones 1024 (4096 x 32,000, 64 entries: 102 us, 105 with 512).
    if (c <= 128 && c % 8 == 0 && a.k <= 64)
        return c <= 64 ? distill_launch<T, 4, 2>(a, n_cu, s) : distill_launch<T, 4, 4>(a, n_cu, s);
    return c <= 64 ? distill_launch<T, 8, 1>(a, n_cu, s) : c <= 128 ? distill_launch<T, 8, 2>(a, n_cu, s) : c <= 256 ? distill_launch<T, 8, 4>(a, n_cu, s)
         : c <= 512 ? distill_launch<T, 16, 4>(a, n_cu, s) : c <= 1024 ? distill_launch<T, 32, 4>(a, n_cu, s)
         : c <= 2048 ? distill_launch<T, 64, 4>(a, n_cu, s) : c <= 4096 ? distill_launch<T, 64, 8>(a, n_cu, s)
         : c <= 8192 ? distill_launch<T, 128, 8>(a, n_cu, s) : c <= 16384 ? distill_launch<T, 256, 8>(a, n_cu, s)
         : c <= 32768 ? distill_launch<T, sizeof(T) == 2 ? 1024 : 512, sizeof(T) == 2 ? 4 : 8>(a, n_cu, s) : distill_wide<T>(a, n_cu, s);
}

}  // namespace

hipError_t launch_train_distill(const DistillArgs& a, bool x_bf16, int n_cu, hipStream_t stream) {
    return x_bf16 ? distill_by_width<uint16_t>(a, n_cu, stream) : distill_by_width<float>(a, n_cu, stream);
}

}  // namespace donerf
