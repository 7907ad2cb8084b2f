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
// High temperatures (NEAR).  p and q differ by parts of 1/T, the loss is T^2 times a sum of
// such differences' squares, and T^2 times the rounding of log p - log q is soon more than
// that.  So the loss is the sum of terms that are never negative,
//   sum_e p_e log(p_e / q_e) = sum_e (p_e log(p_e / q_e) + q_e - p_e) + 1 - sum_e q_e,
// of which, with d = log(p_e / q_e), the terms in brackets are p_e (e^-d - 1 + d) and
// 1 - sum_e q_e is the probability of the classes without an entry, added up without the
// others (where a class comes twice, less its further entries').  d takes the logarithm of
// the sums' ratio from their difference, of the entries' e^u - 1, and the gradient's
// q_e - p_e is p_e (e^-d - 1).  fp32's rounding then stays a part of the result: with 128
// classes and an entry for each, the worst of 300 rows is off by 5e-7 of its loss and of its
// gradient at every T up to 2^16; in the plain form by 2e-5 of its loss at T = 4, 3e-4 at 16,
// 6e-3 at 64 and by more than the loss from 1000 on, and by 7e-3 of its gradient at 2^16.  The
// entries' longer way costs a fifth (160,000 x 128, 4 entries: 23.4 us a call for 19.1), and
// 4096 x 32,000 with 64 of them 161 us for 116.
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

// e^-d - 1 + d for |d| < 1/2, without the cancellation: a series whose next term is 2e-9 of it.
__device__ __forceinline__ float exp_rest(float d) {
    const float x = -d;
    float s = 1.0f / 362880;
    s = __builtin_fmaf(s, x, 1.0f / 40320);
    s = __builtin_fmaf(s, x, 1.0f / 5040);
    s = __builtin_fmaf(s, x, 1.0f / 720);
    s = __builtin_fmaf(s, x, 1.0f / 120);
    s = __builtin_fmaf(s, x, 1.0f / 24);
    s = __builtin_fmaf(s, x, 1.0f / 6);
    s = __builtin_fmaf(s, x, 0.5f);
    return x * x * s;
}
// High temperatures: an entry by its logits less their maxima, e^ of both over the
// temperature, and what its row's sums are of.
struct NearEntry {
    float tn, un, p, q;
    __device__ __forceinline__ NearEntry(const DistillArgs& a, float t, float x)
        : tn(t * a.inv_temp), un(x * a.inv_temp), p(power(a, t)), q(power(a, x)) {}
    __device__ static __forceinline__ float power(const DistillArgs& a, float v) { return __builtin_amdgcn_exp2f(v * a.log2e_over_t); }
    // Its part of the sum of all p less that of all q; of its class's entries one counts q.
    __device__ __forceinline__ float apart(bool first) const { return first ? expm1f(tn) - expm1f(un) : p; }
};
// High temperatures: which classes a row's entries have, a bit each, and which of them come
// again; all bits zero between the rows.
struct NearClasses {
    uint32_t* some;
    uint32_t* again;
    __device__ __forceinline__ void set(int at) const {
        const uint32_t bit = 1u << at % 32;
        if (atomicOr(&some[at / 32], bit) & bit) atomicOr(&again[at / 32], bit);
    }
    __device__ __forceinline__ void clear(int at) const { some[at / 32] = again[at / 32] = 0; }
    // The bits of the 8 columns from k on.
    __device__ __forceinline__ uint32_t chunk(int k) const { return ((const uint8_t*)some)[k / 8]; }
    // Whether entry e is the first one of its class.
    __device__ __forceinline__ bool first(const int32_t* cls, int e) const {
        const int at = cls[e];
        if (again[at / 32] >> at % 32 & 1)
            for (int f = 0; f < e; ++f)
                if (cls[f] == at) return false;
        return true;
    }
};
// A row's sums: of p, of q, and log of their ratio.
struct NearSums {
    float inv_p, inv_q, log_ratio;
    // p's, q's without an entry and with one, and apart() of the entries
    __device__ __forceinline__ NearSums(float sp, float rest, float own, float apart) {
        const float sq = rest + own, d = apart - rest;
        inv_p = 1.0f / sp;
        inv_q = 1.0f / sq;
        log_ratio = __builtin_fabsf(d) < 0.5f * sq ? log1pf(d * inv_q) : logf(sp) - logf(sq);
    }
    // An entry's term of the loss, and q - p.
    __device__ __forceinline__ float term(const NearEntry& e, float* grad) const {
        const float d = e.tn - e.un - log_ratio, p = e.p * inv_p, q = e.q * inv_q;
        const bool close = __builtin_fabsf(d) < 0.5f;
        const float rest = exp_rest(d);
        *grad = close ? p * (rest - d) : q - p;
        return close ? p * rest : p * d + (q - p);
    }
};

// NEAR: for high temperatures.
template <class T, int L, int C, bool NEAR>
__global__ void __launch_bounds__(row_threads(L)) distill_kernel(DistillArgs a) {
    constexpr int kGroups = row_threads(L) / L;
    constexpr int kTurns = L > 64 ? 2 : 1;
    constexpr int kWords = L * C / 4;   // of a row's bits
    __shared__ typename RowReduce<L, 2>::Lds lds;
    __shared__ uint8_t owners[NEAR ? 1 : kGroups * 8 * L * C];   // a byte a column: one of the entries of that class
    __shared__ uint32_t bits[NEAR ? kGroups * 2 * kWords : 1];
    extern __shared__ uint32_t room[];
    RowReduce<L, 2> reduce(&lds);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    // In two places by turns, where a row's waves are several: one that is a row ahead
    // writes to the other.
    int turn = 0;
    uint8_t* const owner = owners + (NEAR ? 0 : group * 8 * L * C);
    uint32_t* const own_bits = bits + (NEAR ? group * 2 * kWords : 0);
    const NearClasses had{own_bits, own_bits + kWords};
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
    if constexpr (NEAR) {
        for (int i = lane; i < 2 * kWords; i += L) own_bits[i] = 0;
        if constexpr (L > 64) lds_barrier();
        else wave_lds_fence();
    }
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
        // more, and at high temperatures, differences first.
        const float base = top * a.log2e_over_t;
        const bool far = NEAR || !(__builtin_fabsf(base) < 1048576.0f);
        auto exponent = [&](float v) { return far ? (v - top) * a.log2e_over_t : __builtin_fmaf(v, a.log2e_over_t, -base); };
        if constexpr (NEAR) {
            // entries first: those of no probability are as if not given
            for (int e = lane; e < a.k; e += L) {
                const int at = en.cls[e];
                const float t = en.power[e] - top_t;
                const bool has = at >= 0 && (NearEntry::power(a, t) != 0.0f || top_t == -neg_inf);   // NaN, too
                const float xe = value_of(x.base[row * x.ld + (at < 0 ? 0 : at)]) - top;
                if (has) had.set(at);
                else en.cls[e] = -1;
                en.power[e] = t;
                en.own[e] = xe;
            }
            if constexpr (L > 64) lds_barrier();
            else wave_lds_fence();
        }
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
        if (NEAR && c.has_single(lane) && had.chunk(c.whole) >> lane & 1) s[0] = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const uint32_t m = NEAR ? had.chunk(8 * (lane + L * j)) : 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += NEAR && m >> i & 1 ? 0.0f : p[j][i];
        }
        float inv, inv_t, loss;
        const float scale = w * a.temp;
        bool twice = false;   // classes that come twice: all but one of their entries find another in their place
        if constexpr (NEAR) {
            if (r0 + step < a.rows) load(row_of(r0 + step));
            float d[2] = {0.0f, 0.0f}, more[2] = {0.0f, 0.0f};   // apart() and q of classes with an entry; q of further entries, their number
            for (int e = lane; e < a.k; e += L) {
                if (en.cls[e] < 0) continue;
                const NearEntry v(a, en.power[e], en.own[e]);
                const bool first = had.first(en.cls, e);
                s[1] += v.p;
                d[0] += v.apart(first);
                d[1] += first ? v.q : 0.0f;
                more[0] += first ? 0.0f : v.q;
                more[1] += first ? 0.0f : 1.0f;
            }
            reduce.template all<Add>(s);
            reduce.template all<Add>(d);
            reduce.template all<Add>(more);
            const NearSums sums(s[1], s[0], d[1], d[0]);
            inv = sums.inv_q;
            inv_t = sums.inv_p;
            twice = more[1] > 0.0f;
            float l[2] = {0.0f, 0.0f};
            for (int e = lane; e < a.k; e += L) {
                const int at = en.cls[e];
                if (at < 0) continue;
                const NearEntry v(a, en.power[e], en.own[e]);
                float grad;
                l[0] += sums.term(v, &grad);
                en.power[e] = twice ? v.p : grad;
                en.own[e] = v.q;
                had.clear(at);   // all have read them, behind the sums
            }
            reduce.template all<Add>(l);
            wave_lds_fence();   // (behind the sums' barrier, too)
            loss = l[0] + (s[0] - more[0]) * inv;
        } else {
            float logit = 0.0f;   // the sum of p (t - x) / (T ln 2), each less its maximum
            float from = 0.0f;    // of the first entry's class
            if (lane < a.k) from = value_of(x.base[row * x.ld + (en.cls[lane] < 0 ? 0 : en.cls[lane])]);
            if (r0 + step < a.rows) load(row_of(r0 + step));
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
            inv = 1.0f / s[0];
            inv_t = 1.0f / s[1];
            wave_lds_fence();   // the entries' powers and owners are there (behind the sums' barrier, too)
            for (int e = lane; e < a.k; e += L) twice |= en.cls[e] >= 0 && owner[en.cls[e]] != (uint8_t)e;
            float l[2] = {logit, twice ? 1.0f : 0.0f};
            reduce.template all<Add>(l);
            twice = l[1] > 0.0f;   // the same for a row's lanes
            loss = l[0] * inv_t * kLn2 + (logf(s[0]) - logf(s[1]));
        }
        if (lane == 0 && live && a.loss) a.loss[row] = empty ? 0.0f : loss * w * a.temp * a.temp;
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
            if (NEAR && !twice) {   // q - p
                store1(a.dx, row, at, pe * scale);
                continue;
            }
            if (twice) {
                pe = 0.0f;
                for (int f = 0; f < a.k; ++f) pe += en.cls[f] == at ? en.power[f] : 0.0f;
            }
            store1(a.dx, row, at, (en.own[e] * inv - pe * inv_t) * scale);
        }
    }
}

// Rows that registers do not hold, by a workgroup each: read three times, from the
// caches but for the first.  107 x 48,791 classes: 15 us a call; 2048 x 65,536 bf16 150 us,
// 538 MB, 3.6 TB/s.
template <class T, bool NEAR>
__global__ void __launch_bounds__(1024) distill_wide_kernel(DistillArgs a) {
    constexpr int L = 1024;
    __shared__ typename RowReduce<L, 2>::Lds lds;
    constexpr int kWords = DONERF_MAX_COLS / 32;   // of a row's bits
    __shared__ uint8_t owner[NEAR ? 1 : DONERF_MAX_COLS];   // a byte a column: one of the entries of that class
    __shared__ uint32_t bits[NEAR ? 2 * kWords : 1];
    __shared__ int32_t cls[kMostEntries];
    __shared__ float power[kMostEntries], own[kMostEntries];
    RowReduce<L, 2> reduce(&lds);
    const int lane = threadIdx.x;
    const RowsIn<T> x((const T*)a.x, a.ldx, a.cols);
    const Columns& c = x.c;
    const float neg_inf = __uint_as_float(kNegInfBits);
    const NearClasses had{bits, bits + (NEAR ? kWords : 0)};
    if constexpr (NEAR) {
        for (int i = lane; i < 2 * kWords; i += L) bits[i] = 0;
        lds_barrier();
    }
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
        float logit = 0.0f;
        const float xe = lane < a.k ? value_of(x.base[row * x.ld + (at < 0 ? 0 : at)]) : 0.0f;
        const NearEntry v(a, t - top_t, xe - top);
        if constexpr (NEAR) {   // entries first: those of no probability are as if not given
            if (at >= 0 && v.p == 0.0f && top_t != -neg_inf) at = -1;
            if (lane < a.k) cls[lane] = (int32_t)at;
            if (at >= 0) had.set((int)at);
            lds_barrier();
        }
        float s[2] = {NEAR && c.has_single(lane) && had.chunk(c.whole) >> lane & 1 ? 0.0f : e1, 0.0f};
        chunks([&](int k, const Raw<T>& r) {
            float f[8];
            r.values(f);
            const uint32_t m = NEAR ? had.chunk(k) : 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += NEAR && m >> i & 1 ? 0.0f : __builtin_amdgcn_exp2f(exponent(f[i]));
        });
        float inv, inv_t, loss;
        const float scale = w * a.temp;
        bool twice;   // whether a class comes twice: all but one of its entries find another in their place
        if constexpr (NEAR) {
            const bool first = at >= 0 && had.first(cls, lane);
            float d[2] = {0.0f, 0.0f}, more[2] = {0.0f, 0.0f};   // apart() and q of classes with an entry; q of further entries, their number
            if (at >= 0) {
                s[1] = v.p;
                d[0] = v.apart(first);
                d[1] = first ? v.q : 0.0f;
                more[0] = first ? 0.0f : v.q;
                more[1] = first ? 0.0f : 1.0f;
            }
            reduce.template all<Add>(s);
            reduce.template all<Add>(d);
            reduce.template all<Add>(more);
            const NearSums sums(s[1], s[0], d[1], d[0]);
            inv = sums.inv_q;
            inv_t = sums.inv_p;
            twice = more[1] > 0.0f;
            float l[2] = {0.0f, 0.0f};
            if (at >= 0) {
                float grad;
                l[0] = sums.term(v, &grad);
                power[lane] = twice ? v.p : grad;
                own[lane] = v.q;
                had.clear((int)at);   // all have read them, behind the sums
            }
            reduce.template all<Add>(l);
            loss = l[0] + (s[0] - more[0]) * inv;
        } else {
            if (lane < a.k) {
                const float d = (t - top_t) * a.log2e_over_t, p = t == neg_inf ? 0.0f : __builtin_amdgcn_exp2f(d);
                const float ex = exponent(xe);
                s[1] = p;
                if (at >= 0 && p != 0.0f) logit = p * (d - ex);
                cls[lane] = (int32_t)at;
                power[lane] = p;
                own[lane] = __builtin_amdgcn_exp2f(ex);
                if (at >= 0) owner[at] = (uint8_t)lane;
            }
            reduce.template all<Add>(s);
            inv = 1.0f / s[0];
            inv_t = 1.0f / s[1];
            float l[2] = {logit, lane < a.k && at >= 0 && owner[at] != (uint8_t)lane ? 1.0f : 0.0f};
            reduce.template all<Add>(l);
            twice = l[1] > 0.0f;
            loss = l[0] * inv_t * kLn2 + (logf(s[0]) - logf(s[1]));
        }
        if (lane == 0 && a.loss) a.loss[row] = empty ? 0.0f : loss * w * a.temp * a.temp;
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
                if (NEAR && !twice) {   // q - p
                    store1(a.dx, row, to, p * scale);
                    continue;
                }
                if (twice) {
                    p = 0.0f;
                    for (int f = 0; f < a.k; ++f) p += cls[f] == to ? power[f] : 0.0f;
                }
                store1(a.dx, row, to, (own[e] * inv - p * inv_t) * scale);
            }
        }
        lds_barrier();   // the next row's entries come into the same place
    }
}

template <class T, bool NEAR, int L, int C>
hipError_t distill_launch(const DistillArgs& a, int n_cu, hipStream_t s) {
    constexpr uint32_t groups = row_threads(L) / L;
    const uint32_t need = (a.rows + groups - 1) / groups, full = (uint32_t)n_cu * (2048 / row_threads(L));
    const dim3 grid(need < full ? need : full), threads(row_threads(L));
    const size_t lds = groups * (L > 64 ? 24 : 12) * a.k;
    hipLaunchKernelGGL((distill_kernel<T, L, C, NEAR>), grid, threads, lds, s, a);
    return hipGetLastError();
}
template <class T, bool NEAR>
hipError_t distill_wide(const DistillArgs& a, int n_cu, hipStream_t s) {
    const uint32_t full = (uint32_t)n_cu * 2;
    const dim3 grid(a.rows < full ? a.rows : full), threads(1024);
    hipLaunchKernelGGL((distill_wide_kernel<T, NEAR>), grid, threads, 0, s, a);
    return hipGetLastError();
}
template <class T, bool NEAR>
hipError_t distill_by_width(const DistillArgs& a, int n_cu, hipStream_t s) {
    const int c = a.cols;
    // Few lanes a row: what they share, the sums and the entries, is then done for more rows at
    // once, and LDS holds their entries (48 KB of it).  33.5 million values, 4 entries a row, in
    // bf16: 64 classes 40 us with 4 lanes, 54 with 8; 512 29 with 16, 34 with 32 and 30 with 8;
    // 4096 26.9 with 64, 30.2 with 128; 16,384 28 with 256, 38 with 512.  Rows of single columns,
    // up to 7, have 8 lanes at least.  From 16,385 classes on fp32 rows have 512 lanes (32,000: 67
    // us, 74 with 1024) and bf16 ones 1024 (4096 x 32,000, 64 entries: 102 us, 105 with 512), but
    // at high temperatures, where the 128 registers of 1024 lanes are too few.
    constexpr int kWidest = sizeof(T) == 2 && !NEAR ? 1024 : 512;
    if (c <= 128 && c % 8 == 0 && a.k <= 64)
        return c <= 64 ? distill_launch<T, NEAR, 4, 2>(a, n_cu, s) : distill_launch<T, NEAR, 4, 4>(a, n_cu, s);
    return c <= 64 ? distill_launch<T, NEAR, 8, 1>(a, n_cu, s) : c <= 128 ? distill_launch<T, NEAR, 8, 2>(a, n_cu, s) : c <= 256 ? distill_launch<T, NEAR, 8, 4>(a, n_cu, s)
         : c <= 512 ? distill_launch<T, NEAR, 16, 4>(a, n_cu, s) : c <= 1024 ? distill_launch<T, NEAR, 32, 4>(a, n_cu, s)
         : c <= 2048 ? distill_launch<T, NEAR, 64, 4>(a, n_cu, s) : c <= 4096 ? distill_launch<T, NEAR, 64, 8>(a, n_cu, s)
         : c <= 8192 ? distill_launch<T, NEAR, 128, 8>(a, n_cu, s) : c <= 16384 ? distill_launch<T, NEAR, 256, 8>(a, n_cu, s)
         : c <= 32768 ? distill_launch<T, NEAR, kWidest, 32768 / 8 / kWidest>(a, n_cu, s) : distill_wide<T, NEAR>(a, n_cu, s);
}

}  // namespace

hipError_t launch_train_distill(const DistillArgs& a, bool x_bf16, int n_cu, hipStream_t stream) {
    // The plain form up to 4, where its loss is off by 2e-5 of itself at worst (a teacher that
    // gives all classes).
    if (a.temp > 4.0f) return x_bf16 ? distill_by_width<uint16_t, true>(a, n_cu, stream) : distill_by_width<float, true>(a, n_cu, stream);
    return x_bf16 ? distill_by_width<uint16_t, false>(a, n_cu, stream) : distill_by_width<float, false>(a, n_cu, stream);
}

}  // namespace donerf
