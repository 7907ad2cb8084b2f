// train_distill.hip - distillation from a teacher's top logits, loss and gradient.
//
//   p = softmax of t / T over a row's given entries, q = softmax of x / T over its
//   classes, loss = w T^2 sum_k p_k (log p_k - log q_{c_k}),
//   dx_j = w T (q_j - sum of p_k over the k with c_k = j).
//
// One pass over x: a row stays in registers between its maximum, its sum and the
// gradient.  Differences to the maximum are taken before they are scaled, so that
// logits of the type's lowest value are as good a mask as -inf.  The entries' few
// columns are written a second time, behind the rest of their row.
#include "rows.h"

namespace donerf {
namespace {

constexpr uint32_t kNegInfBits = 0xff800000u;

template <class T, int L, int C>
__global__ void __launch_bounds__(row_threads(L)) distill_kernel(DistillArgs a) {
    constexpr int kGroups = row_threads(L) / L;
    __shared__ typename RowReduce<L, 1>::Lds lds;
    extern __shared__ uint32_t entries[];   // of each row: k classes, then k probabilities
    RowReduce<L, 1> reduce(&lds);
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    int32_t* const cls = (int32_t*)entries + group * 2 * a.k;
    float* const prob = (float*)(cls + a.k);
    const RowsIn<T> x((const T*)a.x, a.ldx, a.cols);
    const Columns& c = x.c;
    const float neg_inf = __uint_as_float(kNegInfBits);
    auto fence = [] {
        if constexpr (L > 64) __syncthreads();
        else wave_lds_fence();
    };
    for (uint32_t r0 = blockIdx.x * kGroups; r0 < a.rows; r0 += gridDim.x * kGroups) {
        const bool live = r0 + group < a.rows;
        const int64_t row = live ? r0 + group : a.rows - 1;
        Raw<T> raw[C];
#pragma unroll
        for (int j = 0; j < C; ++j) raw[j] = x.load(row, 8 * (lane + L * j));
        float one = neg_inf;
        if (c.any_single()) one = x.load_single(row, lane);
        // the teacher's entries: their maximum, then their sum
        float top_t = neg_inf;
        for (int e = lane; e < a.k; e += L) {
            const int64_t at = a.classes.at(row, e);
            const bool given = at >= 0 && at < a.cols;
            const float t = given ? a.teacher.at(row, e) : neg_inf;
            cls[e] = given ? (int32_t)at : -1;
            prob[e] = t;
            top_t = Max::of(top_t, t);
        }
        top_t = reduce.template one<Max>(top_t);
        float sum_t = 0.0f;
        for (int e = lane; e < a.k; e += L) {
            const float t = prob[e] == neg_inf ? neg_inf : prob[e] - top_t;
            const float p = __builtin_amdgcn_exp2f(t * a.log2e_over_t);
            sum_t += p;
        }
        sum_t = reduce.template one<Add>(sum_t);
        if (!c.has_single(lane)) one = neg_inf;
        float top = one;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if (!c.has(8 * (lane + L * j))) raw[j].fill(kNegInfBits);
            float v[8];
            raw[j].values(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = Max::of(top, v[i]);
            raw[j].hold();
        }
        top = reduce.template one<Max>(top);
        auto power = [&](float v) { return __builtin_amdgcn_exp2f((v - top) * a.log2e_over_t); };
        float sum = power(one);
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float v[8];
            raw[j].values(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += power(v[i]);
            raw[j].hold();
        }
        sum = reduce.template one<Add>(sum);
        const float weight = a.weight ? a.weight[row] : 1.0f;
        // nothing to learn: no weight, no entry, no class
        const bool empty = weight == 0.0f || top_t == neg_inf || top == neg_inf;
        const float inv_sum = 1.0f / sum, inv_t = 1.0f / sum_t, log_ratio = logf(sum) - logf(sum_t);
        float loss = 0.0f;
        for (int e = lane; e < a.k; e += L) {
            if (cls[e] < 0) continue;
            const float t = prob[e];
            const float p = __builtin_amdgcn_exp2f((t - top_t) * a.log2e_over_t) * inv_t;
            const float xc = value_of(x.base[row * x.ld + cls[e]]);
            if (!(p == 0.0f)) loss += p * (((t - top_t) - (xc - top)) * a.inv_temp + log_ratio);
            prob[e] = p;
        }
        loss = reduce.template one<Add>(loss);
        fence();
        if (live && lane == 0 && a.loss) a.loss[row] = empty ? 0.0f : loss * weight * a.temp * a.temp;
        if (a.dx.base) {
            const float scale = weight * a.temp;
            if (live) {
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    const int k = 8 * (lane + L * j);
                    if (!c.has(k)) continue;
                    float v[8];
                    raw[j].values(v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = empty ? 0.0f : power(v[i]) * inv_sum * scale;
                    store8(a.dx, row, k, v);
                }
                if (c.has_single(lane)) store1(a.dx, row, c.single(lane), empty ? 0.0f : power(one) * inv_sum * scale);
            }
            // the entries' columns, behind the stores that they overwrite
            if constexpr (L > 64) {
                __syncthreads();
            } else {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            }
            for (int e = lane; e < a.k; e += L) {
                const int at = cls[e];
                if (at < 0 || empty || !live) continue;
                float p = 0.0f;
                for (int f = 0; f < a.k; ++f)
                    if (cls[f] == at) p += prob[f];
                store1(a.dx, row, at, (power(value_of(x.base[row * x.ld + at])) * inv_sum - p) * scale);
            }
        }
        fence();   // the next row's entries come into the same place
    }
}

template <class T, int L, int C>
hipError_t distill_launch(const DistillArgs& a, int n_cu, hipStream_t s) {
    constexpr uint32_t groups = row_threads(L) / L;
    const uint32_t need = (a.rows + groups - 1) / groups, full = (uint32_t)n_cu * (2048 / row_threads(L));
    hipLaunchKernelGGL((distill_kernel<T, L, C>), dim3(need < full ? need : full), dim3(row_threads(L)), groups * 8 * a.k, s, a);
    return hipGetLastError();
}
template <class T>
hipError_t distill_by_width(const DistillArgs& a, int n_cu, hipStream_t s) {
    const int c = a.cols;
    return c <= 64 ? distill_launch<T, 8, 1>(a, n_cu, s) : c <= 128 ? distill_launch<T, 16, 1>(a, n_cu, s)
         : c <= 256 ? distill_launch<T, 32, 1>(a, n_cu, s) : c <= 512 ? distill_launch<T, 64, 1>(a, n_cu, s)
         : c <= 1024 ? distill_launch<T, 64, 2>(a, n_cu, s) : c <= 2048 ? distill_launch<T, 64, 4>(a, n_cu, s)
         : c <= 4096 ? distill_launch<T, 256, 2>(a, n_cu, s) : c <= 8192 ? distill_launch<T, 256, 4>(a, n_cu, s)
         : c <= 16384 ? distill_launch<T, 512, 4>(a, n_cu, s) : c <= 32768 ? distill_launch<T, 1024, 4>(a, n_cu, s)
         : distill_launch<T, 1024, 8>(a, n_cu, s);
}

}  // namespace

hipError_t launch_train_distill(const DistillArgs& a, bool x_bf16, int n_cu, hipStream_t stream) {
    return x_bf16 ? distill_by_width<uint16_t>(a, n_cu, stream) : distill_by_width<float>(a, n_cu, stream);
}

}  // namespace donerf
