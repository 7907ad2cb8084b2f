// train_embedding.hip - lookup of a table's rows by ids, and the table's gradient.
//
//   forward   y_i = s table[id_i], zeros where id_i names no row.
//   backward  row v of the gradient is s times the sum of dy_i over the i with
//             id_i = v, in the order of i.  The rows' numbers are sorted by their ids
//             (stable, 10 bits or less a pass), the sorted rows are summed in parts of
//             equal length, and runs of one id that cross from part to part are joined
//             from the parts' sums.
#include "rows.h"

namespace donerf {
namespace {

// ---------------------------------------------------------------- forward

template <class T, int L>
__global__ void __launch_bounds__(256) embedding_kernel(EmbeddingArgs a) {
    constexpr int kGroups = 256 / L;
    const int lane = threadIdx.x % L;
    const RowsIn<T> table((const T*)a.table, a.ldt, a.cols);
    const Columns& c = table.c;
    for (int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / L; row < a.rows; row += (int64_t)gridDim.x * kGroups) {
        const int64_t id = a.ids.at(row, 0);
        const bool given = id >= 0 && id < a.n;
        for (int k = 8 * lane; c.has(k); k += 8 * L) {
            float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (given) {
                table.load(id, k).values(v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= a.scale;
            }
            store8(a.y, row, k, v);
        }
        if (c.has_single(lane)) store1(a.y, row, c.single(lane), given ? table.load_single(id, lane) * a.scale : 0.0f);
    }
}

// ---------------------------------------------------------------- sort

constexpr int kSortThreads = 256;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 16;                            // of a thread in one step of its tile
constexpr int kSortStep = kSortThreads * kSortItems;
constexpr int kMostBins = 1 << kSortBits;

// The key that a pass reads: the first one makes it of the ids, n for those without a row.
__device__ __forceinline__ uint32_t sort_key(const SortPass& s, uint32_t i) {
    if (s.keys_in) return s.keys_in[i];
    const int64_t id = s.ids.at(i, 0);
    return id >= 0 && id < s.n ? (uint32_t)id : (uint32_t)s.n;
}

// counts[bin][tile]: the keys of each tile by their digit.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(SortPass s) {
    __shared__ uint32_t bins[kMostBins];
    const uint32_t n_bins = 1u << s.bits;
    for (uint32_t b = threadIdx.x; b < n_bins; b += kSortThreads) bins[b] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * s.tile, end = s.rows - first < s.tile ? s.rows : first + s.tile;
    for (uint32_t i = first + threadIdx.x; i < end; i += kSortThreads)
        atomicAdd(&bins[sort_key(s, i) >> s.shift & (n_bins - 1)], 1u);
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < n_bins; b += kSortThreads) s.counts[(size_t)b * gridDim.x + blockIdx.x] = bins[b];
}

// The sum of v over a workgroup's threads before this one, and all of them.
template <int THREADS>
__device__ __forceinline__ uint32_t scan_before(uint32_t v, uint32_t* lds, uint32_t& total) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(x, d, 64);
        if (lane >= d) x += o;
    }
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    __syncthreads();
    return before + x - v;
}

// A workgroup per bin: counts become the keys of the bin in the tiles before.
__global__ void __launch_bounds__(kSortThreads) sort_scan_kernel(SortPass s, uint32_t tiles) {
    __shared__ uint32_t lds[kSortWaves];
    uint32_t* const row = s.counts + (size_t)blockIdx.x * tiles;
    uint32_t sum = 0;
    for (uint32_t t0 = 0; t0 < tiles; t0 += kSortThreads) {
        const uint32_t t = t0 + threadIdx.x;
        const uint32_t v = t < tiles ? row[t] : 0;
        uint32_t total;
        const uint32_t before = scan_before<kSortThreads>(v, lds, total);
        if (t < tiles) row[t] = sum + before;
        sum += total;
    }
    if (threadIdx.x == 0) s.totals[blockIdx.x] = sum;
}

// Moves a tile's keys and rows to their places.
__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(SortPass s) {
    __shared__ uint32_t at[kMostBins];                  // where the tile's next key of each bin goes
    __shared__ uint32_t waves[kSortWaves][kMostBins];   // keys of each wave, then of the waves before
    __shared__ uint32_t lds[kSortWaves];
    const uint32_t n_bins = 1u << s.bits;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t sum = 0;
    for (uint32_t b0 = 0; b0 < n_bins; b0 += kSortThreads) {
        const uint32_t b = b0 + threadIdx.x;
        const uint32_t v = b < n_bins ? s.totals[b] : 0;
        uint32_t total;
        const uint32_t before = scan_before<kSortThreads>(v, lds, total);
        if (b < n_bins) at[b] = sum + before + s.counts[(size_t)b * gridDim.x + blockIdx.x];
        sum += total;
    }
    const uint32_t first = blockIdx.x * s.tile, end = s.rows - first < s.tile ? s.rows : first + s.tile;
    // steps of kSortStep keys: a wave takes consecutive ones, 64 at a time
    for (uint32_t step = first; step < end; step += kSortStep) {
        for (uint32_t b = threadIdx.x; b < kSortWaves * n_bins; b += kSortThreads) waves[b / n_bins][b % n_bins] = 0;
        __syncthreads();
        uint32_t key[kSortItems], rank[kSortItems];
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            const uint32_t i = step + (wave * kSortItems + j) * 64 + lane;
            key[j] = i < end ? sort_key(s, i) : 0;
        }
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            const bool live = step + (wave * kSortItems + j) * 64 + lane < end;
            const uint32_t bin = key[j] >> s.shift & (n_bins - 1);
            uint64_t same = __ballot(live);   // the live lanes with this lane's digit
            for (int b = 0; b < s.bits; ++b) {
                const uint64_t ones = __ballot(bin >> b & 1);
                same &= bin >> b & 1 ? ones : ~ones;
            }
            const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1));
            const uint32_t seen = live ? waves[wave][bin] : 0;
            wave_lds_fence();
            if (live && before == 0) waves[wave][bin] = seen + (uint32_t)__popcll(same);
            wave_lds_fence();
            rank[j] = seen + before;
        }
        __syncthreads();
        for (uint32_t b = threadIdx.x; b < n_bins; b += kSortThreads) {
            uint32_t run = at[b];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t v = waves[w][b];
                waves[w][b] = run;
                run += v;
            }
            at[b] = run;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            const uint32_t i = step + (wave * kSortItems + j) * 64 + lane;
            if (i < end) {
                const uint32_t to = waves[wave][key[j] >> s.shift & (n_bins - 1)] + rank[j];
                s.keys_out[to] = key[j];
                s.rows_out[to] = s.rows_in ? s.rows_in[i] : i;
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- sums

// Rows of a part are read this many at a time.
constexpr int kAhead = 8;

// Parts of `part` sorted rows; a run of one id that lies within one is the result, one
// that comes from the part before leaves its sum in ends[2 p], one that goes on into
// the next part in ends[2 p + 1].
template <class T, int L>
__global__ void __launch_bounds__(256) embedding_sum_kernel(EmbeddingGradArgs a) {
    const int lane = threadIdx.x % L;
    const int64_t p = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int k = 8 * (int)(blockIdx.y * L + lane);
    const RowsIn<T> dy((const T*)a.dy, a.lddy, a.cols);
    const Columns& c = dy.c;
    const bool single = blockIdx.y == 0 && c.has_single(lane);
    if (p * a.part >= a.rows || !(c.has(k) || single)) return;
    const uint32_t first = (uint32_t)(p * a.part), end = a.rows - first < a.part ? a.rows : first + a.part;
    uint32_t cur = a.keys[first];
    bool from_before = first > 0 && a.keys[first - 1] == cur;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum1 = 0.0f;
    auto leave = [&](bool goes_on) {
        if (cur >= a.n) return;   // rows without an id
        const bool part = from_before || goes_on;
        float* const to = part ? a.ends + (2 * p + (from_before ? 0 : 1)) * a.cols : a.dtable + cur * a.lddt;
        const float scale = part ? 1.0f : a.scale;
        const bool add = !part && a.accumulate;
        if (c.has(k)) {
            float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (add) __builtin_memcpy(v, to + k, 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += sum[i] * scale;
            __builtin_memcpy(to + k, v, 32);
        }
        if (single) to[c.single(lane)] = (add ? to[c.single(lane)] : 0.0f) + sum1 * scale;
    };
    for (uint32_t i0 = first; i0 < end; i0 += kAhead) {
        uint32_t key[kAhead], row[kAhead];
        Raw<T> raw[kAhead];
        float one[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint32_t i = i0 + j < end ? i0 + j : end - 1;
            key[j] = a.keys[i];
            row[j] = a.order[i];
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            raw[j] = dy.load(row[j], k);
            one[j] = c.any_single() ? dy.load_single(row[j], lane) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 + j >= end) break;
            if (key[j] != cur) {
                leave(false);
                cur = key[j];
                from_before = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
                sum1 = 0.0f;
            }
            float v[8];
            raw[j].values(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
            sum1 += one[j];
        }
    }
    leave(end < a.rows && a.keys[end] == cur);
}

// Joins a run that begins in part blockIdx.x and goes on: 64 columns a workgroup, 16
// threads each.
__global__ void __launch_bounds__(1024) embedding_join_kernel(EmbeddingGradArgs a) {
    __shared__ float lds[16][64];
    const int64_t p = blockIdx.x, first = p * a.part, end = first + a.part;
    if (end >= a.rows) return;
    const uint32_t cur = a.keys[end - 1];
    if (cur >= a.n || a.keys[end] != cur) return;                                  // none goes on
    if (first > 0 && a.keys[first] == cur && a.keys[first - 1] == cur) return;     // it began before
    const int group = threadIdx.x / 64, k = (int)(blockIdx.y * 64 + threadIdx.x % 64);
    float sum = 0.0f;
    if (k < a.cols) {
        if (group == 0) sum = a.ends[(2 * p + 1) * a.cols + k];
        for (int64_t q = p + 1 + group; q * a.part < a.rows && a.keys[q * a.part] == cur; q += 16) sum += a.ends[2 * q * a.cols + k];
    }
    lds[group][threadIdx.x % 64] = sum;
    __syncthreads();
    if (group > 0 || k >= a.cols) return;
#pragma unroll
    for (int g = 1; g < 16; ++g) sum += lds[g][threadIdx.x];
    float* const to = a.dtable + cur * a.lddt + k;
    *to = (a.accumulate ? *to : 0.0f) + sum * a.scale;
}

template <int L>
__global__ void __launch_bounds__(256) embedding_zero_kernel(EmbeddingGradArgs a) {
    constexpr int kGroups = 256 / L;
    const int lane = threadIdx.x % L;
    const Columns c(a.cols);
    const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / L; row < a.n; row += (int64_t)gridDim.x * kGroups) {
        float* const to = a.dtable + row * a.lddt;
        for (int k = 8 * lane; c.has(k); k += 8 * L) __builtin_memcpy(to + k, zero, 32);
        if (c.has_single(lane)) to[c.single(lane)] = 0.0f;
    }
}

// ---------------------------------------------------------------- launches

template <class T, int L>
hipError_t lookup_launch(const EmbeddingArgs& a, int n_cu, hipStream_t s) {
    const int64_t need = (a.rows + 256 / L - 1) / (256 / L), full = (int64_t)n_cu * 32;
    hipLaunchKernelGGL((embedding_kernel<T, L>), dim3((uint32_t)(need < full ? need : full)), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <class T>
hipError_t lookup_by_width(const EmbeddingArgs& a, int n_cu, hipStream_t s) {
    return a.cols <= 64 ? lookup_launch<T, 8>(a, n_cu, s) : a.cols <= 128 ? lookup_launch<T, 16>(a, n_cu, s)
         : a.cols <= 256 ? lookup_launch<T, 32>(a, n_cu, s) : a.cols <= 512 ? lookup_launch<T, 64>(a, n_cu, s)
         : lookup_launch<T, 256>(a, n_cu, s);
}

// How the gradient's rows are sorted and summed, and where its workspace's parts are.
struct GradPlan {
    int passes, bits;        // of the sort
    uint32_t tile, tiles;    // keys of a workgroup
    uint32_t part, parts;    // sorted rows of a sum
    size_t keys[2], order[2], counts, totals, ends, bytes;
};
GradPlan grad_plan(int64_t rows, int64_t n, int cols) {
    GradPlan p{};
    int bits = 1;
    while (bits < 32 && ((int64_t)1 << bits) <= n) ++bits;   // keys 0..n
    p.passes = (bits + kSortBits - 1) / kSortBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    auto cut = [&](int64_t least, int64_t most_parts) {
        const int64_t per = (rows + most_parts - 1) / most_parts;
        const int64_t v = per < least ? least : (per + least - 1) / least * least;
        return (uint32_t)v;
    };
    p.tile = cut(kSortStep, 8192);
    p.tiles = (uint32_t)((rows + p.tile - 1) / p.tile);
    p.part = cut(32, 65536);
    p.parts = (uint32_t)((rows + p.part - 1) / p.part);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = take((size_t)rows * 4);
        p.order[i] = take((size_t)rows * 4);
    }
    p.counts = take(((size_t)p.tiles << p.bits) * 4);
    p.totals = take(((size_t)1 << p.bits) * 4);
    p.ends = take((size_t)p.parts * 2 * (size_t)cols * 4);
    p.bytes = at;
    return p;
}

template <int L>
hipError_t zero_launch(const EmbeddingGradArgs& a, int n_cu, hipStream_t s) {
    const int64_t need = (a.n + 256 / L - 1) / (256 / L), full = (int64_t)n_cu * 32;
    hipLaunchKernelGGL((embedding_zero_kernel<L>), dim3((uint32_t)(need < full ? need : full)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <class T, int L>
hipError_t sum_launch(const EmbeddingGradArgs& a, uint32_t parts, hipStream_t s) {
    const uint32_t slabs = (uint32_t)((a.cols + 8 * L - 1) / (8 * L));
    hipLaunchKernelGGL((embedding_sum_kernel<T, L>), dim3((parts + 256 / L - 1) / (256 / L), slabs), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts < 2) return e;
    hipLaunchKernelGGL(embedding_join_kernel, dim3(parts - 1, (uint32_t)((a.cols + 63) / 64)), dim3(1024), 0, s, a);
    return hipGetLastError();
}
template <class T>
hipError_t sum_by_width(const EmbeddingGradArgs& a, uint32_t parts, hipStream_t s) {
    return a.cols <= 64 ? sum_launch<T, 8>(a, parts, s) : a.cols <= 128 ? sum_launch<T, 16>(a, parts, s)
         : a.cols <= 256 ? sum_launch<T, 32>(a, parts, s) : sum_launch<T, 64>(a, parts, s);
}

}  // namespace

hipError_t launch_train_embedding(const EmbeddingArgs& a, bool table_bf16, int n_cu, hipStream_t stream) {
    return table_bf16 ? lookup_by_width<uint16_t>(a, n_cu, stream) : lookup_by_width<float>(a, n_cu, stream);
}

size_t embedding_backward_workspace(int64_t rows, int64_t n, int cols) { return rows ? grad_plan(rows, n, cols).bytes : 0; }

hipError_t launch_train_embedding_backward(EmbeddingGradArgs a, const IntRows& ids, bool dy_bf16, void* workspace, int n_cu,
                                           hipStream_t stream) {
    if (!a.accumulate) {
        const hipError_t e = a.cols <= 64 ? zero_launch<8>(a, n_cu, stream) : a.cols <= 256 ? zero_launch<32>(a, n_cu, stream)
                                                                                           : zero_launch<256>(a, n_cu, stream);
        if (e != hipSuccess) return e;
    }
    if (a.rows == 0) return hipSuccess;
    const GradPlan p = grad_plan(a.rows, a.n, a.cols);
    uint8_t* const ws = (uint8_t*)workspace;
    SortPass s{};
    s.ids = ids;
    s.rows = (uint32_t)a.rows;
    s.n = a.n;
    s.bits = p.bits;
    s.tile = p.tile;
    s.counts = (uint32_t*)(ws + p.counts);
    s.totals = (uint32_t*)(ws + p.totals);
    for (int i = 0; i < p.passes; ++i) {
        s.shift = i * p.bits;
        s.keys_out = (uint32_t*)(ws + p.keys[i % 2]);
        s.rows_out = (uint32_t*)(ws + p.order[i % 2]);
        hipLaunchKernelGGL(sort_count_kernel, dim3(p.tiles), dim3(kSortThreads), 0, stream, s);
        hipLaunchKernelGGL(sort_scan_kernel, dim3(1u << p.bits), dim3(kSortThreads), 0, stream, s, p.tiles);
        hipLaunchKernelGGL(sort_scatter_kernel, dim3(p.tiles), dim3(kSortThreads), 0, stream, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        s.keys_in = s.keys_out;
        s.rows_in = s.rows_out;
    }
    a.keys = s.keys_in;
    a.order = s.rows_in;
    a.ends = (float*)(ws + p.ends);
    a.part = p.part;
    return dy_bf16 ? sum_by_width<uint16_t>(a, p.parts, stream) : sum_by_width<float>(a, p.parts, stream);
}

}  // namespace donerf
