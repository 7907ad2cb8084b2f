// train_embedding.hip - lookup of a table's rows by ids, and the table's gradient.
//
//   forward   y_i = s table[id_i], zeros where id_i names no row.
//   backward  row v of the gradient is s times the sum of dy_i over the i with
//             id_i = v.  The rows' numbers are sorted by their ids (rows of one id stay in
//             the order of i), the sorted rows are summed in parts of equal length, and
//             runs of one id that cross from part to part are joined from the parts'
//             sums: no part is longer where all ids are alike (the sort in one launch
//             is, below), and nothing depends on the order in which workgroups come.
//
// Both are bound by memory where rows are many (dy is read once and the table written,
// twice where a row has an id), and by their launches where they are few.
#include "rows.h"

namespace donerf {
namespace {

// ---------------------------------------------------------------- forward

// 16,384 rows of 2048 columns, fp32 to bf16: 25.4 us, 67 MB written and as much or less read
// (ids that come often are found in the caches).  One row of 2048: 1.7 us.
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

// ---------------------------------------------------------------- zeros

constexpr int kThreads = 1024;        // of the gradient's workgroups
constexpr int kWaves = kThreads / 64;

// Zeros into rows [begin, end) by workgroup `at` of `all`, in turns, but for rows whose flag
// is set (by row - begin).
__device__ __forceinline__ void fill_rows(const ZeroFill& z, int64_t begin, int64_t end, uint32_t at, uint32_t all, const uint32_t* flags) {
    // 4 columns a lane; a row's lanes a power of two, up to a wave
    int bits = 0;
    while (bits < 6 && 4 << bits < z.cols) ++bits;
    const int lane = threadIdx.x & ((1 << bits) - 1), per = kThreads >> bits;
    const int quads = z.cols & ~3;
    typedef float Zeros __attribute__((ext_vector_type(4), aligned(4)));
    for (int64_t row = begin + (int64_t)at * per + (threadIdx.x >> bits); row < end; row += (int64_t)all * per) {
        const uint32_t f = (uint32_t)(row - begin);
        if (flags && flags[f / 32] >> f % 32 & 1) continue;
        float* const to = z.table + row * z.ld;
        // (one loop with both stores is compiled to the plain one)
        if (z.past)
            for (int k = 4 * lane; k < quads; k += 4 << bits) __builtin_nontemporal_store(Zeros{0, 0, 0, 0}, (Zeros*)(to + k));
        else
            for (int k = 4 * lane; k < quads; k += 4 << bits) *(Zeros*)(to + k) = Zeros{0, 0, 0, 0};
        for (int k = quads + lane; k < z.cols; k += 1 << bits) to[k] = 0.0f;
    }
}
// A workgroup's share of the rows of a fill.
__device__ __forceinline__ void fill_share(const ZeroFill& z, uint32_t at, uint32_t all) { fill_rows(z, z.begin, z.end, at, all, nullptr); }

// ---------------------------------------------------------------- sort

constexpr int kMostBins = 1 << kSortBits;

// The key of an id: n for those without a row.
__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t n) { return id >= 0 && id < n ? (uint32_t)id : (uint32_t)n; }
// The key that a pass reads.
__device__ __forceinline__ uint32_t sort_key(const SortPass& s, uint32_t i) {
    return s.keys_in ? s.keys_in[i] : key_of(s.ids.at(i, 0), s.n);
}

// One more in each live lane's bin.  Lanes that agree, as sorted or repeated ids
// do, add once: the same address is served lane by lane.
__device__ __forceinline__ void count_bin(uint32_t* bins, uint32_t bin, bool live) {
    const uint64_t all = __ballot(live);
    if (all == 0) return;
    const int leader = __ffsll((unsigned long long)all) - 1;
    const uint32_t first = __builtin_amdgcn_readlane(bin, leader);
    if (__ballot(live && bin == first) == all) {
        if ((threadIdx.x & 63) == leader) atomicAdd(&bins[first], (uint32_t)__popcll(all));
    } else if (live) {
        atomicAdd(&bins[bin], 1u);
    }
}

// counts[tile][bin]: the keys of each tile by their digit.  160,000 keys: 3 us.
__global__ void __launch_bounds__(kThreads) sort_count_kernel(SortPass s, ZeroFill z) {
    __shared__ uint32_t bins[kMostBins];
    if (blockIdx.x >= s.tiles) return fill_share(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    const uint32_t n_bins = 1u << s.bits;
    for (uint32_t b = threadIdx.x; b < n_bins; b += kThreads) bins[b] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * s.tile, end = s.rows - first < s.tile ? s.rows : first + s.tile;
    for (uint32_t i0 = first; i0 < end; i0 += kThreads) {
        const uint32_t i = i0 + threadIdx.x;
        const bool live = i < end;
        count_bin(bins, (live ? sort_key(s, i) : 0) >> s.shift & (n_bins - 1), live);
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < n_bins; b += kThreads) s.counts[((size_t)blockIdx.x << s.bits) + b] = bins[b];
}

// 64 bins a workgroup: counts become the keys of the bin in the tiles before, a wave a
// share of the tiles.
__global__ void __launch_bounds__(kThreads) sort_scan_kernel(SortPass s) {
    __shared__ uint32_t sums[kWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t bin = blockIdx.x * 64 + lane, per = (s.tiles + kWaves - 1) / kWaves;
    const uint32_t t0 = wave * per, t1 = t0 + per < s.tiles ? t0 + per : s.tiles;
    const bool live = bin < 1u << s.bits;
    uint32_t sum = 0;
    if (live)
        for (uint32_t t = t0; t < t1; ++t) sum += s.counts[((size_t)t << s.bits) + bin];
    sums[wave][lane] = sum;
    __syncthreads();
    uint32_t run = 0, total = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) run += sums[w][lane];
        total += sums[w][lane];
    }
    if (!live) return;
    for (uint32_t t = t0; t < t1; ++t) {
        uint32_t* const at = s.counts + ((size_t)t << s.bits) + bin;
        const uint32_t v = *at;
        *at = run;
        run += v;
    }
    if (wave == 0) s.totals[bin] = total;
}

// LDS of a workgroup that puts keys in order.
struct SortLds {
    uint32_t at[kMostBins];               // where the next key of each bin goes
    uint32_t before[kMostBins];
    alignas(16) uint16_t waves[kWaves][kMostBins];    // keys of each wave, then of the waves before
    uint32_t sums[kWaves];
};

// at[b] becomes the sum of totals before bin b, and before[b].
__device__ __forceinline__ void bin_starts(SortLds& l, uint32_t total, uint32_t before, uint32_t n_bins) {
    // a thread a bin: kMostBins of them at most
    static_assert(kMostBins <= kThreads);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t x = total;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(x, d, 64);
        if (lane >= d) x += o;
    }
    if (lane == 63) l.sums[wave] = x;
    __syncthreads();
    uint32_t run = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        if (w < wave) run += l.sums[w];
    if (threadIdx.x < n_bins) l.at[threadIdx.x] = run + x - total + before;
    __syncthreads();
}

// Where a workgroup's next kThreads keys go, one a thread (those of live threads);
// at[] moves on.  Keys of one bin keep their order.
__device__ __forceinline__ uint32_t place_keys(SortLds& l, uint32_t bin, bool live, int bits) {
    const uint32_t n_bins = 1u << bits;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (uint32_t i = threadIdx.x; i < sizeof(l.waves) / 16; i += kThreads) ((u32x4*)l.waves)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
    uint64_t same = __ballot(live);   // the live lanes with this lane's bin
    for (int b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot(bin >> b & 1);
        same &= bin >> b & 1 ? ones : ~ones;
    }
    const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
    if (live && rank == 0) l.waves[wave][bin] = (uint16_t)__popcll(same);
    __syncthreads();
    if (threadIdx.x < n_bins) {
        uint32_t run = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t v = l.waves[w][threadIdx.x];
            l.waves[w][threadIdx.x] = (uint16_t)run;
            run += v;
        }
        l.before[threadIdx.x] = run;
    }
    __syncthreads();
    const uint32_t to = live ? l.at[bin] + l.waves[wave][bin] + rank : 0;
    __syncthreads();
    if (threadIdx.x < n_bins) l.at[threadIdx.x] += l.before[threadIdx.x];
    return to;   // at[] is read behind the next call's barriers
}

// Moves a tile's keys and rows to their places: 9.3 us for 160,000 keys of 7 bits, most of it
// round trips, of the keys, the tiles' counts and through LDS.
__global__ void __launch_bounds__(kThreads) sort_scatter_kernel(SortPass s, ZeroFill z) {
    __shared__ SortLds l;
    if (blockIdx.x >= s.tiles) return fill_share(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    const uint32_t n_bins = 1u << s.bits, bin = threadIdx.x;
    const uint32_t first = blockIdx.x * s.tile, end = s.rows - first < s.tile ? s.rows : first + s.tile;
    // the first step's, on their way early
    const uint32_t i1 = first + threadIdx.x < end ? first + threadIdx.x : end - 1;
    uint32_t key = sort_key(s, i1), row = s.rows_in ? s.rows_in[i1] : i1;
    uint32_t total = 0, before = 0;   // keys of this thread's bin: all, and those of the tiles before
    if (s.scanned) {
        if (bin < n_bins) total = s.totals[bin], before = s.counts[((size_t)blockIdx.x << s.bits) + bin];
    } else {
        for (uint32_t b = threadIdx.x; b < n_bins; b += kThreads) l.at[b] = l.before[b] = 0;
        __syncthreads();
        const uint32_t per = kThreads >> s.bits, b = threadIdx.x & (n_bins - 1);   // tiles at a time
        constexpr int kTogether = 16;
        for (uint32_t t0 = threadIdx.x >> s.bits; t0 < s.tiles; t0 += kTogether * per) {
            uint32_t v[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const uint32_t t = t0 + j * per < s.tiles ? t0 + j * per : 0;
                v[j] = s.counts[((size_t)t << s.bits) + b];
            }
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const uint32_t t = t0 + j * per;
                total += t < s.tiles ? v[j] : 0;
                before += t < blockIdx.x ? v[j] : 0;
            }
        }
        atomicAdd(&l.at[b], total);
        atomicAdd(&l.before[b], before);
        __syncthreads();
        if (bin < n_bins) {
            before = l.before[bin];
            total = l.at[bin];
        }
        __syncthreads();
    }
    bin_starts(l, total, before, n_bins);
    for (uint32_t i0 = first; i0 < end; i0 += kThreads) {
        const uint32_t i = i0 + threadIdx.x;
        const bool live = i < end;
        if (i0 > first && live) {
            key = sort_key(s, i);
            row = s.rows_in ? s.rows_in[i] : i;
        }
        const uint32_t to = place_keys(l, key >> s.shift & (n_bins - 1), live, s.bits);
        if (live) {
            s.keys_out[to] = key;
            s.rows_out[to] = row;
        }
    }
}

// Up to ITEMS keys a thread in one launch.  Keys are dealt to workgroups by their low
// bits; each reads all of them, keeps its own in their order, sorts them by the other
// bits, and knows from the others' number where they go: equal keys end up side by side,
// which is all that the sums ask for.  The remaining workgroups write zeros meanwhile: 16,384
// keys of 32,000 beside 131 MB 24.3 us, 5.4 TB/s.  Against counts and moves in two passes whole
// calls are shorter: 1500 rows of 32,000 x 256 20.5 us for 30, 4096 of 32,000 x 1024 31 for 43,
// 16,000 of 60,000 x 64 24.5 for 31; of few ids they are not, 12,000 of 100 x 256 22.2 for 20.3.
// A workgroup's time goes with its bucket's keys, and equal ids are one bucket's, as are all
// rows without an id: 16,000 x 64 of 100 ids 19.5 us, of 4 ids 27, of one 44; of 32,000 ids 22,
// and 47 with nine in ten rows without one.
template <int ITEMS>
struct BucketLds {
    SortLds sort;
    uint32_t mine[kWaves], before[kWaves];   // each wave's keys of this bucket, and of those before
    uint16_t keys[ITEMS * kThreads];         // the bits above the bucket's
    uint16_t rows[ITEMS * kThreads];
};
template <int ITEMS>
__global__ void __launch_bounds__(kThreads) sort_buckets_kernel(SortPass s, ZeroFill z) {
    static_assert(ITEMS * kThreads <= 65536 && kSortBits <= 16);
    __shared__ BucketLds<ITEMS> l;
    if (blockIdx.x >= s.tiles) return fill_share(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    const uint32_t n_bins = 1u << s.bits, bucket = blockIdx.x, buckets = 1u << s.shift;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t at0 = wave * ITEMS * 64 + lane;   // a wave takes consecutive keys, 64 at a time
    uint32_t key[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) key[j] = sort_key(s, at0 + 64 * j < s.rows ? at0 + 64 * j : s.rows - 1);
    uint32_t mine = 0, less = 0;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        const bool live = at0 + 64 * j < s.rows;
        const uint32_t b = key[j] & (buckets - 1);
        mine += (uint32_t)__popcll(__ballot(live && b == bucket));
        less += (uint32_t)__popcll(__ballot(live && b < bucket));
    }
    if (lane == 0) l.mine[wave] = mine, l.before[wave] = less;
    if (threadIdx.x < n_bins) l.sort.before[threadIdx.x] = 0;
    __syncthreads();
    uint32_t to = 0, n = 0, base = 0;   // this wave's place, the bucket's keys, and where they go
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) to += l.mine[w];
        n += l.mine[w];
        base += l.before[w];
    }
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        const bool own = at0 + 64 * j < s.rows && (key[j] & (buckets - 1)) == bucket;
        const uint64_t m = __ballot(own);
        if (own) {
            const uint32_t i = to + (uint32_t)__popcll(m & ((1ull << lane) - 1));
            l.keys[i] = (uint16_t)(key[j] >> s.shift);
            l.rows[i] = (uint16_t)(at0 + 64 * j);
        }
        to += (uint32_t)__popcll(m);
    }
    __syncthreads();
    for (uint32_t i0 = 0; i0 < n; i0 += kThreads) {
        const uint32_t i = i0 + threadIdx.x;
        count_bin(l.sort.before, i < n ? l.keys[i] : 0, i < n);
    }
    __syncthreads();
    const uint32_t total = threadIdx.x < n_bins ? l.sort.before[threadIdx.x] : 0;
    bin_starts(l.sort, total, 0, n_bins);
    for (uint32_t i0 = 0; i0 < n; i0 += kThreads) {
        const uint32_t i = i0 + threadIdx.x;
        const uint32_t k = i < n ? l.keys[i] : 0;
        const uint32_t out = base + place_keys(l.sort, k, i < n, s.bits);
        if (i < n) {
            s.keys_out[out] = k << s.shift | bucket;
            s.rows_out[out] = l.rows[i];
        }
    }
}

// ---------------------------------------------------------------- sums

// Rows of a part are read this many at a time.
constexpr int kAhead = 8;

// Sums sorted rows [first, end) of dy at this lane's 8 columns from k on (c.has(k)) and its
// single column (if `single`).  Each run of one id that lies within them is left as the
// result; one that comes from before, or goes on, is put by end(0, ...) or end(1, ...).
template <class T, class Keys, class End>
__device__ __forceinline__ void sum_runs(const EmbeddingGradArgs& a, const RowsIn<T>& dy, const Keys& keys, const Keys& order, uint32_t first,
                                         uint32_t end, int k, int lane, bool single, End put_end) {
    const Columns& c = dy.c;
    uint32_t cur = keys[first];
    bool from_before = first > 0 && keys[first - 1] == cur;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, sum1 = 0.0f;
    auto leave = [&](bool goes_on) {
        if (cur >= a.n) return;   // rows without an id
        if (from_before || goes_on) return put_end(from_before ? 0 : 1, sum, sum1);
        float* const to = a.dtable + cur * a.lddt;
        if (c.has(k)) {
            float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (a.accumulate) __builtin_memcpy(v, to + k, 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += sum[i] * a.scale;
            __builtin_memcpy(to + k, v, 32);
        }
        if (single) to[c.single(lane)] = (a.accumulate ? to[c.single(lane)] : 0.0f) + sum1 * a.scale;
    };
    for (uint32_t i0 = first; i0 < end; i0 += kAhead) {
        uint32_t key[kAhead], row[kAhead];
        Raw<T> raw[kAhead];
        float one[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint32_t i = i0 + j < end ? i0 + j : end - 1;
            key[j] = keys[i];
            row[j] = order[i];
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
    leave(end < a.rows && keys[end] == cur);
}

// Parts of `part` sorted rows, 8 L columns a workgroup: what comes from the part before is
// left in ends[2 p], what goes on into the next one in ends[2 p + 1].  160,000 rows of 256 bf16
// columns 17 us, 82 MB, 4.8 TB/s.
// A workgroup's parts are a block.  One that is all of one id, before and behind it as well,
// leaves the sum of its parts as that of the first: long runs have fewer to join (153,824 rows
// of 2 ids 46 us a call, 114 with a sum for each part).
template <class T, int L>
__global__ void __launch_bounds__(256) embedding_sum_kernel(EmbeddingGradArgs a) {
    constexpr int kParts = 256 / L;
    __shared__ float lds[kParts][8 * L], lds1[kParts][8];
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int64_t p0 = (int64_t)blockIdx.x * kParts, p = p0 + group;
    const int k0 = 8 * (int)(blockIdx.y * L), k = k0 + 8 * lane;
    const RowsIn<T> dy((const T*)a.dy, a.lddy, a.cols);
    const Columns& c = dy.c;
    const bool single = blockIdx.y == 0 && c.has_single(lane);
    const int64_t begin = p0 * a.part, behind = (p0 + kParts) * a.part;
    const bool whole = begin > 0 && behind < a.rows && a.keys[begin - 1] == a.keys[behind];   // the same for all
    if (p * a.part < a.rows && (c.has(k) || single)) {
        const uint32_t first = (uint32_t)(p * a.part), end = (uint32_t)a.rows - first < a.part ? (uint32_t)a.rows : first + a.part;
        sum_runs(a, dy, a.keys, a.order, first, end, k, lane, single, [&](int which, const float* sum, float sum1) {
            if (whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) lds[group][8 * lane + i] = sum[i];
                if (single) lds1[group][lane] = sum1;
                return;
            }
            float* const to = a.ends + (2 * p + which) * a.cols;
            if (c.has(k)) __builtin_memcpy(to + k, sum, 32);
            if (single) to[c.single(lane)] = sum1;
        });
    }
    if (!whole || a.keys[behind] >= a.n) return;
    __syncthreads();
    float* const to = a.ends + 2 * p0 * a.cols;
    for (int t = threadIdx.x; t < 8 * L && c.has(k0 + t); t += 256) {
        float sum = lds[0][t];
#pragma unroll
        for (int g = 1; g < kParts; ++g) sum += lds[g][t];
        to[k0 + t] = sum;
    }
    if (group == 0 && single) {
        float sum = lds1[0][lane];
        for (int g = 1; g < kParts; ++g) sum += lds1[g][lane];
        to[c.single(lane)] = sum;
    }
}

// Where a run's sums are: parts p + 1 up to last, but for one of each block (of 2^bits
// parts) that they hold with the part behind it.
struct Run {
    int64_t first, head, blocks, n;   // first part; parts before the blocks, blocks, sums in all
    int bits;
    __device__ __forceinline__ Run(int64_t p, int64_t last, int b) : first(p + 1), bits(b) {
        const int64_t start = ((p >> bits) + 1) << bits;   // of the first block behind p
        blocks = start < last ? (last - start) >> bits : 0;
        head = blocks ? start - first : last - p;
        n = last - p - (blocks << bits) + blocks;
    }
    // The part of sum i.
    __device__ __forceinline__ int64_t part(int64_t i) const {
        return first + (i < head ? i : i < head + blocks ? head + ((i - head) << bits) : i + (blocks << bits) - blocks);
    }
};
// Joins the runs that begin in 16 parts, a wave each, and go on: 256 columns a workgroup.
// Runs of more than kLongRun further sums are added up by all waves together.  5 us for 5000
// parts of 120 ids, 7.4 us for 2048 of tokens whose commonest has a hundred parts and more, 16 us
// for 4800 of 2 ids: round trips, of the keys, the search for a run's end and its sums.
constexpr int kLongRun = 8;
__global__ void __launch_bounds__(kThreads) embedding_join_kernel(EmbeddingGradArgs a) {
    __shared__ int64_t first_of[kWaves], last_of[kWaves];   // parts of each wave's run, and its id
    __shared__ uint32_t id_of[kWaves], longs;
    __shared__ float lds[kWaves][256];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t p = (int64_t)blockIdx.x * kWaves + wave, parts = (a.rows + a.part - 1) / a.part;
    const int k = (int)(blockIdx.y * 256) + 4 * lane;
    const bool four = k + 4 <= a.cols;
    if (threadIdx.x == 0) longs = 0;
    int64_t last = p;   // the run's last part
    uint32_t cur = 0;
    if (p + 1 < parts) {
        const int64_t first = p * a.part, end = first + a.part;
        // loaded together, whether they are asked for or not
        const int64_t q1 = p + 1 + lane;
        const uint32_t next = a.keys[end], head = a.keys[first], before = a.keys[first > 0 ? first - 1 : 0];
        const uint32_t ahead = a.keys[(q1 < parts ? q1 : parts - 1) * a.part];
        cur = a.keys[end - 1];
        if (cur < a.n && next == cur && !(first > 0 && head == cur && before == cur)) {
            const uint64_t same = __ballot(q1 < parts && ahead == cur);
            last += same == ~0ull ? 64 : __ffsll((unsigned long long)~same) - 1;
            // a run of more: 64 places of the rest at a time, a 64th of it left each time
            for (int64_t rest = parts - 1 - last; same == ~0ull && rest > 0;) {
                const int64_t step = (rest + 63) / 64, q = last + (lane + 1) * step;
                const uint64_t more = __ballot(q < parts && a.keys[(q < parts ? q : parts - 1) * a.part] == cur);
                const int n = more == ~0ull ? 64 : __ffsll((unsigned long long)~more) - 1;
                last += n * step;
                rest = step - 1 < parts - 1 - last ? step - 1 : parts - 1 - last;
            }
        }
    }
    auto load = [&](float* v, int64_t q, int which) {
        const float* const from = a.ends + (2 * q + which) * a.cols + k;
        if (four) {
            __builtin_memcpy(v, from, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = k + i < a.cols ? from[i] : 0.0f;
        }
    };
    // adds a run's sums from, from + step, ..., kLongRun at a time
    auto add = [&](float* sum, const Run& run, int64_t from, int step) {
        for (; from < run.n; from += kLongRun * step) {
            float v[kLongRun][4];
#pragma unroll
            for (int j = 0; j < kLongRun; ++j)
                if (from + j * step < run.n) load(v[j], run.part(from + j * step), 0);
#pragma unroll
            for (int j = 0; j < kLongRun; ++j)
                if (from + j * step < run.n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] += v[j][i];
        }
    };
    auto finish = [&](const float* sum, uint32_t id) {
        float* const to = a.dtable + id * a.lddt + k;
        float v[4] = {0, 0, 0, 0};
        if (a.accumulate)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = k + i < a.cols ? to[i] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += sum[i] * a.scale;
        if (four) {
            __builtin_memcpy(to, v, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k + i < a.cols) to[i] = v[i];
        }
    };
    __syncthreads();
    const Run own(p, last, a.block_bits);
    if (own.n > kLongRun) {
        if (lane == 0) {
            first_of[wave] = p, last_of[wave] = last, id_of[wave] = cur;
            atomicOr(&longs, 1u << wave);
        }
    } else if (last > p) {
        float sum[4];
        load(sum, p, 1);
        add(sum, own, 0, 1);
        finish(sum, cur);
    }
    __syncthreads();
    for (uint32_t left = longs; left; left &= left - 1) {   // the same for all waves
        const int w = __ffs(left) - 1;
        float sum[4] = {0, 0, 0, 0};
        if (wave == 0) load(sum, first_of[w], 1);
        add(sum, Run(first_of[w], last_of[w], a.block_bits), wave, kWaves);
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[wave][4 * lane + i] = sum[i];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int v = 1; v < kWaves; ++v)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += lds[v][4 * lane + i];
            finish(sum, id_of[w]);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- all at once

// Up to kThreads rows in one launch.  Workgroups below a.slabs take 64 columns each: they
// sort the ids in LDS and sum the rows in parts of `part`, ends in LDS, too.  The others
// write zeros into the table's rows that have no id.  100 rows of 32,000 x 1024: 20 us, 6.5 TB/s.
constexpr int kSmallLanes = 8, kSmallGroups = kThreads / kSmallLanes;
struct SmallLds {
    union {
        SortLds sort;
        float ends[kSmallGroups][2][8 * kSmallLanes];
        uint32_t flags[kMostBins];
    };
    float ends1[kSmallGroups][2][8];   // of the single columns
    uint32_t keys[kThreads], order[kThreads];
};
template <class T>
__global__ void __launch_bounds__(kThreads) embedding_small_kernel(EmbeddingGradArgs a, IntRows ids, ZeroFill z, int passes, int bits) {
    __shared__ SmallLds l;
    const int t = threadIdx.x;
    const uint32_t rows = (uint32_t)a.rows;
    const bool live = t < (int)rows;
    uint32_t key = live ? key_of(ids.at(t, 0), a.n) : 0;
    if (blockIdx.x >= a.slabs) {
        // 32 rows a word of flags
        const uint32_t at = blockIdx.x - a.slabs, all = gridDim.x - a.slabs;
        const int64_t begin = a.n * at / all, end = a.n * (at + 1) / all;
        for (int64_t v0 = begin; v0 < end; v0 += 32 * kMostBins) {
            const int64_t v1 = v0 + 32 * kMostBins < end ? v0 + 32 * kMostBins : end;
            for (int w = t; w < kMostBins; w += kThreads) l.flags[w] = 0;
            __syncthreads();
            if (live && key >= v0 && key < v1) atomicOr(&l.flags[(uint32_t)(key - v0) / 32], 1u << (uint32_t)(key - v0) % 32);
            __syncthreads();
            fill_rows(z, v0, v1, 0, 1, l.flags);
            __syncthreads();
        }
        return;
    }
    uint32_t row = t;
    for (int p = 0; p < passes; ++p) {
        const uint32_t n_bins = 1u << bits, bin = key >> (p * bits) & (n_bins - 1);
        if (t < (int)n_bins) l.sort.before[t] = 0;
        __syncthreads();
        count_bin(l.sort.before, bin, live);
        __syncthreads();
        const uint32_t total = t < (int)n_bins ? l.sort.before[t] : 0;
        bin_starts(l.sort, total, 0, n_bins);
        const uint32_t to = place_keys(l.sort, bin, live, bits);
        if (live) l.keys[to] = key, l.order[to] = row;
        __syncthreads();
        if (live) key = l.keys[t], row = l.order[t];
        __syncthreads();
    }
    const int lane = t % kSmallLanes, group = t / kSmallLanes;
    const int k = 8 * (int)(blockIdx.x * kSmallLanes + lane);
    const RowsIn<T> dy((const T*)a.dy, a.lddy, a.cols);
    const Columns& c = dy.c;
    const bool single = blockIdx.x == 0 && c.has_single(lane);
    const uint32_t first = group * a.part;
    if (first < rows && (c.has(k) || single)) {
        const uint32_t end = rows - first < a.part ? rows : first + a.part;
        sum_runs(a, dy, l.keys, l.order, first, end, k, lane, single, [&](int which, const float* sum, float sum1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) l.ends[group][which][8 * lane + i] = sum[i];
            if (single) l.ends1[group][which][lane] = sum1;
        });
    }
    __syncthreads();
    // a group joins the run that begins in its part and goes on
    const uint32_t end = first + a.part;
    if (end >= rows || !(c.has(k) || single)) return;
    const uint32_t cur = l.keys[end - 1];
    if (cur >= a.n || l.keys[end] != cur || (first > 0 && l.keys[first] == cur && l.keys[first - 1] == cur)) return;
    float sum[8], sum1 = single ? l.ends1[group][1][lane] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = l.ends[group][1][8 * lane + i];
    for (uint32_t q = group + 1; q * a.part < rows && l.keys[q * a.part] == cur; ++q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += l.ends[q][0][8 * lane + i];
        if (single) sum1 += l.ends1[q][0][lane];
    }
    float* const to = a.dtable + cur * a.lddt;
    if (c.has(k))
#pragma unroll
        for (int i = 0; i < 8; ++i) to[k + i] = (a.accumulate ? to[k + i] : 0.0f) + sum[i] * a.scale;
    if (single) to[c.single(lane)] = (a.accumulate ? to[c.single(lane)] : 0.0f) + sum1 * a.scale;
}

// ---------------------------------------------------------------- launches

// Rows and buckets (as a power of two) of a sort in one launch (each bucket's workgroup reads
// all keys), and counts of all tiles that each tile's workgroup adds up by itself, from 16 loads
// at a time, rather than in a launch between.
constexpr int64_t kMostSortedAtOnce = 16 * kThreads, kMostTileCounts = 65536;
constexpr int kMostBucketBits = 8;

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
    bool at_once;            // in one launch
    int bucket_bits;         // of its workgroups
    uint32_t tile, tiles;    // keys of a workgroup, workgroups
    int scanned;             // the tiles' counts are added up in a launch of their own
    int lanes;               // of a row in the sums
    uint32_t part, parts;    // sorted rows of a sum
    size_t keys[2], order[2], counts, totals, ends, bytes;
};
GradPlan grad_plan(int64_t rows, int64_t n, int cols) {
    GradPlan p{};
    int bits = 1;
    while (bits < 32 && ((int64_t)1 << bits) <= n) ++bits;   // keys 0..n
    p.passes = (bits + kSortBits - 1) / kSortBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    if (rows <= kThreads) {
        p.part = (uint32_t)((rows + kSmallGroups - 1) / kSmallGroups);
        return p;            // all at once, without a workspace
    }
    auto cut = [&](int64_t least, int64_t most_parts) {
        const int64_t per = (rows + most_parts - 1) / most_parts;
        return (uint32_t)(per < least ? least : (per + least - 1) / least * least);
    };
    p.tile = cut(kThreads, 2048);
    p.tiles = (uint32_t)((rows + p.tile - 1) / p.tile);
    p.at_once = rows <= kMostSortedAtOnce && bits <= kMostBucketBits + kSortBits;
    if (p.at_once) {
        // so many buckets that one pass sorts each, and that they hold 256 keys or so (level with 1024
        // each where zeros are written beside them)
        p.bucket_bits = bits > kSortBits ? bits - kSortBits : 0;
        while (p.bucket_bits < bits - 1 && p.bucket_bits < 7 && (kThreads / 4) << p.bucket_bits < rows) ++p.bucket_bits;
        p.bits = bits - p.bucket_bits;
        p.tiles = 1u << p.bucket_bits;
    }
    p.scanned = (int64_t)p.tiles << p.bits > kMostTileCounts;
    p.lanes = cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : 64;
    // Parts of 8 to 32 rows, for 131,072 lanes: fewer leave the chip idle (60,000 rows of 32
    // columns in 2048 parts 40 us, in 7500 35), more take longer to join than they save (160,000
    // of 32: the 10,000 parts of this rule 30 us, 5000 29).  Beyond 2 million rows, 65,536
    // longer ones.
    p.part = cut(kAhead, 2048 * 64 / p.lanes);
    if (p.part > 32) p.part = 32;
    if (rows > 32 * 65536) p.part = cut(kAhead, 65536);
    p.parts = (uint32_t)((rows + p.part - 1) / p.part);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 15) / 16 * 16;
        return here;
    };
    for (int i = 0; i < (p.passes > 1 && !p.at_once ? 2 : 1); ++i) {
        p.keys[i] = take((size_t)rows * 4);
        p.order[i] = take((size_t)rows * 4);
    }
    if (!p.at_once) p.counts = take(((size_t)p.tiles << p.bits) * 4);
    if (!p.at_once && p.scanned) p.totals = take(((size_t)1 << p.bits) * 4);
    p.ends = take((size_t)p.parts * 2 * (size_t)cols * 4);
    p.bytes = at;
    return p;
}

template <class T, int L>
hipError_t sum_launch(EmbeddingGradArgs a, uint32_t parts, hipStream_t s) {
    a.block_bits = __builtin_ctz(256 / L);
    const uint32_t slabs = (uint32_t)((a.cols + 8 * L - 1) / (8 * L));
    hipLaunchKernelGGL((embedding_sum_kernel<T, L>), dim3((parts + 256 / L - 1) / (256 / L), slabs), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts < 2) return e;
    hipLaunchKernelGGL(embedding_join_kernel, dim3((parts + kWaves - 1) / kWaves, (uint32_t)((a.cols + 255) / 256)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}
template <class T>
hipError_t sum_by_width(const EmbeddingGradArgs& a, const GradPlan& p, hipStream_t s) {
    return p.lanes == 8 ? sum_launch<T, 8>(a, p.parts, s) : p.lanes == 16 ? sum_launch<T, 16>(a, p.parts, s)
         : p.lanes == 32 ? sum_launch<T, 32>(a, p.parts, s) : sum_launch<T, 64>(a, p.parts, s);
}

// Whether zeros pass the caches (bytes of dy and of the table).  Where both do not fit into
// the last level beside what else is there (256 MB in all), zeros that stay push dy out of it
// and are themselves pushed out while the sums read and write: 24,000 rows of 32,000 x 1024
// (49 and 131 MB) 65 us, 52 past the caches, and with a pass over the result behind the call 103
// and 95; 65,536 of 128,000 x 512 95 and 78, with the pass 190 and 178; 8192 of 32,000 x 1024
// (148 MB) 38 and 40, with the pass 80 and 82.  With few rows of dy there is little to push out,
// and what reads the result finds a part of it: 4096 of 32,000 x 1024 31 us and 37, with the pass
// 65 and 72.
bool zeros_past_caches(int64_t dy, int64_t table) { return dy >= table / 8 && dy + table >= (int64_t)144 << 20; }
// Workgroups that write zeros into n rows.
uint32_t fill_groups(int64_t n, int cols, int n_cu) {
    const int64_t need = (n * cols + 16383) / 16384;   // 64 KB each, or more
    const int64_t most = (int64_t)n_cu * 2;
    return (uint32_t)(need < 1 ? 1 : need < most ? need : most);
}

}  // namespace

hipError_t launch_train_embedding(const EmbeddingArgs& a, bool table_bf16, int n_cu, hipStream_t stream) {
    return table_bf16 ? lookup_by_width<uint16_t>(a, n_cu, stream) : lookup_by_width<float>(a, n_cu, stream);
}

size_t embedding_backward_workspace(int64_t rows, int64_t n, int cols) { return grad_plan(rows, n, cols).bytes; }

hipError_t launch_train_embedding_backward(EmbeddingGradArgs a, const IntRows& ids, bool dy_bf16, void* workspace, int n_cu,
                                           hipStream_t stream) {
    if (a.rows == 0 && a.accumulate) return hipSuccess;
    const GradPlan p = grad_plan(a.rows, a.n, a.cols);
    ZeroFill z{a.dtable, a.lddt, a.cols, zeros_past_caches(a.rows * a.cols * (dy_bf16 ? 2 : 4), a.n * a.cols * 4), 0, a.n};
    a.part = p.part;
    if (a.rows <= kThreads) {
        a.slabs = a.rows ? (uint32_t)((a.cols + 8 * kSmallLanes - 1) / (8 * kSmallLanes)) : 0;
        const dim3 grid(a.slabs + (a.accumulate ? 0 : fill_groups(a.n, a.cols, n_cu)));
        if (dy_bf16) hipLaunchKernelGGL((embedding_small_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a, ids, z, p.passes, p.bits);
        else hipLaunchKernelGGL((embedding_small_kernel<float>), grid, dim3(kThreads), 0, stream, a, ids, z, p.passes, p.bits);
        return hipGetLastError();
    }
    uint8_t* const ws = (uint8_t*)workspace;
    SortPass s{};
    s.ids = ids;
    s.rows = (uint32_t)a.rows;
    s.n = a.n;
    s.bits = p.bits;
    s.tile = p.tile;
    s.tiles = p.tiles;
    s.scanned = p.scanned;
    s.counts = (uint32_t*)(ws + p.counts);
    s.totals = (uint32_t*)(ws + p.totals);
    // the zeros are written beside the sort, whose launches leave most of the chip idle
    const int launches = p.at_once ? 1 : 2 * p.passes;
    int launch = 0;
    auto share = [&] {
        z.begin = a.n * launch / launches;
        z.end = a.n * (launch + 1) / launches;
        ++launch;
        return a.accumulate ? 0 : fill_groups(z.end - z.begin, a.cols, n_cu);
    };
    hipError_t e = hipSuccess;
    for (int i = 0; i < (p.at_once ? 1 : p.passes) && e == hipSuccess; ++i) {
        s.shift = i * p.bits;
        s.keys_out = (uint32_t*)(ws + p.keys[i % 2]);
        s.rows_out = (uint32_t*)(ws + p.order[i % 2]);
        const dim3 threads(kThreads);
        if (p.at_once) {
            const dim3 grid(p.tiles + share());
            s.shift = p.bucket_bits;
            if (a.rows <= 4 * kThreads) hipLaunchKernelGGL((sort_buckets_kernel<4>), grid, threads, 0, stream, s, z);
            else hipLaunchKernelGGL((sort_buckets_kernel<16>), grid, threads, 0, stream, s, z);
        } else {
            const dim3 counters(p.tiles + share());
            hipLaunchKernelGGL(sort_count_kernel, counters, threads, 0, stream, s, z);
            if (p.scanned) hipLaunchKernelGGL(sort_scan_kernel, dim3(((1u << p.bits) + 63) / 64), threads, 0, stream, s);
            const dim3 movers(p.tiles + share());
            hipLaunchKernelGGL(sort_scatter_kernel, movers, threads, 0, stream, s, z);
        }
        e = hipGetLastError();
        s.keys_in = s.keys_out;
        s.rows_in = s.rows_out;
    }
    if (e != hipSuccess) return e;
    a.keys = s.keys_in;
    a.order = s.rows_in;
    a.ends = (float*)(ws + p.ends);
    return dy_bf16 ? sum_by_width<uint16_t>(a, p, stream) : sum_by_width<float>(a, p, stream);
}

}  // namespace donerf
