// rows.h - rows of a matrix in registers, for operators that need a whole row at
// once: L lanes share a row and hold C chunks of 8 columns each, lane l those at
// columns 8 (l + L j), j < C.  The up to 7 columns behind the last whole chunk are held
// one by one, by the row's first lanes.
#pragma once

#include "internal.h"
#include "mx.h"

namespace donerf {
namespace {

// Threads of a workgroup whose rows have L lanes each.
constexpr int row_threads(int L) { return L > 256 ? L : 256; }

// 8 consecutive values of a row as they are in memory.
template <class T>
struct Raw;
template <>
struct Raw<uint16_t> {   // bf16
    u32x4 v;
    __device__ __forceinline__ void values(float* f) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    // The value with these fp32 bits (one that bf16 has) in all places.
    __device__ __forceinline__ void fill(uint32_t bits) {
        const uint32_t two = bits | bits >> 16;
        v = u32x4{two, two, two, two};
    }
    // Nothing computed of the values before this is kept behind it: they are taken
    // apart again there, instead of being held twice.
    __device__ __forceinline__ void hold() { asm volatile("" : "+v"(v)); }
};
template <>
struct Raw<float> {
    u32x4 v[2];
    __device__ __forceinline__ void values(float* f) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i / 4][i % 4]);
    }
    __device__ __forceinline__ void fill(uint32_t bits) { v[0] = v[1] = u32x4{bits, bits, bits, bits}; }
    __device__ __forceinline__ void hold() { asm volatile("" : "+v"(v[0]), "+v"(v[1])); }
};

__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// How a row's columns are shared out.
struct Columns {
    int cols, whole;   // all of them, and those of whole chunks
    __device__ __forceinline__ explicit Columns(int n) : cols(n), whole(n & ~7) {}
    __device__ __forceinline__ bool has(int k) const { return k < whole; }
    // Whether a lane holds a single column, and which (one of the row's in any case).
    __device__ __forceinline__ bool any_single() const { return whole < cols; }
    __device__ __forceinline__ bool has_single(int lane) const { return lane < cols - whole; }
    __device__ __forceinline__ int single(int lane) const { return has_single(lane) ? whole + lane : cols - 1; }
};

// Rows of any stride, at any address that their type's size divides (gfx950 takes wide
// loads at such addresses).  Loads have no conditions: guarded ones would each be waited
// for before the next.
template <class T>
struct RowsIn {
    typedef Raw<T> Held;
    const T* base;
    int64_t ld;
    Columns c;
    __device__ __forceinline__ RowsIn(const T* p, int64_t ld_, int cols) : base(p), ld(ld_), c(cols) {}
    // The chunk at column k of a row; one behind the last whole chunk reads the first.
    __device__ __forceinline__ Held load(int64_t row, int k) const {
        Held r;
        if (c.whole == 0) r.fill(0);   // the same for all lanes
        else __builtin_memcpy(&r, base + row * ld + (c.has(k) ? k : 0), sizeof r);
        return r;
    }
    __device__ __forceinline__ float load_single(int64_t row, int lane) const { return value_of(base[row * ld + c.single(lane)]); }
    __device__ __forceinline__ bool single_is_zero(float v, int64_t, int) const { return v == 0.0f; }
};

// E4M3 rows in the same chunks.
struct Mx8Raw {
    u32x2 p;
    int code;
    __device__ __forceinline__ void values(float* f) const {
        from_e4m3x4(p[0], code, f);
        from_e4m3x4(p[1], code, f + 4);
    }
    __device__ __forceinline__ void hold() { asm volatile("" : "+v"(p), "+v"(code)); }
};
struct Mx8In {
    typedef Mx8Raw Held;
    MxIn q;
    Columns c;
    __device__ __forceinline__ Mx8In(const MxIn& q_, int cols) : q(q_), c(cols) {}
    __device__ __forceinline__ Held load(int64_t row, int k) const {
        const int at = c.has(k) ? k : 0;   // rows have whole blocks
        return Mx8Raw{*(const u32x2*)(q.codes + row * q.ld + at), (int)q.scales[row * q.ld_scales + at / kMxBlock]};
    }
    __device__ __forceinline__ float load_single(int64_t row, int lane) const {
        const int at = c.single(lane);
        float f[4];
        from_e4m3x4(q.codes[row * q.ld + at], q.scales[row * q.ld_scales + at / kMxBlock], f);
        return f[0];
    }
    __device__ __forceinline__ bool single_is_zero(float, int64_t row, int lane) const {
        return (q.codes[row * q.ld + c.single(lane)] & 0x7f) == 0;
    }
};

// Whether value i of a chunk is zero; of an E4M3 one the element, whatever its scale.
__device__ __forceinline__ bool is_zero(const Mx8Raw& h, const float*, int i) { return ((h.p[i / 4] >> (8 * (i % 4))) & 0x7fu) == 0; }
template <class T>
__device__ __forceinline__ bool is_zero(const Raw<T>&, const float* v, int i) { return v[i] == 0.0f; }

// 8 values from column k on, or one, in the result's type.
__device__ __forceinline__ void store8(const RowsOut& y, int64_t row, int k, const float* v) {
    if (y.bf16) {
        const u32x4 p = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        __builtin_memcpy((uint16_t*)y.base + row * y.ld + k, &p, 16);
    } else {
        __builtin_memcpy((float*)y.base + row * y.ld + k, v, 32);
    }
}
__device__ __forceinline__ void store1(const RowsOut& y, int64_t row, int k, float v) {
    if (y.bf16) ((uint16_t*)y.base)[row * y.ld + k] = (uint16_t)pack_bf16x2(v, v);
    else ((float*)y.base)[row * y.ld + k] = v;
}

// 8 values from column k on as E4M3: a block's four chunks are in a quad of lanes.  All
// four call it; columns behind the last one hold zeros.
__device__ __forceinline__ void store_mx8(const MxOut& q, int64_t row, int k, int cols, const float* v) {
    uint32_t top = quad_max(top_bits<8>(v));
    const bool bad = top >= kInfBits;   // the same over a quad
    if (bad) top = quad_max(finite_top_bits<8>(v));
    const int code = mx8_code(top);
    u32x2 p = {to_e4m3x4(v, code), to_e4m3x4(v + 4, code)};
    if (bad) p = u32x2{e4m3_not_finite(p[0], v), e4m3_not_finite(p[1], v + 4)};
    const int block = k / kMxBlock;
    if (block * kMxBlock >= cols) return;
    *(u32x2*)(q.codes + row * q.ld + k) = p;
    if (k % kMxBlock == 0) q.scales[row * q.ld_scales + block] = (uint8_t)code;
}

// ---------------------------------------------------------------- sums and maxima over a row's lanes

struct Add {
    __device__ static __forceinline__ float of(float a, float b) { return a + b; }
};
// NaN kept.
struct Max {
    __device__ static __forceinline__ float of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Over each L neighbouring lanes of a wave, L a power of two up to 64; every lane gets
// the same bits, as each step combines the same two values on either side.
template <int L, class F>
__device__ __forceinline__ float lanes_all(float v) {
    if constexpr (L > 1) v = F::of(v, dpp<0xB1>(v));    // lanes 1 0 3 2
    if constexpr (L > 2) v = F::of(v, dpp<0x4E>(v));    // lanes 2 3 0 1
    if constexpr (L > 4) v = F::of(v, dpp<0x141>(v));   // 7 .. 0 of each 8
    if constexpr (L > 8) v = F::of(v, dpp<0x140>(v));   // 15 .. 0 of each 16
    if constexpr (L > 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = F::of(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if constexpr (L > 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = F::of(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    return v;
}

// Over the L lanes of a row, N values at once, in registers: steps of a few cycles where LDS
// would take a hundred each.  Rows of several waves meet in LDS,
// in two places by turns: a wave that is a call ahead writes to the other one, and
// cannot be two ahead.
template <int L, int N, int THREADS = row_threads(L)>
struct RowReduce {
    static constexpr int kWaves = L > 64 ? THREADS / 64 : 0;
    struct Lds {
        float v[2][N][kWaves > 0 ? kWaves : 1];
    };
    Lds* lds;
    int turn = 0;
    __device__ __forceinline__ RowReduce(Lds* l) : lds(l) {}
    template <class F>
    __device__ __forceinline__ void all(float (&v)[N]) {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = lanes_all<(L < 64 ? L : 64), F>(v[n]);
        if constexpr (L > 64) {
            constexpr int W = L / 64;   // waves of a row
            const int wave = threadIdx.x / 64, first = wave / W * W;
            if (threadIdx.x % 64 == 0)
#pragma unroll
                for (int n = 0; n < N; ++n) lds->v[turn][n][wave] = v[n];
            lds_barrier();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                v[n] = lds->v[turn][n][first];
#pragma unroll
                for (int i = 1; i < W; ++i) v[n] = F::of(v[n], lds->v[turn][n][first + i]);
            }
            turn ^= 1;
        }
    }
    template <class F>
    __device__ __forceinline__ float one(float x) {
        static_assert(N == 1);
        float v[1] = {x};
        all<F>(v);
        return v[0];
    }
};

}  // namespace
}  // namespace donerf
