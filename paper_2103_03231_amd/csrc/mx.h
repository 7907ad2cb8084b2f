// mx.h - microscaled formats on gfx950 (include/donerf.h donerf_type): blocks of
// 32 consecutive columns of a row share one power of two, 2^(c - 127) with c one
// byte (E8M0, 255 = NaN).
//
// The scale of a block is the smallest 2^s that holds its largest value,
// max|v| <= M 2^s with M the elements' largest (6 for E2M1, 448 for E4M3), as
// the fp8 networks choose theirs: nothing is clamped, so every element is off by
// at most half a step of its own binade or of the smallest one.  Both
// conversions, to elements (rounded to nearest even) and back, are single
// instructions that take the scale as the exponent field of an fp32.
#pragma once

#include "device.h"

namespace donerf {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

constexpr int kMxBlock = 32;      // columns that share a scale
constexpr int kMxNaN = 255;       // scale code

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t kInfBits = 0x7f800000u;   // and above: NaN

// Largest |v| as its bits, NaN if there is one (v_maximum3_f32 keeps it).
template <int N>
__device__ __forceinline__ uint32_t top_bits(const float* v) {
    float t = __builtin_fabsf(v[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) t = __builtin_elementwise_maximum(t, __builtin_fabsf(v[i]));
    return abs_bits(t);
}
// The same among finite values only.
template <int N>
__device__ __forceinline__ uint32_t finite_top_bits(const float* v) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) t = max(t, abs_bits(v[i]) < kInfBits ? abs_bits(v[i]) : 0u);
    return t;
}

// The largest of v over a quad of lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
}

// Scale code of a block whose largest |v| has the bits top: the exponent of
// 1.5 * 2^2 (E2M1) or 1.75 * 2^8 (E4M3) below it, one more where its mantissa is
// larger; at least 0, where every fp32 below the smallest normal number fits.
__device__ __forceinline__ int mx4_code(uint32_t top) {
    if (top >= kInfBits) return kMxNaN;   // a block that holds an infinity or NaN reads as NaN
    return max(0, (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u));
}
__device__ __forceinline__ int mx8_code(uint32_t top) {
    return max(0, (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u));
}
__device__ __forceinline__ float scale_arg(int code) { return __uint_as_float((uint32_t)code << 23); }

// 8 values as E2M1, the first in the lowest nibble.
__device__ __forceinline__ uint32_t to_e2m1x8(const float* v, int code) {
    const float s = scale_arg(code);
    uint32_t p = 0;
    p = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(p, v[0], v[1], s, 0);
    p = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(p, v[2], v[3], s, 1);
    p = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(p, v[4], v[5], s, 2);
    p = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(p, v[6], v[7], s, 3);
    return code == kMxNaN ? 0u : p;
}
// 8 E2M1 codes with those of negative values, and -0, zero.
__device__ __forceinline__ uint32_t relu_e2m1x8(uint32_t p) {
    const uint32_t s = p & 0x88888888u;
    return p & ~(s | (s - (s >> 3)));
}

// 4 finite values as E4M3, the first in the lowest byte.
__device__ __forceinline__ uint32_t round_e4m3x4(const float* v, int code) {
    const float s = scale_arg(code);
    s16x2 p = {0, 0};
    p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[0], v[1], s, false);
    p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, v[2], v[3], s, true);
    return __builtin_bit_cast(uint32_t, p);
}
// The smallest element, 2^-9 of the scale; below the normal numbers as far as fp32
// goes.
__device__ __forceinline__ float least_e4m3(int code) { return ldexpf(1.0f, code - 127 - 9); }
// The same, where a value other than zero keeps at least the smallest code (2^-17.8
// of the block's largest value), so a checkpoint still tells which units a ReLU let
// through.
__device__ __forceinline__ uint32_t to_e4m3x4(const float* v, int code) {
    const float least = least_e4m3(code);
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float m = v[i] == 0.0f ? 0.0f : fmaxf(fabsf(v[i]), least);
        w[i] = copysignf(m, v[i]);
    }
    return round_e4m3x4(w, code);
}
// The codes p of 4 values with NaN in the place of those that are not finite
// (E4M3 has no infinity).
__device__ __forceinline__ uint32_t e4m3_not_finite(uint32_t p, const float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (abs_bits(v[i]) >= kInfBits) p |= 0x7fu << (8 * i);
    return p;
}

// 8 E2M1 or 4 E4M3 elements as fp32; a NaN scale gives NaN.
__device__ __forceinline__ void from_e2m1x8(uint32_t p, int code, float* v) {
    sfor<4>([&](auto I) {
        const f32x2 t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(p, scale_arg(code), CV(I));
        v[2 * CV(I)] = t[0];
        v[2 * CV(I) + 1] = t[1];
    });
}
__device__ __forceinline__ void from_e4m3x4(uint32_t p, int code, float* v) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)p, scale_arg(code), false);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)p, scale_arg(code), true);
    v[0] = a[0];
    v[1] = a[1];
    v[2] = b[0];
    v[3] = b[1];
}
// The same as bf16, 8 elements: exact, but for results below bf16's smallest
// numbers and overflow.
__device__ __forceinline__ u32x4 e2m1x8_as_bf16(uint32_t p, int code) {
    const float s = scale_arg(code);
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(p, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(p, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(p, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(p, s, 3))};
}
__device__ __forceinline__ u32x4 e4m3x8_as_bf16(u32x2 p, int code) {
    const float s = scale_arg(code);
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)p[0], s, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)p[0], s, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)p[1], s, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)p[1], s, true))};
}

// 8 consecutive values of a row from column k on as fp32, zeros behind the last
// of `cols`.  Rows may start at any multiple of their type's size: gfx950 takes
// wide loads at such addresses.
template <class T>
struct Row8;
template <>
struct Row8<float> {
    __device__ static __forceinline__ void load(const float* row, int k, int cols, float* v) {
        if (k + 8 <= cols) {
            __builtin_memcpy(v, row + k, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = row[k + i < cols ? k + i : cols - 1];   // loads without conditions
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < cols ? v[i] : 0.0f;
        }
    }
    __device__ static __forceinline__ void store(float* row, int k, int cols, const float* v) {
        if (k + 8 <= cols) {
            __builtin_memcpy(row + k, v, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < cols) row[k + i] = v[i];
        }
    }
};
template <>
struct Row8<uint16_t> {   // bf16
    __device__ static __forceinline__ u32x4 load_raw(const uint16_t* row, int k, int cols) {
        u32x4 p = {0, 0, 0, 0};
        if (k + 8 <= cols) {
            __builtin_memcpy(&p, row + k, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v = row[k + i < cols ? k + i : cols - 1];
                p[i / 2] |= k + i < cols ? v << (16 * (i & 1)) : 0u;
            }
        }
        return p;
    }
    __device__ static __forceinline__ void load(const uint16_t* row, int k, int cols, float* v) {
        const u32x4 p = load_raw(row, k, cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(p[i] << 16);
            v[2 * i + 1] = __uint_as_float(p[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ void store_raw(uint16_t* row, int k, int cols, u32x4 p) {
        if (k + 8 <= cols) {
            __builtin_memcpy(row + k, &p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < cols) row[k + i] = (uint16_t)(p[i / 2] >> (16 * (i & 1)));
        }
    }
};

// bf16 rows of any stride and address (2-byte aligned), read in chunks of 8
// columns by unconditional 16-byte loads: guarded ones would each be waited for
// before the next.  A chunk that reaches behind its row's end reads on into what
// follows, except at the very end of the matrix, where the load stays within it;
// fix() brings the chunk's columns into place and clears what is not the row's.
struct Bf16Rows {
    const uint16_t* base;
    int64_t ld;
    int64_t rows;
    int cols;
    int64_t last;    // offset of the last 16 bytes of the matrix; negative if it has fewer
    __device__ __forceinline__ Bf16Rows() {}
    __device__ __forceinline__ Bf16Rows(const uint16_t* p, int64_t ld_, int64_t rows_, int cols_)
        : base(p), ld(ld_), rows(rows_), cols(cols_), last((rows_ - 1) * ld_ + cols_ - 8) {}
    // The chunk at column k of a row < rows; k may lie behind the last column.
    __device__ __forceinline__ u32x4 load(int64_t row, int k) const { return load_at(row * ld + k, k); }
    // The same by its offset in the matrix, which may lie behind its end.
    __device__ __forceinline__ u32x4 load_at(int64_t at, int k) const {
        if (last < 0) {   // fewer than 16 bytes
            const int64_t row = at - k;
            return row <= last + 8 - cols ? Row8<uint16_t>::load_raw(base + row, k, cols) : u32x4{0, 0, 0, 0};
        }
        u32x4 v;
        __builtin_memcpy(&v, base + (at < last ? at : last), 16);
        return v;
    }
    __device__ __forceinline__ u32x4 fix(u32x4 v, int64_t row, int k) const {
        if (last >= 0) {
            const int64_t past = row * ld + k - last;
            const int s = past < 0 ? 0 : past > 8 ? 8 : (int)past;
            if (s & 8) v = u32x4{0, 0, 0, 0};
            if (s & 4) v = u32x4{v[2], v[3], 0, 0};
            if (s & 2) v = u32x4{v[1], v[2], v[3], 0};
            if (s & 1) v = u32x4{(v[0] >> 16) | (v[1] << 16), (v[1] >> 16) | (v[2] << 16), (v[2] >> 16) | (v[3] << 16), v[3] >> 16};
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int left = cols - k - 2 * i;
            v[i] &= left >= 2 ? 0xffffffffu : left == 1 ? 0xffffu : 0u;
        }
        return v;
    }
};

}  // namespace
}  // namespace donerf
