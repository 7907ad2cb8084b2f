// mx_convert.hip - fp32 and bf16 rows to microscaled ones and back (mx.h).
//
// Four lanes share a block of 32 columns, eight columns each: a wave's loads and
// stores then cover whole cache lines, and the block's largest value takes two
// exchanges within a quad of lanes.  One pass, nothing kept: bound by memory
// (160,000 x 256 bf16 to E4M3 24 us, back 19 us: 5.2 and 6.4 TB/s, the buffers partly
// in the last-level cache; 2049 x 4100 fp32 to E2M1 8.3 us).
#include "internal.h"
#include "mx.h"

namespace donerf {
namespace {

constexpr int kConvThreads = 256;

template <class T, bool FP8>
__global__ void __launch_bounds__(kConvThreads) mx_quantize_kernel(const T* x, int64_t ldx, MxOut q, uint32_t rows,
                                                                   int cols, uint32_t per_row) {
    // per_row = 4 lanes per block: quads are whole at the end too
    const uint32_t total = rows * per_row;
    for (uint32_t i = blockIdx.x * kConvThreads + threadIdx.x; i < total; i += gridDim.x * kConvThreads) {
        const uint32_t row = i / per_row, c = i % per_row;
        float v[8];
        Row8<T>::load(x + row * ldx, (int)c * 8, cols, v);
        uint32_t top = quad_max(top_bits<8>(v));
        uint8_t* dst = q.codes + row * q.ld;
        int code;
        if (FP8) {
            const bool bad = __any(top >= kInfBits);
            if (bad && top >= kInfBits) top = quad_max(finite_top_bits<8>(v));   // whole quads
            code = mx8_code(top);
            u32x2 p = {to_e4m3x4(v, code), to_e4m3x4(v + 4, code)};
            if (bad) p = u32x2{e4m3_not_finite(p[0], v), e4m3_not_finite(p[1], v + 4)};
            *(u32x2*)(dst + (size_t)c * 8) = p;
        } else {
            code = mx4_code(top);
            *(uint32_t*)(dst + (size_t)c * 4) = to_e2m1x8(v, code);
        }
        if ((c & 3) == 0) q.scales[row * q.ld_scales + (c >> 2)] = (uint8_t)code;
    }
}

template <class T, bool FP8>
__global__ void __launch_bounds__(kConvThreads) mx_dequantize_kernel(MxIn q, T* y, int64_t ldy, uint32_t rows, int cols,
                                                                     uint32_t per_row) {
    const uint32_t total = rows * per_row;
    for (uint32_t i = blockIdx.x * kConvThreads + threadIdx.x; i < total; i += gridDim.x * kConvThreads) {
        const uint32_t row = i / per_row, c = i % per_row;
        if ((int)c * 8 >= cols) continue;
        const uint8_t* src = q.codes + row * q.ld;
        const int code = q.scales[row * q.ld_scales + (c >> 2)];
        u32x2 p = {0, 0};
        if (FP8) p = *(const u32x2*)(src + (size_t)c * 8);
        else p[0] = *(const uint32_t*)(src + (size_t)c * 4);
        if constexpr (sizeof(T) == 2) {
            Row8<T>::store_raw(y + row * ldy, (int)c * 8, cols, FP8 ? e4m3x8_as_bf16(p, code) : e2m1x8_as_bf16(p[0], code));
        } else {
            float v[8];
            if (FP8) {
                from_e4m3x4(p[0], code, v);
                from_e4m3x4(p[1], code, v + 4);
            } else {
                from_e2m1x8(p[0], code, v);
            }
            Row8<T>::store(y + row * ldy, (int)c * 8, cols, v);
        }
    }
}

// Calls f(first row, rows, workgroups) for slices of the rows whose lanes a
// 32-bit index counts.
template <class F>
hipError_t by_slices(int64_t rows, int cols, int n_cu, F f) {
    const uint32_t per_row = 4u * (uint32_t)((cols + kMxBlock - 1) / kMxBlock);
    const int64_t most = ((int64_t)1 << 30) / per_row;
    for (int64_t r0 = 0; r0 < rows; r0 += most) {
        const uint32_t n = (uint32_t)(rows - r0 < most ? rows - r0 : most);
        const uint32_t wg = (n * per_row + kConvThreads - 1) / kConvThreads;
        const uint32_t full = (uint32_t)n_cu * 32;
        f(r0, n, per_row, dim3(wg < full ? wg : full));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_mx_quantize(const void* x, int64_t ldx, bool x_bf16, const MxOut& q, bool fp8, int64_t rows, int cols,
                              int n_cu, hipStream_t stream) {
    return by_slices(rows, cols, n_cu, [&](int64_t r0, uint32_t n, uint32_t per_row, dim3 grid) {
        const MxOut o{q.codes + r0 * q.ld, q.ld, q.scales + r0 * q.ld_scales, q.ld_scales};
        const float* xf = (const float*)x + (x_bf16 ? 0 : r0 * ldx);
        const uint16_t* xh = (const uint16_t*)x + (x_bf16 ? r0 * ldx : 0);
        const dim3 th(kConvThreads);
        if (x_bf16 && fp8) hipLaunchKernelGGL((mx_quantize_kernel<uint16_t, true>), grid, th, 0, stream, xh, ldx, o, n, cols, per_row);
        else if (x_bf16) hipLaunchKernelGGL((mx_quantize_kernel<uint16_t, false>), grid, th, 0, stream, xh, ldx, o, n, cols, per_row);
        else if (fp8) hipLaunchKernelGGL((mx_quantize_kernel<float, true>), grid, th, 0, stream, xf, ldx, o, n, cols, per_row);
        else hipLaunchKernelGGL((mx_quantize_kernel<float, false>), grid, th, 0, stream, xf, ldx, o, n, cols, per_row);
    });
}

hipError_t launch_mx_dequantize(const MxIn& q, bool fp8, void* y, int64_t ldy, bool y_bf16, int64_t rows, int cols,
                                int n_cu, hipStream_t stream) {
    return by_slices(rows, cols, n_cu, [&](int64_t r0, uint32_t n, uint32_t per_row, dim3 grid) {
        const MxIn o{q.codes + r0 * q.ld, q.ld, q.scales + r0 * q.ld_scales, q.ld_scales};
        float* yf = (float*)y + (y_bf16 ? 0 : r0 * ldy);
        uint16_t* yh = (uint16_t*)y + (y_bf16 ? r0 * ldy : 0);
        const dim3 th(kConvThreads);
        if (y_bf16 && fp8) hipLaunchKernelGGL((mx_dequantize_kernel<uint16_t, true>), grid, th, 0, stream, o, yh, ldy, n, cols, per_row);
        else if (y_bf16) hipLaunchKernelGGL((mx_dequantize_kernel<uint16_t, false>), grid, th, 0, stream, o, yh, ldy, n, cols, per_row);
        else if (fp8) hipLaunchKernelGGL((mx_dequantize_kernel<float, true>), grid, th, 0, stream, o, yf, ldy, n, cols, per_row);
        else hipLaunchKernelGGL((mx_dequantize_kernel<float, false>), grid, th, 0, stream, o, yf, ldy, n, cols, per_row);
    });
}

}  // namespace donerf
