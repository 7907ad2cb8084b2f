// mx_linear.hip - y = act(x W^T + b) with x and W microscaled E2M1.
#include "layer_gemm.h"

namespace donerf {
namespace {

template <int SRC>
hipError_t launch_converting(const GemmArgs& g, int out, int n_cu, hipStream_t stream) {
    switch (out) {
        case kOutF32: return launch_layer_rows<kOpMx4, 1, false, SRC, kEpiF32>(g, n_cu, stream);
        case kOutMx4: return launch_layer_rows<kOpMx4, 1, false, SRC, kEpiMx4>(g, n_cu, stream);
        default: return launch_layer_rows<kOpMx4, 1, false, SRC, kEpiBf16>(g, n_cu, stream);
    }
}

}  // namespace

bool mx_linear_converts(const GemmArgs& g, int n_cu) { return fits_rows(g, 256, n_cu); }

hipError_t launch_mx_linear_convert(const GemmArgs& g, bool x_bf16, int out, int n_cu, hipStream_t stream) {
    return x_bf16 ? launch_converting<kSrcBf16>(g, out, n_cu, stream) : launch_converting<kSrcF32>(g, out, n_cu, stream);
}

hipError_t launch_mx_linear(const GemmArgs& g, int out, int n_cu, hipStream_t stream) {
    switch (out) {
        case kOutF32: return launch_layer_gemm<kOpMx4, false, true, true, kEpiF32>(g, n_cu, stream);
        case kOutMx4: return launch_layer_gemm<kOpMx4, false, true, true, kEpiMx4>(g, n_cu, stream);
        default: return launch_layer_gemm<kOpMx4, false, true, true, kEpiBf16>(g, n_cu, stream);
    }
}

}  // namespace donerf
