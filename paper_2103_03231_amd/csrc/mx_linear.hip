// mx_linear.hip - y = act(x W^T + b) with x and W microscaled E2M1.
#include "layer_gemm.h"

namespace donerf {

hipError_t launch_mx_linear(const GemmArgs& g, int out, int n_cu, hipStream_t stream) {
    switch (out) {
        case kOutF32: return launch_layer_gemm<kOpMx4, false, true, true, kEpiF32>(g, n_cu, stream);
        case kOutMx4: return launch_layer_gemm<kOpMx4, false, true, true, kEpiMx4>(g, n_cu, stream);
        default: return launch_layer_gemm<kOpMx4, false, true, true, kEpiBf16>(g, n_cu, stream);
    }
}

}  // namespace donerf
