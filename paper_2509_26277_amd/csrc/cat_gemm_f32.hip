// Instances of the tile kernel for float operands.
#include "cat_gemm_kernel.h"

namespace cat {

cat_status launch_gemm_f32(GemmKind kind, const GemmArgs& a, hipStream_t st) {
    if (kind == kForward) return launch_gemm_tiles<float, float, kForward, 128, 128, 32>(a, st);
    if (kind == kInputGrad) return launch_gemm_tiles<float, float, kInputGrad, 128, 128, 32>(a, st);
    if (kind == kGated) return launch_gemm_tiles<float, float, kGated, 128, 128, 32>(a, st);
    return launch_gemm_tiles<float, float, kWeightGrad, 128, 128, 32>(a, st);
}

}  // namespace cat
