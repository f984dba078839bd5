// Instances of the tile kernel for bfloat16 operands.
#include "cat_gemm_kernel.h"

namespace cat {

cat_status launch_gemm_bf16(GemmKind kind, bool large, const GemmArgs& a, hipStream_t st) {
    if (large) {
        if (kind == kForward) return launch_gemm_tiles<bf16_t, bf16_t, kForward, 256, 256, 64>(a, st);
        if (kind == kInputGrad) return launch_gemm_tiles<bf16_t, bf16_t, kInputGrad, 256, 256, 64>(a, st);
        if (kind == kGated) return launch_gemm_tiles<bf16_t, bf16_t, kGated, 256, 256, 64>(a, st);
        return launch_gemm_tiles<bf16_t, bf16_t, kWeightGrad, 256, 256, 64>(a, st);
    }
    if (kind == kForward) return launch_gemm_tiles<bf16_t, bf16_t, kForward, 128, 128, 32>(a, st);
    if (kind == kInputGrad) return launch_gemm_tiles<bf16_t, bf16_t, kInputGrad, 128, 128, 32>(a, st);
    if (kind == kGated) return launch_gemm_tiles<bf16_t, bf16_t, kGated, 128, 128, 32>(a, st);
    return launch_gemm_tiles<bf16_t, bf16_t, kWeightGrad, 128, 128, 32>(a, st);
}

}  // namespace cat
