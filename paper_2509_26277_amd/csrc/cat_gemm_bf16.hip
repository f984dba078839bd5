// Instances of the tile kernel for bfloat16 operands.
#include "cat_gemm_kernel.h"

namespace cat {

template <int EDGE, int WM>
static cat_status launch_gate_grad(const GemmArgs& a, hipStream_t st) {
    if (a.n % 8 == 0 && !a.parts) switch (a.e.act) {
            case CAT_ACT_NONE: return launch_gemm_tiles<bf16_t, bf16_t, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_NONE>(a, st);
            case CAT_ACT_RELU: return launch_gemm_tiles<bf16_t, bf16_t, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_RELU>(a, st);
            case CAT_ACT_GELU: return launch_gemm_tiles<bf16_t, bf16_t, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_GELU>(a, st);
            case CAT_ACT_GELU_TANH: return launch_gemm_tiles<bf16_t, bf16_t, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_GELU_TANH>(a, st);
            default: return launch_gemm_tiles<bf16_t, bf16_t, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_SILU>(a, st);
        }
    return launch_gemm_tiles<bf16_t, bf16_t, kGatedGrad, EDGE, EDGE, WM>(a, st);
}
cat_status launch_gemm_bf16(GemmKind kind, bool large, const GemmArgs& a, hipStream_t st) {
    if (large) {
        if (kind == kForward) return launch_gemm_tiles<bf16_t, bf16_t, kForward, 256, 256, 64>(a, st);
        if (kind == kInputGrad) return launch_gemm_tiles<bf16_t, bf16_t, kInputGrad, 256, 256, 64>(a, st);
        if (kind == kGated) return launch_gemm_tiles<bf16_t, bf16_t, kGated, 256, 256, 64>(a, st);
        if (kind == kGatedGrad) return launch_gate_grad<256, 64>(a, st);
        return launch_gemm_tiles<bf16_t, bf16_t, kWeightGrad, 256, 256, 64>(a, st);
    }
    if (kind == kForward) return launch_gemm_tiles<bf16_t, bf16_t, kForward, 128, 128, 32>(a, st);
    if (kind == kInputGrad) return launch_gemm_tiles<bf16_t, bf16_t, kInputGrad, 128, 128, 32>(a, st);
    if (kind == kGated) return launch_gemm_tiles<bf16_t, bf16_t, kGated, 128, 128, 32>(a, st);
    if (kind == kGatedGrad) return launch_gate_grad<128, 32>(a, st);
    return launch_gemm_tiles<bf16_t, bf16_t, kWeightGrad, 128, 128, 32>(a, st);
}

}  // namespace cat
