// Instances of the tile kernel for operands of 8-bit integers.
#include "cat_gemm_kernel.h"

namespace cat {

template <typename T>
static cat_status launch(GemmKind kind, bool large, const GemmArgs& a, hipStream_t st) {
    if (large) {
        if (kind == kForward) return launch_gemm_tiles<int8_t, T, kForward, 256, 256, 64>(a, st);
        return launch_gemm_tiles<int8_t, T, kGated, 256, 256, 64>(a, st);
    }
    if (kind == kForward) return launch_gemm_tiles<int8_t, T, kForward, 128, 128, 32>(a, st);
    return launch_gemm_tiles<int8_t, T, kGated, 128, 128, 32>(a, st);
}
cat_status launch_gemm_i8(GemmKind kind, bool large, cat_dtype out, const GemmArgs& a, hipStream_t st) {
    return out == CAT_F32 ? launch<float>(kind, large, a, st) : launch<bf16_t>(kind, large, a, st);
}

}  // namespace cat
