// Instances of the tile kernel for the gradients of a gate, bfloat16 operands.
#include "cat_gemm_kernel.h"

namespace cat {

cat_status launch_gate_grad_bf16(bool large, const GemmArgs& a, hipStream_t st) {
    return large ? launch_gate_grad<bf16_t, 256, 64>(a, st) : launch_gate_grad<bf16_t, 128, 32>(a, st);
}

}  // namespace cat
