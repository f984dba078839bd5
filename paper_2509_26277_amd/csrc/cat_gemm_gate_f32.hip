// Instances of the tile kernel for the gradients of a gate, float operands.
#include "cat_gemm_kernel.h"

namespace cat {

cat_status launch_gate_grad_f32(const GemmArgs& a, hipStream_t st) { return launch_gate_grad<float, 128, 32>(a, st); }

}  // namespace cat
