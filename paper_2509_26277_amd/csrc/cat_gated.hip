// The gated feed-forward half: both projections, the activation and the product in one pass, and the gradients behind the gate
// from its checkpoints.
//
//   g = x Wg^T + bg, v = x Wv^T + bv, h = act(g) * v      w = [Wg; Wv]; 4 M F K operations; reads x, w, writes h (and codes of g, v)
//   dh = dy W2, dz = [dh v act'(g) | dh act(g)]           W2: N x F; 2 M N F; reads dy, W2, the codes, writes dz
//   db = sum over rows of dz                              from the fp32 values on their way out
//   dW2 = dy^T (act(g) * v), db2 = sum over rows of dy    2 M N F (bfloat16: twice, act(g) * v being two terms)
//
// A wave of the tile kernel works on 64 columns of the gate and the same 64 of the value, so that both meet in a lane's registers:
// neither projection, nor dh, goes to memory.
//
// The products bound them and, on top, what a tile's end reads and writes (us, bfloat16: 16384 x 2 x 4096 over 1024 212, with checkpoints 270;
// both gradients of 16384 x 4096 over 1024 203, where the products alone take 117; dW2 of the same, both terms, 233, its shares' join 13, act(g) * v
// laid out 70; float, 8192 x 1000 over 256: 52, and 38, 7, 12).
#include "cat_product.h"

namespace cat {
namespace {

// Shares of k of dh joined and the gate's gradients: a workgroup 128 columns of a share of the rows, 16 rows at a time, 16 lanes of
// 8 columns each; the sums over its rows are its row of e.col_sums.
template <typename T>
__global__ __launch_bounds__(256) void k_join_gate_grad(const float* __restrict__ parts, int splits, int64_t M, int64_t N, int64_t rows, const Epilogue e) {
    __shared__ float s[4][16][17];
    const int lane = threadIdx.x & 15, slot = threadIdx.x / 16;
    const int64_t n = (int64_t)blockIdx.x * kPackGroup + lane * 8, G = gridDim.x;
    const int64_t m0 = (int64_t)blockIdx.y * rows, m1 = m0 + rows < M ? m0 + rows : M;
    float sums[16];
#pragma unroll
    for (int i = 0; i < 16; i++) sums[i] = 0.f;
    if (n < N)
        for (int64_t m = m0 + slot; m < m1; m += 16) {
            float d[8], gate[8], value[8];
            ld_parts<T, 8>(parts + m * N, splits, M * N, n, N, d);
            ld_codes<8>(e.codes_in + m * N, n, N, e.scales_in[m * G + blockIdx.x], gate);
            ld_codes<8>(e.codes_in + (M + m) * N, n, N, e.scales_in[(M + m) * G + blockIdx.x], value);
            with_act(e.act, [&](auto which) {
                constexpr int ACT = decltype(which)::value;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float z = gate[i];
                    float a, da;
                    act_both<ACT, kFast<T>>(z, a, da);
                    gate[i] = d[i] * value[i] * da;
                    value[i] = d[i] * a;
                }
            });
            T* out = (T*)e.out + m * 2 * N;
            st_entries<T, 8>(out, n, N, gate);
            st_entries<T, 8>(out + N, n, N, value);
#pragma unroll
            for (int i = 0; i < 8; i++) sums[i] += gate[i], sums[8 + i] += value[i];
        }
    if (!e.col_sums) return;
#pragma unroll
    for (int i = 0; i < 16; i++) {  // the four slots of a wave
        sums[i] += __shfl_xor(sums[i], 16, kWave);
        sums[i] += __shfl_xor(sums[i], 32, kWave);
        if (slot % 4 == 0) s[slot / 4][lane][i] = sums[i];
    }
    __syncthreads();
    const int c = threadIdx.x / 16, i = threadIdx.x & 15;
    const int64_t at = (int64_t)blockIdx.x * kPackGroup + c * 8 + (i & 7);
    if (at < N) e.col_sums[((int64_t)blockIdx.y * 2 + (i >> 3)) * N + at] = (s[0][c][i] + s[1][c][i]) + (s[2][c][i] + s[3][c][i]);
}

Plan plan_gated(int64_t M, int64_t F, int64_t K, cat_dtype dt, bool pack) { return plan(kGated, M, F, K, M, K, 2 * F, K, entry_bytes(dt), false, pack); }
Plan plan_gate_grad(int64_t M, int64_t N, int64_t F, cat_dtype dt) { return plan(kGatedGrad, M, F, N, M, N, N, F, entry_bytes(dt), false); }
Plan plan_gate_weight(int64_t M, int64_t N, int64_t F, cat_dtype dt) {
    return plan(kWeightGrad, N, F, M, M, N, M, F, entry_bytes(dt), true, false, dt == CAT_BF16 ? 2 : 1, true);
}

cat_status check_gate(const char* who, int64_t M, const int8_t* codes, const float* scales) {
    CAT_TRY(check_ptr(who, "codes", codes, M > 0));
    return check_ptr(who, "scales", scales, M > 0);
}

}  // namespace
}  // namespace cat

using namespace cat;

extern "C" {

size_t cat_gated_linear_workspace_bytes(int64_t M, int64_t F, int64_t K, cat_dtype dt) {
    if (check_linear("cat_gated_linear_workspace_bytes", M, F, K, dt) != CAT_OK) return 0;
    const size_t a = stated(plan_gated(M - tail_rows(kGated, M, F, K, entry_bytes(dt)), F, K, dt, false)), b = stated(plan_gated(M, F, K, dt, true));
    return a > b ? a : b;
}

cat_status cat_gated_linear(const void* x, const void* w, const float* bias, int64_t M, int64_t F, int64_t K, cat_dtype dt, cat_activation act, void* y,
                            int8_t* codes, float* scales, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "cat_gated_linear";
    CAT_TRY(check_linear(who, M, F, K, dt));
    CAT_TRY(check_act(who, act));
    CAT_TRY(check_ptr(who, "x", x, M > 0));
    CAT_TRY(check_ptr(who, "w", w, true));
    CAT_TRY(check_ptr(who, "bias", bias, false));
    CAT_TRY(check_ptr(who, "y", y, M > 0));
    CAT_TRY(check_checkpoint(who, codes, scales));
    if (M > 0 && (y == x || y == w || y == bias)) return set_error(CAT_ERR_INVALID_ARG, "%s: y may not alias an input", who);
    const int64_t tail = codes ? 0 : tail_rows(kGated, M, F, K, entry_bytes(dt));  // (a checkpoint's halves are one behind the other)
    const Plan pl = plan_gated(M - tail, F, K, dt, codes != nullptr);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    if (M == 0) return CAT_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    char* ws = (char*)workspace;
    Epilogue e = {};
    e.out = y, e.bias = bias, e.codes_out = codes, e.scales_out = scales, e.act = (int)act;
    if (pl.few)
        return dt == CAT_F32 ? few_rows<float, float, true>(pl, x, K, w, K, M, F, K, e, ws, st) : few_rows<bf16_t, bf16_t, true>(pl, x, K, w, K, M, F, K, e, ws, st);
    if (tail) CAT_TRY((dt == CAT_F32 ? few_tail<float, float, true>(x, K, w, K, M, tail, F, K, e, st) : few_tail<bf16_t, bf16_t, true>(x, K, w, K, M, tail, F, K, e, st)));
    M -= tail;
    CAT_TRY(lay_out(dt, pl, x, M, K, w, nullptr, nullptr, false, 0, 2 * F, K, ws, st));
    const GemmArgs a = gemm_args(pl, entry_bytes(dt), pl.lay_q ? ws + pl.at_q : x, M, pl.lay_p ? ws + pl.at_p : w, 2 * F, M, F, K, e, ws);
    CAT_TRY(dt == CAT_F32 ? launch_gemm_f32(kGated, a, st) : launch_gemm_bf16(kGated, pl.large, a, st));
    if (!pl.joined) return CAT_OK;
    return dt == CAT_F32 ? join<float, float, kGated>(a.parts, pl.splits, M, F, e, st) : join<bf16_t, bf16_t, kGated>(a.parts, pl.splits, M, F, e, st);
}

size_t cat_gated_backward_workspace_bytes(int64_t M, int64_t N, int64_t F, cat_dtype dt) {
    if (check_linear("cat_gated_backward_workspace_bytes", M, N, F, dt) != CAT_OK) return 0;
    const size_t a = stated(plan_gate_grad(M, N, F, dt)), b = stated(plan_gate_weight(M, N, F, dt));
    return a > b ? a : b;
}

cat_status cat_gated_backward_input(const void* dy, const void* w, const int8_t* codes, const float* scales, int64_t M, int64_t N, int64_t F, cat_dtype dt,
                                    cat_activation act, void* dz, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "cat_gated_backward_input";
    CAT_TRY(check_linear(who, M, N, F, dt));
    CAT_TRY(check_act(who, act));
    CAT_TRY(check_ptr(who, "dy", dy, M > 0));
    CAT_TRY(check_ptr(who, "w", w, true));
    CAT_TRY(check_gate(who, M, codes, scales));
    CAT_TRY(check_ptr(who, "dz", dz, M > 0));
    CAT_TRY(check_ptr(who, "dbias", dbias, false));
    if (M > 0 && (dz == dy || dz == w || dz == codes || dz == scales)) return set_error(CAT_ERR_INVALID_ARG, "%s: dz may not alias an input", who);
    const Plan pl = plan_gate_grad(M, N, F, dt);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    hipStream_t st = (hipStream_t)hip_stream;
    char* ws = (char*)workspace;
    if (M == 0) return dbias ? launch_fill_zero(dbias, (size_t)2 * F * 4, st) : CAT_OK;
    Epilogue e = {};
    e.out = dz, e.codes_in = codes, e.scales_in = scales, e.act = (int)act, e.col_sums = dbias ? (float*)(ws + pl.at_sums) : nullptr;
    CAT_TRY(lay_out(dt, pl, dy, M, N, w, nullptr, nullptr, false, 0, N, F, ws, st));
    const GemmArgs a = gemm_args(pl, entry_bytes(dt), pl.lay_q ? ws + pl.at_q : dy, M, pl.lay_p ? ws + pl.at_p : w, N, M, F, N, e, ws);
    CAT_TRY(dt == CAT_F32 ? launch_gate_grad_f32(a, st) : launch_gate_grad_bf16(pl.large, a, st));
    if (pl.joined) {
        const dim3 grid((unsigned)((F + kPackGroup - 1) / kPackGroup), (unsigned)pl.sum_parts);
        if (dt == CAT_F32)
            hipLaunchKernelGGL(k_join_gate_grad<float>, grid, dim3(256), 0, st, (const float*)a.parts, pl.splits, M, F, pl.sum_rows, e);
        else
            hipLaunchKernelGGL(k_join_gate_grad<bf16_t>, grid, dim3(256), 0, st, (const float*)a.parts, pl.splits, M, F, pl.sum_rows, e);
        CAT_LAUNCH_CHECK("k_join_gate_grad");
    }
    return dbias ? launch_sum_parts(e.col_sums, pl.sum_parts, 2 * F, 2 * F, dbias, nullptr, st) : CAT_OK;
}

cat_status cat_gated_backward_weight(const void* dy, const int8_t* codes, const float* scales, int64_t M, int64_t N, int64_t F, cat_dtype dt,
                                     cat_activation act, void* dw, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "cat_gated_backward_weight";
    CAT_TRY(check_linear(who, M, N, F, dt));
    CAT_TRY(check_act(who, act));
    CAT_TRY(check_ptr(who, "dy", dy, M > 0));
    CAT_TRY(check_gate(who, M, codes, scales));
    CAT_TRY(check_ptr(who, "dw", dw, true));
    CAT_TRY(check_ptr(who, "dbias", dbias, false));
    if (dw == dy || dw == codes || dw == scales) return set_error(CAT_ERR_INVALID_ARG, "%s: dw may not alias an input", who);
    const Plan pl = plan_gate_weight(M, N, F, dt);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    return weight_gradient(pl, dy, nullptr, codes, scales, true, M, N, F, dt, (int)act, dw, dbias, (char*)workspace, (hipStream_t)hip_stream);
}

}  // extern "C"
