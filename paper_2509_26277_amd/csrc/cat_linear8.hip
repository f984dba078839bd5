// Products of 8-bit integers with a scale for every row of either operand, and their gated form.
//
//   z = (sum_k x_mk w_nk) * xs_m * ws_n + b_n        the sum exact, in 32-bit integers; what follows in fp32
//   y = act(z) + res                                 2 M N K operations; reads x, w, res, writes y
//   y = act(z_gate) * z_value                        4 M F K
//
// The tile kernel and the one for few rows are those of the other products: 16 integers fill the registers of 8 bfloat16 entries and
// a matrix instruction takes the same time over twice as many, so a step of 128 bytes is 128 entries of k.
//
// With many rows the matrix cores bound it and, where k is short, the tiles' ends (us: 16384 x 8192 over 2048 to bfloat16 235, with GELU 267;
// 65536 x 2048 over 512 with GELU 135; 65536 x 1000 over 512 to float 68; gated 16384 x 2 x 4096 over 2048 224); with few the bytes of w
// (8192 x 2048, one row 5.8; gated 2 x 8192 x 2048 8.5).
#include "cat_product.h"

namespace cat {
namespace {

constexpr int64_t kMaxK8 = 131071;  // the largest magnitudes, 128 * 128 each, still sum up to less than 2^31

// 8-bit integers: bytes, 16 a thread
__global__ __launch_bounds__(256) void k_lay_out8(const Layout<int8_t> first, const Layout<int8_t> second) {
    const bool other = blockIdx.x >= first.blocks;
    const Layout<int8_t>& a = other ? second : first;
    const int64_t block = other ? blockIdx.x - first.blocks : blockIdx.x;
    const int64_t per = a.ld / 16, n = a.rows * per;
    for (int64_t t = block * 256 + threadIdx.x; t < n; t += (int64_t)a.blocks * 256) {
        const int64_t row = n < (1ll << 32) ? (uint32_t)t / (uint32_t)per : t / per, j = (t - row * per) * 16;
        *(f32x4*)(a.dst + row * a.ld + j) = few_load(a.src + row * a.from, j, a.cols);
    }
}

// ld: from a row of codes to the next
cat_status check_ld(const char* who, const char* name, int64_t ld, int64_t K) {
    if (ld == K || (ld > K && ld % 16 == 0 && ld <= kGemmMaxRowBytes)) return CAT_OK;
    return set_error(CAT_ERR_INVALID_ARG, "%s: rows of %s of %lld entries lie %lld apart: as many, or a larger multiple of 16", who, name, (long long)K, (long long)ld);
}
cat_status check8(const char* who, int64_t M, int64_t N, int64_t K, cat_dtype dt, int act) {
    CAT_TRY(check_linear(who, M, N, 1, dt));
    CAT_TRY(check_rows(who, M, K, dt));
    CAT_TRY(check_act(who, act));
    if (K > kMaxK8)
        return set_error(CAT_ERR_UNSUPPORTED, "%s: rows of %lld entries: sums of 8-bit products stay in 32 bits up to %lld", who, (long long)K, (long long)kMaxK8);
    return CAT_OK;
}
int64_t tail8(bool gated, int64_t M, int64_t N, int64_t K) { return tail_rows(gated ? kGated : kForward, M, N, K, 1); }
// Of the rows before the tail.  Rows of x that start on 16-byte boundaries are used where they are, whatever their last 16 bytes hold
// behind K: w's hold zeros there, being laid out anew unless K is a multiple of 16.
Plan plan8(bool gated, int64_t M, int64_t N, int64_t K, int64_t ldx, int64_t ldw) {
    return plan(gated ? kGated : kForward, M, N, K, M, ldx, gated ? 2 * N : N, K % 16 ? K : ldw, 1, false);
}
// (whatever the result's type: of bfloat16, rows of out may be the longest)
size_t workspace8(const char* who, bool gated, int64_t M, int64_t N, int64_t K) {
    if (check8(who, M, N, K, CAT_BF16, 0) != CAT_OK) return 0;
    return stated(plan8(gated, M - tail8(gated, M, N, K), N, K, K, K));
}

template <typename T, bool GATED>
cat_status product8(const Plan& pl, const int8_t* x, int64_t ldx, const int8_t* w, int64_t ldw, int64_t M, int64_t N, int64_t K, const Epilogue& e, char* ws,
                    hipStream_t st) {
    constexpr GemmKind kind = GATED ? kGated : kForward;
    if (pl.few) return few_rows<int8_t, T, GATED>(pl, x, ldx, w, ldw, M, N, K, e, ws, st);
    const int64_t rows_w = GATED ? 2 * N : N;
    Layout<int8_t> lq = layout_of<int8_t>(x, nullptr, nullptr, M, K, pl.ldq, ws + pl.at_q), lp = layout_of<int8_t>(w, nullptr, nullptr, rows_w, K, pl.ldp, ws + pl.at_p);
    lq.from = (int)ldx, lp.from = (int)ldw;
    if (pl.lay_p) {  // (and x with it, or not)
        const Layout<int8_t> none = {};
        hipLaunchKernelGGL(k_lay_out8, dim3(lp.blocks + (pl.lay_q ? lq.blocks : 0)), dim3(256), 0, st, lp, pl.lay_q ? lq : none);
        CAT_LAUNCH_CHECK("k_lay_out8");
    }
    GemmArgs a = gemm_args(pl, 1, pl.lay_q ? ws + pl.at_q : (const char*)x, M, pl.lay_p ? ws + pl.at_p : (const char*)w, rows_w, M, N, K, e, ws);
    if (!pl.lay_q) a.q_bytes = (M - 1) * pl.ldq + whole(K, 1);
    if (!pl.lay_p) a.p_bytes = (rows_w - 1) * pl.ldp + K;
    CAT_TRY(launch_gemm_i8(kind, pl.large, sizeof(T) == 4 ? CAT_F32 : CAT_BF16, a, st));
    return pl.joined ? join<int8_t, T, kind>(a.parts, pl.splits, M, N, e, st) : CAT_OK;
}
template <bool GATED>
cat_status product8(const char* who, const int8_t* x, int64_t ldx, const float* x_scales, const int8_t* w, int64_t ldw, const float* w_scales,
                    const float* bias, const void* residual, int64_t M, int64_t N, int64_t K, cat_dtype dt, int act, void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    CAT_TRY(check8(who, M, N, K, dt, act));
    CAT_TRY(check_ld(who, "x", ldx, K));
    CAT_TRY(check_ld(who, "w", ldw, K));
    CAT_TRY(check_ptr(who, "x", x, M > 0));
    CAT_TRY(check_ptr(who, "x_scales", x_scales, M > 0));
    CAT_TRY(check_ptr(who, "w", w, true));
    CAT_TRY(check_ptr(who, "w_scales", w_scales, true));
    CAT_TRY(check_ptr(who, "bias", bias, false));
    CAT_TRY(check_ptr(who, "residual", residual, false));
    CAT_TRY(check_ptr(who, "y", y, M > 0));
    if (M > 0 && (y == x || y == w || y == residual || y == x_scales || y == w_scales || y == bias))
        return set_error(CAT_ERR_INVALID_ARG, "%s: y may not alias an input", who);
    const int64_t tail = tail8(GATED, M, N, K);
    const Plan pl = plan8(GATED, M - tail, N, K, ldx, ldw);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    if (M == 0) return CAT_OK;
    Epilogue e = {};
    e.out = y, e.bias = bias, e.residual = residual, e.act = act, e.row_scales = x_scales, e.col_scales = w_scales;
    hipStream_t st = (hipStream_t)hip_stream;
    if (tail) CAT_TRY((dt == CAT_F32 ? few_tail<int8_t, float, GATED>(x, ldx, w, ldw, M, tail, N, K, e, st) : few_tail<int8_t, bf16_t, GATED>(x, ldx, w, ldw, M, tail, N, K, e, st)));
    return dt == CAT_F32 ? product8<float, GATED>(pl, x, ldx, w, ldw, M - tail, N, K, e, (char*)workspace, st)
                         : product8<bf16_t, GATED>(pl, x, ldx, w, ldw, M - tail, N, K, e, (char*)workspace, st);
}

}  // namespace
}  // namespace cat

using namespace cat;

extern "C" {

size_t cat_linear8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    return workspace8("cat_linear8_workspace_bytes", false, M, N, K);
}
cat_status cat_linear8(const int8_t* x, int64_t ldx, const float* x_scales, const int8_t* w, int64_t ldw, const float* w_scales, const float* bias, const void* residual, int64_t M,
                       int64_t N, int64_t K, cat_dtype dt, cat_activation act, void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    return product8<false>("cat_linear8", x, ldx, x_scales, w, ldw, w_scales, bias, residual, M, N, K, dt, (int)act, y, workspace, workspace_bytes, hip_stream);
}

size_t cat_gated_linear8_workspace_bytes(int64_t M, int64_t F, int64_t K) {
    return workspace8("cat_gated_linear8_workspace_bytes", true, M, F, K);
}
cat_status cat_gated_linear8(const int8_t* x, int64_t ldx, const float* x_scales, const int8_t* w, int64_t ldw, const float* w_scales, const float* bias, int64_t M, int64_t F,
                             int64_t K, cat_dtype dt, cat_activation act, void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    return product8<true>("cat_gated_linear8", x, ldx, x_scales, w, ldw, w_scales, bias, nullptr, M, F, K, dt, (int)act, y, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
