// Rows to 8-bit integers with a scale a row, for the products of 8-bit integers; as they are, or through layer norm.  Kernels,
// launchers and entry points.
//
//   h = x, or h = (x - mu) rstd w + b;  a = max |h|, scale = a / 127, code = h * (127 / a) rounded to the nearest integer
//
// One pass over memory and bound by it, 3 bytes an entry of bfloat16 rows, 5 of float ones: a row is read once and stays in
// registers for its statistics, its largest magnitude and its codes, the next one requested ahead, as in layer norm.  Rows of more
// than 8192 entries have a workgroup each that reads the row again for every use.
//
// Measured (us, inputs from memory): 65536 x 1024 bfloat16 33 (6.1 TB/s), fp32 63 (5.3); through the norm 49 and 66: the bfloat16 norm is bound
// by its instructions.  One row of 2048: 2.7.
#include "cat_rows.h"

namespace cat {
namespace {

// The largest magnitude over the TPR threads of a row; as row_sums.
template <int TPR>
__device__ __forceinline__ uint32_t row_max(uint32_t a, float (*slots)[2][8], int& slot) {
    a = lanes_max<(TPR < kWave ? TPR : kWave)>(a);
    if constexpr (TPR > kWave) {
        static_assert(TPR == 256, "");
        if ((threadIdx.x & (kWave - 1)) == 0) slots[slot][0][threadIdx.x / kWave] = __uint_as_float(a);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++) a = mag_max(a, slots[slot][0][i]);
        slot ^= 1;
    }
    return a;
}

template <typename T, int TPR, int VPL, bool NORM>
__global__ __launch_bounds__(kThreads<TPR>) void k_rows8(const T* __restrict__ x, int64_t N, int64_t D, const float* __restrict__ weight,
                                                         const float* __restrict__ bias, float eps, int8_t* __restrict__ codes,
                                                         int64_t ld, float* __restrict__ scales) {
    constexpr int V = kVec<T>, RPB = kThreads<TPR> / TPR;
    __shared__ float slots[2][2][8];
    int slot = 0;
    const int sub = threadIdx.x % TPR;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t own_row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Part<T, false> next[VPL];
#pragma unroll
    for (int k = 0; k < VPL; k++) next[k].load(x, nullptr, nullptr, own_row < N ? own_row : N - 1, ((int64_t)k * TPR + sub) * V, D, 0);
    float w[NORM ? VPL : 1][V], b[NORM ? VPL : 1][V];
    if constexpr (NORM) {
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            ld_params<V>(weight, ((int64_t)k * TPR + sub) * V, D, 1.f, w[k]);
            ld_params<V>(bias, ((int64_t)k * TPR + sub) * V, D, 0.f, b[k]);
        }
    }
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < N; r0 += stride, own_row += stride) {
        const bool mine = own_row < N;
        const int64_t row = mine ? own_row : N - 1;
        Part<T, false> v[VPL];
#pragma unroll
        for (int k = 0; k < VPL; k++) v[k] = next[k];
        if (r0 + stride < N) {
            const int64_t r = own_row + stride < N ? own_row + stride : N - 1;
#pragma unroll
            for (int k = 0; k < VPL; k++) next[k].load(x, nullptr, nullptr, r, ((int64_t)k * TPR + sub) * V, D, 0);
        }
        float h[VPL][V];
#pragma unroll
        for (int k = 0; k < VPL; k++)
#pragma unroll
            for (int e = 0; e < V; e++) h[k][e] = v[k].at(e);
        if constexpr (NORM) {
            float s[1] = {0.f};
#pragma unroll
            for (int k = 0; k < VPL; k++)
#pragma unroll
                for (int e = 0; e < V; e++) s[0] += h[k][e];
            row_sums<TPR>(s, slots, slot);
            const float mu = s[0] / (float)D;
            float q[1] = {0.f};
            // (one comparison a group: those of eight entries were a third of the instructions of a row's statistics)
#pragma unroll
            for (int k = 0; k < VPL; k++) {
                const int64_t j = ((int64_t)k * TPR + sub) * V;
                const int n = j + V <= D ? V : j < D ? (int)(D - j) : 0;
                if (n == V) {
#pragma unroll
                    for (int e = 0; e < V; e++) h[k][e] -= mu, q[0] = fmaf(h[k][e], h[k][e], q[0]);
                } else {
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        h[k][e] = e < n ? h[k][e] - mu : 0.f;
                        q[0] = fmaf(h[k][e], h[k][e], q[0]);
                    }
                }
            }
            row_sums<TPR>(q, slots, slot);
            const float rs = 1.f / sqrtf(q[0] / (float)D + eps);
            // (behind the row's end: zeros; with rs an infinity a NaN, as the row has them then)
#pragma unroll
            for (int k = 0; k < VPL; k++)
#pragma unroll
                for (int e = 0; e < V; e++) h[k][e] = fmaf(h[k][e] * rs, w[k][e], b[k][e]);
        }
        uint32_t a = 0;
#pragma unroll
        for (int k = 0; k < VPL; k++)
#pragma unroll
            for (int e = 0; e < V; e++) a = mag_max(a, h[k][e]);
        const PackScale s = pack_scale(row_max<TPR>(a, slots, slot));
        if (!mine) continue;
        if (sub == 0) scales[row] = s.step;
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            if (j < D) st_codes<V>(codes + row * ld, j, D, h[k], s.up);
        }
    }
}

template <typename T, bool NORM>
__global__ __launch_bounds__(kNormThreads) void k_rows8_long(const T* __restrict__ x, int64_t N, int64_t D, const float* __restrict__ weight,
                                                             const float* __restrict__ bias, float eps, int8_t* __restrict__ codes,
                                                             int64_t ld, float* __restrict__ scales) {
    constexpr int V = kVec<T>;
    __shared__ float slots[2][2][8];
    int slot = 0;
    for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
        const T* xr = x + row * D;
        float mu = 0.f, rs = 1.f;
        if constexpr (NORM) {
            float s[1] = {0.f};
            for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
                float v[V];
                ld_group_to(xr, j, D, v);
#pragma unroll
                for (int e = 0; e < V; e++) s[0] += v[e];
            }
            row_sums<kNormThreads>(s, slots, slot);
            mu = s[0] / (float)D;
            float q[1] = {0.f};
            for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
                float v[V];
                ld_group_to(xr, j, D, v);
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (j + e < D) q[0] = fmaf(v[e] - mu, v[e] - mu, q[0]);
            }
            row_sums<kNormThreads>(q, slots, slot);
            rs = 1.f / sqrtf(q[0] / (float)D + eps);
        }
        const auto values = [&](int64_t j, float (&v)[V]) {
            ld_group_to(xr, j, D, v);
            if constexpr (NORM) {
                float w[V], b[V];
                ld_params<V>(weight, j, D, 1.f, w);
                ld_params<V>(bias, j, D, 0.f, b);
#pragma unroll
                for (int e = 0; e < V; e++) v[e] = fmaf((v[e] - mu) * rs, w[e], b[e]);
            }
        };
        uint32_t a = 0;
        for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
            float v[V];
            values(j, v);
#pragma unroll
            for (int e = 0; e < V; e++)
                if (j + e < D) a = mag_max(a, v[e]);
        }
        const PackScale s = pack_scale(row_max<kNormThreads>(a, slots, slot));
        if (threadIdx.x == 0) scales[row] = s.step;
        for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
            float v[V];
            values(j, v);
            st_codes<V>(codes + row * ld, j, D, v, s.up);
        }
    }
}

// How many threads share a row: four 16-byte groups each (three, where those are enough), so that a wave has up to 4 KB of rows under
// way and few lanes to reduce over; 8 threads of the shortest rows, and more than a wave's from 257 groups on, as in layer norm.
// (us, 65536 x 512 bf16 through the norm: 36 with a wave a row and a group a lane, 26 so; 65536 x 512 fp32 47 and 26.)
template <typename T>
NormShape rows8_shape(int64_t D) {
    const int64_t n = (D + kVec<T> - 1) / kVec<T>;
    if (n > 256) return norm_shape<T, false>(D);
    const int tpr = n <= 32 ? 8 : n <= 64 ? 16 : n <= 128 ? 32 : 64;
    return {tpr, (int)((n + tpr - 1) / tpr)};
}
constexpr int kRows8Groups = 1024;  // workgroups; further rows by stride
template <typename T, bool NORM>
cat_status launch_rows8(const T* x, int64_t N, int64_t D, const float* weight, const float* bias, float eps, int8_t* codes, int64_t ld, float* scales, hipStream_t st) {
    const NormShape s = rows8_shape<T>(D);
    const int64_t rpb = s.tpr && s.tpr < kNormThreads ? kNormThreads / s.tpr : 1, blocks = (N + rpb - 1) / rpb;
    const dim3 grid((unsigned)(blocks < kRows8Groups ? blocks : kRows8Groups));
#define CAT_X(TPR, VPL)               \
    if (s.tpr == TPR && s.vpl == VPL) \
        hipLaunchKernelGGL((k_rows8<T, TPR, VPL, NORM>), grid, dim3(kThreads<TPR>), 0, st, x, N, D, weight, bias, eps, codes, ld, scales);
    CAT_X(8, 1) CAT_X(8, 2) CAT_X(8, 3) CAT_X(8, 4) CAT_X(16, 3) CAT_X(16, 4) CAT_X(32, 3) CAT_X(32, 4) CAT_X(64, 3) CAT_X(64, 4) CAT_X(256, 4)
    if constexpr (sizeof(T) == 4) {
        CAT_X(64, 8) CAT_X(256, 8)
    } else {
        CAT_X(256, 2)
    }
#undef CAT_X
    if (!s.tpr) hipLaunchKernelGGL((k_rows8_long<T, NORM>), grid, dim3(kNormThreads), 0, st, x, N, D, weight, bias, eps, codes, ld, scales);
    CAT_LAUNCH_CHECK("k_rows8");
    return CAT_OK;
}

cat_status check_rows8(const char* who, const void* x, int64_t N, int64_t D, cat_dtype dt, const int8_t* codes, int64_t ld, const float* scales) {
    CAT_TRY(check_rows(who, N, D, dt));
    if (ld < D || ld >= (1ll << 31)) return set_error(CAT_ERR_INVALID_ARG, "%s: rows of %lld codes lie %lld apart", who, (long long)D, (long long)ld);
    CAT_TRY(check_ptr(who, "x", x, N > 0));
    CAT_TRY(check_ptr(who, "codes", codes, N > 0));
    CAT_TRY(check_ptr(who, "scales", scales, N > 0));
    if (N > 0 && (codes == x || scales == x)) return set_error(CAT_ERR_INVALID_ARG, "%s: codes and scales may not alias x", who);
    return CAT_OK;
}

}  // namespace
}  // namespace cat

using namespace cat;

extern "C" {

cat_status cat_quantize_rows(const void* x, int64_t N, int64_t D, cat_dtype dt, int8_t* codes, int64_t ld, float* scales, void* hip_stream) {
    CAT_TRY(check_rows8("cat_quantize_rows", x, N, D, dt, codes, ld, scales));
    if (N == 0) return CAT_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    return dt == CAT_F32 ? launch_rows8<float, false>((const float*)x, N, D, nullptr, nullptr, 0.f, codes, ld, scales, st)
                         : launch_rows8<bf16_t, false>((const bf16_t*)x, N, D, nullptr, nullptr, 0.f, codes, ld, scales, st);
}

cat_status cat_layer_norm_quantize(const void* x, int64_t N, int64_t D, cat_dtype dt, const float* weight, const float* bias, float eps, int8_t* codes,
                                   int64_t ld, float* scales, void* hip_stream) {
    const char* who = "cat_layer_norm_quantize";
    CAT_TRY(check_rows8(who, x, N, D, dt, codes, ld, scales));
    CAT_TRY(check_ptr(who, "weight", weight, false));
    CAT_TRY(check_ptr(who, "bias", bias, false));
    if (!(eps >= 0.f) || isinf(eps)) return set_error(CAT_ERR_INVALID_ARG, "%s: eps = %g is not finite and >= 0", who, (double)eps);
    if (N == 0) return CAT_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    return dt == CAT_F32 ? launch_rows8<float, true>((const float*)x, N, D, weight, bias, eps, codes, ld, scales, st)
                         : launch_rows8<bf16_t, true>((const bf16_t*)x, N, D, weight, bias, eps, codes, ld, scales, st);
}

}  // extern "C"
