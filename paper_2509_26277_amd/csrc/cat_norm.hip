// Layer norm of a row, forward (from rows, or again from their checkpoint) and backward, with the sums over rows that the
// gradients of its parameters are.  Kernels, launchers and entry points.
//
//   forward    mu = mean x, v = mean (x - mu)^2, rstd = 1 / sqrt(v + eps), y = (x - mu) rstd w + b
//   backward   xhat = (x - mu) rstd, g = dy w:  dx = rstd (g - mean g - xhat mean(g xhat)) [+ gradient over the residual]
//              dw = sum_rows dy xhat, db = sum_rows dy
//
// All of it is bound by memory: a row is read once, stays in registers for both of its statistics (the variance is that
// of the centred entries, not a difference of large sums) and for the result.  TPR threads share a row, each with VPL
// 16-byte groups of it: 8 lanes for the shortest rows (8 rows a wave), a wave up to four groups a lane, a workgroup of
// four waves (sums over LDS) up to 8192 entries, and beyond that a workgroup that reads the row again for every use.
#include "cat_block.h"

namespace cat {
namespace {

constexpr int kNormThreads = 256;
constexpr int64_t kNormMaxBlocks = 1 << 22;  // further rows by stride

// the sum over the TPR threads of a row (TPR = 256: the workgroup; `slot` alternates, so that one barrier a sum is enough)
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float (*slots)[4], int& slot) {
    if constexpr (TPR <= kWave) {
        return lanes_sum<TPR>(v);
    } else {
        v = lanes_sum<kWave>(v);
        if ((threadIdx.x & (kWave - 1)) == 0) slots[slot][threadIdx.x / kWave] = v;
        __syncthreads();
        v = (slots[slot][0] + slots[slot][1]) + (slots[slot][2] + slots[slot][3]);
        slot = slot == 2 ? 0 : slot + 1;
        return v;
    }
}

// ---- forward ----
// PACK: also the checkpoint of x.  FROM8: x is a checkpoint, and mean and rstd are given.
template <typename T, int TPR, int VPL, bool PACK, bool FROM8>
__global__ __launch_bounds__(kNormThreads) void k_norm(const T* __restrict__ x, int64_t N, int64_t D, const float* __restrict__ weight,
                                                       const float* __restrict__ bias, float eps, T* __restrict__ y, float* __restrict__ mean,
                                                       float* __restrict__ rstd, int8_t* __restrict__ codes, float* __restrict__ scales) {
    constexpr int V = kVec<T>, RPB = kNormThreads / TPR, GL = kPackGroup / V;  // GL: neighbouring lanes that share a scale
    __shared__ float slots[3][4];
    int slot = 0;
    const int sub = threadIdx.x % TPR;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < N; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t own_row = r0 + threadIdx.x / TPR;
        const bool mine = own_row < N;
        const int64_t row = mine ? own_row : N - 1;
        float v[VPL][V];
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            if constexpr (FROM8)
                ld_codes<V>(codes + row * D, j, D, j < D ? scales[row * G + j / kPackGroup] : 0.f, v[k]);
            else
                ld_group_to(x + row * D, j, D, v[k]);
        }
        if constexpr (PACK) {
#pragma unroll
            for (int k = 0; k < VPL; k++) {
                const int64_t j = ((int64_t)k * TPR + sub) * V;
                float a = 0.f;
#pragma unroll
                for (int e = 0; e < V; e++) a = max_nan(a, fabsf(v[k][e]));
                a = lanes_max<(TPR < GL ? TPR : GL)>(a);
                const PackScale s = pack_scale(a);
                if (mine && j < D) {
                    st_codes<V>(codes + row * D, j, D, v[k], s.up);
                    if (j % kPackGroup == 0) scales[row * G + j / kPackGroup] = s.step;
                }
            }
        }
        float mu, rs;
        if constexpr (FROM8) {
            mu = mean[row], rs = rstd[row];
        } else {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < VPL; k++)
#pragma unroll
                for (int e = 0; e < V; e++) s += v[k][e];
            mu = row_sum<TPR>(s, slots, slot) / (float)D;
            float q = 0.f;
#pragma unroll
            for (int k = 0; k < VPL; k++) {
                const int64_t j = ((int64_t)k * TPR + sub) * V;
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const float c = v[k][e] - mu;
                    if (j + e < D) q = fmaf(c, c, q);
                }
            }
            rs = 1.f / sqrtf(row_sum<TPR>(q, slots, slot) / (float)D + eps);
            if (mine && sub == 0) {
                if (mean) mean[row] = mu;
                if (rstd) rstd[row] = rs;
            }
        }
        if (!mine) continue;
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            if (j >= D) continue;
            float w[V], b[V], o[V];
            ld_params<V>(weight, j, D, 1.f, w);
            ld_params<V>(bias, j, D, 0.f, b);
#pragma unroll
            for (int e = 0; e < V; e++) o[e] = fmaf((v[k][e] - mu) * rs, w[e], b[e]);
            st_group_to(y + row * D, j, D, o);
        }
    }
}

// rows of more than 8192 entries: a workgroup each, the row read again (from the caches) for every use
template <typename T, bool FROM8>
__global__ __launch_bounds__(kNormThreads) void k_norm_long(const T* __restrict__ x, int64_t N, int64_t D, const float* __restrict__ weight,
                                                            const float* __restrict__ bias, float eps, T* __restrict__ y,
                                                            float* __restrict__ mean, float* __restrict__ rstd,
                                                            const int8_t* __restrict__ codes, const float* __restrict__ scales) {
    constexpr int V = kVec<T>;
    __shared__ float slots[3][4];
    int slot = 0;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
        const T* xr = x + row * D;
        auto load = [&](int64_t j, float (&v)[V]) {
            if constexpr (FROM8)
                ld_codes<V>(codes + row * D, j, D, scales[row * G + j / kPackGroup], v);
            else
                ld_group_to(xr, j, D, v);
        };
        float mu, rs;
        if constexpr (FROM8) {
            mu = mean[row], rs = rstd[row];
        } else {
            float s = 0.f, q = 0.f;
            for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
                float v[V];
                load(j, v);
#pragma unroll
                for (int e = 0; e < V; e++) s += v[e];
            }
            mu = row_sum<kNormThreads>(s, slots, slot) / (float)D;
            for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
                float v[V];
                load(j, v);
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (j + e < D) q = fmaf(v[e] - mu, v[e] - mu, q);
            }
            rs = 1.f / sqrtf(row_sum<kNormThreads>(q, slots, slot) / (float)D + eps);
            if (threadIdx.x == 0) {
                if (mean) mean[row] = mu;
                if (rstd) rstd[row] = rs;
            }
        }
        for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
            float v[V], w[V], b[V];
            load(j, v);
            ld_params<V>(weight, j, D, 1.f, w);
            ld_params<V>(bias, j, D, 0.f, b);
#pragma unroll
            for (int e = 0; e < V; e++) v[e] = fmaf((v[e] - mu) * rs, w[e], b[e]);
            st_group_to(y + row * D, j, D, v);
        }
    }
}

// ---- backward ----
// A workgroup goes through its rows by stride and keeps its threads' channels of dw and db in registers; at its end the
// rows' slots (RPB of them share the channels) are added in LDS in a fixed order and written as the workgroup's part, which
// k_norm_params adds up: no atomics, the same bits on every run.
template <typename T, int TPR, int VPL, bool FROM8>
__global__ __launch_bounds__(kNormThreads) void k_norm_backward(const T* __restrict__ dy, const T* __restrict__ x,
                                                                const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                                const float* __restrict__ mean, const float* __restrict__ rstd, int64_t N,
                                                                int64_t D, const float* __restrict__ weight, const T* __restrict__ radd,
                                                                T* __restrict__ dx, float* __restrict__ parts) {
    constexpr int V = kVec<T>, RPB = kNormThreads / TPR;
    __shared__ float slots[3][4];
    __shared__ float sums[RPB > 1 ? kNormThreads * V : 1];
    int slot = 0;
    const int sub = threadIdx.x % TPR;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    const float inv = 1.f / (float)D;
    float aw[VPL][V], ab[VPL][V], w[VPL][V];
#pragma unroll
    for (int k = 0; k < VPL; k++) {
        ld_params<V>(weight, ((int64_t)k * TPR + sub) * V, D, 1.f, w[k]);
#pragma unroll
        for (int e = 0; e < V; e++) aw[k][e] = ab[k][e] = 0.f;
    }
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < N; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t own_row = r0 + threadIdx.x / TPR;
        const bool mine = own_row < N;
        const int64_t row = mine ? own_row : N - 1;
        const float mu = mean[row], rs = rstd[row];
        float h[VPL][V], g[VPL][V];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            if constexpr (FROM8)
                ld_codes<V>(codes + row * D, j, D, j < D ? scales[row * G + j / kPackGroup] : 0.f, h[k]);
            else
                ld_group_to(x + row * D, j, D, h[k]);
            ld_group_to(dy + row * D, j, D, g[k]);  // (zero behind the row's end, so that xhat there does not count)
        }
#pragma unroll
        for (int k = 0; k < VPL; k++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                h[k][e] = (h[k][e] - mu) * rs;
                const float d = mine ? g[k][e] : 0.f;
                ab[k][e] += d;
                aw[k][e] = fmaf(d, mine ? h[k][e] : 0.f, aw[k][e]);
                g[k][e] *= w[k][e];
                s1 += g[k][e];
                s2 = fmaf(g[k][e], h[k][e], s2);
            }
        s1 = row_sum<TPR>(s1, slots, slot) * inv;
        s2 = row_sum<TPR>(s2, slots, slot) * inv;
        if (!mine) continue;
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            if (j >= D) continue;
            float o[V];
            if (radd)
                ld_group_to(radd + row * D, j, D, o);
            else
#pragma unroll
                for (int e = 0; e < V; e++) o[e] = 0.f;
#pragma unroll
            for (int e = 0; e < V; e++) o[e] = fmaf(rs, g[k][e] - s1 - h[k][e] * s2, o[e]);
            st_group_to(dx + row * D, j, D, o);
        }
    }
    if (!parts) return;
    // parts: gridDim.x x 2 x D
    float* pw = parts + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int q = 0; q < 2; q++) {
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            float(&a)[V] = q == 0 ? aw[k] : ab[k];
            if constexpr (RPB > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < V; e++) sums[e * kNormThreads + threadIdx.x] = a[e];
                __syncthreads();
                if (threadIdx.x < TPR) {
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        float t = 0.f;
                        for (int r = 0; r < RPB; r++) t += sums[e * kNormThreads + r * TPR + threadIdx.x];
                        if (j + e < D) pw[q * D + j + e] = t;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (j + e < D) pw[q * D + j + e] = a[e];
            }
        }
    }
}

// rows of more than 8192 entries: dx by a workgroup a row, the sums over rows by k_norm_columns
template <typename T, bool FROM8>
__global__ __launch_bounds__(kNormThreads) void k_norm_backward_long(const T* __restrict__ dy, const T* __restrict__ x,
                                                                     const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                                     const float* __restrict__ mean, const float* __restrict__ rstd, int64_t N,
                                                                     int64_t D, const float* __restrict__ weight, const T* __restrict__ radd,
                                                                     T* __restrict__ dx) {
    constexpr int V = kVec<T>;
    __shared__ float slots[3][4];
    int slot = 0;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
        const float mu = mean[row], rs = rstd[row];
        float s1 = 0.f, s2 = 0.f;
        auto load = [&](int64_t j, float (&h)[V], float (&g)[V]) {
            float w[V];
            if constexpr (FROM8)
                ld_codes<V>(codes + row * D, j, D, scales[row * G + j / kPackGroup], h);
            else
                ld_group_to(x + row * D, j, D, h);
            ld_group_to(dy + row * D, j, D, g);
            ld_params<V>(weight, j, D, 1.f, w);
#pragma unroll
            for (int e = 0; e < V; e++) h[e] = (h[e] - mu) * rs, g[e] *= w[e];
        };
        for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
            float h[V], g[V];
            load(j, h, g);
#pragma unroll
            for (int e = 0; e < V; e++) s1 += g[e], s2 = fmaf(g[e], h[e], s2);
        }
        s1 = row_sum<kNormThreads>(s1, slots, slot) / (float)D;
        s2 = row_sum<kNormThreads>(s2, slots, slot) / (float)D;
        for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
            float h[V], g[V], o[V];
            load(j, h, g);
            if (radd)
                ld_group_to(radd + row * D, j, D, o);
            else
#pragma unroll
                for (int e = 0; e < V; e++) o[e] = 0.f;
#pragma unroll
            for (int e = 0; e < V; e++) o[e] = fmaf(rs, g[e] - s1 - h[e] * s2, o[e]);
            st_group_to(dx + row * D, j, D, o);
        }
    }
}
// a thread a channel, blockIdx.y a share of the rows
template <typename T, bool FROM8>
__global__ __launch_bounds__(kNormThreads) void k_norm_columns(const T* __restrict__ dy, const T* __restrict__ x,
                                                               const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                               const float* __restrict__ mean, const float* __restrict__ rstd, int64_t N,
                                                               int64_t D, float* __restrict__ parts) {
    const int64_t j = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    if (j >= D) return;
    float aw = 0.f, ab = 0.f;
    for (int64_t row = blockIdx.y; row < N; row += gridDim.y) {
        float v;
        if constexpr (FROM8)
            v = (float)codes[row * D + j] * scales[row * G + j / kPackGroup];
        else
            v = ld_elem(x + row * D + j);
        const float d = ld_elem(dy + row * D + j);
        aw = fmaf(d, (v - mean[row]) * rstd[row], aw);
        ab += d;
    }
    parts[(int64_t)blockIdx.y * 2 * D + j] = aw;
    parts[(int64_t)blockIdx.y * 2 * D + D + j] = ab;
}

// dweight and dbias from the workgroups' parts (P x 2 x D): 64 channels a workgroup, four waves share the parts, a fixed order
__global__ __launch_bounds__(256) void k_norm_params(const float* __restrict__ parts, int P, int64_t D, float* __restrict__ dweight,
                                                     float* __restrict__ dbias) {
    __shared__ float s[4][kWave];
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
    const int64_t c = (int64_t)blockIdx.x * kWave + lane;  // of 2 D
    float t = 0.f;
    if (c < 2 * D)
        for (int p = wv; p < P; p += 4) t += parts[(int64_t)p * 2 * D + c];
    s[wv][lane] = t;
    __syncthreads();
    if (wv || c >= 2 * D) return;
    t = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
    if (c < D) {
        if (dweight) dweight[c] = t;
    } else if (dbias) {
        dbias[c - D] = t;
    }
}

// ---- the instance for a row length ----
// TPR threads with VPL groups each hold a row; 0 threads: the kernels for long rows.
struct NormShape {
    int tpr, vpl;
};
template <typename T>
NormShape norm_shape(int64_t D) {
    const int64_t n = (D + kVec<T> - 1) / kVec<T>;  // 16-byte groups of a row
    if (n <= 8) return {8, 1};
    if (n <= 16) return {16, 1};
    if (n <= 32) return {32, 1};
    if (n <= 64) return {64, 1};
    if (n <= 128) return {64, 2};
    if (n <= 256) return {64, 4};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return {256, 4};
    if (n <= 2048 && sizeof(T) == 4) return {256, 8};
    return {0, 0};
}
#define CAT_NORM_SHAPES(X) X(8, 1) X(16, 1) X(32, 1) X(64, 1) X(64, 2) X(64, 4) X(256, 2) X(256, 4) X(256, 8)

// workgroups of the backward pass: their parts are written and read again, so no more than fill the card
constexpr int kNormParts = 1024;
int norm_parts(int64_t N, NormShape s) {
    const int64_t rpb = s.tpr ? kNormThreads / s.tpr : 1, b = (N + rpb - 1) / rpb;
    return (int)(b < kNormParts ? b : kNormParts);
}
// long rows: shares of the rows that k_norm_columns takes
constexpr int kColumnParts = 64;

unsigned norm_blocks(int64_t N, int rpb) {
    const int64_t b = (N + rpb - 1) / rpb;
    return (unsigned)(b < kNormMaxBlocks ? b : kNormMaxBlocks);
}

template <typename T, bool PACK, bool FROM8>
cat_status launch_norm(const T* x, int64_t N, int64_t D, const float* weight, const float* bias, float eps, T* y, float* mean, float* rstd,
                       int8_t* codes, float* scales, hipStream_t st) {
    const NormShape s = norm_shape<T>(D);
#define CAT_X(TPR, VPL)                                                                                                                  \
    if (s.tpr == TPR && s.vpl == VPL)                                                                                                    \
        hipLaunchKernelGGL((k_norm<T, TPR, VPL, PACK, FROM8>), dim3(norm_blocks(N, kNormThreads / TPR)), dim3(kNormThreads), 0, st, x, N, \
                           D, weight, bias, eps, y, mean, rstd, codes, scales);
    CAT_NORM_SHAPES(CAT_X)
#undef CAT_X
    if (!s.tpr) {
        if (PACK) {
            const cat_status r = cat_pack8(x, N, D, sizeof(T) == 4 ? CAT_F32 : CAT_BF16, codes, scales, (void*)st);
            if (r != CAT_OK) return r;
        }
        hipLaunchKernelGGL((k_norm_long<T, FROM8>), dim3(norm_blocks(N, 1)), dim3(kNormThreads), 0, st, x, N, D, weight, bias, eps, y, mean,
                           rstd, codes, scales);
    }
    CAT_LAUNCH_CHECK("k_norm");
    return CAT_OK;
}

template <typename T, bool FROM8>
cat_status launch_norm_backward(const T* dy, const T* x, const int8_t* codes, const float* scales, const float* mean, const float* rstd,
                                int64_t N, int64_t D, const float* weight, const T* radd, T* dx, float* dweight, float* dbias, float* parts,
                                hipStream_t st) {
    const NormShape s = norm_shape<T>(D);
    int P = norm_parts(N, s);
    if (!dweight && !dbias) parts = nullptr;
#define CAT_X(TPR, VPL)                                                                                                                \
    if (s.tpr == TPR && s.vpl == VPL)                                                                                                  \
        hipLaunchKernelGGL((k_norm_backward<T, TPR, VPL, FROM8>), dim3((unsigned)P), dim3(kNormThreads), 0, st, dy, x, codes, scales, mean, \
                           rstd, N, D, weight, radd, dx, parts);
    CAT_NORM_SHAPES(CAT_X)
#undef CAT_X
    if (!s.tpr) {
        hipLaunchKernelGGL((k_norm_backward_long<T, FROM8>), dim3(norm_blocks(N, 1)), dim3(kNormThreads), 0, st, dy, x, codes, scales, mean,
                           rstd, N, D, weight, radd, dx);
        CAT_LAUNCH_CHECK("k_norm_backward_long");
        if (parts) {
            P = (int)(N < kColumnParts ? N : kColumnParts);
            hipLaunchKernelGGL((k_norm_columns<T, FROM8>), dim3((unsigned)((D + kNormThreads - 1) / kNormThreads), (unsigned)P),
                               dim3(kNormThreads), 0, st, dy, x, codes, scales, mean, rstd, N, D, parts);
        }
    }
    CAT_LAUNCH_CHECK("k_norm_backward");
    if (parts) {
        hipLaunchKernelGGL(k_norm_params, dim3((unsigned)((2 * D + kWave - 1) / kWave)), dim3(256), 0, st, parts, P, D, dweight, dbias);
        CAT_LAUNCH_CHECK("k_norm_params");
    }
    return CAT_OK;
}

}  // namespace
}  // namespace cat

using namespace cat;

extern "C" {

cat_status cat_layer_norm(const void* x, int64_t N, int64_t D, cat_dtype dt, const float* weight, const float* bias, float eps, void* y,
                          float* mean, float* rstd, int8_t* codes, float* scales, void* hip_stream) {
    const char* who = "cat_layer_norm";
    CAT_TRY(check_rows(who, N, D, dt));
    CAT_TRY(check_ptr(who, "x", x, N > 0));
    CAT_TRY(check_ptr(who, "weight", weight, false));
    CAT_TRY(check_ptr(who, "bias", bias, false));
    CAT_TRY(check_ptr(who, "y", y, N > 0));
    CAT_TRY(check_ptr(who, "mean", mean, false));
    CAT_TRY(check_ptr(who, "rstd", rstd, false));
    CAT_TRY(check_ptr(who, "codes", codes, scales != nullptr));
    CAT_TRY(check_ptr(who, "scales", scales, codes != nullptr));
    if (!(eps >= 0.f) || isinf(eps)) return set_error(CAT_ERR_INVALID_ARG, "%s: eps = %g is not finite and >= 0", who, (double)eps);
    if (N > 0 && y == x) return set_error(CAT_ERR_INVALID_ARG, "%s: y may not alias x", who);
    if (N == 0) return CAT_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    if (dt == CAT_F32)
        return codes ? launch_norm<float, true, false>((const float*)x, N, D, weight, bias, eps, (float*)y, mean, rstd, codes, scales, st)
                     : launch_norm<float, false, false>((const float*)x, N, D, weight, bias, eps, (float*)y, mean, rstd, codes, scales, st);
    return codes ? launch_norm<bf16_t, true, false>((const bf16_t*)x, N, D, weight, bias, eps, (bf16_t*)y, mean, rstd, codes, scales, st)
                 : launch_norm<bf16_t, false, false>((const bf16_t*)x, N, D, weight, bias, eps, (bf16_t*)y, mean, rstd, codes, scales, st);
}

cat_status cat_layer_norm_packed(const int8_t* codes, const float* scales, const float* mean, const float* rstd, int64_t N, int64_t D,
                                 cat_dtype dt, const float* weight, const float* bias, void* y, void* hip_stream) {
    const char* who = "cat_layer_norm_packed";
    CAT_TRY(check_rows(who, N, D, dt));
    CAT_TRY(check_ptr(who, "codes", codes, N > 0));
    CAT_TRY(check_ptr(who, "scales", scales, N > 0));
    CAT_TRY(check_ptr(who, "mean", mean, N > 0));
    CAT_TRY(check_ptr(who, "rstd", rstd, N > 0));
    CAT_TRY(check_ptr(who, "weight", weight, false));
    CAT_TRY(check_ptr(who, "bias", bias, false));
    CAT_TRY(check_ptr(who, "y", y, N > 0));
    if (N == 0) return CAT_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    // (the kernel of the forward pass only reads these with FROM8)
    int8_t* c = const_cast<int8_t*>(codes);
    float *s = const_cast<float*>(scales), *m = const_cast<float*>(mean), *r = const_cast<float*>(rstd);
    if (dt == CAT_F32) return launch_norm<float, false, true>(nullptr, N, D, weight, bias, 0.f, (float*)y, m, r, c, s, st);
    return launch_norm<bf16_t, false, true>(nullptr, N, D, weight, bias, 0.f, (bf16_t*)y, m, r, c, s, st);
}

size_t cat_layer_norm_backward_workspace_bytes(int64_t N, int64_t D, cat_dtype dt) {
    if (check_rows("cat_layer_norm_backward_workspace_bytes", N, D, dt) != CAT_OK) return 0;
    const NormShape s = dt == CAT_F32 ? norm_shape<float>(D) : norm_shape<bf16_t>(D);
    const int P = s.tpr ? norm_parts(N, s) : kColumnParts;
    return ((size_t)(P > 0 ? P : 1) * 2 * (size_t)D * sizeof(float) + 255) & ~(size_t)255;
}

cat_status cat_layer_norm_backward(const void* dy, const void* x, const int8_t* codes, const float* scales, const float* mean,
                                   const float* rstd, int64_t N, int64_t D, cat_dtype dt, const float* weight, const void* residual_grad,
                                   void* dx, float* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "cat_layer_norm_backward";
    CAT_TRY(check_rows(who, N, D, dt));
    CAT_TRY(check_ptr(who, "dy", dy, N > 0));
    if (N > 0 && (x == nullptr) == (codes == nullptr)) return set_error(CAT_ERR_INVALID_ARG, "%s: give x or its checkpoint, one of the two", who);
    CAT_TRY(check_ptr(who, "x", x, false));
    CAT_TRY(check_ptr(who, "codes", codes, scales != nullptr));
    CAT_TRY(check_ptr(who, "scales", scales, codes != nullptr));
    CAT_TRY(check_ptr(who, "mean", mean, N > 0));
    CAT_TRY(check_ptr(who, "rstd", rstd, N > 0));
    CAT_TRY(check_ptr(who, "weight", weight, false));
    CAT_TRY(check_ptr(who, "residual_grad", residual_grad, false));
    CAT_TRY(check_ptr(who, "dx", dx, N > 0));
    CAT_TRY(check_ptr(who, "dweight", dweight, false));
    CAT_TRY(check_ptr(who, "dbias", dbias, false));
    if (N > 0 && (dx == dy || dx == x || dx == residual_grad)) return set_error(CAT_ERR_INVALID_ARG, "%s: dx may not alias an input", who);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, cat_layer_norm_backward_workspace_bytes(N, D, dt)));
    hipStream_t st = (hipStream_t)hip_stream;
    if (N == 0) {
        if (dweight) CAT_TRY(launch_fill_zero(dweight, (size_t)D * sizeof(float), st));
        if (dbias) CAT_TRY(launch_fill_zero(dbias, (size_t)D * sizeof(float), st));
        return CAT_OK;
    }
    float* parts = (float*)workspace;
    if (dt == CAT_F32) {
        using T = float;
        return codes ? launch_norm_backward<T, true>((const T*)dy, (const T*)x, codes, scales, mean, rstd, N, D, weight,
                                                     (const T*)residual_grad, (T*)dx, dweight, dbias, parts, st)
                     : launch_norm_backward<T, false>((const T*)dy, (const T*)x, codes, scales, mean, rstd, N, D, weight,
                                                      (const T*)residual_grad, (T*)dx, dweight, dbias, parts, st);
    }
    using T = bf16_t;
    return codes ? launch_norm_backward<T, true>((const T*)dy, (const T*)x, codes, scales, mean, rstd, N, D, weight, (const T*)residual_grad,
                                                 (T*)dx, dweight, dbias, parts, st)
                 : launch_norm_backward<T, false>((const T*)dy, (const T*)x, codes, scales, mean, rstd, N, D, weight,
                                                  (const T*)residual_grad, (T*)dx, dweight, dbias, parts, st);
}

}  // extern "C"
