// Layer norm of a row, forward (from rows, or again from their checkpoint) and backward, with the sums over rows that the
// gradients of its parameters are.  Kernels, launchers and entry points.
//
//   forward    mu = mean x, v = mean (x - mu)^2, rstd = 1 / sqrt(v + eps), y = (x - mu) rstd w + b
//   backward   xhat = (x - mu) rstd, g = dy w:  dx = rstd (g - mean g - xhat mean(g xhat)) [+ gradient over the residual]
//              dw = sum_rows dy xhat, db = sum_rows dy
//
// All of it is bound by memory: a row is read once, stays in registers for both of its statistics (the variance is that
// of the centred entries, not a difference of large sums) and for the result.  TPR threads share a row, each with VPL
// 16-byte groups of it: 8 lanes for the shortest rows (8 rows a wave); forward a wave up to 2048 entries (32 a lane) and a
// workgroup of four waves (sums over LDS) up to 8192; backward, with its sums and two or three rows ahead, a wave up to 1024,
// four waves up to 4096 and eight up to 8192.  Longer rows have a workgroup each that reads the row again for every use.
//
// Measured, with a large copy at 5.2 TB/s: forward 131072 x 2048 bf16 201 us (5.3 TB/s); 65536 x 1024 bf16 forward with
// checkpoint 58 us, backward from it 101 (4.7 TB/s) and 5 for its sums; fp32 the same rows 138 us (4.4) and 174 with its sums
// (5.0).  16411 x 1001 fp32 41 us and 57 with the sums (3.6 and 3.7): 1000 columns take as long, 1024, where no lane stands idle,
// 36 and 49.  One row: 4 us, a launch.
#include "cat_block.h"

namespace cat {
namespace {

constexpr int kNormThreads = 256;
constexpr int64_t kNormMaxBlocks = 1 << 22;  // long rows: further ones by stride

// A lane's 16-byte group of a row as it lies in memory: the next row's are requested while the present one's are worked on,
// so they have to be few registers.
template <typename T, bool FROM8>
struct Part {
    uint32_t w[FROM8 ? kVec<T> / 4 : 4];
    float step;
    // entries [j, j + V) of a row of D entries, zero behind its end
    __device__ __forceinline__ void load(const T* x, const int8_t* codes, const float* scales, int64_t row, int64_t j, int64_t D, int64_t G) {
        constexpr int V = kVec<T>;
        if constexpr (FROM8) {
            const int8_t* c = codes + row * D + j;
            step = j < D ? scales[row * G + j / kPackGroup] : 0.f;
            if (j + V <= D) {
                const std::conditional_t<V == 8, Codes8, Codes4> q = *(const std::conditional_t<V == 8, Codes8, Codes4>*)c;
#pragma unroll
                for (int e = 0; e < V / 4; e++) w[e] = q.w[e];
            } else {
#pragma unroll
                for (int e = 0; e < V / 4; e++) w[e] = 0;
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (j + e < D) w[e / 4] |= (uint32_t)(uint8_t)c[e] << (8 * (e % 4));
            }
        } else {
            const T* c = x + row * D + j;
            if (j + V <= D) {
                const Group16<T> q = *(const Group16<T>*)c;
#pragma unroll
                for (int e = 0; e < 4; e++) w[e] = q.w[e];
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) w[e] = 0;
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (j + e < D) {
                        if constexpr (sizeof(T) == 4)
                            w[e] = __float_as_uint(c[e]);
                        else
                            w[e / 2] |= (uint32_t)c[e] << (16 * (e % 2));
                    }
            }
        }
    }
    __device__ __forceinline__ float at(int e) const {
        if constexpr (FROM8) return code_value(w[e / 4], e % 4) * step;
        else if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
};

// Sums over the TPR threads of a row, Q of them at a time.  TPR > 64: over the workgroup's waves by LDS; `slot` alternates, so
// that one barrier a time is enough.
template <int TPR, int Q>
__device__ __forceinline__ void row_sums(float (&v)[Q], float (*slots)[2][8], int& slot) {
#pragma unroll
    for (int q = 0; q < Q; q++) v[q] = lanes_sum<(TPR < kWave ? TPR : kWave)>(v[q]);
    if constexpr (TPR > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
            for (int q = 0; q < Q; q++) slots[slot][q][threadIdx.x / kWave] = v[q];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const float* s = slots[slot][q];
            v[q] = (s[0] + s[1]) + (s[2] + s[3]);
            if constexpr (TPR > 256) v[q] += (s[4] + s[5]) + (s[6] + s[7]);
        }
        slot ^= 1;
    }
}
template <int TPR>
constexpr int kThreads = TPR > kNormThreads ? TPR : kNormThreads;

// ---- forward ----
// PACK: also the checkpoint of x.  FROM8: x is a checkpoint, and mean and rstd are given.  Workgroups go through the rows
// by stride: weight and bias stay in registers, and a row is requested while the one before it is worked on.
template <typename T, int TPR, int VPL, bool PACK, bool FROM8>
__global__ __launch_bounds__(kThreads<TPR>) void k_norm(const T* __restrict__ x, int64_t N, int64_t D, const float* __restrict__ weight,
                                                        const float* __restrict__ bias, float eps, T* __restrict__ y, float* __restrict__ mean,
                                                        float* __restrict__ rstd, int8_t* __restrict__ codes, float* __restrict__ scales) {
    constexpr int V = kVec<T>, RPB = kThreads<TPR> / TPR, GL = kPackGroup / V;  // GL: neighbouring lanes that share a scale
    __shared__ float slots[2][2][8];
    int slot = 0;
    const int sub = threadIdx.x % TPR;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup, stride = (int64_t)gridDim.x * RPB;
    int64_t own_row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Part<T, FROM8> next[VPL];
#pragma unroll
    for (int k = 0; k < VPL; k++) next[k].load(x, codes, scales, own_row < N ? own_row : N - 1, ((int64_t)k * TPR + sub) * V, D, G);
    float w[VPL][V], b[VPL][V];
#pragma unroll
    for (int k = 0; k < VPL; k++) {
        ld_params<V>(weight, ((int64_t)k * TPR + sub) * V, D, 1.f, w[k]);
        ld_params<V>(bias, ((int64_t)k * TPR + sub) * V, D, 0.f, b[k]);
    }
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < N; r0 += stride, own_row += stride) {
        const bool mine = own_row < N;
        const int64_t row = mine ? own_row : N - 1;
        Part<T, FROM8> v[VPL];
#pragma unroll
        for (int k = 0; k < VPL; k++) v[k] = next[k];
        if (r0 + stride < N) {
            const int64_t r = own_row + stride < N ? own_row + stride : N - 1;
#pragma unroll
            for (int k = 0; k < VPL; k++) next[k].load(x, codes, scales, r, ((int64_t)k * TPR + sub) * V, D, G);
        }
        if constexpr (PACK) {
#pragma unroll
            for (int k = 0; k < VPL; k++) {
                const int64_t j = ((int64_t)k * TPR + sub) * V;
                uint32_t a = 0;
                float f[V];
#pragma unroll
                for (int e = 0; e < V; e++) f[e] = v[k].at(e), a = mag_max(a, f[e]);
                a = lanes_max<(TPR < GL ? TPR : GL)>(a);
                const PackScale s = pack_scale(a);
                if (mine && j < D) {
                    st_codes<V>(codes + row * D, j, D, f, s.up);
                    if (j % kPackGroup == 0) scales[row * G + j / kPackGroup] = s.step;
                }
            }
        }
        float mu, rs;
        if constexpr (FROM8) {
            mu = mean[row], rs = rstd[row];
        } else {
            float s[1] = {0.f};
#pragma unroll
            for (int k = 0; k < VPL; k++)
#pragma unroll
                for (int e = 0; e < V; e++) s[0] += v[k].at(e);
            row_sums<TPR>(s, slots, slot);
            mu = s[0] / (float)D;
            float q[1] = {0.f};
#pragma unroll
            for (int k = 0; k < VPL; k++) {
                const int64_t j = ((int64_t)k * TPR + sub) * V;
#pragma unroll
                for (int e = 0; e < V; e++) {
                    const float c = v[k].at(e) - mu;
                    if (j + e < D) q[0] = fmaf(c, c, q[0]);
                }
            }
            row_sums<TPR>(q, slots, slot);
            rs = 1.f / sqrtf(q[0] / (float)D + eps);
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
            float o[V];
#pragma unroll
            for (int e = 0; e < V; e++) o[e] = fmaf((v[k].at(e) - mu) * rs, w[k][e], b[k][e]);
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
    __shared__ float slots[2][2][8];
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
            float t[1] = {s};
            row_sums<kNormThreads>(t, slots, slot);
            mu = t[0] / (float)D;
            for (int64_t j = (int64_t)threadIdx.x * V; j < D; j += kNormThreads * V) {
                float v[V];
                load(j, v);
#pragma unroll
                for (int e = 0; e < V; e++)
                    if (j + e < D) q = fmaf(v[e] - mu, v[e] - mu, q);
            }
            t[0] = q;
            row_sums<kNormThreads>(t, slots, slot);
            rs = 1.f / sqrtf(t[0] / (float)D + eps);
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
// A workgroup goes through its rows by stride, a row ahead as above, and keeps its threads' channels of dw and db in registers;
// at its end the rows' slots (RPB of them share the channels) are added in LDS in a fixed order and written as the workgroup's
// part, which launch_sum_parts adds up: no atomics, the same bits on every run.
template <typename T, int TPR, int VPL, bool FROM8>
__global__ __launch_bounds__(kThreads<TPR>) void k_norm_backward(const T* __restrict__ dy, const T* __restrict__ x,
                                                                 const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                                 const float* __restrict__ mean, const float* __restrict__ rstd, int64_t N,
                                                                 int64_t D, const float* __restrict__ weight, const T* __restrict__ radd,
                                                                 T* __restrict__ dx, float* __restrict__ parts) {
    constexpr int V = kVec<T>, RPB = kThreads<TPR> / TPR;
    __shared__ float slots[2][2][8];
    __shared__ float sums[RPB > 1 ? kThreads<TPR> * V : 1];
    int slot = 0;
    const int sub = threadIdx.x % TPR;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup, stride = (int64_t)gridDim.x * RPB;
    const float inv = 1.f / (float)D;
    int64_t own_row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Part<T, FROM8> next_x[VPL];
    Part<T, false> next_g[VPL], next_a[VPL];
    float next_mu, next_rs;
    auto request = [&](int64_t r) {
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            next_x[k].load(x, codes, scales, r, j, D, G);
            next_g[k].load(dy, nullptr, nullptr, r, j, D, G);  // (zero behind the row's end, so that xhat there does not count)
            if (radd) next_a[k].load(radd, nullptr, nullptr, r, j, D, G);
        }
        next_mu = mean[r], next_rs = rstd[r];
    };
    request(own_row < N ? own_row : N - 1);
    float aw[VPL][V], ab[VPL][V], w[VPL][V];
#pragma unroll
    for (int k = 0; k < VPL; k++) {
        ld_params<V>(weight, ((int64_t)k * TPR + sub) * V, D, 1.f, w[k]);
#pragma unroll
        for (int e = 0; e < V; e++) aw[k][e] = ab[k][e] = 0.f;
    }
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < N; r0 += stride, own_row += stride) {
        const bool mine = own_row < N;
        Part<T, FROM8> px[VPL];
        Part<T, false> pg[VPL], pa[VPL];
        const float mu = next_mu, rs = next_rs;
#pragma unroll
        for (int k = 0; k < VPL; k++) px[k] = next_x[k], pg[k] = next_g[k], pa[k] = next_a[k];
        if (r0 + stride < N) request(own_row + stride < N ? own_row + stride : N - 1);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < VPL; k++)
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float h = (px[k].at(e) - mu) * rs, d = mine ? pg[k].at(e) : 0.f, g = d * w[k][e];
                ab[k][e] += d;
                aw[k][e] = fmaf(d, mine ? h : 0.f, aw[k][e]);
                s[0] += g;
                s[1] = fmaf(g, h, s[1]);
            }
        row_sums<TPR>(s, slots, slot);
        const float s1 = s[0] * inv, s2 = s[1] * inv;
        if (!mine) continue;
#pragma unroll
        for (int k = 0; k < VPL; k++) {
            const int64_t j = ((int64_t)k * TPR + sub) * V;
            if (j >= D) continue;
            float o[V];
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float h = (px[k].at(e) - mu) * rs, g = pg[k].at(e) * w[k][e];
                o[e] = fmaf(rs, g - s1 - h * s2, radd ? pa[k].at(e) : 0.f);
            }
            st_group_to(dx + own_row * D, j, D, o);
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
    __shared__ float slots[2][2][8];
    int slot = 0;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    for (int64_t row = blockIdx.x; row < N; row += gridDim.x) {
        const float mu = mean[row], rs = rstd[row];
        float s[2] = {0.f, 0.f};
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
            for (int e = 0; e < V; e++) s[0] += g[e], s[1] = fmaf(g[e], h[e], s[1]);
        }
        row_sums<kNormThreads>(s, slots, slot);
        const float s1 = s[0] / (float)D, s2 = s[1] / (float)D;
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

// ---- the instance for a row length ----
// TPR threads with VPL 16-byte groups each hold a row; 0 threads: the kernels for long rows.  A wave takes up to 32 entries
// a lane in the forward pass and up to 16 in the backward pass, whose sums and rows ahead need more registers.
struct NormShape {
    int tpr, vpl;
};
constexpr int64_t kNormLong = 8192;
template <typename T, bool BACK>
NormShape norm_shape(int64_t D) {
    constexpr int wide = kVec<T> == 8 ? 1 : 2;  // groups of 8 entries
    const int64_t n = (D + kVec<T> - 1) / kVec<T>;
    if (D > kNormLong) return {0, 0};
    if (n <= 8) return {8, 1};
    if (n <= 16) return {16, 1};
    if (n <= 32) return {32, 1};
    if (n <= 64) return {64, 1};
    if (D <= 512) return {64, wide};
    if (D <= 1024) return {64, 2 * wide};
    if (!BACK) return D <= 2048 ? NormShape{64, 4 * wide} : D <= 4096 ? NormShape{256, 2 * wide} : NormShape{256, 4 * wide};
    return D <= 2048 ? NormShape{256, wide} : D <= 4096 ? NormShape{256, 2 * wide} : NormShape{512, 2 * wide};
}

// workgroups: as many as the card holds at a time, and of the backward pass, whose parts are written and read again, no more
constexpr int kNormGroups = 1024, kNormParts = 512;
int norm_groups(int64_t N, NormShape s, int most) {
    const int64_t rpb = s.tpr && s.tpr < kNormThreads ? kNormThreads / s.tpr : 1, b = (N + rpb - 1) / rpb;
    return (int)(b < most ? b : most);
}
// long rows: shares of the rows that k_norm_columns takes
int column_parts(int64_t N) { return (int)(N < 64 ? N : 64); }

unsigned norm_blocks(int64_t N) { return (unsigned)(N < kNormMaxBlocks ? N : kNormMaxBlocks); }

template <typename T, int TPR, int VPL, bool PACK, bool FROM8>
void norm_instance(const T* x, int64_t N, int64_t D, const float* weight, const float* bias, float eps, T* y, float* mean, float* rstd, int8_t* codes,
                   float* scales, hipStream_t st) {
    hipLaunchKernelGGL((k_norm<T, TPR, VPL, PACK, FROM8>), dim3((unsigned)norm_groups(N, {TPR, VPL}, kNormGroups)), dim3(kThreads<TPR>), 0, st, x, N, D,
                       weight, bias, eps, y, mean, rstd, codes, scales);
}
template <typename T, bool PACK, bool FROM8>
cat_status launch_norm(const T* x, int64_t N, int64_t D, const float* weight, const float* bias, float eps, T* y, float* mean, float* rstd,
                       int8_t* codes, float* scales, hipStream_t st) {
    const NormShape s = norm_shape<T, false>(D);
#define CAT_X(TPR, VPL) \
    if (s.tpr == TPR && s.vpl == VPL) norm_instance<T, TPR, VPL, PACK, FROM8>(x, N, D, weight, bias, eps, y, mean, rstd, codes, scales, st);
    CAT_X(8, 1) CAT_X(16, 1) CAT_X(32, 1) CAT_X(64, 1) CAT_X(64, 2) CAT_X(64, 4) CAT_X(256, 4)
    if constexpr (sizeof(T) == 4) {
        CAT_X(64, 8) CAT_X(256, 8)
    } else {
        CAT_X(256, 2)
    }
#undef CAT_X
    if (!s.tpr) {
        if (PACK) CAT_TRY(cat_pack8(x, N, D, sizeof(T) == 4 ? CAT_F32 : CAT_BF16, codes, scales, (void*)st));
        hipLaunchKernelGGL((k_norm_long<T, FROM8>), dim3(norm_blocks(N)), dim3(kNormThreads), 0, st, x, N, D, weight, bias, eps, y, mean, rstd, codes,
                           scales);
    }
    CAT_LAUNCH_CHECK("k_norm");
    return CAT_OK;
}

template <typename T, int TPR, int VPL, bool FROM8>
void norm_backward_instance(const T* dy, const T* x, const int8_t* codes, const float* scales, const float* mean, const float* rstd, int64_t N, int64_t D,
                            const float* weight, const T* radd, T* dx, float* parts, int P, hipStream_t st) {
    hipLaunchKernelGGL((k_norm_backward<T, TPR, VPL, FROM8>), dim3((unsigned)P), dim3(kThreads<TPR>), 0, st, dy, x, codes, scales, mean, rstd, N, D, weight,
                       radd, dx, parts);
}
template <typename T, bool FROM8>
cat_status launch_norm_backward(const T* dy, const T* x, const int8_t* codes, const float* scales, const float* mean, const float* rstd,
                                int64_t N, int64_t D, const float* weight, const T* radd, T* dx, float* dweight, float* dbias, float* parts,
                                hipStream_t st) {
    const NormShape s = norm_shape<T, true>(D);
    int P = norm_groups(N, s, kNormParts);
    if (!dweight && !dbias) parts = nullptr;
#define CAT_X(TPR, VPL) \
    if (s.tpr == TPR && s.vpl == VPL) norm_backward_instance<T, TPR, VPL, FROM8>(dy, x, codes, scales, mean, rstd, N, D, weight, radd, dx, parts, P, st);
    CAT_X(8, 1) CAT_X(16, 1) CAT_X(32, 1) CAT_X(64, 1) CAT_X(64, 2) CAT_X(256, 2)
    if constexpr (sizeof(T) == 4) {
        CAT_X(64, 4) CAT_X(256, 4) CAT_X(512, 4)
    } else {
        CAT_X(256, 1) CAT_X(512, 2)
    }
#undef CAT_X
    if (!s.tpr) {
        hipLaunchKernelGGL((k_norm_backward_long<T, FROM8>), dim3(norm_blocks(N)), dim3(kNormThreads), 0, st, dy, x, codes, scales, mean, rstd, N, D,
                           weight, radd, dx);
        CAT_LAUNCH_CHECK("k_norm_backward_long");
        if (parts) {
            P = column_parts(N);
            hipLaunchKernelGGL((k_norm_columns<T, FROM8>), dim3((unsigned)((D + kNormThreads - 1) / kNormThreads), (unsigned)P), dim3(kNormThreads), 0,
                               st, dy, x, codes, scales, mean, rstd, N, D, parts);
        }
    }
    CAT_LAUNCH_CHECK("k_norm_backward");
    return parts ? launch_sum_parts(parts, P, 2 * D, D, dweight, dbias, st) : CAT_OK;
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
    const NormShape s = dt == CAT_F32 ? norm_shape<float, true>(D) : norm_shape<bf16_t, true>(D);
    const int P = s.tpr ? norm_groups(N, s, kNormParts) : column_parts(N);
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
    // (the workspace holds the parts of the parameters' gradients alone)
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, dweight || dbias ? cat_layer_norm_backward_workspace_bytes(N, D, dt) : 256));
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
