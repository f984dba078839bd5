// What the kernels share that hold whole rows in registers (layer norm, rows to 8 bits): a lane's part of a row, sums over the
// threads of a row, and how many threads take one.
#pragma once
#include "cat_block.h"

namespace cat {

constexpr int kNormThreads = 256;
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

}  // namespace cat
