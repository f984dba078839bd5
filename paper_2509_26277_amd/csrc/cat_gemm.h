// Matrix products of the block's operators: what the launchers and the kernels agree on.
//
//   out[m][n] = sum_k Q(m, k) P(n, k)        followed by an epilogue on rows of out
//
// Either operand lies with k contiguous (element (r, k) at r * ld + k) or "turned" (at k * ld + r):
//   forward          x w^T       Q = x,           P = w
//   input gradient   dy w        Q = dy,          P = w turned
//   weight gradient  dy^T u      Q = dy turned,   P = u turned
#pragma once
#include "cat_block.h"

namespace cat {

enum GemmKind { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

// What happens to out on its way to memory, by kind:
//   kForward     z = out + bias; codes_out: the checkpoint of z; y = act(z) + residual
//   kInputGrad   out * act'(codes_in)
//   kWeightGrad  nothing
struct Epilogue {
    void* out;
    const float* bias;
    const void* residual;
    int8_t* codes_out;
    float* scales_out;
    const int8_t* codes_in;
    const float* scales_in;
    int act;
};

struct GemmArgs {
    const void *p, *q;
    int64_t ldp, ldq;          // entries; rows start on 16-byte boundaries
    int64_t p_bytes, q_bytes;  // what may be read from p, q on
    int64_t m, n, k;
    int64_t k_split;  // entries of k a share takes (a multiple of the kernel's step); shares beyond the first: blockIdx.y
    int splits;
    float* parts;  // splits > 1: splits x m x n
    Epilogue e;
};

constexpr int64_t kGemmMaxRowBytes = 1 << 23;  // offsets inside a tile of 256 rows stay below 2^31

// E (4 or 8) neighbouring entries of a row of out, from column n on (a multiple of E), through the epilogue.  PACK: the 16 lanes of
// a DPP row hold 128 columns of one row of out, all of them active.
template <typename T, int E>
__device__ __forceinline__ void ld_entries(const T* row, int64_t n, int64_t N, float (&v)[E]) {
    if constexpr (E == kVec<T>) {
        ld_group_to(row, n, N, v);
    } else if constexpr (E > kVec<T>) {
        float a[4], b[4];
        ld_group_to(row, n, N, a);
        ld_group_to(row, n + 4, N, b);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = a[e], v[4 + e] = b[e];
    } else {
#pragma unroll
        for (int e = 0; e < E; e++) v[e] = n + e < N ? ld_elem(row + n + e) : 0.f;
    }
}
template <typename T, int E>
__device__ __forceinline__ void st_entries(T* row, int64_t n, int64_t N, const float (&v)[E]) {
    if constexpr (E == kVec<T>) {
        st_group_to(row, n, N, v);
    } else if constexpr (E > kVec<T>) {
        const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
        st_group_to(row, n, N, a);
        st_group_to(row, n + 4, N, b);
    } else {
#pragma unroll
        for (int e = 0; e < E; e++)
            if (n + e < N) st_round(row + n + e, v[e]);
    }
}
template <typename T, int KIND, int E, bool PACK>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t m, int64_t n, int64_t N, bool valid, float (&v)[E]) {
    const int64_t at = m * N;
    if constexpr (KIND == kForward) {
        if (e.bias) {
            float b[E];
            ld_params<E>(e.bias, valid ? n : 0, N, 0.f, b);
#pragma unroll
            for (int i = 0; i < E; i++) v[i] += b[i];
        }
        if constexpr (PACK) {
            if (e.codes_out) {
                uint32_t a = 0;
#pragma unroll
                for (int i = 0; i < E; i++) a = mag_max(a, valid && n + i < N ? v[i] : 0.f);
                const PackScale s = pack_scale(lanes_max<kPackGroup / E>(a));
                if (valid && n < N) {
                    st_codes<E>(e.codes_out + at, n, N, v, s.up);
                    if (n % kPackGroup == 0) e.scales_out[m * ((N + kPackGroup - 1) / kPackGroup) + n / kPackGroup] = s.step;
                }
            }
        }
        if (!valid || n >= N) return;
        with_act(e.act, [&](auto which) {
#pragma unroll
            for (int i = 0; i < E; i++) v[i] = act_value<decltype(which)::value, sizeof(T) == 2>(v[i]);
        });
        if (e.residual) {
            float r[E];
            ld_entries<T, E>((const T*)e.residual + at, n, N, r);
#pragma unroll
            for (int i = 0; i < E; i++) v[i] += r[i];
        }
    } else {
        if (!valid || n >= N) return;
        if constexpr (KIND == kInputGrad) {
            if (e.act != CAT_ACT_NONE) {
                float c[E];
                const float step = e.scales_in[m * ((N + kPackGroup - 1) / kPackGroup) + n / kPackGroup];
                ld_codes<E>(e.codes_in + at, n, N, step, c);
                with_act(e.act, [&](auto which) {
#pragma unroll
                    for (int i = 0; i < E; i++) v[i] *= act_grad<decltype(which)::value, sizeof(T) == 2>(c[i]);
                });
            }
        }
    }
    st_entries<T, E>((T*)e.out + at, n, N, v);
}

// launchers of the tile kernels, one translation unit a type; `large`: tiles of 256 x 256 (bfloat16 only)
cat_status launch_gemm_f32(GemmKind kind, const GemmArgs& a, hipStream_t st);
cat_status launch_gemm_bf16(GemmKind kind, bool large, const GemmArgs& a, hipStream_t st);

}  // namespace cat
