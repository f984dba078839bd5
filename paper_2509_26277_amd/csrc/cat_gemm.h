// Matrix products of the block's operators: what the launchers and the kernels agree on.
//
//   out[m][n] = sum_k Q(m, k) P(n, k)        followed by an epilogue on rows of out
//
// Either operand lies with k contiguous (element (r, k) at r * ld + k) or "turned" (at k * ld + r):
//   forward          x w^T       Q = x,           P = w
//   input gradient   dy w        Q = dy,          P = w turned
//   weight gradient  dy^T u      Q = dy turned,   P = u turned
//   gated            x w^T       Q = x,           P = w, whose first n rows are the gate's and whose last n the value's: out
//                                has n columns, of both products at once
//   gate's gradient  dy w        Q = dy,          P = w turned
// Operands are float, bfloat16 or, forward and gated, 8-bit integers, whose sums are 32-bit integers.
#pragma once
#include "cat_block.h"

namespace cat {

typedef int i32x4 __attribute__((ext_vector_type(4)));
// four sums of E's products
template <typename E>
using Sums = std::conditional_t<sizeof(E) == 1, i32x4, f32x4>;

enum GemmKind { kForward = 0, kInputGrad = 1, kWeightGrad = 2, kGated = 3, kGatedGrad = 4 };

// What happens to out on its way to memory, by kind:
//   kForward     z = out + bias; codes_out: the checkpoint of z; y = act(z) + residual
//   kInputGrad   out * act'(codes_in)
//   kWeightGrad  nothing
//   kGated       g, v = out + bias (2 n entries); codes_out: the checkpoints of g and v, one behind the other; act(g) * v
//   kGatedGrad   g, v = codes_in (as above): rows of 2 n entries, out * v * act'(g) and out * act(g); their sums over the rows
//                of a wave, or of a joining workgroup: a row of col_sums each (2 n entries)
// Sums of 8-bit integers are multiplied by row_scales (of q's row) and col_scales (of p's row) first.
struct Epilogue {
    void* out;
    const float* bias;
    const void* residual;
    int8_t* codes_out;
    float* scales_out;
    const int8_t* codes_in;
    const float* scales_in;
    int act;
    const float* row_scales;
    const float* col_scales;
    float* col_sums;
};

struct GemmArgs {
    const void *p, *q;
    int64_t ldp, ldq;          // entries; rows start on 16-byte boundaries
    int64_t p_bytes, q_bytes;  // what may be read from p (of a term), q on
    int64_t m, n, k;
    int64_t k_split;  // entries of k a share takes (a multiple of the kernel's step)
    int splits, k_shares;  // all shares, and those of k: where p has two terms, upper bits and rest, one behind the other, each has its own
    void* parts;  // instead of an epilogue: sums as they are, splits x m x n (gated: x 2 n), float or 32-bit integers
    bool tiled;   // those of weight gradients tile by tile, as the registers hold them (splits x tiles x TM x TN)
    Epilogue e;
};

// Tiles in the order in which the XCDs take them: eight columns at a time.
__host__ __device__ inline void tile_place(uint32_t tile, uint32_t tm, uint32_t tn, uint32_t& row, uint32_t& column) {
    const uint32_t band = tile / (8 * tm), in = tile - band * 8 * tm, width = tn - band * 8 < 8 ? tn - band * 8 : 8;
    row = in / width, column = band * 8 + in % width;
}
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
template <typename T, int KIND, int E, bool PACK, int FAST = sizeof(T) == 2>
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
            for (int i = 0; i < E; i++) v[i] = act_value<decltype(which)::value, FAST>(v[i]);
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
                    for (int i = 0; i < E; i++) v[i] *= act_grad<decltype(which)::value, FAST>(c[i]);
                });
            }
        }
    }
    st_entries<T, E>((T*)e.out + at, n, N, v);
}

// launchers of the tile kernels, one translation unit a type, the gate's gradients, which are many, in others (and not in
// launch_gemm_*); `large`: tiles of 256 x 256 (not float)
cat_status launch_gemm_f32(GemmKind kind, const GemmArgs& a, hipStream_t st);
cat_status launch_gemm_bf16(GemmKind kind, bool large, const GemmArgs& a, hipStream_t st);
cat_status launch_gate_grad_f32(const GemmArgs& a, hipStream_t st);
cat_status launch_gate_grad_bf16(bool large, const GemmArgs& a, hipStream_t st);
cat_status launch_gemm_i8(GemmKind kind, bool large, cat_dtype out, const GemmArgs& a, hipStream_t st);

}  // namespace cat
