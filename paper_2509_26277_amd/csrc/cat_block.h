// What the operators of a transformer block's training step share (layer norm, product with epilogue, checkpoints in
// 8 bits): vector access to rows of any length, reductions over some lanes, the format of a checkpoint, activations.
#pragma once
#include <math.h>

#include <type_traits>

#include "cat_common.h"

namespace cat {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two floats to two bfloat16 values, ties to even; NaN and infinities stay what they are (one v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ void st_round(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_round(bf16_t* p, float v) { *p = (bf16_t)pack_bf16(v, 0.f); }

// 16 bytes of a row: 8 bfloat16 or 4 float entries.  Rows whose length is no whole number of such groups start anywhere
// on an element's boundary; the memory system takes 16-byte accesses there, only their address has to be declared so.
template <typename T>
constexpr int kVec = (int)(16 / sizeof(T));
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Group16 {
    uint32_t w[4];
};
template <typename T>
__device__ __forceinline__ void ld_group(const T* p, float (&v)[kVec<T>]) {
    const Group16<T> g = *(const Group16<T>*)p;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = __uint_as_float(g.w[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            v[2 * e] = __uint_as_float(g.w[e] << 16);
            v[2 * e + 1] = __uint_as_float(g.w[e] & 0xFFFF0000u);
        }
    }
}
template <typename T>
__device__ __forceinline__ void st_group(T* p, const float (&v)[kVec<T>]) {
    Group16<T> g;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; e++) g.w[e] = __float_as_uint(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) g.w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
    }
    *(Group16<T>*)p = g;
}
// the entries [j, j + kVec) of a row of D entries, zero behind its end
template <typename T>
__device__ __forceinline__ void ld_group_to(const T* row, int64_t j, int64_t D, float (&v)[kVec<T>]) {
    constexpr int V = kVec<T>;
    if (j + V <= D) {
        ld_group(row + j, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = j + e < D ? ld_elem(row + j + e) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void st_group_to(T* row, int64_t j, int64_t D, const float (&v)[kVec<T>]) {
    constexpr int V = kVec<T>;
    if (j + V <= D) {
        st_group(row + j, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; e++)
            if (j + e < D) st_round(row + j + e, v[e]);
    }
}
// V parameters from index j on (nullptr: `other`); the array itself starts on a 16-byte boundary and j is a multiple of V
template <int V>
__device__ __forceinline__ void ld_params(const float* p, int64_t j, int64_t D, float other, float (&v)[V]) {
    if (p == nullptr) {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = other;
    } else if (j + V <= D) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const float4 q = *(const float4*)(p + j + e);
            v[e] = q.x, v[e + 1] = q.y, v[e + 2] = q.z, v[e + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = j + e < D ? p[j + e] : other;
    }
}

// ---- reductions over L = 8, 16, 32 or 64 neighbouring lanes, the result in each of them ----
// Up to 16 lanes as permutations inside a row of 16 lanes, beyond that as exchanges between those rows.  All 64 lanes of
// the wave must be active.
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
    v += dpp_f32<0xB1>(v);                                    // quad_perm [1, 0, 3, 2]
    v += dpp_f32<0x4E>(v);                                    // quad_perm [2, 3, 0, 1]
    if constexpr (L >= 8) v += dpp_f32<0x141>(v);             // row_half_mirror
    if constexpr (L >= 16) v += dpp_f32<0x140>(v);            // row_mirror
    if constexpr (L >= 32) v += __shfl_xor(v, 16, kWave);
    if constexpr (L >= 64) v += __shfl_xor(v, 32, kWave);
    return v;
}
// The largest magnitude, as bits: those of finite values are ordered as integers, infinity's above them and NaN's above that,
// so a NaN stays (v_max_f32 drops it).
__device__ __forceinline__ uint32_t mag_max(uint32_t a, float v) {
    const uint32_t m = __float_as_uint(v) & 0x7FFFFFFFu;
    return a > m ? a : m;
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
    return v > o ? v : o;
}
template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    v = dpp_max<0xB1>(v);
    v = dpp_max<0x4E>(v);
    if constexpr (L >= 8) v = dpp_max<0x141>(v);
    if constexpr (L >= 16) v = dpp_max<0x140>(v);
    if constexpr (L >= 32) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, 16, kWave);
        v = v > o ? v : o;
    }
    return v;
}

// ---- checkpoints in 8 bits ----
// Groups of 128 consecutive channels of a row share a scale s = a / 127 with a the group's largest magnitude; a channel's
// code is x * (127 / a), rounded to the nearest integer (ties to even), its value code * s.  Both quotients are correctly
// rounded, so a group's codes do not depend on which kernel wrote them.  a < 2^-100 (where 127 / a comes near the largest
// float): zeros.  A NaN or an infinity makes the group's scale one, and every value of the group NaN (0 * inf too).  The
// largest float's 127th, rounded up, times 127 would be an infinity: the float below it is that group's scale.
constexpr int kPackGroup = CAT_PACK_GROUP;
struct PackScale {
    float up, step;
};
__device__ __forceinline__ PackScale pack_scale(uint32_t magnitude) {
    const float amax = __uint_as_float(magnitude);
    PackScale s;
    const bool held = !(amax < 0x1p-100f);
    s.up = held ? __fdiv_rn(127.f, amax) : 0.f;
    s.step = magnitude == 0x7F7FFFFFu ? 0x1.020406p+121f : held ? __fdiv_rn(amax, 127.f) : 0.f;
    return s;
}
// Codes in the low bytes: |x| * (127 / a) rounds to at most 127, and the sum with 1.5 * 2^23, whose last place is 1, rounds it
// to the nearest integer, ties to even, in two's complement.  (Not one fma: the product is rounded by itself.)
__device__ __forceinline__ uint32_t pack_code(float x, float up) {
#pragma clang fp contract(off)
    const float p = x * up;
    return __float_as_uint(p + 12582912.f);
}
__device__ __forceinline__ uint32_t pack_codes4(const float* v, float up) {
    const uint32_t lo = __builtin_amdgcn_perm(pack_code(v[1], up), pack_code(v[0], up), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(pack_code(v[3], up), pack_code(v[2], up), 0x04000C0Cu);
    return lo | hi;
}
__device__ __forceinline__ float code_value(uint32_t w, int e) { return (float)(int8_t)(w >> (8 * e)); }
struct __attribute__((packed, aligned(1))) Codes4 {
    uint32_t w[1];
};
struct __attribute__((packed, aligned(1))) Codes8 {
    uint32_t w[2];
};
// V codes from index j of a row on
template <int V>
__device__ __forceinline__ void st_codes(int8_t* row, int64_t j, int64_t D, const float (&v)[V], float up) {
    std::conditional_t<V == 8, Codes8, Codes4> c;
#pragma unroll
    for (int e = 0; e < V / 4; e++) c.w[e] = pack_codes4(v + 4 * e, up);
    if (j + V <= D) {
        *(decltype(c)*)(row + j) = c;
    } else {
#pragma unroll
        for (int e = 0; e < V; e++)
            if (j + e < D) row[j + e] = (int8_t)(c.w[e / 4] >> (8 * (e % 4)));
    }
}
// V values from index j of a row on, zero behind its end
template <int V>
__device__ __forceinline__ void ld_codes(const int8_t* row, int64_t j, int64_t D, float step, float (&v)[V]) {
    if (j + V <= D) {
        const std::conditional_t<V == 8, Codes8, Codes4> c = *(const std::conditional_t<V == 8, Codes8, Codes4>*)(row + j);
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = code_value(c.w[e / 4], e % 4) * step;
    } else {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = j + e < D ? (float)row[j + e] * step : 0.f;
    }
}

// ---- activations ----
// In fp32 throughout.  The saturated ends come out of the exponentials by themselves (exp -> inf gives 1 / inf = 0); a NaN
// stays, and of -infinity GELU and SiLU are -inf * 0, a NaN, whatever the type (a sum that left the floats is not hidden).
// FAST, for bfloat16 results: the epilogue of a product is bound by these instructions (its matrix cores wait), and the
// library's erf is some forty of them.
// The hardware's exponential is off by half a step of fp32 for every unit of its argument: nothing to a bfloat16 result, but 44
// half steps of a float SiLU at z = -80, which therefore takes the library's and the correctly rounded quotient (us, derivative
// of 65536 x 1000: 113 -> 121).  The other float forms keep it, being no worse for it: over [-9, 9] GELU' is off by 1.9 half
// steps of one (1.8 with an exact exponential), tanh GELU by 157 of its value (149: the rounding of its cubic argument).
template <bool HARDWARE>
__device__ __forceinline__ float logistic(float z) {
    if constexpr (HARDWARE) return __fdividef(1.f, 1.f + __expf(-z));
    else return __fdiv_rn(1.f, 1.f + expf(-z));
}
constexpr float kInvSqrt2 = 0.70710678118654752f, kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kTanhIn = 0.79788456080286536f, kTanhCube = 0.044715f;
// gelu with tanh: 0.5 z (1 + tanh u) = z * logistic(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3)
__device__ __forceinline__ float tanh_arg2(float z) { return 2.f * kTanhIn * z * fmaf(kTanhCube * z, z, 1.f); }
// The normal distribution's tail, Phi(-x) = exp(-x^2 / 2) G(x) for x >= 0: G as a polynomial of degree 7 in 1 / (1 + 0.36 x)
// without a constant term, fitted for the smallest largest relative error over [0, 14] (8.8e-7; beyond 14 the exponential is
// below the smallest float).
__device__ __forceinline__ float tail_factor(float x) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.36f, x, 1.f));
    float g = fmaf(t, 0.04705369665f, -0.17975622158f);
    g = fmaf(t, g, 0.18094301977f);
    g = fmaf(t, g, 0.02655653377f);
    g = fmaf(t, g, 0.13971675770f);
    g = fmaf(t, g, 0.14177289019f);
    g = fmaf(t, g, 0.14371301576f);
    return t * g;
}
__device__ __forceinline__ float normal_exp(float z) { return __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f); }
template <int ACT, bool FAST>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == CAT_ACT_RELU) {
        return z > 0.f ? z : (z != z ? z : 0.f);
    } else if constexpr (ACT == CAT_ACT_GELU && FAST) {  // z - z Phi(-z), or z Phi(z)
        const float x = fabsf(fminf(z, 1e30f));           // (no inf * 0 for +inf)
        return fmaf(-x, normal_exp(z) * tail_factor(x), fmaxf(z, 0.f));
    } else if constexpr (ACT == CAT_ACT_GELU) {
        return 0.5f * z * (1.f + erff(z * kInvSqrt2));
    } else if constexpr (ACT == CAT_ACT_GELU_TANH) {
        return z * logistic<true>(tanh_arg2(z));
    } else if constexpr (ACT == CAT_ACT_SILU) {
        return z * logistic<FAST>(z);
    } else {
        return z;
    }
}
template <int ACT, bool FAST>
__device__ __forceinline__ float act_grad(float z) {
    if constexpr (ACT == CAT_ACT_RELU) {
        return z > 0.f ? 1.f : (z != z ? z : 0.f);
    } else if constexpr (ACT == CAT_ACT_GELU && FAST) {  // Phi + z phi: s below zero, 1 - s above
        const float x = fminf(fabsf(z), 1e30f), s = normal_exp(z) * fmaf(-kInvSqrt2Pi, x, tail_factor(x));
        return z > 0.f ? 1.f - s : s;
    } else if constexpr (ACT == CAT_ACT_GELU) {
        return fmaf(z * kInvSqrt2Pi, __expf(-0.5f * z * z), 0.5f * (1.f + erff(z * kInvSqrt2)));
    } else if constexpr (ACT == CAT_ACT_GELU_TANH) {
        // (beyond |z| = 32 the factor p (1 - p) is zero in fp32, and z * z must not turn it into 0 * inf)
        const float p = logistic<true>(tanh_arg2(z)), c = fminf(fmaxf(z, -32.f), 32.f);
        return fmaf(c * p * (1.f - p), 2.f * kTanhIn * fmaf(3.f * kTanhCube * c, c, 1.f), p);
    } else if constexpr (ACT == CAT_ACT_SILU) {
        const float p = logistic<FAST>(z);
        return p * fmaf(z, 1.f - p, 1.f);
    } else {
        return 1.f;
    }
}
// f(std::integral_constant<int, act>) for the activation: one branch, outside the loops over entries
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case CAT_ACT_RELU: f(std::integral_constant<int, CAT_ACT_RELU>()); break;
        case CAT_ACT_GELU: f(std::integral_constant<int, CAT_ACT_GELU>()); break;
        case CAT_ACT_GELU_TANH: f(std::integral_constant<int, CAT_ACT_GELU_TANH>()); break;
        case CAT_ACT_SILU: f(std::integral_constant<int, CAT_ACT_SILU>()); break;
        default: f(std::integral_constant<int, CAT_ACT_NONE>()); break;
    }
}

// ---- checks of arguments (cat_pack.hip); `who` is the entry point's name ----
cat_status check_rows(const char* who, int64_t N, int64_t D, cat_dtype dt);  // 0 <= N, 1 <= D, known type
cat_status check_ptr(const char* who, const char* name, const void* p, bool needed);  // 16-byte aligned, and there if needed
cat_status check_act(const char* who, int act);
cat_status check_workspace(const char* who, const void* ws, size_t have, size_t need);

}  // namespace cat

// out[c] = sum over P parts of parts[p][c], c < n: to `lo` below `split`, to `hi` from there on (each nullable); cat_pack.hip
namespace cat {
cat_status launch_sum_parts(const float* parts, int P, int64_t n, int64_t split, float* lo, float* hi, hipStream_t st);
}

#define CAT_TRY(expr)                       \
    do {                                    \
        const cat_status _s = (expr);       \
        if (_s != CAT_OK) return _s;        \
    } while (0)
