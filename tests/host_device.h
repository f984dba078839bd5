// The few device functions and builtins that the kernels' tile ends use, for a build on the host: one lane at a time, an exchange between
// lanes gives a lane its own value back.  What is computed is not looked at there, only which addresses are formed.
#pragma once
#include <math.h>
#include <stdint.h>
#include <string.h>

#define __device__
#define __host__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
typedef void* hipStream_t;
struct uint2 { uint32_t x, y; };
struct alignas(16) uint4 { uint32_t x, y, z, w; };
struct alignas(16) float4 { float x, y, z, w; };
inline uint2 make_uint2(uint32_t x, uint32_t y) { return {x, y}; }
inline uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return {x, y, z, w}; }
inline float __uint_as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
inline uint32_t __float_as_uint(float v) { return __builtin_bit_cast(uint32_t, v); }
inline long long __double_as_longlong(double v) { return __builtin_bit_cast(long long, v); }
inline double __longlong_as_double(long long v) { return __builtin_bit_cast(double, v); }
template <typename V> inline V __shfl_xor(V v, int, int) { return v; }
inline float __fdiv_rn(float a, float b) { return a / b; }
inline float __fdividef(float a, float b) { return a / b; }
inline float __expf(float v) { return expf(v); }
#define __builtin_amdgcn_update_dpp(old, v, ...) (v)
#define __builtin_amdgcn_readlane(v, lane) (v)
#define __builtin_amdgcn_perm(hi, lo, which) ((hi) ^ (lo))
#define __builtin_amdgcn_rcpf(v) (1.f / (v))
#define __builtin_amdgcn_exp2f(v) exp2f(v)
#define __builtin_amdgcn_sched_barrier(v)
#define __builtin_amdgcn_s_barrier()
struct HostSwap {
    uint32_t a;
    uint32_t operator[](int) const { return a; }
};
#define __builtin_amdgcn_permlane16_swap(a, b, ...) (HostSwap{a})
#define __builtin_amdgcn_permlane32_swap(a, b, ...) (HostSwap{a})
struct HostIndex {
    unsigned x;
};
static HostIndex threadIdx;
