// Checkpoints in 8 bits: rows to codes and back, and the gradient of an activation whose argument is held so.  The checks
// of arguments that the block's operators share are here too.  Kernels, launchers and entry points.
//
// Measured: 65536 x 1000 fp32 to codes 75 us (4.4 TB/s), back 60 (5.5); 16384 x 4096 bf16 back 36 (5.6).
// All three are one pass over memory and bound by it: a thread holds one 16-byte group of a row (8 bfloat16 or 4 float
// entries), so a scale's 128 channels are 16 or 32 neighbouring lanes, whose largest magnitude is found by lane exchanges.
// The threads of a launch go through (row, scale group, part) in that order, so short last groups cost the lanes behind a
// row's end and nothing else.
#include "cat_block.h"

namespace cat {

cat_status check_rows(const char* who, int64_t N, int64_t D, cat_dtype dt) {
    if (dt != CAT_F32 && dt != CAT_BF16) return set_error(CAT_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    if (N < 0 || N >= (1ll << 31) || D < 1 || D >= (1ll << 31))
        return set_error(CAT_ERR_INVALID_ARG, "%s: need 0 <= rows < 2^31 and 1 <= row length < 2^31 (got %lld and %lld)", who,
                         (long long)N, (long long)D);
    return CAT_OK;
}
cat_status check_ptr(const char* who, const char* name, const void* p, bool needed) {
    if (!p) return needed ? set_error(CAT_ERR_INVALID_ARG, "%s: %s is NULL", who, name) : CAT_OK;
    if ((uintptr_t)p % 16) return set_error(CAT_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", who, name);
    return CAT_OK;
}
cat_status check_act(const char* who, int act) {
    if (act < CAT_ACT_NONE || act > CAT_ACT_SILU) return set_error(CAT_ERR_INVALID_ARG, "%s: unknown activation %d", who, act);
    return CAT_OK;
}
cat_status check_workspace(const char* who, const void* ws, size_t have, size_t need) {
    if (!ws) return set_error(CAT_ERR_WORKSPACE, "%s: workspace is NULL (need %zu bytes)", who, need);
    if ((uintptr_t)ws % 256) return set_error(CAT_ERR_WORKSPACE, "%s: workspace is not 256-byte aligned", who);
    if (have < need) return set_error(CAT_ERR_WORKSPACE, "%s: workspace has %zu bytes, need %zu", who, have, need);
    return CAT_OK;
}

// Sums of the workgroups' parts (P x n), columns below `split` to `lo`, the others to `hi`: a workgroup 32 columns at a time, its
// 32 half-waves every 32nd part each, a fixed order.  (512 parts of 2048 columns: see the measurements in the norm's file)
__global__ __launch_bounds__(1024) void k_sum_parts(const float* __restrict__ parts, int P, int64_t n, int64_t split, float* __restrict__ lo,
                                                    float* __restrict__ hi) {
    __shared__ float s[32][33];
    const int c = threadIdx.x % 32, h = threadIdx.x / 32;
    for (int64_t first = (int64_t)blockIdx.x * 32;;) {
        const int64_t at = first + c;
        float t = 0.f;
        if (at < n) {
#pragma unroll 8
            for (int p = h; p < P; p += 32) t += parts[(int64_t)p * n + at];
        }
        s[h][c] = t;
        __syncthreads();
        t = s[c][h];  // the 32 sums of a column side by side
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t += __shfl_xor(t, o, 32);
        const int64_t out = first + h;
        float* to = out < split ? lo : hi;
        if (c == 0 && out < n && to) to[out < split ? out : out - split] = t;
        first += (int64_t)gridDim.x * 32;
        if (first >= n) break;
        __syncthreads();
    }
}
// (a launch has fewer than 2^32 threads: 2^21 workgroups, further columns by stride)
cat_status launch_sum_parts(const float* parts, int P, int64_t n, int64_t split, float* lo, float* hi, hipStream_t st) {
    const int64_t blocks = (n + 31) / 32;
    hipLaunchKernelGGL(k_sum_parts, dim3((unsigned)(blocks < (1 << 21) ? blocks : 1 << 21)), dim3(1024), 0, st, parts, P, n, split, lo, hi);
    CAT_LAUNCH_CHECK("k_sum_parts");
    return CAT_OK;
}

namespace {

// What a thread of these kernels works on: the V entries from channel j of a row on, in scale group g (numbered through all
// rows).  parts = 128 / V threads share a group.
template <typename T>
struct Place {
    int64_t row, j, group;
};
template <typename T>
__device__ __forceinline__ Place<T> place_of(int64_t t, int64_t G) {
    constexpr int parts = kPackGroup / kVec<T>;
    Place<T> p;
    p.group = t / parts;
    if (p.group < (1ll << 32)) {  // a 64-bit division is some forty instructions
        p.row = (uint32_t)p.group / (uint32_t)G;
    } else {
        p.row = p.group / G;
    }
    p.j = (p.group - p.row * G) * kPackGroup + (t % parts) * kVec<T>;
    return p;
}

// Codes of 2^31 * 2^24 groups would need more workgroups than a launch has; a launch's threads go on by its size.
constexpr int64_t kPackMaxBlocks = 1 << 22;
// Places a thread of k_unpack8 reads before it writes the first.  Float rows: four codes a place are too little under way (65536 x
// 1000: 72 us with one, 61 with four).  bfloat16 rows: one (16384 x 4096: 37 us, 39 with four).
template <typename T>
constexpr int kUnpackAhead = sizeof(T) == 4 ? 4 : 1;

template <typename T>
__global__ __launch_bounds__(256) void k_pack8(const T* __restrict__ x, int64_t groups, int64_t G, int64_t D, int8_t* __restrict__ codes,
                                               float* __restrict__ scales) {
    constexpr int V = kVec<T>, parts = kPackGroup / V;
    // (whole waves stay in the loop together: groups * parts counts threads, and lanes past it only lack their stores)
    const int64_t n = groups * parts, n64 = (n + 63) & ~63ll;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < n64; t += (int64_t)gridDim.x * 256) {
        const bool mine = t < n;
        const Place<T> p = place_of<T>(mine ? t : n - 1, G);
        float v[V];
        ld_group_to(x + p.row * D, p.j, D, v);
        uint32_t a = 0;
#pragma unroll
        for (int e = 0; e < V; e++) a = mag_max(a, v[e]);
        a = lanes_max<parts>(a);
        const PackScale s = pack_scale(a);
        if (!mine) continue;
        if (p.j < D) st_codes<V>(codes + p.row * D, p.j, D, v, s.up);
        if (p.j % kPackGroup == 0) scales[p.group] = s.step;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_unpack8(const int8_t* __restrict__ codes, const float* __restrict__ scales, int64_t groups,
                                                 int64_t G, int64_t D, T* __restrict__ x) {
    constexpr int V = kVec<T>, parts = kPackGroup / V, kAhead = kUnpackAhead<T>;
    const int64_t n = groups * parts;
    for (int64_t t0 = (int64_t)blockIdx.x * 256 * kAhead + threadIdx.x; t0 < n; t0 += (int64_t)gridDim.x * 256 * kAhead) {
        Place<T> p[kAhead];
        float v[kAhead][V];
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const int64_t t = t0 + u * 256;
            p[u] = place_of<T>(t < n ? t : n - 1, G);
            if (t >= n) p[u].j = D;
            if (p[u].j < D) ld_codes<V>(codes + p[u].row * D, p[u].j, D, scales[p[u].group], v[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; u++)
            if (p[u].j < D) st_group_to(x + p[u].row * D, p[u].j, D, v[u]);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_activation_backward(const T* __restrict__ dy, const int8_t* __restrict__ codes,
                                                             const float* __restrict__ scales, int64_t groups, int64_t G, int64_t D,
                                                             int act, T* __restrict__ dz) {
    constexpr int V = kVec<T>, parts = kPackGroup / V;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < groups * parts; t += (int64_t)gridDim.x * 256) {
        const Place<T> p = place_of<T>(t, G);
        if (p.j >= D) continue;
        float d[V], z[V];
        ld_group_to(dy + p.row * D, p.j, D, d);
        ld_codes<V>(codes + p.row * D, p.j, D, scales[p.group], z);
        with_act(act, [&](auto which) {
#pragma unroll
            for (int e = 0; e < V; e++) d[e] *= act_grad<decltype(which)::value, sizeof(T) == 2>(z[e]);
        });
        st_group_to(dz + p.row * D, p.j, D, d);
    }
}

template <typename T>
dim3 pack_grid(int64_t groups, int each = 1) {
    const int64_t threads = groups * (kPackGroup / kVec<T>), blocks = (threads + 256 * each - 1) / (256 * each);
    return dim3((unsigned)(blocks < kPackMaxBlocks ? blocks : kPackMaxBlocks));
}

}  // namespace
}  // namespace cat

using namespace cat;

#define CAT_BY_TYPE(dt, CALL)               \
    do {                                    \
        if ((dt) == CAT_F32) {              \
            using T = float;                \
            CALL;                           \
        } else {                            \
            using T = bf16_t;               \
            CALL;                           \
        }                                   \
    } while (0)

extern "C" {

cat_status cat_pack8(const void* x, int64_t N, int64_t D, cat_dtype dt, int8_t* codes, float* scales, void* hip_stream) {
    const char* who = "cat_pack8";
    CAT_TRY(check_rows(who, N, D, dt));
    CAT_TRY(check_ptr(who, "x", x, N > 0));
    CAT_TRY(check_ptr(who, "codes", codes, N > 0));
    CAT_TRY(check_ptr(who, "scales", scales, N > 0));
    if (N == 0) return CAT_OK;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    CAT_BY_TYPE(dt, hipLaunchKernelGGL(k_pack8<T>, pack_grid<T>(N * G), dim3(256), 0, (hipStream_t)hip_stream, (const T*)x, N * G, G, D,
                                       codes, scales));
    CAT_LAUNCH_CHECK("k_pack8");
    return CAT_OK;
}

cat_status cat_unpack8(const int8_t* codes, const float* scales, int64_t N, int64_t D, cat_dtype dt, void* x, void* hip_stream) {
    const char* who = "cat_unpack8";
    CAT_TRY(check_rows(who, N, D, dt));
    CAT_TRY(check_ptr(who, "codes", codes, N > 0));
    CAT_TRY(check_ptr(who, "scales", scales, N > 0));
    CAT_TRY(check_ptr(who, "x", x, N > 0));
    if (N == 0) return CAT_OK;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    CAT_BY_TYPE(dt, hipLaunchKernelGGL(k_unpack8<T>, pack_grid<T>(N * G, kUnpackAhead<T>), dim3(256), 0, (hipStream_t)hip_stream, codes, scales, N * G, G,
                                       D, (T*)x));
    CAT_LAUNCH_CHECK("k_unpack8");
    return CAT_OK;
}

cat_status cat_activation_backward(const void* dy, const int8_t* codes, const float* scales, int64_t N, int64_t D, cat_dtype dt,
                                   cat_activation act, void* dz, void* hip_stream) {
    const char* who = "cat_activation_backward";
    CAT_TRY(check_rows(who, N, D, dt));
    CAT_TRY(check_act(who, act));
    CAT_TRY(check_ptr(who, "dy", dy, N > 0));
    CAT_TRY(check_ptr(who, "codes", codes, N > 0));
    CAT_TRY(check_ptr(who, "scales", scales, N > 0));
    CAT_TRY(check_ptr(who, "dz", dz, N > 0));
    if (N > 0 && dz == dy) return set_error(CAT_ERR_INVALID_ARG, "%s: dz may not alias dy", who);
    if (N == 0) return CAT_OK;
    const int64_t G = (D + kPackGroup - 1) / kPackGroup;
    CAT_BY_TYPE(dt, hipLaunchKernelGGL(k_activation_backward<T>, pack_grid<T>(N * G), dim3(256), 0, (hipStream_t)hip_stream, (const T*)dy,
                                       codes, scales, N * G, G, D, (int)act, (T*)dz));
    CAT_LAUNCH_CHECK("k_activation_backward");
    return CAT_OK;
}

}  // extern "C"
