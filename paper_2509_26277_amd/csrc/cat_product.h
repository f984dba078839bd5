// What the entry points of the products share: the choice of a kernel and its workspace, and the kernels beside the tile kernel
// (few rows, joining shares of k, operands laid out anew).
#pragma once
#include "cat_gemm.h"

namespace cat {

// ---- plans (cat_linear.hip) ----
constexpr int64_t kFewRows = 64;
struct Plan {
    bool few, wide, large;     // wide: few rows of x, 32 rows of w a workgroup
    int splits, terms;         // shares, and of how many terms of p (of both, where there are two)
    bool joined, tiled;        // the tile kernel writes its sums as they are, and the joining kernel goes on with them; tile by tile
    int64_t k_split;
    int64_t ldq, ldp;          // row lengths of the operands as the kernel reads them
    bool lay_q, lay_p;         // laid out anew in the workspace
    size_t at_q, at_p, at_parts, at_sums, total;
    bool writes;               // to the workspace at all
    int sum_parts;
    int64_t sum_rows;
};
// The size that a call states.  256 bytes mean that nothing is written there, so that all calls, on whatever streams, may be given the
// same 256: one that does write, be it less, states more.
inline size_t stated(const Plan& pl) { return pl.writes && pl.total <= 256 ? 512 : pl.total; }
// q: rows_q x cols_q, p: rows_p x cols_p as they lie in memory, entries of so many bytes; out is m x n, contracted over k.
// pack: out's checkpoint is written (of a gated product: small tiles leave that to the joining kernel).  terms: of p, of a weight's
// gradient.  tiled: a weight's gradient may take the memory of whole tiles for its shares.
Plan plan(GemmKind kind, int64_t m, int64_t n, int64_t k, int64_t rows_q, int64_t cols_q, int64_t rows_p, int64_t cols_p, int entry, bool from_codes,
          bool pack = false, int terms = 1, bool tiled = false);
// How many of m rows, behind the last whole tile, are better off in the kernel for few rows (forward and gated, without a checkpoint):
// none, unless the tiles then need a round of workgroups less.
int64_t tail_rows(GemmKind kind, int64_t m, int64_t n, int64_t k, int entry);
inline int entry_bytes(cat_dtype dt) { return dt == CAT_F32 ? 4 : 2; }
// cols in whole 16-byte groups
inline int64_t whole(int64_t cols, int entry) {
    const int64_t v = 16 / entry;
    return (cols + v - 1) / v * v;
}
inline size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
constexpr int64_t kMaxBlocks = 1 << 22;
inline unsigned blocks_of(int64_t threads) {
    const int64_t b = (threads + 255) / 256;
    return (unsigned)(b < 1 ? 1 : b < kMaxBlocks ? b : kMaxBlocks);
}
cat_status check_linear(const char* who, int64_t M, int64_t N, int64_t K, cat_dtype dt);
cat_status check_checkpoint(const char* who, const int8_t* codes, const float* scales);
// the weight's gradient and the sums over the rows of dy, as cat_linear_backward_weight gives them (its checks made); gated: the
// product's input was act(gate) * value of the two checkpoints
cat_status weight_gradient(const Plan& pl, const void* dy, const void* x, const int8_t* codes, const float* scales, bool gated, int64_t M, int64_t N,
                           int64_t K, cat_dtype dt, int act, void* dw, float* dbias, char* ws, hipStream_t st);

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// W sums as they are to what the epilogue starts from; c: their first column among p's rows (gated: the value's lie behind the
// gate's).  Sums of 8-bit integers: times both scales, plus the bias.
template <typename E, int W>
__device__ __forceinline__ void scaled(const Epilogue& e, int64_t m, int64_t c, int64_t end, float (&v)[W]) {
    float b[W];
#pragma unroll
    for (int i = 0; i < W; i++) b[i] = 0.f;
    if (e.bias) ld_entries<float, W>(e.bias, c, end, b);
    if constexpr (sizeof(E) == 1) {
        float s[W];
        ld_entries<float, W>(e.col_scales, c, end, s);
        const float scale = e.row_scales[m];
#pragma unroll
        for (int i = 0; i < W; i++) v[i] = fmaf((float)(int)__float_as_uint(v[i]), scale * s[i], b[i]);
    } else {
#pragma unroll
        for (int i = 0; i < W; i++) v[i] += b[i];
    }
}
// The gated product's epilogue on W neighbouring columns, the bias added.  PACK: as in finish.
template <typename T, int W, bool PACK>
__device__ __forceinline__ void finish_gate(const Epilogue& e, int64_t m, int64_t M, int64_t n, int64_t N, bool valid, const float (&gate)[W], const float (&value)[W]) {
    if constexpr (PACK) {
        if (e.codes_out) {
            const auto part = [&](const float(&v)[W], int64_t row) {
                uint32_t a = 0;
#pragma unroll
                for (int i = 0; i < W; i++) a = mag_max(a, valid && n + i < N ? v[i] : 0.f);
                const PackScale s = pack_scale(lanes_max<kPackGroup / W>(a));
                if (valid && n < N) {
                    st_codes<W>(e.codes_out + row * N, n, N, v, s.up);
                    if (n % kPackGroup == 0) e.scales_out[row * ((N + kPackGroup - 1) / kPackGroup) + n / kPackGroup] = s.step;
                }
            };
            part(gate, m), part(value, M + m);
        }
    }
    if (!valid || n >= N) return;
    float v[W];
    with_act(e.act, [&](auto which) {
#pragma unroll
        for (int i = 0; i < W; i++) v[i] = act_value<decltype(which)::value, kFast<T>>(gate[i]) * value[i];
    });
    st_entries<T, W>((T*)e.out + m * N, n, N, v);
}

// ---- few rows ----
// A workgroup takes 16 rows of w (gated: 16 of the gate and the same 16 of the value), its waves shares of k (blockIdx.y: shares of
// it).  w goes through the registers in the layout of the matrix instruction's first operand, 64 bytes of a row a load; rows of x
// are the second operand, from the caches.  The waves' sums meet in LDS.  (One row, 8192 x 2048 bf16: 8.4 us, 4.0 TB/s of w; the
// bytes alone 6.5.)
constexpr int kFewWaves = 4;
template <typename E>
__device__ __forceinline__ f32x4 few_load(const E* row, int64_t k, int64_t K) {
    if (k + kVec<E> <= K) {
        const Group16<E> g = *(const Group16<E>*)(row + k);
        return f32x4{__uint_as_float(g.w[0]), __uint_as_float(g.w[1]), __uint_as_float(g.w[2]), __uint_as_float(g.w[3])};
    }
    union {
        E t[kVec<E>];
        f32x4 f;
    } u;
#pragma unroll
    for (int e = 0; e < kVec<E>; e++) u.t[e] = k + e < K ? row[k + e] : (E)0;
    return u.f;
}
template <typename E>
__device__ __forceinline__ Sums<E> few_multiply(f32x4 a, f32x4 b, Sums<E> c) {
    if constexpr (sizeof(E) == 1) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    } else if constexpr (sizeof(E) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
}
template <typename E, typename T, int MB, bool GATED, int R>
__global__ __launch_bounds__(kFewWaves * kWave) void k_few_rows(const E* __restrict__ x, const E* __restrict__ w, int64_t ldx, int64_t ldw, int64_t M, int64_t N,
                                                                int64_t K, int64_t k_split, void* __restrict__ parts, const Epilogue e) {
    constexpr int kStep = 4 * kVec<E>, U = MB == 1 ? 8 : 4, P = GATED ? 2 : 1, Q = P * R;
    __shared__ Sums<E> sums[kFewWaves][Q * MB][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * R);
    const E *wr[Q], *xr[MB];  // [part * R + 16 rows]
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int64_t n = n0 + q % R * 16 + r;
        wr[q] = w + (q / R * N + (n < N ? n : N - 1)) * ldw;
    }
#pragma unroll
    for (int b = 0; b < MB; b++) xr[b] = x + (b * 16 + r < M ? b * 16 + r : M - 1) * ldx;
    Sums<E> acc[Q][MB];
#pragma unroll
    for (int i = 0; i < Q * MB; i++) acc[i / MB][i % MB] = Sums<E>{0, 0, 0, 0};

    const int64_t s0 = (int64_t)blockIdx.y * k_split, s1 = s0 + k_split < K ? s0 + k_split : K;
    const int64_t mine = ((s1 - s0 + kFewWaves - 1) / kFewWaves + kStep - 1) / kStep * kStep;
    int64_t k = s0 + wave * mine;
    const int64_t end = k + mine < s1 ? k + mine : s1;
    for (; k + U * kStep <= end; k += U * kStep) {
        f32x4 a[U][Q], b[U][MB];
#pragma unroll
        for (int u = 0; u < U; u++) {
#pragma unroll
            for (int p = 0; p < Q; p++) a[u][p] = few_load(wr[p], k + u * kStep + g * kVec<E>, K);
#pragma unroll
            for (int j = 0; j < MB; j++) b[u][j] = few_load(xr[j], k + u * kStep + g * kVec<E>, K);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int j = 0; j < MB; j++)
#pragma unroll
                for (int p = 0; p < Q; p++) acc[p][j] = few_multiply<E>(a[u][p], b[u][j], acc[p][j]);
    }
    // (only the last share ends inside a step, at the rows' end, where few_load gives zeros)
    for (; k < end; k += kStep) {
        f32x4 a[Q];
#pragma unroll
        for (int p = 0; p < Q; p++) a[p] = few_load(wr[p], k + g * kVec<E>, K);
#pragma unroll
        for (int j = 0; j < MB; j++) {
            const f32x4 b = few_load(xr[j], k + g * kVec<E>, K);
#pragma unroll
            for (int p = 0; p < Q; p++) acc[p][j] = few_multiply<E>(a[p], b, acc[p][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < Q * MB; i++) sums[wave][i][lane] = acc[i / MB][i % MB];
    __syncthreads();
    // a wave finishes every fourth of the MB x R pieces of 16 rows of x by 16 rows of w
#pragma unroll
    for (int piece = wave; piece < MB * R; piece += kFewWaves) {
        const int block = piece / R, of = piece % R;
        const int64_t m = block * 16 + r, nn = n0 + of * 16 + 4 * g;
        float v[P][4];
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int i = (p * R + of) * MB + block;
            const f32x4 s = __builtin_bit_cast(f32x4, (Sums<E>)((sums[0][i][lane] + sums[1][i][lane]) + (sums[2][i][lane] + sums[3][i][lane])));
#pragma unroll
            for (int q = 0; q < 4; q++) v[p][q] = s[q];
        }
        if (m >= M || nn >= N) continue;
        if (parts) {
#pragma unroll
            for (int p = 0; p < P; p++) st_group_to((float*)parts + ((int64_t)blockIdx.y * M + m) * (P * N) + p * N, nn, N, v[p]);
        } else if constexpr (GATED) {
            scaled<E, 4>(e, m, nn, N, v[0]);
            scaled<E, 4>(e, m, N + nn, 2 * N, v[1]);
            finish_gate<T, 4, false>(e, m, M, nn, N, true, v[0], v[1]);
        } else if constexpr (sizeof(E) == 1) {
            scaled<E, 4>(e, m, nn, N, v[0]);
            Epilogue rest = e;
            rest.bias = nullptr;
            finish<T, kForward, 4, false, kFast<T>>(rest, m, nn, N, true, v[0]);
        } else {
            finish<T, kForward, 4, false>(e, m, nn, N, true, v[0]);
        }
    }
}

// ---- shares of k joined, and the epilogue ----
template <typename E, int W>
__device__ __forceinline__ void ld_parts(const float* parts, int splits, int64_t stride, int64_t n, int64_t N, float (&v)[W]) {
#pragma unroll
    for (int i = 0; i < W; i++) v[i] = 0.f;  // (0 as an integer, too)
    if (n < N)
        for (int s = 0; s < splits; s++) {
            float p[W];
            ld_entries<float, W>(parts + s * stride, n, N, p);
#pragma unroll
            for (int i = 0; i < W; i++) {
                if constexpr (sizeof(E) == 1) v[i] = __uint_as_float(__float_as_uint(v[i]) + __float_as_uint(p[i]));
                else v[i] += p[i];
            }
        }
}
template <typename E, typename T, int KIND>
__global__ __launch_bounds__(256) void k_join(const float* __restrict__ parts, int splits, int64_t M, int64_t N, int64_t groups, const Epilogue e) {
    const int64_t G = (N + kPackGroup - 1) / kPackGroup, n16 = groups * 16, n64 = (n16 + 63) & ~63ll;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < n64; t += (int64_t)gridDim.x * 256) {
        const int64_t gr = t < n16 ? t / 16 : groups - 1, m = gr / G, n = (gr - m * G) * kPackGroup + (t & 15) * 8;
        float v[8];
        if constexpr (KIND == kGated) {
            float value[8];
            ld_parts<E, 8>(parts + m * 2 * N, splits, M * 2 * N, n, N, v);
            ld_parts<E, 8>(parts + m * 2 * N + N, splits, M * 2 * N, n, N, value);
            if (n < N) scaled<E, 8>(e, m, n, N, v), scaled<E, 8>(e, m, N + n, 2 * N, value);
            finish_gate<T, 8, true>(e, m, M, n, N, t < n16, v, value);
        } else {
            ld_parts<E, 8>(parts + m * N, splits, M * N, n, N, v);
            if constexpr (sizeof(E) == 1) {
                if (n < N) scaled<E, 8>(e, m, n, N, v);
                Epilogue rest = e;
                rest.bias = nullptr;
                finish<T, KIND, 8, true, kFast<T>>(rest, m, n, N, t < n16, v);
            } else {
                finish<T, KIND, 8, true>(e, m, n, N, t < n16, v);
            }
        }
    }
}

// ---- operands laid out anew ----
// Rows of whole_lines() (zeros behind a row's end) from rows that are no whole 16-byte groups, or act of a checkpoint.  A launch
// takes up to two operands, the first by the first `blocks` workgroups.
// act(c) is rounded to bfloat16 with bfloat16 rows: the matrix cores take no wider operand at their rate (the rest as a second
// operand is the product over again), and the forward product's rows, whose product is differentiated, were rounded so too.
// Relative error of dw, 4096 x 1024 over 16384 rows: 2.3e-3, of which its own rounding is 1.7e-3.  Float rows keep all of it.
// act(g) * v, of a gate's checkpoints, is not: bfloat16 operands hold it in two terms, its upper 16 bits and what is left of it, rounded, one
// matrix behind the other, and the product is taken with both (2^-15 of a term at most; dw's error is its own rounding's, 1.66e-3, where
// one term left 2.34e-3).  An infinity has no rest.
template <typename T>
struct Layout {
    const T* src;
    const int8_t* codes;  // instead of src: a checkpoint, through act; gated: times the one behind it
    const float* scales;
    int64_t rows, cols;
    int from, ld;  // from a row of src, of dst, to the next (rows are below kGemmMaxRowBytes; 64 bytes in all, a line of the arguments each)
    T* dst;
    unsigned blocks;
};
enum { kFromRows = 0, kFromCodes = 1, kFromGated = 2 };
template <typename T, int FROM>
__global__ __launch_bounds__(256) void k_lay_out(const Layout<T> first, const Layout<T> second, int act) {
    constexpr int V = kVec<T>;
    const bool other = blockIdx.x >= first.blocks;
    const Layout<T>& a = other ? second : first;
    const int64_t block = other ? blockIdx.x - first.blocks : blockIdx.x;
    const int64_t per = a.ld / V, n = a.rows * per, G = (a.cols + kPackGroup - 1) / kPackGroup;
    for (int64_t t = block * 256 + threadIdx.x; t < n; t += (int64_t)a.blocks * 256) {
        const int64_t row = n < (1ll << 32) ? (uint32_t)t / (uint32_t)per : t / per, j = (t - row * per) * V;
        float v[V];
        if constexpr (FROM != kFromRows) {
            ld_codes<V>(a.codes + row * a.cols, j, a.cols, a.scales[row * G + j / kPackGroup], v);
            with_act(act, [&](auto which) {  // act(0) = 0 behind the row's end
#pragma unroll
                for (int e = 0; e < V; e++) v[e] = act_value<decltype(which)::value, FROM == kFromGated ? kFast<T> : sizeof(T) == 2>(v[e]);
            });
            if constexpr (FROM == kFromGated) {
                float value[V];
                ld_codes<V>(a.codes + (a.rows + row) * a.cols, j, a.cols, a.scales[(a.rows + row) * G + j / kPackGroup], value);
#pragma unroll
                for (int e = 0; e < V; e++) v[e] *= value[e];
                if constexpr (sizeof(T) == 2) {
                    float rest[V];
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        const float upper = __uint_as_float(__float_as_uint(v[e]) & 0xFFFF0000u);
                        rest[e] = fabsf(v[e]) < INFINITY ? v[e] - upper : 0.f;
                        v[e] = upper;
                    }
                    st_group(a.dst + (a.rows + row) * a.ld + j, rest);
                }
            }
        } else {
            ld_group_to(a.src + row * a.from, j, a.cols, v);
        }
        st_group(a.dst + row * a.ld + j, v);
    }
}
template <typename T>
Layout<T> layout_of(const void* src, const int8_t* codes, const float* scales, int64_t rows, int64_t cols, int64_t ld, void* dst) {
    static_assert(sizeof(Layout<T>) == 64, "");
    return {(const T*)src, codes, scales, rows, cols, (int)cols, (int)ld, (T*)dst, blocks_of(rows * (ld / kVec<T>))};
}
// q and p as the plan has them, those that lie otherwise; p from a checkpoint if codes are given
template <typename T>
cat_status lay_out(const Plan& pl, const void* q, int64_t rows_q, int64_t cols_q, const void* p, const int8_t* codes, const float* scales, bool gated, int act,
                   int64_t rows_p, int64_t cols_p, char* ws, hipStream_t st) {
    const Layout<T> lq = layout_of<T>(q, nullptr, nullptr, rows_q, cols_q, pl.ldq, ws + pl.at_q);
    const Layout<T> lp = layout_of<T>(p, codes, scales, rows_p, cols_p, pl.ldp, ws + pl.at_p), none = {};
    if (pl.lay_p && codes) {
        if (gated)
            hipLaunchKernelGGL((k_lay_out<T, kFromGated>), dim3(lp.blocks), dim3(256), 0, st, lp, none, act);
        else
            hipLaunchKernelGGL((k_lay_out<T, kFromCodes>), dim3(lp.blocks), dim3(256), 0, st, lp, none, act);
        CAT_LAUNCH_CHECK("k_lay_out");
    }
    const bool more = pl.lay_p && !codes;
    if (pl.lay_q || more) {
        const Layout<T>& first = pl.lay_q ? lq : lp;
        const Layout<T>& second = pl.lay_q && more ? lp : none;
        hipLaunchKernelGGL((k_lay_out<T, kFromRows>), dim3(first.blocks + second.blocks), dim3(256), 0, st, first, second, 0);
        CAT_LAUNCH_CHECK("k_lay_out");
    }
    return CAT_OK;
}
cat_status lay_out(cat_dtype dt, const Plan& pl, const void* q, int64_t rows_q, int64_t cols_q, const void* p, const int8_t* codes,
                   const float* scales, bool gated, int act, int64_t rows_p, int64_t cols_p, char* ws, hipStream_t st) {
    return dt == CAT_F32 ? lay_out<float>(pl, q, rows_q, cols_q, p, codes, scales, gated, act, rows_p, cols_p, ws, st)
                         : lay_out<bf16_t>(pl, q, rows_q, cols_q, p, codes, scales, gated, act, rows_p, cols_p, ws, st);
}

template <typename E, typename T, int KIND>
cat_status join(const void* parts, int splits, int64_t M, int64_t N, const Epilogue& e, hipStream_t st) {
    const int64_t groups = M * ((N + kPackGroup - 1) / kPackGroup);
    hipLaunchKernelGGL((k_join<E, T, KIND>), dim3(blocks_of(groups * 16)), dim3(256), 0, st, (const float*)parts, splits, M, N, groups, e);
    CAT_LAUNCH_CHECK("k_join");
    return CAT_OK;
}

// the tile kernel's arguments, over operands that lie as the plan says
inline GemmArgs gemm_args(const Plan& pl, int entry, const void* q, int64_t rows_q, const void* p, int64_t rows_p, int64_t m, int64_t n, int64_t k, const Epilogue& e,
                          char* ws) {
    GemmArgs a = {};
    a.k_shares = pl.splits / pl.terms;
    a.q = q, a.p = p, a.ldq = pl.ldq, a.ldp = pl.ldp;
    a.q_bytes = rows_q * pl.ldq * entry, a.p_bytes = rows_p * pl.ldp * entry;
    a.m = m, a.n = n, a.k = k, a.k_split = pl.k_split, a.splits = pl.splits, a.parts = pl.joined ? ws + pl.at_parts : nullptr, a.tiled = pl.tiled, a.e = e;
    return a;
}

template <typename E, typename T, bool GATED>
cat_status few_rows(const Plan& pl, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t M, int64_t N, int64_t K, const Epilogue& e, char* ws,
                    hipStream_t st) {
    const int64_t rows = pl.wide ? 32 : 16;
    const dim3 grid((unsigned)((N + rows - 1) / rows), (unsigned)pl.splits), block(kFewWaves * kWave);
    void* parts = pl.splits > 1 || e.codes_out ? ws + pl.at_parts : nullptr;
    const auto launch = [&](auto blocks, auto pieces) {
        hipLaunchKernelGGL((k_few_rows<E, T, decltype(blocks)::value, GATED, decltype(pieces)::value>), grid, block, 0, st, (const E*)x, (const E*)w, ldx, ldw, M,
                           N, K, pl.k_split, parts, e);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    if constexpr (sizeof(E) == 1 && !GATED) {
        if (M <= 16) launch(one, one);
        else if (M <= 32) pl.wide ? launch(two, two) : launch(two, one);
        else pl.wide ? launch(four, two) : launch(four, one);
    } else {
        M <= 16 ? launch(one, one) : M <= 32 ? launch(two, one) : launch(four, one);
    }
    CAT_LAUNCH_CHECK("k_few_rows");
    return parts ? join<E, T, GATED ? kGated : kForward>(parts, pl.splits, M, N, e, st) : CAT_OK;
}
// the last `tail` of M rows (tail_rows), in one launch
template <typename E, typename T, bool GATED>
cat_status few_tail(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t M, int64_t tail, int64_t N, int64_t K, Epilogue e, hipStream_t st) {
    const int64_t m0 = M - tail;
    e.out = (T*)e.out + m0 * N;
    if (e.residual) e.residual = (const T*)e.residual + m0 * N;
    if (e.row_scales) e.row_scales += m0;
    Plan pl = {};
    pl.splits = pl.terms = 1, pl.k_split = K;
    return few_rows<E, T, GATED>(pl, (const E*)x + m0 * ldx, ldx, w, ldw, tail, N, K, e, nullptr, st);
}

}  // namespace
}  // namespace cat
