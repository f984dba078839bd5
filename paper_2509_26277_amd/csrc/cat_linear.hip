// The product with bias, activation and residual in its epilogue, and its two gradients: the choice of a kernel, its
// workspace, and the kernels beside the tile kernel (few rows, joining shares of k, operands laid out anew, sums over rows).
//
//   z = x w^T + b, y = act(z) + res          2 M N K operations; reads x, w, res, writes y (and the checkpoint of z)
//   dx = (dy w) * act'(c)                    c: the checkpoint of the rows whose activation the product took
//   dw = dy^T u, u = x or act(c); db = sum over rows of dy
//
// With many rows the matrix cores bound it, with few the bytes of w: those go from memory to the matrix cores directly.
#include "cat_gemm.h"

namespace cat {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- few rows ----
// A workgroup takes 16 rows of w, its waves shares of k (blockIdx.y: shares of it).  w goes through the registers in the
// layout of the matrix instruction's first operand, 64 bytes of a row a load; rows of x are the second operand, from the
// caches.  The waves' sums meet in LDS.  (One row, 8192 x 2048 bf16: 8.4 us, 4.0 TB/s of w; the bytes alone 6.5.)
constexpr int kFewWaves = 4;
template <typename T>
__device__ __forceinline__ f32x4 few_load(const T* row, int64_t k, int64_t K) {
    if (k + kVec<T> <= K) {
        const Group16<T> g = *(const Group16<T>*)(row + k);
        return f32x4{__uint_as_float(g.w[0]), __uint_as_float(g.w[1]), __uint_as_float(g.w[2]), __uint_as_float(g.w[3])};
    }
    union {
        T t[kVec<T>];
        f32x4 f;
    } u;
#pragma unroll
    for (int e = 0; e < kVec<T>; e++) u.t[e] = k + e < K ? row[k + e] : (T)0;
    return u.f;
}
template <typename T>
__device__ __forceinline__ f32x4 few_multiply(f32x4 a, f32x4 b, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
}
template <typename T, int MB>
__global__ __launch_bounds__(kFewWaves * kWave) void k_few_rows(const T* __restrict__ x, const T* __restrict__ w, int64_t M, int64_t N, int64_t K,
                                                                int64_t k_split, float* __restrict__ parts, const Epilogue e) {
    constexpr int kStep = 4 * kVec<T>, U = MB == 1 ? 8 : 4;
    __shared__ f32x4 sums[kFewWaves][MB][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int64_t n = n0 + r < N ? n0 + r : N - 1;
    const T* wr = w + n * K;
    const T* xr[MB];
#pragma unroll
    for (int b = 0; b < MB; b++) xr[b] = x + (b * 16 + r < M ? b * 16 + r : M - 1) * K;
    f32x4 acc[MB];
#pragma unroll
    for (int b = 0; b < MB; b++) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int64_t s0 = (int64_t)blockIdx.y * k_split, s1 = s0 + k_split < K ? s0 + k_split : K;
    const int64_t mine = ((s1 - s0 + kFewWaves - 1) / kFewWaves + kStep - 1) / kStep * kStep;
    int64_t k = s0 + wave * mine;
    const int64_t end = k + mine < s1 ? k + mine : s1;
    for (; k + U * kStep <= end; k += U * kStep) {
        f32x4 a[U], b[U][MB];
#pragma unroll
        for (int u = 0; u < U; u++) {
            a[u] = few_load(wr, k + u * kStep + g * kVec<T>, K);
#pragma unroll
            for (int j = 0; j < MB; j++) b[u][j] = few_load(xr[j], k + u * kStep + g * kVec<T>, K);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int j = 0; j < MB; j++) acc[j] = few_multiply<T>(a[u], b[u][j], acc[j]);
    }
    // (only the last share ends inside a step, at the rows' end, where few_load gives zeros)
    for (; k < end; k += kStep) {
        const f32x4 a = few_load(wr, k + g * kVec<T>, K);
#pragma unroll
        for (int j = 0; j < MB; j++) acc[j] = few_multiply<T>(a, few_load(xr[j], k + g * kVec<T>, K), acc[j]);
    }
#pragma unroll
    for (int j = 0; j < MB; j++) sums[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave >= MB) return;
    const f32x4 s = (sums[0][wave][lane] + sums[1][wave][lane]) + (sums[2][wave][lane] + sums[3][wave][lane]);
    float v[4] = {s[0], s[1], s[2], s[3]};
    const int64_t m = wave * 16 + r, nn = n0 + 4 * g;
    if (parts) {
        if (m < M && nn < N) st_group_to(parts + ((int64_t)blockIdx.y * M + m) * N, nn, N, v);
    } else {
        finish<T, kForward, 4, false>(e, m, nn, N, m < M, v);
    }
}

// ---- shares of k joined, and the epilogue ----
template <typename T, int KIND>
__global__ __launch_bounds__(256) void k_join(const float* __restrict__ parts, int splits, int64_t M, int64_t N, int64_t groups, const Epilogue e) {
    const int64_t G = (N + kPackGroup - 1) / kPackGroup, n16 = groups * 16, n64 = (n16 + 63) & ~63ll;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < n64; t += (int64_t)gridDim.x * 256) {
        const int64_t gr = t < n16 ? t / 16 : groups - 1, m = gr / G, n = (gr - m * G) * kPackGroup + (t & 15) * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (n < N)
            for (int s = 0; s < splits; s++) {
                float p[8];
                ld_entries<float, 8>(parts + ((int64_t)s * M + m) * N, n, N, p);
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] += p[i];
            }
        finish<T, KIND, 8, true>(e, m, n, N, t < n16, v);
    }
}

// ---- operands laid out anew ----
// Rows of whole_lines() (zeros behind a row's end) from rows that are no whole 16-byte groups, or act of a checkpoint.  A launch
// takes up to two operands, the first by the first `blocks` workgroups.
// act(c) is rounded to bfloat16 with bfloat16 rows: the matrix cores take no wider operand at their rate (the rest as a second
// operand is the product over again), and the forward product's rows, whose product is differentiated, were rounded so too.
// Relative error of dw, 4096 x 1024 over 16384 rows: 2.3e-3, of which its own rounding is 1.7e-3.  Float rows keep all of it.
template <typename T>
struct Layout {
    const T* src;
    const int8_t* codes;  // instead of src: a checkpoint, through act
    const float* scales;
    int64_t rows, cols, ld;
    T* dst;
    unsigned blocks;
};
template <typename T, bool FROM8>
__global__ __launch_bounds__(256) void k_lay_out(const Layout<T> first, const Layout<T> second, int act) {
    constexpr int V = kVec<T>;
    const bool other = blockIdx.x >= first.blocks;
    const Layout<T>& a = other ? second : first;
    const int64_t block = other ? blockIdx.x - first.blocks : blockIdx.x;
    const int64_t per = a.ld / V, n = a.rows * per, G = (a.cols + kPackGroup - 1) / kPackGroup;
    for (int64_t t = block * 256 + threadIdx.x; t < n; t += (int64_t)a.blocks * 256) {
        const int64_t row = n < (1ll << 32) ? (uint32_t)t / (uint32_t)per : t / per, j = (t - row * per) * V;
        float v[V];
        if constexpr (FROM8) {
            ld_codes<V>(a.codes + row * a.cols, j, a.cols, a.scales[row * G + j / kPackGroup], v);
            with_act(act, [&](auto which) {  // act(0) = 0 behind the row's end
#pragma unroll
                for (int e = 0; e < V; e++) v[e] = act_value<decltype(which)::value, sizeof(T) == 2>(v[e]);
            });
        } else {
            ld_group_to(a.src + row * a.cols, j, a.cols, v);
        }
        st_group(a.dst + row * a.ld + j, v);
    }
}

// ---- sums over rows ----
// A thread V neighbouring columns, four waves four rows at a time, blockIdx.y a share of the rows.
template <typename T>
__global__ __launch_bounds__(256) void k_column_sums(const T* __restrict__ x, int64_t M, int64_t N, int64_t rows, float* __restrict__ parts) {
    constexpr int V = kVec<T>;
    __shared__ float s[4][V][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t j = ((int64_t)blockIdx.x * kWave + lane) * V, m0 = (int64_t)blockIdx.y * rows, m1 = m0 + rows < M ? m0 + rows : M;
    float a[V];
#pragma unroll
    for (int e = 0; e < V; e++) a[e] = 0.f;
    if (j < N)
        for (int64_t m = m0 + wave; m < m1; m += 4) {
            float v[V];
            ld_group_to(x + m * N, j, N, v);
#pragma unroll
            for (int e = 0; e < V; e++) a[e] += v[e];
        }
#pragma unroll
    for (int e = 0; e < V; e++) s[wave][e][lane] = a[e];
    __syncthreads();
    if (wave || j >= N) return;
#pragma unroll
    for (int e = 0; e < V; e++)
        if (j + e < N) parts[(int64_t)blockIdx.y * N + j + e] = (s[0][e][lane] + s[1][e][lane]) + (s[2][e][lane] + s[3][e][lane]);
}
// ---- plans ----
constexpr int64_t kMaxBlocks = 1 << 22;
unsigned blocks_of(int64_t threads) {
    const int64_t b = (threads + 255) / 256;
    return (unsigned)(b < 1 ? 1 : b < kMaxBlocks ? b : kMaxBlocks);
}
size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
int64_t entry_bytes(cat_dtype dt) { return dt == CAT_F32 ? 4 : 2; }
int64_t whole(int64_t cols, cat_dtype dt) {
    const int64_t v = 16 / entry_bytes(dt);
    return (cols + v - 1) / v * v;
}
// the row length of an operand laid out anew: whole steps of 128 bytes, so that a step of a row is one line of the caches and
// not parts of two
int64_t whole_lines(int64_t cols, cat_dtype dt) {
    const int64_t v = 128 / entry_bytes(dt);
    return (cols + v - 1) / v * v;
}

constexpr int64_t kFewRows = 64;

struct Plan {
    bool few, large;
    int splits;
    int64_t k_split;
    int64_t ldq, ldp;          // row lengths of the operands as the kernel reads them
    bool lay_q, lay_p;         // laid out anew in the workspace
    size_t at_q, at_p, at_parts, at_sums, total;
    int sum_parts;
    int64_t sum_rows;
};
// Large or small tiles, and the shares of k, by the time that each choice is expected to take.  A CU works on a large tile or
// on one or two small ones, so `rounds` of 256 tiles follow one another, each so many steps of k (128 bytes) and an end; what the
// join of shares moves comes on top.  Measured, us a step: bfloat16 large 1.55, small 0.5 (turned operands 0.52) where two share a
// CU and 0.65 (0.7) where one has it alone; float 1.75.  A tile's end: 6, 2 and 4 us.  Sums of shares: written and read at 4 TB/s,
// and a launch.  (us, the rule's choice and what stands beside it.  bfloat16: weight gradient 4096 x 1024 over 16384 rows, large
// tiles in four shares 142, small in two 153, in one 173; input gradient 1024 x 8192 over 8192, small 132, large in two shares 141; 300 x
// 4096 over 4096, small in two shares 35, in one 42, large 51 at best; weight gradient 5000 x 2000 over 3000 rows, large 72, small
// 83.  Float: 4096 x 1000 over 512, one share 48, two 67; 300 x 4096 over 4096, five shares 122, one 257, eight 128.)
void choose_tiles(GemmKind kind, int64_t m, int64_t n, int64_t steps, cat_dtype dt, bool& large, int& splits) {
    double best = -1.0;
    for (int l = 0; l < (dt == CAT_BF16 ? 2 : 1); l++) {
        const int64_t edge = l ? 256 : 128, tiles = ((m + edge - 1) / edge) * ((n + edge - 1) / edge);
        const double end = dt == CAT_F32 ? 4.0 : l ? 6.0 : 2.0;
        for (int s = 1; s <= 32 && (s == 1 || steps / s >= 4); s++) {
            const int64_t rounds = (tiles * s + 255) / 256;
            const double step = dt == CAT_F32 ? 1.75 : l ? 1.55 : kind == kForward ? (rounds > 1 ? 0.5 : 0.65) : (rounds > 1 ? 0.52 : 0.7);
            const double us = rounds * (((steps + s - 1) / s) * step + end) + (s > 1 ? 4.0 + (double)s * m * n * 2e-6 : 0.0);
            if (best < 0.0 || us < best) best = us, large = l, splits = s;
            if (rounds > 2 && s > 1) break;  // (more shares only add to what is joined)
        }
    }
}
// q: rows_q x cols_q, p: rows_p x cols_p as they lie in memory; out is m x n, contracted over k
Plan plan(GemmKind kind, int64_t m, int64_t n, int64_t k, int64_t rows_q, int64_t cols_q, int64_t rows_p, int64_t cols_p, cat_dtype dt,
          bool from_codes) {
    Plan pl = {};
    const int64_t e = entry_bytes(dt), step = 128 / e;
    pl.few = kind == kForward && m <= kFewRows;
    pl.ldq = cols_q, pl.ldp = cols_p;
    if (pl.few) {
        const int64_t wgs = (n + 15) / 16;
        int64_t s = 512 / wgs;  // few rows of w: shares of k until the card is full, each at least 8 steps a wave
        const int64_t most = k / (kFewWaves * 8 * step);
        s = s < most ? s : most;
        pl.splits = (int)(s < 1 ? 1 : s > 16 ? 16 : s);
        pl.k_split = ((k + pl.splits - 1) / pl.splits + step - 1) / step * step;
        pl.splits = (int)((k + pl.k_split - 1) / pl.k_split);
    } else {
        pl.lay_q = cols_q != whole(cols_q, dt);
        pl.lay_p = from_codes || cols_p != whole(cols_p, dt);
        if (pl.lay_q) pl.ldq = whole_lines(cols_q, dt);
        if (pl.lay_p) pl.ldp = whole_lines(cols_p, dt);
        choose_tiles(kind, m, n, (k + step - 1) / step, dt, pl.large, pl.splits);
        pl.k_split = ((k + pl.splits - 1) / pl.splits + step - 1) / step * step;
        if (pl.k_split < step) pl.k_split = step;
        pl.splits = (int)((k + pl.k_split - 1) / pl.k_split);
        if (pl.splits < 1) pl.splits = 1;
    }
    size_t at = 0;
    pl.at_q = at;
    if (pl.lay_q) at += up256((size_t)rows_q * pl.ldq * e);
    pl.at_p = at;
    if (pl.lay_p) at += up256((size_t)rows_p * pl.ldp * e);
    pl.at_parts = at;
    // (few rows: the checkpoint's groups of 128 columns are found by the joining kernel, whatever the number of shares)
    if (pl.splits > 1 || pl.few) at += up256((size_t)pl.splits * m * n * 4);
    pl.at_sums = at;
    if (kind == kWeightGrad) {  // sums over the rows of dy (k rows, m columns)
        const int64_t v = 16 / e, gx = (m + 64 * v - 1) / (64 * v);
        int64_t P = 1024 / gx;
        const int64_t most = (k + 31) / 32;
        P = P < most ? P : most;
        P = P < 1 ? 1 : P > 256 ? 256 : P;
        pl.sum_rows = (k + P - 1) / P;
        if (pl.sum_rows < 1) pl.sum_rows = 1;
        pl.sum_parts = (int)((k + pl.sum_rows - 1) / pl.sum_rows);
        at += up256((size_t)(pl.sum_parts > 0 ? pl.sum_parts : 1) * m * 4);
    }
    pl.total = at > 256 ? at : 256;
    return pl;
}
Plan plan_forward(int64_t M, int64_t N, int64_t K, cat_dtype dt) { return plan(kForward, M, N, K, M, K, N, K, dt, false); }
Plan plan_input(int64_t M, int64_t N, int64_t K, cat_dtype dt) { return plan(kInputGrad, M, K, N, M, N, N, K, dt, false); }
Plan plan_weight(int64_t M, int64_t N, int64_t K, cat_dtype dt, bool from_codes) {
    return plan(kWeightGrad, N, K, M, M, N, M, K, dt, from_codes);
}

template <typename T>
Layout<T> layout_of(const void* src, const int8_t* codes, const float* scales, int64_t rows, int64_t cols, int64_t ld, void* dst) {
    return {(const T*)src, codes, scales, rows, cols, ld, (T*)dst, blocks_of(rows * (ld / kVec<T>))};
}
// q and p as the plan has them, those that lie otherwise; p from a checkpoint if codes are given
template <typename T>
cat_status lay_out(const Plan& pl, const void* q, int64_t rows_q, int64_t cols_q, const void* p, const int8_t* codes, const float* scales, int act,
                   int64_t rows_p, int64_t cols_p, char* ws, hipStream_t st) {
    const Layout<T> lq = layout_of<T>(q, nullptr, nullptr, rows_q, cols_q, pl.ldq, ws + pl.at_q);
    const Layout<T> lp = layout_of<T>(p, codes, scales, rows_p, cols_p, pl.ldp, ws + pl.at_p), none = {};
    if (pl.lay_p && codes) {
        hipLaunchKernelGGL((k_lay_out<T, true>), dim3(lp.blocks), dim3(256), 0, st, lp, none, act);
        CAT_LAUNCH_CHECK("k_lay_out");
    }
    const bool more = pl.lay_p && !codes;
    if (pl.lay_q || more) {
        const Layout<T>& first = pl.lay_q ? lq : lp;
        const Layout<T>& second = pl.lay_q && more ? lp : none;
        hipLaunchKernelGGL((k_lay_out<T, false>), dim3(first.blocks + second.blocks), dim3(256), 0, st, first, second, 0);
        CAT_LAUNCH_CHECK("k_lay_out");
    }
    return CAT_OK;
}
cat_status lay_out(cat_dtype dt, const Plan& pl, const void* q, int64_t rows_q, int64_t cols_q, const void* p, const int8_t* codes,
                   const float* scales, int act, int64_t rows_p, int64_t cols_p, char* ws, hipStream_t st) {
    return dt == CAT_F32 ? lay_out<float>(pl, q, rows_q, cols_q, p, codes, scales, act, rows_p, cols_p, ws, st)
                         : lay_out<bf16_t>(pl, q, rows_q, cols_q, p, codes, scales, act, rows_p, cols_p, ws, st);
}

template <typename T, int KIND>
cat_status join(const float* parts, int splits, int64_t M, int64_t N, const Epilogue& e, hipStream_t st) {
    const int64_t groups = M * ((N + kPackGroup - 1) / kPackGroup);
    hipLaunchKernelGGL((k_join<T, KIND>), dim3(blocks_of(groups * 16)), dim3(256), 0, st, parts, splits, M, N, groups, e);
    CAT_LAUNCH_CHECK("k_join");
    return CAT_OK;
}
template <typename T>
cat_status join(GemmKind kind, const float* parts, int splits, int64_t M, int64_t N, const Epilogue& e, hipStream_t st) {
    if (kind == kForward) return join<T, kForward>(parts, splits, M, N, e, st);
    if (kind == kInputGrad) return join<T, kInputGrad>(parts, splits, M, N, e, st);
    return join<T, kWeightGrad>(parts, splits, M, N, e, st);
}

// the tile kernel over operands that lie as the plan says
cat_status multiply_tiles(GemmKind kind, const Plan& pl, cat_dtype dt, const void* q, int64_t rows_q, const void* p, int64_t rows_p, int64_t m, int64_t n,
                          int64_t k, const Epilogue& e, char* ws, hipStream_t st) {
    GemmArgs a = {};
    a.q = q, a.p = p, a.ldq = pl.ldq, a.ldp = pl.ldp;
    a.q_bytes = rows_q * pl.ldq * entry_bytes(dt), a.p_bytes = rows_p * pl.ldp * entry_bytes(dt);
    a.m = m, a.n = n, a.k = k, a.k_split = pl.k_split, a.splits = pl.splits, a.parts = (float*)(ws + pl.at_parts), a.e = e;
    CAT_TRY(dt == CAT_F32 ? launch_gemm_f32(kind, a, st) : launch_gemm_bf16(kind, pl.large, a, st));
    if (pl.splits == 1) return CAT_OK;
    return dt == CAT_F32 ? join<float>(kind, a.parts, pl.splits, m, n, e, st) : join<bf16_t>(kind, a.parts, pl.splits, m, n, e, st);
}

template <typename T>
cat_status few_rows(const Plan& pl, const void* x, const void* w, int64_t M, int64_t N, int64_t K, const Epilogue& e, char* ws, hipStream_t st) {
    const dim3 grid((unsigned)((N + 15) / 16), (unsigned)pl.splits), block(kFewWaves * kWave);
    float* parts = pl.splits > 1 || e.codes_out ? (float*)(ws + pl.at_parts) : nullptr;
    if (M <= 16)
        hipLaunchKernelGGL((k_few_rows<T, 1>), grid, block, 0, st, (const T*)x, (const T*)w, M, N, K, pl.k_split, parts, e);
    else if (M <= 32)
        hipLaunchKernelGGL((k_few_rows<T, 2>), grid, block, 0, st, (const T*)x, (const T*)w, M, N, K, pl.k_split, parts, e);
    else
        hipLaunchKernelGGL((k_few_rows<T, 4>), grid, block, 0, st, (const T*)x, (const T*)w, M, N, K, pl.k_split, parts, e);
    CAT_LAUNCH_CHECK("k_few_rows");
    return parts ? join<T, kForward>(parts, pl.splits, M, N, e, st) : CAT_OK;
}

cat_status check_linear(const char* who, int64_t M, int64_t N, int64_t K, cat_dtype dt) {
    CAT_TRY(check_rows(who, M, K, dt));
    CAT_TRY(check_rows(who, M, N, dt));
    if (whole(K, dt) * entry_bytes(dt) > kGemmMaxRowBytes || whole(N, dt) * entry_bytes(dt) > kGemmMaxRowBytes)
        return set_error(CAT_ERR_UNSUPPORTED, "%s: rows of %lld and %lld entries: products take rows of up to %lld bytes", who, (long long)K, (long long)N,
                         (long long)kGemmMaxRowBytes);
    return CAT_OK;
}
cat_status check_checkpoint(const char* who, const int8_t* codes, const float* scales) {
    CAT_TRY(check_ptr(who, "codes", codes, scales != nullptr));
    return check_ptr(who, "scales", scales, codes != nullptr);
}

}  // namespace
}  // namespace cat

using namespace cat;

extern "C" {

size_t cat_linear_workspace_bytes(int64_t M, int64_t N, int64_t K, cat_dtype dt) {
    if (check_linear("cat_linear_workspace_bytes", M, N, K, dt) != CAT_OK) return 0;
    return plan_forward(M, N, K, dt).total;
}

cat_status cat_linear(const void* x, const void* w, const float* bias, const void* residual, int64_t M, int64_t N, int64_t K, cat_dtype dt,
                      cat_activation act, void* y, int8_t* codes, float* scales, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "cat_linear";
    CAT_TRY(check_linear(who, M, N, K, dt));
    CAT_TRY(check_act(who, act));
    CAT_TRY(check_ptr(who, "x", x, M > 0));
    CAT_TRY(check_ptr(who, "w", w, true));
    CAT_TRY(check_ptr(who, "bias", bias, false));
    CAT_TRY(check_ptr(who, "residual", residual, false));
    CAT_TRY(check_ptr(who, "y", y, M > 0));
    CAT_TRY(check_checkpoint(who, codes, scales));
    if (M > 0 && (y == x || y == w || y == residual)) return set_error(CAT_ERR_INVALID_ARG, "%s: y may not alias an input", who);
    const Plan pl = plan_forward(M, N, K, dt);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    if (M == 0) return CAT_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    char* ws = (char*)workspace;
    const Epilogue e = {y, bias, residual, codes, scales, nullptr, nullptr, (int)act};
    if (pl.few) return dt == CAT_F32 ? few_rows<float>(pl, x, w, M, N, K, e, ws, st) : few_rows<bf16_t>(pl, x, w, M, N, K, e, ws, st);
    CAT_TRY(lay_out(dt, pl, x, M, K, w, nullptr, nullptr, 0, N, K, ws, st));
    return multiply_tiles(kForward, pl, dt, pl.lay_q ? ws + pl.at_q : x, M, pl.lay_p ? ws + pl.at_p : w, N, M, N, K, e, ws, st);
}

size_t cat_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, cat_dtype dt) {
    if (check_linear("cat_linear_backward_workspace_bytes", M, N, K, dt) != CAT_OK) return 0;
    const size_t a = plan_input(M, N, K, dt).total, b = plan_weight(M, N, K, dt, true).total;
    return a > b ? a : b;
}

cat_status cat_linear_backward_input(const void* dy, const void* w, const int8_t* codes, const float* scales, int64_t M, int64_t N, int64_t K,
                                     cat_dtype dt, cat_activation act, void* dx, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* who = "cat_linear_backward_input";
    CAT_TRY(check_linear(who, M, N, K, dt));
    CAT_TRY(check_act(who, act));
    CAT_TRY(check_ptr(who, "dy", dy, M > 0));
    CAT_TRY(check_ptr(who, "w", w, true));
    CAT_TRY(check_checkpoint(who, codes, scales));
    CAT_TRY(check_ptr(who, "dx", dx, M > 0));
    if (M > 0 && act != CAT_ACT_NONE && !codes) return set_error(CAT_ERR_INVALID_ARG, "%s: an activation needs the checkpoint of its argument", who);
    if (M > 0 && (dx == dy || dx == w)) return set_error(CAT_ERR_INVALID_ARG, "%s: dx may not alias an input", who);
    const Plan pl = plan_input(M, N, K, dt);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    if (M == 0) return CAT_OK;
    hipStream_t st = (hipStream_t)hip_stream;
    char* ws = (char*)workspace;
    const Epilogue e = {dx, nullptr, nullptr, nullptr, nullptr, codes, scales, (int)act};
    CAT_TRY(lay_out(dt, pl, dy, M, N, w, nullptr, nullptr, 0, N, K, ws, st));
    return multiply_tiles(kInputGrad, pl, dt, pl.lay_q ? ws + pl.at_q : dy, M, pl.lay_p ? ws + pl.at_p : w, N, M, K, N, e, ws, st);
}

cat_status cat_linear_backward_weight(const void* dy, const void* x, const int8_t* codes, const float* scales, int64_t M, int64_t N, int64_t K,
                                      cat_dtype dt, cat_activation act, void* dw, float* dbias, void* workspace, size_t workspace_bytes,
                                      void* hip_stream) {
    const char* who = "cat_linear_backward_weight";
    CAT_TRY(check_linear(who, M, N, K, dt));
    CAT_TRY(check_act(who, act));
    CAT_TRY(check_ptr(who, "dy", dy, M > 0));
    if (M > 0 && (x == nullptr) == (codes == nullptr)) return set_error(CAT_ERR_INVALID_ARG, "%s: give x or a checkpoint, one of the two", who);
    CAT_TRY(check_ptr(who, "x", x, false));
    CAT_TRY(check_checkpoint(who, codes, scales));
    CAT_TRY(check_ptr(who, "dw", dw, true));
    CAT_TRY(check_ptr(who, "dbias", dbias, false));
    if (M > 0 && act != CAT_ACT_NONE && !codes) return set_error(CAT_ERR_INVALID_ARG, "%s: an activation needs the checkpoint of its argument", who);
    if (dw == dy || dw == x) return set_error(CAT_ERR_INVALID_ARG, "%s: dw may not alias an input", who);
    const Plan pl = plan_weight(M, N, K, dt, codes != nullptr);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    hipStream_t st = (hipStream_t)hip_stream;
    char* ws = (char*)workspace;
    if (M == 0) {  // (an odd number of bfloat16 entries is no whole number of words)
        const Epilogue e = {dw, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0};
        if (dbias) CAT_TRY(launch_fill_zero(dbias, (size_t)N * 4, st));
        return dt == CAT_F32 ? join<float, kWeightGrad>(nullptr, 0, N, K, e, st) : join<bf16_t, kWeightGrad>(nullptr, 0, N, K, e, st);
    }
    if (dbias) {
        float* parts = (float*)(ws + pl.at_sums);
        const int64_t v = 16 / entry_bytes(dt);
        const dim3 grid((unsigned)((N + 64 * v - 1) / (64 * v)), (unsigned)pl.sum_parts);
        if (dt == CAT_F32)
            hipLaunchKernelGGL(k_column_sums<float>, grid, dim3(256), 0, st, (const float*)dy, M, N, pl.sum_rows, parts);
        else
            hipLaunchKernelGGL(k_column_sums<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)dy, M, N, pl.sum_rows, parts);
        CAT_LAUNCH_CHECK("k_column_sums");
        CAT_TRY(launch_sum_parts(parts, pl.sum_parts, N, N, dbias, nullptr, st));
    }
    CAT_TRY(lay_out(dt, pl, dy, M, N, x, codes, scales, (int)act, M, K, ws, st));
    const Epilogue e = {dw, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0};
    return multiply_tiles(kWeightGrad, pl, dt, pl.lay_q ? ws + pl.at_q : dy, M, pl.lay_p ? ws + pl.at_p : x, M, N, K, M, e, ws, st);
}

}  // extern "C"
