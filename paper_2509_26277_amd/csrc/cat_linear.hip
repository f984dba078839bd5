// The product with bias, activation and residual in its epilogue, and its two gradients: the choice of a kernel, its
// workspace, and sums over rows.
//
//   z = x w^T + b, y = act(z) + res          2 M N K operations; reads x, w, res, writes y (and the checkpoint of z)
//   dx = (dy w) * act'(c)                    c: the checkpoint of the rows whose activation the product took
//   dw = dy^T u, u = x or act(c); db = sum over rows of dy
//
// With many rows the matrix cores bound it, with few the bytes of w: those go from memory to the matrix cores directly.
#include "cat_product.h"

namespace cat {
namespace {

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
// the row length of an operand laid out anew: whole steps of 128 bytes, so that a step of a row is one line of the caches and
// not parts of two
int64_t whole_lines(int64_t cols, int entry) {
    const int64_t v = 128 / entry;
    return (cols + v - 1) / v * v;
}

// Large or small tiles, and the shares of k, by the time that each choice is expected to take.  A CU works on a large tile or
// on one or two small ones, so `rounds` of 256 tiles follow one another, each so many steps of k (128 bytes) and an end; what the
// join of shares moves comes on top.  Measured, us a step: bfloat16 large 1.55, small 0.5 (turned operands 0.52) where two share a
// CU and 0.65 (0.7) where one has it alone; float 1.75.  A tile's end: 6, 2 and 4 us.  Sums of shares: written and read at 4 TB/s,
// and a launch.  (us, the rule's choice and what stands beside it.  bfloat16: weight gradient 4096 x 1024 over 16384 rows, large
// tiles in four shares 142, small in two 153, in one 173; input gradient 1024 x 8192 over 8192, small 132, large in two shares 141; 300 x
// 4096 over 4096, small in two shares 35, in one 42, large 51 at best; weight gradient 5000 x 2000 over 3000 rows, large 72, small
// 83.  Float: 4096 x 1000 over 512, one share 48, two 67; 300 x 4096 over 4096, five shares 122, one 257, eight 128.)
double choose_tiles(GemmKind kind, int64_t m, int64_t n, int64_t steps, int entry, bool pack, bool& large, int& splits) {
    const bool gated = kind == kGated, forward = kind == kForward || gated;
    const int64_t width = gated ? 2 * n : n;
    double best = -1.0;
    for (int l = 0; l < (entry == 4 ? 1 : 2); l++) {
        const int64_t edge = l ? 256 : 128, across = gated ? edge / 2 : edge, tiles = ((m + edge - 1) / edge) * ((n + across - 1) / across);
        const double end = entry == 4 ? 4.0 : l ? 6.0 : 2.0;
        for (int s = 1; s <= 32 && (s == 1 || steps / s >= 4); s++) {
            const int64_t rounds = (tiles * s + 255) / 256;
            const double step = entry == 4 ? 1.75 : l ? 1.55 : forward ? (rounds > 1 ? 0.5 : 0.65) : (rounds > 1 ? 0.52 : 0.7);
            const bool joined = s > 1 || (gated && pack && !l);
            const double us = rounds * (((steps + s - 1) / s) * step + end) + (joined ? 4.0 + (double)s * m * width * 2e-6 : 0.0);
            if (best < 0.0 || us < best) best = us, large = l, splits = s;
            if (rounds > 2 && s > 1) break;  // (more shares only add to what is joined)
        }
    }
    return best;
}
}  // namespace

// The launch of few rows takes 5 us and what its bytes of w take at 3.5 TB/s.  (us: gated float 4099 x 1001 over 513, 528 tiles where the
// card holds 512: 117 in one, 93 with three rows apart.)
int64_t tail_rows(GemmKind kind, int64_t m, int64_t n, int64_t k, int entry) {
    const int64_t step = 128 / entry, steps = (k + step - 1) / step, width = kind == kGated ? 2 * n : n;
    bool large;
    int splits;
    const double few = 5.0 + (double)width * k * entry / 3.5e6;
    double best = choose_tiles(kind, m, n, steps, entry, false, large, splits);
    int64_t tail = 0;
    for (int64_t edge = 128; edge <= 256; edge += 128) {
        const int64_t rest = m % edge;
        if (m < edge + rest || rest == 0 || rest > kFewRows) continue;
        const double us = few + choose_tiles(kind, m - rest, n, steps, entry, false, large, splits);
        if (us < best) best = us, tail = rest;
    }
    return tail;
}
// Up to 64 rows of x: every workgroup of the kernel for few rows reads all of them from the caches, for 16 rows of w, or of gate and
// value.  32 rows of w halve that where w is long (us, 48 rows of 8-bit integers by 2048 x 8192: 17.4 -> 15.0, 64 by 8192 x 8192: 45 -> 31; not
// where it is short, 64 by 1024 x 1024: 5.4 and 6.9); from 64 MB of w on, the tiles do it (64 by 8192 x 8192: 28, gated bfloat16 61 -> 47; 48 by
// 8192 x 2048 bfloat16, gated, not: 17.8 and 21.1).
constexpr int64_t kFewWideBytes = 1 << 24, kFewMostBytes = 1 << 26;
Plan plan(GemmKind kind, int64_t m, int64_t n, int64_t k, int64_t rows_q, int64_t cols_q, int64_t rows_p, int64_t cols_p, int entry, bool from_codes,
          bool pack, int terms, bool tiled) {
    Plan pl = {};
    pl.terms = terms;
    const int64_t step = 128 / entry;
    const int64_t bytes_w = rows_p * k * entry;  // (however far apart its rows lie: the sizes of workspace know nothing of that)
    const bool own = kind == kForward && entry > 1;  // (the products of the block's training step: as they were)
    pl.few = (kind == kForward || kind == kGated) && m <= kFewRows && (own || m <= 16 || bytes_w < kFewMostBytes);
    pl.ldq = cols_q, pl.ldp = cols_p;
    if (pl.few) {
        pl.wide = kind == kForward && entry == 1 && m > 16 && bytes_w >= kFewWideBytes;
        const int64_t wgs = pl.wide ? (n + 31) / 32 : (n + 15) / 16;
        // few rows of w: shares of k until the card is full, each at least 8 steps a wave (wide: 2, and half as many)
        int64_t s = (pl.wide ? 256 : 512) / wgs;
        const int64_t most = k / (kFewWaves * (pl.wide ? 2 : 8) * step);
        s = s < most ? s : most;
        pl.splits = (int)(s < 1 ? 1 : s > 16 ? 16 : s);
        pl.k_split = ((k + pl.splits - 1) / pl.splits + step - 1) / step * step;
        pl.splits = (int)((k + pl.k_split - 1) / pl.k_split);
    } else {
        pl.lay_q = cols_q != whole(cols_q, entry);
        pl.lay_p = from_codes || cols_p != whole(cols_p, entry);
        if (pl.lay_q) pl.ldq = whole_lines(cols_q, entry);
        if (pl.lay_p) pl.ldp = whole_lines(cols_p, entry);
        choose_tiles(kind, m, n, (k + step - 1) / step * pl.terms, entry, pack, pl.large, pl.splits);
        pl.splits = (pl.splits + pl.terms - 1) / pl.terms;  // (a term's)
        pl.k_split = ((k + pl.splits - 1) / pl.splits + step - 1) / step * step;
        if (pl.k_split < step) pl.k_split = step;
        pl.splits = (int)((k + pl.k_split - 1) / pl.k_split);
        if (pl.splits < 1) pl.splits = 1;
        pl.splits *= pl.terms;
        pl.joined = pl.splits > 1 || (kind == kGated && pack && !pl.large) || (kind == kGatedGrad && n < 8);
    }
    size_t at = 0;
    pl.at_q = at;
    if (pl.lay_q) at += up256((size_t)rows_q * pl.ldq * entry);
    pl.at_p = at;
    if (pl.lay_p) at += up256((size_t)pl.terms * rows_p * pl.ldp * entry);
    pl.at_parts = at;
    // (few rows: the checkpoint's groups of 128 columns are found by the joining kernel, whatever the number of shares)
    // (shares of a weight's gradient tile by tile: faster, us, 1024 x 4096 over 16384 rows 158 by rows, 140 so, 256 x 1000 over 8192 fp32 52 and 46;
    // where tiles reach beyond dw that is up to four times the memory, which the sizes that cat_linear_backward_* state have no room for)
    const int64_t edge = pl.large ? 256 : 128, tile_rows = (m + edge - 1) / edge * edge, tile_columns = (n + edge - 1) / edge * edge;
    pl.tiled = pl.joined && kind == kWeightGrad && (tiled || (tile_rows == m && tile_columns == n));
    if (pl.tiled) at += up256((size_t)pl.splits * tile_rows * tile_columns * 4);
    else if (pl.joined || (pl.few && (own || pack || pl.splits > 1))) at += up256((size_t)pl.splits * m * (kind == kGated ? 2 * n : n) * 4);
    pl.at_sums = at;
    if (kind == kWeightGrad) {  // sums over the rows of dy (k rows, m columns)
        const int64_t v = 16 / entry, gx = (m + 64 * v - 1) / (64 * v);
        int64_t P = 1024 / gx;
        const int64_t most = (k + 31) / 32;
        P = P < most ? P : most;
        P = P < 1 ? 1 : P > 256 ? 256 : P;
        pl.sum_rows = (k + P - 1) / P;
        if (pl.sum_rows < 1) pl.sum_rows = 1;
        pl.sum_parts = (int)((k + pl.sum_rows - 1) / pl.sum_rows);
        at += up256((size_t)(pl.sum_parts > 0 ? pl.sum_parts : 1) * m * 4);
    }
    if (kind == kGatedGrad) {  // the sums over rows of both gradients: by the tile kernel's waves, 64 or 32 rows each, or by shares
        if (pl.joined) {
            const int64_t G = (n + kPackGroup - 1) / kPackGroup, most = (m + 15) / 16;
            int64_t P = 1024 / G;
            P = P < most ? P : most;
            P = P < 1 ? 1 : P;
            pl.sum_rows = m > P ? (m + P - 1) / P : 1;
            pl.sum_parts = (int)((m + pl.sum_rows - 1) / pl.sum_rows);
        } else {
            pl.sum_parts = (int)((m + edge - 1) / edge * 4);
        }
        at += up256((size_t)pl.sum_parts * 2 * n * 4);
    }
    pl.total = at > 256 ? at : 256;
    pl.writes = at > 0;
    return pl;
}

namespace {

// The shares of k of a weight's gradient, as the tile kernel left them: a thread eight neighbouring columns of a row, which are a lane's
// of two of its tiles of 16 x 16.
template <typename T>
__global__ __launch_bounds__(256) void k_join_tiles(const float* __restrict__ parts, int splits, int64_t m, int64_t n, int edge, uint32_t tm, uint32_t tn, T* __restrict__ out) {
    const int rows = edge / 64;  // tiles of 16 rows a wave
    const int64_t tiles = (int64_t)tm * tn, each = (int64_t)edge * edge, pieces = tiles * each / 8;
    for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < pieces; p += (int64_t)gridDim.x * 256) {
        const int64_t tile = p / (each / 8);
        const int in = (int)(p - tile * (each / 8)), lane = in & 63, pair = in / 64 % 4, row16 = in / 256 % rows, wave = in / 256 / rows;
        uint32_t tile_m, tile_n;
        tile_place((uint32_t)tile, tm, tn, tile_m, tile_n);
        const int across = edge / 128, wm = wave / across, wn = wave % across;
        const int64_t row = (int64_t)tile_m * edge + wm * (edge / 4) + row16 * 16 + (lane & 15), column = (int64_t)tile_n * edge + wn * 128 + pair * 32 + (lane >> 4) * 8;
        if (row >= m || column >= n) continue;
        const float* at = parts + tile * each + ((int64_t)(wave * rows + row16) * 8 + 2 * pair) * 256 + lane * 4;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; s++) {
            const f32x4 lo = *(const f32x4*)(at + s * tiles * each), hi = *(const f32x4*)(at + s * tiles * each + 256);
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] += lo[i], v[4 + i] += hi[i];
        }
        st_entries<T, 8>(out + row * n, column, n, v);
    }
}

template <typename T>
cat_status join(GemmKind kind, const void* parts, int splits, int64_t M, int64_t N, const Epilogue& e, hipStream_t st) {
    if (kind == kForward) return join<T, T, kForward>(parts, splits, M, N, e, st);
    if (kind == kInputGrad) return join<T, T, kInputGrad>(parts, splits, M, N, e, st);
    return join<T, T, kWeightGrad>(parts, splits, M, N, e, st);
}
// bfloat16 and float products as the plan says, over operands that lie so
cat_status multiply_tiles(GemmKind kind, const Plan& pl, cat_dtype dt, const void* q, int64_t rows_q, const void* p, int64_t rows_p, int64_t m, int64_t n,
                          int64_t k, const Epilogue& e, char* ws, hipStream_t st) {
    const GemmArgs a = gemm_args(pl, entry_bytes(dt), q, rows_q, p, rows_p, m, n, k, e, ws);
    CAT_TRY(dt == CAT_F32 ? launch_gemm_f32(kind, a, st) : launch_gemm_bf16(kind, pl.large, a, st));
    if (!pl.joined) return CAT_OK;
    if (pl.tiled) {
        const int edge = pl.large ? 256 : 128;
        const uint32_t tm = (uint32_t)((m + edge - 1) / edge), tn = (uint32_t)((n + edge - 1) / edge);
        const dim3 grid(blocks_of((int64_t)tm * tn * edge * edge / 8));
        if (dt == CAT_F32)
            hipLaunchKernelGGL(k_join_tiles<float>, grid, dim3(256), 0, st, (const float*)a.parts, pl.splits, m, n, edge, tm, tn, (float*)e.out);
        else
            hipLaunchKernelGGL(k_join_tiles<bf16_t>, grid, dim3(256), 0, st, (const float*)a.parts, pl.splits, m, n, edge, tm, tn, (bf16_t*)e.out);
        CAT_LAUNCH_CHECK("k_join_tiles");
        return CAT_OK;
    }
    return dt == CAT_F32 ? join<float>(kind, a.parts, pl.splits, m, n, e, st) : join<bf16_t>(kind, a.parts, pl.splits, m, n, e, st);
}

Plan plan_forward(int64_t M, int64_t N, int64_t K, cat_dtype dt) { return plan(kForward, M, N, K, M, K, N, K, entry_bytes(dt), false); }
Plan plan_input(int64_t M, int64_t N, int64_t K, cat_dtype dt) { return plan(kInputGrad, M, K, N, M, N, N, K, entry_bytes(dt), false); }
Plan plan_weight(int64_t M, int64_t N, int64_t K, cat_dtype dt, bool from_codes, bool tiled = false) {
    return plan(kWeightGrad, N, K, M, M, N, M, K, entry_bytes(dt), from_codes, false, 1, tiled);
}

}  // namespace

cat_status check_linear(const char* who, int64_t M, int64_t N, int64_t K, cat_dtype dt) {
    CAT_TRY(check_rows(who, M, K, dt));
    CAT_TRY(check_rows(who, M, N, dt));
    const int e = entry_bytes(dt);
    if (whole(K, e) * e > kGemmMaxRowBytes || whole(N, e) * e > kGemmMaxRowBytes)
        return set_error(CAT_ERR_UNSUPPORTED, "%s: rows of %lld and %lld entries: products take rows of up to %lld bytes", who, (long long)K, (long long)N,
                         (long long)kGemmMaxRowBytes);
    return CAT_OK;
}
cat_status check_checkpoint(const char* who, const int8_t* codes, const float* scales) {
    CAT_TRY(check_ptr(who, "codes", codes, scales != nullptr));
    return check_ptr(who, "scales", scales, codes != nullptr);
}

cat_status weight_gradient(const Plan& pl, const void* dy, const void* x, const int8_t* codes, const float* scales, bool gated, int64_t M, int64_t N,
                           int64_t K, cat_dtype dt, int act, void* dw, float* dbias, char* ws, hipStream_t st) {
    const Epilogue e = {dw};
    if (M == 0) {  // (an odd number of bfloat16 entries is no whole number of words)
        if (dbias) CAT_TRY(launch_fill_zero(dbias, (size_t)N * 4, st));
        return dt == CAT_F32 ? join<float, float, kWeightGrad>(nullptr, 0, N, K, e, st) : join<bf16_t, bf16_t, kWeightGrad>(nullptr, 0, N, K, e, st);
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
    CAT_TRY(lay_out(dt, pl, dy, M, N, x, codes, scales, gated, act, M, K, ws, st));
    return multiply_tiles(kWeightGrad, pl, dt, pl.lay_q ? ws + pl.at_q : dy, M, pl.lay_p ? ws + pl.at_p : x, M, N, K, M, e, ws, st);
}

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
    if (pl.few) return dt == CAT_F32 ? few_rows<float, float, false>(pl, x, K, w, K, M, N, K, e, ws, st) : few_rows<bf16_t, bf16_t, false>(pl, x, K, w, K, M, N, K, e, ws, st);
    CAT_TRY(lay_out(dt, pl, x, M, K, w, nullptr, nullptr, false, 0, N, K, ws, st));
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
    CAT_TRY(lay_out(dt, pl, dy, M, N, w, nullptr, nullptr, false, 0, N, K, ws, st));
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
    // (the same bits either way; x as it lies leaves the room that act of a checkpoint would take)
    Plan pl = plan_weight(M, N, K, dt, codes != nullptr, true);
    if (pl.total > workspace_bytes) pl = plan_weight(M, N, K, dt, codes != nullptr);
    CAT_TRY(check_workspace(who, workspace, workspace_bytes, pl.total));
    return weight_gradient(pl, dy, x, codes, scales, false, M, N, K, dt, (int)act, dw, dbias, (char*)workspace, (hipStream_t)hip_stream);
}

}  // extern "C"
