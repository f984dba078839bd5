// Every tile end of the matrix products (what a wave does with its sums), lane by lane on the host, on arrays exactly as long as their
// matrices: an access outside of one ends the program (address sanitizer), an entry that no lane writes shows.  tile_ends.inc: the functions
// out of cat_gemm_kernel.h as they are, without their empty asm statements.  Arguments: pairs of M and N (rows and columns of out).
#include <stdio.h>
#include <stdlib.h>

#include "cat_gemm.h"
namespace cat {
typedef char* lds_char;
typedef volatile uint32_t* lds_words;
#include "tile_ends.inc"
}  // namespace cat
using namespace cat;

template <typename T>
T* array(int64_t n) {  // (malloc: on a 16-byte boundary)
    T* p = (T*)malloc(n * sizeof(T));
    memset((void*)p, 0x11, n * sizeof(T));
    return p;
}
template <typename T>
void written(const T* p, int64_t n, const char* what) {
    for (int64_t i = 0; i < n; i++) {
        bool same = true;
        for (size_t b = 0; b < sizeof(T); b++) same = same && ((const unsigned char*)(p + i))[b] == 0x11;
        if (same) printf("%s: entry %lld is not written\n", what, (long long)i), exit(1);
    }
}
template <typename T, int KIND, int TM, int ACT, bool I8, bool PACK, bool RES>
void run(int64_t M, int64_t N) {
    constexpr bool GATED = KIND == kGated, GRAD = KIND == kGatedGrad;
    constexpr int TN = TM, WM = TM / 4, MT = WM / 16, WN = 128, TO = GATED ? TN / 2 : TN, WO = GATED ? 64 : WN;
    const int64_t G = (N + 127) / 128, tm = (M + TM - 1) / TM, tn = (N + TO - 1) / TO, two = GATED || GRAD ? 2 : 1;
    Epilogue e = {};
    T* out = array<T>(M * N * (GRAD ? 2 : 1));
    int8_t* codes = array<int8_t>(two * M * N);
    float* scales = array<float>(two * M * G);
    float* sums = GRAD ? array<float>(tm * 4 * 2 * N) : nullptr;
    T* residual = RES ? array<T>(M * N) : nullptr;
    e.out = out, e.residual = residual, e.act = ACT;
    if (PACK) e.codes_out = codes, e.scales_out = scales;
    else if (GRAD || KIND == kInputGrad) e.codes_in = codes, e.scales_in = scales;
    if (GRAD || KIND == kInputGrad)
        for (int64_t i = 0; i < two * M * G; i++) scales[i] = 1.f;
    for (int64_t tile_m = 0; tile_m < tm; tile_m++)
        for (int64_t tile_n = 0; tile_n < tn; tile_n++)
            for (int wave = 0; wave < 4 * (TN / WN); wave++)
                for (int lane = 0; lane < 64; lane++) {
                    threadIdx.x = wave * 64 + lane;
                    const int r = lane & 15, g = lane >> 4, wm = wave / (TN / WN), wn = wave % (TN / WN);
                    const int64_t nw = tile_n * TO + wn * WO, nl = nw + 8 * g, m = tile_m * TM + wm * WM + r;
                    f32x4 acc[MT][8];
                    for (int i = 0; i < MT * 8; i++) acc[i / 8][i % 8] = f32x4{1.5f, 2.5f, 3.5f, 4.5f};
                    if (nw >= N) continue;
                    if constexpr (GRAD) {
                        float* part = sums + (tile_m * (TM / WM) + wm) * 2 * N;
                        if (N % 8) finish_gate_grad<T, ACT, MT, false>(e, acc, m, M, nl, N, r, part);
                        else finish_gate_grad<T, ACT, MT, true>(e, acc, m, M, nl, N, r, part);
                    } else if constexpr (GATED) {
                        PackScale s[MT][2];
                        for (int i = 0; i < MT * 2; i++) s[i / 2][i % 2] = {1.f, 1.f};
                        if (nw + WO <= N && N % 8 == 0) finish_gated<T, MT, true>(e, acc, m, M, nl, N, g, PACK ? s : nullptr);
                        else finish_gated<T, MT, false>(e, acc, m, M, nl, N, g, PACK ? s : nullptr);
                    } else {  // (as the kernel chooses)
                        if (nw + WN <= N && N % 8 == 0) finish_rows<T, KIND, I8, MT, true>(e, acc, m, M, nl, N, g);
                        else if (I8 && N % 8 == 0) finish_rows<T, KIND, I8, MT, true, I8>(e, acc, m, M, nl, N, g);
                        else if (I8 && nw + WN <= N) finish_rows<T, KIND, I8, MT, true, false, !I8>(e, acc, m, M, nl, N, g);
                        else finish_rows<T, KIND, I8, MT, false>(e, acc, m, M, nl, N, g);
                    }
                }
    written(out, M * N * (GRAD ? 2 : 1), "out");
    if (GRAD) written(sums, tm * 4 * 2 * N, "sums");
    if (PACK) written(codes, two * M * N, "codes"), written(scales, two * M * G, "scales");
    free(out), free(codes), free(scales), free(sums), free(residual);
}
template <typename T, int TM>
void all(int64_t M, int64_t N) {
    run<T, kForward, TM, CAT_ACT_SILU, true, false, false>(M, N);
    run<T, kForward, TM, CAT_ACT_SILU, true, false, true>(M, N);
    run<T, kForward, TM, CAT_ACT_SILU, false, true, true>(M, N);
    run<T, kInputGrad, TM, CAT_ACT_SILU, false, false, false>(M, N);
    run<T, kWeightGrad, TM, CAT_ACT_NONE, false, false, false>(M, N);
    run<T, kGated, TM, CAT_ACT_SILU, false, false, false>(M, N);
    if (TM == 256) run<T, kGated, TM, CAT_ACT_SILU, false, true, false>(M, N);  // (smaller tiles' checkpoints: the joining kernel)
    if (N >= 8) run<T, kGatedGrad, TM, CAT_ACT_SILU, false, false, false>(M, N), run<T, kGatedGrad, TM, CAT_ACT_NONE, false, false, false>(M, N);
}
int main(int argc, char** argv) {
    for (int i = 1; i + 1 < argc; i += 2) {
        const int64_t M = atoll(argv[i]), N = atoll(argv[i + 1]);
        printf("%lld x %lld\n", (long long)M, (long long)N), fflush(stdout);
        all<uint16_t, 128>(M, N), all<uint16_t, 256>(M, N), all<float, 128>(M, N);
        run<float, kForward, 256, CAT_ACT_SILU, true, false, true>(M, N);
        run<float, kGated, 256, CAT_ACT_SILU, true, false, false>(M, N);
    }
    return 0;
}
