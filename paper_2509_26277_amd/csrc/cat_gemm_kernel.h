// The tile kernel of the block's matrix products on the matrix cores (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32:
// exact products, fp32 sums).
//
// A workgroup computes TM x TN entries of out, each of its waves WM x 128.  A step takes 128 bytes of k (64 bfloat16 or 32
// float entries) of both operands into LDS by loads that go there directly (no registers, no stores; what lies outside an
// operand arrives as zeros by the bounds of its buffer), two steps' worth of LDS in turn.
//   k contiguous: 128 bytes of a row, its eight 16-byte chunks c at position c ^ (row & 7), so that the 16 rows of a
//                 fragment are read without bank conflicts; the load's lane order does the exchange.
//   turned:       the rows of k as they lie, chunk c at c ^ f(k).  bfloat16 fragments are read by ds_read_b64_tr_b16,
//                 which hands a lane four k of its column; float ones entry by entry.
// The n side is the matrix instruction's first operand: a lane then holds four neighbouring columns of one row of out, and
// a wave whole scale groups of 128 columns.  At the end each wave passes its rows, 16 at a time, through a patch of LDS of
// its own, from which a lane takes 8 neighbouring columns: loads and stores of the epilogue are whole lines.
#pragma once
#include "cat_gemm.h"

namespace cat {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
typedef __attribute__((address_space(3))) void* lds_void;
typedef __attribute__((address_space(3))) char* lds_char;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kStepBytes = 128;
constexpr uint32_t kOutside = 0x80000000u;  // an offset that no operand's buffer reaches

// One operand's way into LDS: ROWS rows (columns of a turned operand) x one step, by W waves.
template <typename T, bool TURNED, int ROWS, int W>
struct Stage {
    static constexpr int kLoads = ROWS * kStepBytes / 1024 / W;  // 1 KB a load of a wave
    static constexpr int kStep = kStepBytes / (int)sizeof(T);
    static constexpr int kRowBytes = TURNED ? ROWS * (int)sizeof(T) : kStepBytes;  // in LDS
    uint32_t off[kLoads];
    int kc;  // k contiguous: this lane's first k of a step
    const char* base;
    int64_t left, step_bytes;

    static __device__ __forceinline__ int swizzle(int k) { return sizeof(T) == 2 ? 2 * ((k + (k >> 3)) & 3) : 4 * ((k >> 2) & 3); }

    __device__ __forceinline__ void init(const void* ptr, int64_t ld, int64_t bytes, int64_t r0, int64_t rows, int64_t k0, int wave, int lane) {
        const int64_t pitch = ld * (int64_t)sizeof(T);
        const int64_t at = TURNED ? k0 * pitch + r0 * (int64_t)sizeof(T) : r0 * pitch + k0 * (int64_t)sizeof(T);
        base = (const char*)ptr + at;
        left = bytes - at;
        step_bytes = TURNED ? kStep * pitch : kStepBytes;
        kc = 0;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int byte = (wave * kLoads + i) * 1024 + lane * 16;
            const int line = byte / kRowBytes, pos = byte % kRowBytes / 16;
            if constexpr (TURNED) {
                const int c = pos ^ swizzle(line);
                off[i] = r0 + c * kVec<T> < rows ? (uint32_t)(line * pitch + c * 16) : kOutside;
            } else {
                const int c = pos ^ (line & 7);
                kc = c * kVec<T>;  // (line & 7 is the same for all loads of a lane)
                off[i] = r0 + line < rows ? (uint32_t)(line * pitch + c * 16) : kOutside;
            }
        }
    }
    // k_left: entries of k from this step on; the last step may be short
    __device__ __forceinline__ void load(lds_char lds, int wave, int64_t k_left) {
        const uint32_t n = left <= 0 ? 0u : left < (int64_t)kOutside ? (uint32_t)left : kOutside;
        auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, n, 0x00027000);
        const bool cut = !TURNED && k_left < kStep && kc >= k_left;  // (turned: rows behind the last lie behind the buffer's end)
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds + (wave * kLoads + i) * 1024), 16, cut ? kOutside : off[i], 0, 0, 0);
        base += step_bytes;
        left -= step_bytes;
    }
};

// Fragments of one operand: 16 rows x half a step.  Lane (r = lane % 16, g = lane / 16) holds bfloat16 k = 32 h + 8 g .. + 7
// or float k = 16 h + 4 g .. + 3 of row r.
template <typename T, bool TURNED, int ROWS>
struct Fragments {
    uint32_t at[TURNED ? 4 : 2];
    // tile16: the wave's first tile of 16 rows
    __device__ __forceinline__ void init(int tile16, int lane) {
        const int r = lane & 15, g = lane >> 4;
        if constexpr (!TURNED) {
#pragma unroll
            for (int h = 0; h < 2; h++) at[h] = (tile16 * 16 + r) * kStepBytes + ((h * 4 + g) ^ (r & 7)) * 16;
        } else if constexpr (sizeof(T) == 2) {
            const int f = 2 * (((r >> 2) + g) & 3);  // swizzle(k) for k = 8 g + r / 4 (+ 4, + 32)
#pragma unroll
            for (int t = 0; t < 4; t++) {
                const int tile = tile16 + t;
                at[t] = (8 * g + (r >> 2)) * (ROWS * 2) + (((2 * (tile & 3) + ((r & 3) >> 1)) ^ f) + 8 * (tile >> 2)) * 16 + (r & 1) * 8;
            }
        } else {
#pragma unroll
            for (int t = 0; t < 4; t++) {
                const int tile = tile16 + t;
                at[t] = 4 * g * (ROWS * 4) + (4 * ((tile & 3) ^ g) + 16 * (tile >> 2)) * 16 + r * 4;
            }
        }
    }
    __device__ __forceinline__ f32x4 read(lds_char lds, int t, int h) const {
        if constexpr (!TURNED) {
            return *(__attribute__((address_space(3))) f32x4*)(lds + at[h] + t * 16 * kStepBytes);
        } else if constexpr (sizeof(T) == 2) {
            const lds_char p = lds + at[t & 3] + (t >> 2) * 128 + h * 32 * (ROWS * 2);
            union {
                i16x4 s[2];
                f32x4 f;
            } u;
            u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)p);
            u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(p + 4 * (ROWS * 2)));
            return u.f;
        } else {
            const lds_char p = lds + at[t & 3] + (t >> 2) * 256 + h * 16 * (ROWS * 4);
            f32x4 f;
#pragma unroll
            for (int j = 0; j < 4; j++) f[j] = *(__attribute__((address_space(3))) float*)(p + j * (ROWS * 4));
            return f;
        }
    }
};

template <typename T>
__device__ __forceinline__ f32x4 multiply(f32x4 a, f32x4 b, f32x4 c) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
}

template <typename T, int KIND, int TM, int TN, int WM>
__global__ __launch_bounds__((TM / WM) * (TN / 128) * 64) void k_gemm(const GemmArgs a) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass does not know all of the builtins, and would leave out the kernel's stub)
    constexpr bool PT = KIND != kForward, QT = KIND == kWeightGrad;
    constexpr int WN = 128, W = (TM / WM) * (TN / WN), MT = WM / 16, NT = WN / 16;
    constexpr int kStep = kStepBytes / (int)sizeof(T);
    constexpr int kBuf = (TM + TN) * kStepBytes;
    constexpr int kPatchPitch = WN * 4 + 16, kPatch = 16 * kPatchPitch;
    static_assert(W * kPatch <= 2 * kBuf, "the waves' patches fit the stages");
    __shared__ __attribute__((aligned(1024))) char lds_mem[2 * kBuf];
    const lds_char lds = (lds_char)lds_mem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (TN / WN), wn = wave % (TN / WN);

    // Workgroups go to the eight XCDs in turn; each XCD takes a run of neighbouring tiles, eight columns of them at a time, so
    // that what its L2 holds of either operand serves many of them.
    const int64_t tm = (a.m + TM - 1) / TM, tn = (a.n + TN - 1) / TN, tiles = tm * tn;
    const int64_t b = blockIdx.x, share = tiles / 8, more = tiles % 8, x = b % 8, i = b / 8;
    const int64_t t = x * share + (x < more ? x : more) + i;
    const int64_t band = t / (8 * tm), in = t - band * 8 * tm, width = tn - band * 8 < 8 ? tn - band * 8 : 8;
    const int64_t m0 = in / width * TM, n0 = (band * 8 + in % width) * TN;

    const int64_t k0 = (int64_t)blockIdx.y * a.k_split;
    int64_t k_left = a.k - k0 < a.k_split ? a.k - k0 : a.k_split;
    Stage<T, PT, TN, W> sp;
    Stage<T, QT, TM, W> sq;
    sp.init(a.p, a.ldp, a.p_bytes, n0, a.n, k0, wave, lane);
    sq.init(a.q, a.ldq, a.q_bytes, m0, a.m, k0, wave, lane);
    Fragments<T, PT, TN> fp;
    Fragments<T, QT, TM> fq;
    fp.init(wn * NT, lane);
    fq.init(wm * MT, lane);

    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; mt++)
#pragma unroll
        for (int nt = 0; nt < NT; nt++) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};

    int cur = 0;
    if (k_left > 0) {
        sp.load(lds, wave, k_left);
        sq.load(lds + TN * kStepBytes, wave, k_left);
    }
    __syncthreads();
    for (; k_left > 0; k_left -= kStep, cur ^= kBuf) {
        if (k_left > kStep) {
            sp.load(lds + (cur ^ kBuf), wave, k_left - kStep);
            sq.load(lds + (cur ^ kBuf) + TN * kStepBytes, wave, k_left - kStep);
        }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            f32x4 p[NT], q[MT];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) p[nt] = fp.read(lds + cur, nt, h);
#pragma unroll
            for (int mt = 0; mt < MT; mt++) q[mt] = fq.read(lds + cur + TN * kStepBytes, mt, h);
#pragma unroll
            for (int mt = 0; mt < MT; mt++)
#pragma unroll
                for (int nt = 0; nt < NT; nt++) acc[mt][nt] = multiply<T>(p[nt], q[mt], acc[mt][nt]);
        }
        __syncthreads();
    }

    const int r = lane & 15, g = lane >> 4;
    if (a.splits > 1) {  // the sum of a share of k: fp32, joined by a kernel of its own
        float* part = a.parts + (int64_t)blockIdx.y * a.m * a.n;
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int64_t m = m0 + wm * WM + mt * 16 + r;
            if (m >= a.m) continue;
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                const int64_t n = n0 + wn * WN + nt * 16 + 4 * g;
                const float v[4] = {acc[mt][nt][0], acc[mt][nt][1], acc[mt][nt][2], acc[mt][nt][3]};
                if (n < a.n) st_group_to(part + m * a.n, n, a.n, v);
            }
        }
        return;
    }
    const lds_char patch = lds + wave * kPatch;
#pragma unroll 1
    for (int mt = 0; mt < MT; mt++) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) *(__attribute__((address_space(3))) f32x4*)(patch + r * kPatchPitch + nt * 64 + g * 16) = acc[0][nt];
#pragma unroll
        for (int j = 0; j + 1 < MT; j++)  // (so that the loop need not be unrolled: the epilogue is long)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) acc[j][nt] = acc[j + 1][nt];
        // the patch is the wave's own, and a wave's LDS accesses are done in order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int64_t n = n0 + wn * WN + r * 8;
#pragma unroll 1
        for (int s = 0; s < 4; s++) {
            const int64_t m = m0 + wm * WM + mt * 16 + s * 4 + g;
            const lds_char from = patch + (s * 4 + g) * kPatchPitch + r * 32;
            const f32x4 lo = *(__attribute__((address_space(3))) f32x4*)from, hi = *(__attribute__((address_space(3))) f32x4*)(from + 16);
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            finish<T, KIND, 8, true>(a.e, m, n, a.n, m < a.m, v);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
#endif
}

template <typename T, int KIND, int TM, int TN, int WM>
cat_status launch_gemm_tiles(const GemmArgs& a, hipStream_t st) {
    const int64_t tiles = ((a.m + TM - 1) / TM) * ((a.n + TN - 1) / TN);
    if (tiles >= (1ll << 31)) return set_error(CAT_ERR_UNSUPPORTED, "product of %lld x %lld entries has too many tiles", (long long)a.m, (long long)a.n);
    hipLaunchKernelGGL((k_gemm<T, KIND, TM, TN, WM>), dim3((unsigned)tiles, (unsigned)a.splits), dim3((TM / WM) * (TN / 128) * 64), 0, st, a);
    CAT_LAUNCH_CHECK("k_gemm");
    return CAT_OK;
}

}  // namespace cat
