// The tile kernel of the block's matrix products on the matrix cores (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32:
// exact products, fp32 sums).
//
// A workgroup computes TM x TN entries of out, each of its waves WM x 128.  A step takes 128 bytes of k (64 bfloat16 or 32
// float entries) of both operands into LDS by loads that go there directly (no registers, no stores; what lies outside an
// operand arrives as zeros by the bounds of its buffer), two steps' worth of LDS in turn.
//   k contiguous: 128 bytes of a row, its eight 16-byte chunks c at position c ^ key(row), so that the 16 rows of a
//                 fragment are read without bank conflicts; the load's lane order does the exchange.
//   turned:       the rows of k as they lie, chunk c at c ^ f(k).  bfloat16 fragments are read by ds_read_b64_tr_b16,
//                 which hands a lane four k of its column; float ones entry by entry.
// The n side is the matrix instruction's first operand: a lane then holds four columns of one row of out a tile, and a wave
// whole scale groups of 128 columns.  Its tiles are paired, tile 2 t taking columns 0..3, 8..11, 16..19, 24..27 of 32 and
// tile 2 t + 1 the others, so that a lane's eight columns of a pair are neighbours: the epilogue works on them where they are,
// with 16-byte loads and stores.
//
// Measured (TFLOP/s; a library product of 8192^3: bfloat16 1385, float 154).  bfloat16, tiles of 256 x 256: forward 8192^3 1400 to
// 1490, 4096^3 1370 to 1410; input gradient 8192^3 1380, weight gradient 1360 (1260 and 1220 with the places of both operands two
// chunks apart, where paired tiles met on the same banks).  Float: 2048^3 128.  The matrix cores are busy in 57 % of the cycles of
// 16384 x 8192 over 2048 with GELU, at 2.0 GHz; what comes on top of the steps is the epilogue, whose instructions they wait for:
// GELU 21 us of 16384 x 4096 over 1024 (126 without), codes 14, a derivative 40 (121 without).  (Through LDS, 16 rows at a time, a tile's epilogue took 11 to
// 27 us, as long as 8 to 16 steps of k.)
#pragma once
#include "cat_gemm.h"

namespace cat {

typedef __attribute__((address_space(3))) void* lds_void;
typedef __attribute__((address_space(3))) char* lds_char;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kStepBytes = 128;
constexpr uint32_t kOutside = 0x80000000u;  // an offset that no operand's buffer reaches

// One operand's way into LDS: ROWS rows (columns of a turned operand) x one step, by W waves.
template <typename T, bool TURNED, bool PAIRED, int ROWS, int W>
struct Stage {
    static constexpr int kLoads = ROWS * kStepBytes / 1024 / W;  // 1 KB a load of a wave
    static constexpr int kStep = kStepBytes / (int)sizeof(T);
    static constexpr int kRowBytes = TURNED ? ROWS * (int)sizeof(T) : kStepBytes;  // in LDS
    uint32_t off[kLoads];
    int kc[2];  // k contiguous: this lane's first k of a step, even and odd loads
    int64_t pitch;
    const char* base;
    int64_t left;

    static __device__ __forceinline__ int key(int row) { return (row & 3) | ((row >> 1) & 4); }
    // f(k).  A bfloat16 fragment's 16 lanes read four k of four chunks each (paired tiles: half of every chunk) or of two whole
    // ones: places 64 and 32 bytes apart keep them on banks of their own.
    static __device__ __forceinline__ int swizzle(int k) {
        return sizeof(T) == 2 ? (PAIRED ? 4 : 2) * ((k + (k >> 3)) & 3) : 4 * ((k >> 2) & 3);
    }

    // Offsets inside a tile.  Rows behind the operand's last and rows of k behind its last lie behind the buffer's end.  Columns
    // of a turned operand behind its last do not; like those rows, they only reach entries of out that are not stored.
    __device__ __forceinline__ void init(int64_t ld, int wave, int lane) {
        pitch = ld * (int64_t)sizeof(T);
        kc[0] = kc[1] = 0;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int byte = (wave * kLoads + i) * 1024 + lane * 16;
            const int line = byte / kRowBytes, pos = byte % kRowBytes / 16;
            const int c = pos ^ (TURNED ? swizzle(line) : key(line));
            if (!TURNED) kc[i & 1] = c * kVec<T>;  // (the key depends on a row's place among 16, two loads' worth)
            off[i] = (uint32_t)(line * pitch + c * 16);
        }
    }
    // where a tile's first step begins, and what may be read from there on (never nothing: a tile begins inside)
    __device__ __forceinline__ void tile(const void* ptr, int64_t bytes, int64_t r0, int64_t k0, const char*& from, int64_t& much) const {
        const int64_t at = TURNED ? k0 * pitch + r0 * (int64_t)sizeof(T) : r0 * pitch + k0 * (int64_t)sizeof(T);
        from = (const char*)ptr + at;
        much = bytes - at;
    }
    // One step's loads: begin(), then one() for each of them.  kl: entries of k in this step (the last may be short).
    __amdgpu_buffer_rsrc_t rsrc;
    bool cut[2];
    __device__ __forceinline__ void begin(int kl) {
        const uint32_t n = (uint64_t)left >> 31 ? kOutside : (uint32_t)left;
        rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, n, 0x00027000);
        // (turned: rows behind the last lie behind the buffer's end)
        cut[0] = !TURNED && kc[0] >= kl, cut[1] = !TURNED && kc[1] >= kl;
        const int64_t step = TURNED ? kStep * pitch : kStepBytes;
        base += step;
        left -= step;
    }
    __device__ __forceinline__ void one(lds_char lds, int wave, int i) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds + (wave * kLoads + i) * 1024), 16, cut[i & 1] ? kOutside : off[i], 0, 0, 0);
    }
};

// Fragments of one operand: 16 rows x half a step.  Lane (r = lane % 16, g = lane / 16) holds bfloat16 k = 32 h + 8 g .. + 7
// or float k = 16 h + 4 g .. + 3 of row r.  PAIRED: row r of tiles 2 t and 2 t + 1 is row 32 t + 8 (r / 4) + r % 4 (+ 4).
template <typename T, bool TURNED, bool PAIRED, int ROWS>
struct Fragments {
    static constexpr int kAt = TURNED || PAIRED ? 4 : 2;
    uint32_t at[kAt];
    // tile16: the wave's first tile of 16 rows (PAIRED: an even one)
    __device__ __forceinline__ void init(int tile16, int lane) {
        const int r = lane & 15, g = lane >> 4;
        using S = Stage<T, TURNED, PAIRED, ROWS, 4>;
        if constexpr (!TURNED && !PAIRED) {
#pragma unroll
            for (int h = 0; h < 2; h++) at[h] = (tile16 * 16 + r) * kStepBytes + ((h * 4 + g) ^ S::key(r)) * 16;
        } else if constexpr (!TURNED) {  // [odd tile][h]; the key of rows 8 (r / 4) + r % 4 (+ 4) is that of r / 4's parity and r % 4
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int row = 8 * (r >> 2) + (r & 3) + 4 * (i >> 1);
                at[i] = (tile16 * 16 + row) * kStepBytes + (((i & 1) * 4 + g) ^ S::key(row)) * 16;
            }
        } else if constexpr (sizeof(T) == 2 && PAIRED) {
            // turned: this lane supplies columns 8 q .. 8 q + 3 (odd tile: + 4) of 32 at k (+ 4, + 32), 8 bytes; f(k) changes the
            // place of 32 columns among 128
            const int k = 8 * (lane >> 4) + (r >> 2), q = r & 3;
#pragma unroll
            for (int i = 0; i < 4; i++) at[i] = k * (ROWS * 2) + ((4 * ((tile16 >> 1) + i) + q) ^ S::swizzle(k)) * 16;
        } else {
            // turned: columns are addressed in pieces of 4 (bfloat16, 8 bytes, supplied by one lane) or by themselves (float);
            // bits 5 and 6 of a column's place change with f(k), so tiles 0..3 of every 64 columns have an address each
#pragma unroll
            for (int t = 0; t < 4; t++) {
                const int tile = tile16 + t;
                if constexpr (sizeof(T) == 2) {
                    const int k = 8 * g + (r >> 2), q = r & 3;  // this lane supplies columns 4 q .. 4 q + 3 of the tile at k (+ 4, + 32)
                    const int col = 16 * tile + 4 * q;
                    at[t] = k * (ROWS * 2) + ((col >> 3) ^ S::swizzle(k)) * 16 + (col & 7) * 2;
                } else {
                    const int k = 4 * g;
                    const int col = PAIRED ? 32 * (tile >> 1) + 8 * (r >> 2) + (r & 3) + 4 * (tile & 1) : 16 * tile + r;
                    at[t] = k * (ROWS * 4) + ((col >> 2) ^ S::swizzle(k)) * 16 + (col & 3) * 4;
                }
            }
        }
    }
    // tiles FROM, FROM + 1 of half step H
    template <int H, int FROM, int NF>
    __device__ __forceinline__ void read2(lds_char lds, f32x4 (&f)[NF]) const {
        if constexpr (TURNED && sizeof(T) == 2 && PAIRED) {
            turned2<H * 32 * ROWS * 2, 4 * ROWS * 2, 8>((uint32_t)(uintptr_t)lds, at[FROM / 2], at[FROM / 2], f[FROM], f[FROM + 1]);
        } else if constexpr (TURNED && sizeof(T) == 2) {
            turned2<H * 32 * ROWS * 2 + (FROM >> 2) * 128, 4 * ROWS * 2, 0>((uint32_t)(uintptr_t)lds, at[FROM & 3], at[(FROM & 3) + 1], f[FROM], f[FROM + 1]);
        } else {
#pragma unroll
            for (int t = FROM; t < FROM + 2; t++) {
                if constexpr (!TURNED) {
                    const uint32_t a = PAIRED ? at[(t & 1) * 2 + H] + (t >> 1) * 32 * kStepBytes : at[H] + t * 16 * kStepBytes;
                    f[t] = *(__attribute__((address_space(3))) f32x4*)(lds + a);
                } else {
                    const lds_char p = lds + at[t & 3] + (t >> 2) * 256 + H * 16 * (ROWS * 4);
#pragma unroll
                    for (int j = 0; j < 4; j++) f[t][j] = *(__attribute__((address_space(3))) float*)(p + j * (ROWS * 4));
                }
            }
        }
    }
    template <int H, int NF>
    __device__ __forceinline__ void read(lds_char lds, f32x4 (&f)[NF]) const {
        if constexpr (TURNED && sizeof(T) == 2 && NF % 4 == 0) {
            const uint32_t base = (uint32_t)(uintptr_t)lds;
            constexpr int off = H * 32 * ROWS * 2, next = 4 * ROWS * 2;
            if constexpr (PAIRED) {
                turned4<off, next, 8>(base, at[0], at[0], at[1], at[1], f[0], f[1], f[2], f[3]);
                if constexpr (NF == 8) turned4<off, next, 8>(base, at[2], at[2], at[3], at[3], f[4], f[5], f[6], f[7]);
            } else {
                static_assert(NF == 4, "");
                turned4<off, next, 0>(base, at[0], at[1], at[2], at[3], f[0], f[1], f[2], f[3]);
            }
        } else {
            read2<H, 0>(lds, f);
            if constexpr (NF > 2) read2<H, 2>(lds, f);
            if constexpr (NF > 4) read2<H, 4>(lds, f), read2<H, 6>(lds, f);
        }
    }
    // The turning reads as blocks that end with their own wait: behind the builtin the compiler puts a wait for all loads into
    // LDS under way, the next step's among them, which was a third of the time of a gradient's step.
    // (ODD: what an odd tile's address has more)
    template <int OFF, int NEXT, int ODD>
    __device__ __forceinline__ void turned2(uint32_t base, uint32_t at0, uint32_t at1, f32x4& f0, f32x4& f1) const {
        f32x2 a0, a1, b0, b1;
        asm volatile(
            "ds_read_b64_tr_b16 %0, %4 offset:%6\n\t"
            "ds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
            "ds_read_b64_tr_b16 %2, %5 offset:%8\n\t"
            "ds_read_b64_tr_b16 %3, %5 offset:%9\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1)
            : "v"(base + at0), "v"(base + at1), "n"(OFF), "n"(OFF + NEXT), "n"(OFF + ODD), "n"(OFF + NEXT + ODD)
            : "memory");
        f0 = f32x4{a0[0], a0[1], a1[0], a1[1]}, f1 = f32x4{b0[0], b0[1], b1[0], b1[1]};
    }
    template <int OFF, int NEXT, int ODD>
    __device__ __forceinline__ void turned4(uint32_t base, uint32_t at0, uint32_t at1, uint32_t at2, uint32_t at3, f32x4& f0, f32x4& f1, f32x4& f2, f32x4& f3) const {
        f32x2 a0, a1, b0, b1, c0, c1, d0, d1;
        asm volatile(
            "ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
            "ds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
            "ds_read_b64_tr_b16 %2, %9 offset:%14\n\t"
            "ds_read_b64_tr_b16 %3, %9 offset:%15\n\t"
            "ds_read_b64_tr_b16 %4, %10 offset:%12\n\t"
            "ds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
            "ds_read_b64_tr_b16 %6, %11 offset:%14\n\t"
            "ds_read_b64_tr_b16 %7, %11 offset:%15\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1), "=&v"(c0), "=&v"(c1), "=&v"(d0), "=&v"(d1)
            : "v"(base + at0), "v"(base + at1), "v"(base + at2), "v"(base + at3), "n"(OFF), "n"(OFF + NEXT), "n"(OFF + ODD), "n"(OFF + NEXT + ODD)
            : "memory");
        f0 = f32x4{a0[0], a0[1], a1[0], a1[1]}, f1 = f32x4{b0[0], b0[1], b1[0], b1[1]};
        f2 = f32x4{c0[0], c0[1], c1[0], c1[1]}, f3 = f32x4{d0[0], d0[1], d1[0], d1[1]};
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

// The epilogue of a wave's MT x 16 rows by 128 columns.  Lane (r, g): rows m + 16 mt, columns n + 32 t .. + 7, t = 0..3, in
// acc[mt][2 t] and acc[mt][2 t + 1].  WHOLE: all columns lie inside out, whose rows are whole 16-byte groups.  Otherwise the
// eight columns are read and written where they lie (16-byte accesses on an element's boundary), entry by entry where they
// cross the row's end.
template <typename T, bool WHOLE>
__device__ __forceinline__ void ld8(const T* row, int64_t n, int64_t N, float (&v)[8]) {
    if constexpr (!WHOLE) {
        ld_entries<T, 8>(row, n, N, v);
    } else if constexpr (sizeof(T) == 2) {
        const uint4 q = *(const uint4*)(row + n);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; e++) v[2 * e] = __uint_as_float(w[e] << 16), v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    } else {
        const f32x4 lo = *(const f32x4*)(row + n), hi = *(const f32x4*)(row + n + 4);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] = lo[e], v[4 + e] = hi[e];
    }
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void st8(T* row, int64_t n, int64_t N, const float (&v)[8]) {
    if constexpr (!WHOLE) {
        st_entries<T, 8>(row, n, N, v);
    } else if constexpr (sizeof(T) == 2) {
        *(uint4*)(row + n) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
        *(f32x4*)(row + n) = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4*)(row + n + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
}
template <typename T, int KIND, int MT, bool WHOLE>
__device__ __forceinline__ void finish_rows(const Epilogue& e, f32x4 (&acc)[MT][8], int64_t m, int64_t M, int64_t n, int64_t N, int g) {
    const int64_t G = (N + kPackGroup - 1) / kPackGroup, group = n / kPackGroup;
    if constexpr (KIND == kForward) {
        if (e.codes_out) {
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                uint32_t a = 0;
#pragma unroll
                for (int nt = 0; nt < 8; nt++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (WHOLE || n + 32 * (nt >> 1) + 4 * (nt & 1) + i < N) a = mag_max(a, acc[mt][nt][i]);
                // (the four lanes of a row of out, 16 apart)
                const auto by16 = __builtin_amdgcn_permlane16_swap(a, a, false, false);
                a = by16[0] > by16[1] ? by16[0] : by16[1];
                const auto by32 = __builtin_amdgcn_permlane32_swap(a, a, false, false);
                const PackScale s = pack_scale(by32[0] > by32[1] ? by32[0] : by32[1]);
                const int64_t row = m + 16 * mt;
                if (row < M) {
#pragma unroll
                    for (int t = 0; t < 4; t++) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; i++) v[i] = acc[mt][2 * t + (i >> 2)][i & 3];
                        if constexpr (WHOLE)
                            *(uint2*)(e.codes_out + row * N + n + 32 * t) = make_uint2(pack_codes4(v, s.up), pack_codes4(v + 4, s.up));
                        else
                            st_codes<8>(e.codes_out + row * N, n + 32 * t, N, v, s.up);
                    }
                    if (g == 0) e.scales_out[row * G + group] = s.step;
                }
                __builtin_amdgcn_sched_barrier(0);  // (a row at a time: all of them together do not fit the registers)
            }
        }
    }
    // What the tile reads besides its sums (the residual; the argument of the derivative), as it lies, for all of its rows at
    // once: they come from memory, and row by row each of them would be waited for.
    constexpr bool kAhead = WHOLE && (KIND == kInputGrad || KIND == kForward);
    constexpr int kWords = !kAhead ? 1 : KIND == kInputGrad ? 2 : 2 * (int)sizeof(T);
    uint32_t raw[kAhead ? MT : 1][4][kWords];
    float steps[MT];
    const auto request = [&] {
        if constexpr (kAhead) {
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                const int64_t row = m + 16 * mt < M ? m + 16 * mt : M - 1;
#pragma unroll
                for (int t = 0; t < 4; t++) {
                    if constexpr (KIND == kInputGrad) {
                        const uint2 c = *(const uint2*)(e.codes_in + row * N + n + 32 * t);
                        raw[mt][t][0] = c.x, raw[mt][t][1] = c.y;
                    } else {
                        const uint4* q = (const uint4*)((const T*)e.residual + row * N + n + 32 * t);
#pragma unroll
                        for (int i = 0; i < kWords / 4; i++)
                            raw[mt][t][4 * i] = q[i].x, raw[mt][t][4 * i + 1] = q[i].y, raw[mt][t][4 * i + 2] = q[i].z, raw[mt][t][4 * i + 3] = q[i].w;
                    }
                }
                if constexpr (KIND == kInputGrad) steps[mt] = e.scales_in[row * G + group];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto rows = [&](auto which, auto with_residual) {
        constexpr int ACT = decltype(which)::value;
        constexpr bool fast = sizeof(T) == 2, res = decltype(with_residual)::value;
        if constexpr (KIND == kInputGrad ? ACT != CAT_ACT_NONE : res) request();
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int64_t row = m + 16 * mt;
            if (row >= M) continue;
            float more[4][8];
            if constexpr (kAhead && res) {
#pragma unroll
                for (int t = 0; t < 4; t++)
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        more[t][i] = sizeof(T) == 4 ? __uint_as_float(raw[mt][t][i % kWords])
                                                    : __uint_as_float(i % 2 ? raw[mt][t][i / 2] & 0xFFFF0000u : raw[mt][t][i / 2] << 16);
            } else if constexpr (res) {
#pragma unroll
                for (int t = 0; t < 4; t++) ld8<T, WHOLE>((const T*)e.residual + row * N, n + 32 * t, N, more[t]);
            }
            if constexpr (KIND == kInputGrad && ACT != CAT_ACT_NONE) {
#pragma unroll
                for (int t = 0; t < 4; t++) {
                    if constexpr (WHOLE) {
#pragma unroll
                        for (int i = 0; i < 8; i++) more[t][i] = code_value(raw[mt][t][i / 4], i % 4) * steps[mt];
                    } else {
                        ld_codes<8>(e.codes_in + row * N, n + 32 * t, N, e.scales_in[row * G + group], more[t]);
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 4; t++) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    v[i] = acc[mt][2 * t + (i >> 2)][i & 3];
                    if constexpr (KIND == kForward) v[i] = act_value<ACT, fast>(v[i]);
                    if constexpr (KIND == kInputGrad) v[i] *= act_grad<ACT, fast>(more[t][i]);
                    if constexpr (res) v[i] += more[t][i];
                }
                st8<T, WHOLE>((T*)e.out + row * N, n + 32 * t, N, v);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if constexpr (KIND == kWeightGrad)
        rows(std::integral_constant<int, CAT_ACT_NONE>(), std::false_type());
    else if (KIND == kForward && e.residual)
        with_act(e.act, [&](auto which) { rows(which, std::true_type()); });
    else
        with_act(e.act, [&](auto which) { rows(which, std::false_type()); });
}

// Workgroups stay for all of their tiles: a tile's first loads are under way while the one before it is finished and stored.
template <typename T, int KIND, int TM, int TN, int WM>
__global__ __launch_bounds__((TM / WM) * (TN / 128) * 64, 2) void k_gemm(const GemmArgs a) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass does not know all of the builtins, and would leave out the kernel's stub)
    constexpr bool PT = KIND != kForward, QT = KIND == kWeightGrad;
    constexpr int WN = 128, W = (TM / WM) * (TN / WN), MT = WM / 16, NT = WN / 16;
    constexpr int kStep = kStepBytes / (int)sizeof(T);
    constexpr int kBuf = (TM + TN) * kStepBytes;
    __shared__ __attribute__((aligned(1024))) char lds_mem[2 * kBuf + 2 * 1024];
    const lds_char lds = (lds_char)lds_mem, lds_bias = lds + 2 * kBuf;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (TN / WN), wn = wave % (TN / WN);

    // Workgroups go to the eight XCDs in turn; each XCD takes a run of neighbouring tiles, eight columns of them at a time, so
    // that what its L2 holds of either operand serves many of them.
    const uint32_t tm = (uint32_t)((a.m + TM - 1) / TM), tn = (uint32_t)((a.n + TN - 1) / TN), tiles = tm * tn;
    const uint32_t xcd = blockIdx.x & 7, share = tiles / 8, more = tiles % 8;
    const uint32_t stride = (gridDim.x - xcd + 7) / 8, end = (xcd + 1) * share + (xcd + 1 < more ? xcd + 1 : more);
    uint32_t t = xcd * share + (xcd < more ? xcd : more) + blockIdx.x / 8;
    if (t >= end) return;
    const auto place = [&](uint32_t tile, uint32_t& m0, uint32_t& n0) {
        const uint32_t band = tile / (8 * tm), in = tile - band * 8 * tm, width = tn - band * 8 < 8 ? tn - band * 8 : 8;
        m0 = in / width, n0 = band * 8 + in % width;
    };

    const int64_t k0 = (int64_t)blockIdx.y * a.k_split, k_all = a.k - k0 < a.k_split ? a.k - k0 : a.k_split;
    Stage<T, PT, true, TN, W> sp;
    Stage<T, QT, false, TM, W> sq;
    Fragments<T, PT, true, TN> fp;
    Fragments<T, QT, false, TM> fq;
    const auto addresses = [&](int of_lane) {
        sp.init(a.ldp, wave, of_lane);
        sq.init(a.ldq, wave, of_lane);
        fp.init(wn * NT, of_lane);
        fq.init(wm * MT, of_lane);
    };
    addresses(lane);
    constexpr int kAll = MT * NT, kLoads = decltype(sp)::kLoads;
    static_assert(kLoads == 4 && decltype(sq)::kLoads == 4, "");

    // The next step to be requested, of this tile or of the next one (behind the last tile: of that one again, not used).
    const int steps = (int)((k_all + kStep - 1) / kStep), tail = (int)(k_all - (int64_t)(steps - 1) * kStep);
    uint32_t tile_m, tile_n;
    place(t, tile_m, tile_n);
    int ahead = steps;
    sp.tile(a.p, a.p_bytes, (int64_t)tile_n * TN, k0, sp.base, sp.left);
    sq.tile(a.q, a.q_bytes, (int64_t)tile_m * TM, k0, sq.base, sq.left);
    const char *next_p, *next_q;
    int64_t next_p_left, next_q_left;
    const auto look_ahead = [&](uint32_t next) {
        uint32_t next_m, next_n;
        place(next < end ? next : t, next_m, next_n);
        sp.tile(a.p, a.p_bytes, (int64_t)next_n * TN, k0, next_p, next_p_left);
        sq.tile(a.q, a.q_bytes, (int64_t)next_m * TM, k0, next_q, next_q_left);
    };
    const auto begin = [&] {
        const bool turn = ahead == 0;
        ahead = turn ? steps : ahead;
        sp.base = turn ? next_p : sp.base, sp.left = turn ? next_p_left : sp.left;
        sq.base = turn ? next_q : sq.base, sq.left = turn ? next_q_left : sq.left;
        const int kl = ahead == 1 ? tail : kStep;
        sp.begin(kl), sq.begin(kl);
        ahead--;
    };
    look_ahead(t + stride);
    begin();
#pragma unroll
    for (int i = 0; i < 4; i++) sp.one(lds, wave, i), sq.one(lds + TN * kStepBytes, wave, i);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (as before the barrier of a step below)
    __syncthreads();
    begin();
#pragma unroll
    for (int i = 0; i < 4; i++) sp.one(lds + kBuf, wave, i), sq.one(lds + kBuf + TN * kStepBytes, wave, i);

    int cur = 0, odd = 0;
    for (;; t += stride, odd ^= 1024) {
        const int64_t m0 = (int64_t)tile_m * TM, n0 = (int64_t)tile_n * TN;
        // The addresses are made anew for every tile, from a lane number that the compiler takes for another one: kept over a
        // tile's end they would not fit the registers, and their way back from memory would wait for that tile's stores.
        int lane_again = lane;
        asm volatile("" : "+v"(lane_again));
        addresses(lane_again);
        look_ahead(t + (steps > 1 ? 1 : 2) * stride);  // (tiles of one step: the next one's is requested already)
        // the tile's bias into LDS, for its end (without one, and with shares of k, which the joining kernel finishes: zeros)
        if (KIND == kForward && wave == 0) {
            const int64_t there = a.e.bias && a.splits == 1 ? (a.n - n0) * 4 : 0;
            auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.e.bias + n0), 0, there < TN * 4 ? (uint32_t)there : TN * 4, 0x00027000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds_bias + odd), 16, lane_again * 16, 0, 0, 0);
        }
        f32x4 acc[MT][NT];
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) acc[mt][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
        // A step's second half is read while the first is multiplied, and the next step's first half while the second half's last
        // rows are: the wait for the next step's loads, and for the waves that still read this one's, stands before those rows, and
        // the loads of the step after it follow, one by one between the products.
        const auto multiply_rows = [&](const f32x4(&p)[NT], const f32x4(&q)[MT], int from, int to) {  // products from .. to - 1
#pragma unroll
            for (int i = from; i < to; i++) acc[i / NT][i % NT] = multiply<T>(p[i % NT], q[i / NT], acc[i / NT][i % NT]);
        };
        f32x4 p0[NT], q0[MT], p1[NT], q1[MT];
        fp.template read<0>(lds + cur, p0);
        fq.template read<0>(lds + cur + TN * kStepBytes, q0);
        for (int step = 0; step < steps; step++, cur ^= kBuf) {
            begin();
            fp.template read<1>(lds + cur, p1);
            fq.template read<1>(lds + cur + TN * kStepBytes, q1);
            multiply_rows(p0, q0, 0, kAll);
            multiply_rows(p1, q1, 0, kAll / 2);
#pragma unroll
            for (int i = 0; i < NT + MT; i++) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // a DS read
            }
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next step's loads, of this wave: not left to the compiler, which
            __syncthreads();                                  // does not see what the turning reads read
            // (after the last step: of the next tile, and read again there)
            const lds_char then_p = lds + (cur ^ kBuf), then_q = then_p + TN * kStepBytes;
            const auto part = [&](auto which) {
                constexpr int i = decltype(which)::value;
                multiply_rows(p1, q1, kAll / 2 + kAll / 16 * i, kAll / 2 + kAll / 16 * (i + 1));
                if constexpr (i < NT / 2) fp.template read2<0, 2 * i>(then_p, p0);
                if constexpr (i >= 4 && i < 4 + MT / 2) fq.template read2<0, 2 * (i - 4)>(then_q, q0);
                if constexpr (i < kLoads) sp.one(lds + cur, wave, i);
                if constexpr (i >= kLoads) sq.one(lds + cur + TN * kStepBytes, wave, i - kLoads);
                __builtin_amdgcn_sched_barrier(0);
            };
            part(std::integral_constant<int, 0>()), part(std::integral_constant<int, 1>());
            part(std::integral_constant<int, 2>()), part(std::integral_constant<int, 3>());
            part(std::integral_constant<int, 4>()), part(std::integral_constant<int, 5>());
            part(std::integral_constant<int, 6>()), part(std::integral_constant<int, 7>());
            // (keeps the compiler from moving these reads behind the products, to where the loop uses them)
#pragma unroll
            for (int i = 0; i < NT; i++) asm volatile("" : "+v"(p0[i]));
#pragma unroll
            for (int i = 0; i < MT; i++) asm volatile("" : "+v"(q0[i]));
        }

        int lane_end = lane;
        asm volatile("" : "+v"(lane_end));
        const int r = lane_end & 15, g = lane_end >> 4;
        const int64_t nw = n0 + wn * WN, nl = nw + 8 * g;  // the wave's first column; this lane's of pair t: nl + 32 t
        if (KIND == kForward) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                const f32x4 b = *(__attribute__((address_space(3))) f32x4*)(lds_bias + odd + (wn * WN + 8 * g + (nt >> 1) * 32 + 4 * (nt & 1)) * 4);
#pragma unroll
                for (int mt = 0; mt < MT; mt++) acc[mt][nt] += b;
            }
        }
        if (a.splits > 1) {  // the sum of a share of k: fp32, joined by a kernel of its own
            float* part = a.parts + (int64_t)blockIdx.y * a.m * a.n;
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                const int64_t m = m0 + wm * WM + mt * 16 + r;
                if (m >= a.m) continue;
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    const int64_t n = nl + (nt >> 1) * 32 + 4 * (nt & 1);
                    const float v[4] = {acc[mt][nt][0], acc[mt][nt][1], acc[mt][nt][2], acc[mt][nt][3]};
                    if (n < a.n) st_group_to(part + m * a.n, n, a.n, v);
                }
            }
        } else if (nw + WN <= a.n && a.n % 8 == 0) {
            finish_rows<T, KIND, MT, true>(a.e, acc, m0 + wm * WM + r, a.m, nl, a.n, g);
        } else if (nw < a.n) {
            finish_rows<T, KIND, MT, false>(a.e, acc, m0 + wm * WM + r, a.m, nl, a.n, g);
        }
        if (t + stride >= end) break;
        place(t + stride, tile_m, tile_n);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loads ahead: no wave ends while LDS is still written for it
#endif
}

template <typename T, int KIND, int TM, int TN, int WM>
cat_status launch_gemm_tiles(const GemmArgs& a, hipStream_t st) {
    const int64_t tiles = ((a.m + TM - 1) / TM) * ((a.n + TN - 1) / TN);
    if (tiles >= (1ll << 31)) return set_error(CAT_ERR_UNSUPPORTED, "product of %lld x %lld entries has too many tiles", (long long)a.m, (long long)a.n);
    // as many workgroups as the card holds at a time (256 CUs, by LDS one large tile's or two small ones' each)
    const int64_t most = 256 * (TM == 256 ? 1 : 2);
    hipLaunchKernelGGL((k_gemm<T, KIND, TM, TN, WM>), dim3((unsigned)(a.splits > 1 || tiles < most ? tiles : most), (unsigned)a.splits), dim3((TM / WM) * (TN / 128) * 64), 0, st, a);
    CAT_LAUNCH_CHECK("k_gemm");
    return CAT_OK;
}

}  // namespace cat
