// The tile kernel of the block's matrix products on the matrix cores (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32:
// exact products, fp32 sums; v_mfma_i32_16x16x64_i8: exact sums).
//
// A workgroup computes TM x TN entries of out, each of its waves WM x 128.  A step takes 128 bytes of k (64 bfloat16, 32
// float or 128 8-bit entries) of both operands into LDS by loads that go there directly (no registers, no stores; what lies outside an
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
// 8-bit integers (TOP/s; the library 2050 at 8192^3): 8192^3 2270 to 2510, gated 2730; 16384 x 8192 over 2048 2300, with GELU 2060.  Gated bfloat16
// 8192 x 2 x 4096 over 8192 1450 to 1490, checkpoints 4 % more time; 16384 x 2 x 4096 over 1024 212 us, with checkpoints 255 to 270.
#pragma once
#include "cat_gemm.h"

namespace cat {

typedef __attribute__((address_space(3))) void* lds_void;
typedef __attribute__((address_space(3))) char* lds_char;
typedef __attribute__((address_space(3))) volatile uint32_t* lds_words;
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
__device__ __forceinline__ Sums<T> multiply(f32x4 a, f32x4 b, Sums<T> c) {
    if constexpr (sizeof(T) == 1) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    } else if constexpr (sizeof(T) == 2) {
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
// Not ALIGNED, WHOLE: all columns lie inside out, whose rows start anywhere.
template <typename T, bool WHOLE, bool ALIGNED = true>
__device__ __forceinline__ void ld8(const T* row, int64_t n, int64_t N, float (&v)[8]) {
    if constexpr (!WHOLE || !ALIGNED) {
        ld_entries<T, 8>(row, n, WHOLE ? n + 8 : N, v);
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
template <typename T, bool WHOLE, bool ALIGNED = true>
__device__ __forceinline__ void st8(T* row, int64_t n, int64_t N, const float (&v)[8]) {
    if constexpr (!WHOLE || !ALIGNED) {
        st_entries<T, 8>(row, n, WHOLE ? n + 8 : N, v);
    } else if constexpr (sizeof(T) == 2) {
        *(uint4*)(row + n) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
        *(f32x4*)(row + n) = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4*)(row + n + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
}
// Float results: eight columns a lane are two stores of 16 bytes, each of which would leave gaps as wide.  Lanes r and r + 8 exchange
// halves, so that one store has the whole 128 bytes of rows 0..7 of 16 and the other those of rows 8..15.  to: columns n .. n + 7 of
// the lane's own row, r of 16; `left` rows from the first of the 16 on are there.  All lanes of a row of 16 take part.
// (us: gate's gradients 8192 x 1000 over 256 60 -> 57, 65536 x 1000 over 512 8-bit integers 90 -> 83; of long rows it is the slower one, 16384 x
// 8192 over 1024 8-bit integers 236 -> 243, and of the gated float product, bound by its products, neither.)
constexpr int64_t kExchangeMost = 1024;  // columns of out, of 8-bit integers
__device__ __forceinline__ void st_float_rows(float* to, int64_t pitch, int64_t left, int r, f32x4 lo, f32x4 hi) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int a = (int)__float_as_uint(lo[i]), b = (int)__float_as_uint(hi[i]);
        lo[i] = __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(a, b, 0x128, 0xF, 0xC, false));  // row_ror 8, lanes 8..15
        hi[i] = __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(b, a, 0x128, 0xF, 0x3, false));  // lanes 0..7
    }
    const int row = r & 7;
    float* at = to + (row - r) * pitch + 4 * (r >> 3);
    if (row < left) *(Group16<float>*)at = __builtin_bit_cast(Group16<float>, lo);
    if (row + 8 < left) *(Group16<float>*)(at + 8 * pitch) = __builtin_bit_cast(Group16<float>, hi);
}

// I8: of 8-bit integers, whose products leave no checkpoint.  CUT (with WHOLE): rows are whole groups of eight columns, of which some
// lie behind the row's end.  Not ALIGNED (with WHOLE): all columns inside, rows that start anywhere (us, 16384 x 8198 over 1024 to fp32: 325
// with every group compared with the row's end, 269; bfloat16 with a residual 253 and 241.  The gated product gains nothing so).
template <typename T, int KIND, bool I8, int MT, bool WHOLE, bool CUT = false, bool ALIGNED = true>
__device__ __forceinline__ void finish_rows(const Epilogue& e, f32x4 (&acc)[MT][8], int64_t m, int64_t M, int64_t n, int64_t N, int g) {
    const int64_t G = (N + kPackGroup - 1) / kPackGroup, group = n / kPackGroup;
    constexpr int FAST = I8 ? kFast<T> : sizeof(T) == 2;
    if constexpr (KIND == kForward && !I8) {
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
    constexpr bool kAhead = WHOLE && ALIGNED && (KIND == kInputGrad || (KIND == kForward && MT * sizeof(T) <= 8));  // (what the registers hold)
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
                        const uint4* q = (const uint4*)((const T*)e.residual + row * N + (!CUT || n + 32 * t < N ? n + 32 * t : 0));
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
        constexpr bool res = decltype(with_residual)::value;
        if constexpr (KIND == kInputGrad ? ACT != CAT_ACT_NONE : res) request();
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            constexpr bool kExchange = I8 && sizeof(T) == 4 && WHOLE;
            const int64_t row = kExchange && m + 16 * mt >= M ? M - 1 : m + 16 * mt;
            if (!kExchange && row >= M) continue;
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
                for (int t = 0; t < 4; t++)
                    if (!CUT || n + 32 * t < N) ld8<T, WHOLE, ALIGNED>((const T*)e.residual + row * N, n + 32 * t, N, more[t]);
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
                    if constexpr (KIND == kForward) v[i] = act_value<ACT, FAST>(v[i]);
                    if constexpr (KIND == kInputGrad) v[i] *= act_grad<ACT, FAST>(more[t][i]);
                    if constexpr (res) v[i] += more[t][i];
                }
                if constexpr (kExchange) {
                    const int r = threadIdx.x & 15;
                    if (CUT && n + 32 * t >= N) continue;
                    if (N > kExchangeMost) {
                        if (m + 16 * mt < M) st8<T, WHOLE, ALIGNED>((T*)e.out + row * N, n + 32 * t, N, v);
                    } else
                        st_float_rows((float*)e.out + (m + 16 * mt) * N + n + 32 * t, N, M - (m + 16 * mt - r), r, f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]});
                } else {
                    if (!CUT || n + 32 * t < N) st8<T, WHOLE, ALIGNED>((T*)e.out + row * N, n + 32 * t, N, v);
                }
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

// The gated product's.  Lane (r, g) holds columns n + 32 t .. + 7, t = 0, 1, of the gate in acc[mt][0..3], of the value in
// acc[mt][4..7].
// Its checkpoints: the largest magnitudes of a wave's 64 columns of both go to LDS (four words a row of the tile: gate and value of
// one wave's columns and of the other's, which share a scale with them; gated_top) and come back as the scales of 128 (gated_scales).
// The barrier between waits for LDS alone: the next tile's loads stay under way.
template <int MT, bool WHOLE>
__device__ __forceinline__ void gated_top(const f32x4 (&acc)[MT][8], int64_t n, int64_t N, lds_char row0, int half, int g) {
#pragma unroll
    for (int mt = 0; mt < MT; mt++)
#pragma unroll
        for (int part = 0; part < 2; part++) {
            float top = 0.f;  // (maximum: a NaN stays)
#pragma unroll
            for (int nt = 0; nt < 4; nt++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (WHOLE || n + 32 * (nt >> 1) + 4 * (nt & 1) + i < N) top = __builtin_elementwise_maximum(top, fabsf(acc[mt][part * 4 + nt][i]));
            uint32_t a = __float_as_uint(top) & 0x7FFFFFFFu;
            const auto by16 = __builtin_amdgcn_permlane16_swap(a, a, false, false);
            a = by16[0] > by16[1] ? by16[0] : by16[1];
            const auto by32 = __builtin_amdgcn_permlane32_swap(a, a, false, false);
            a = by32[0] > by32[1] ? by32[0] : by32[1];
            if (g == 0) ((lds_words)(row0 + mt * 16 * 16))[half * 2 + part] = a;
        }
}
template <int MT>
__device__ __forceinline__ void gated_scales(lds_char row0, PackScale (&s)[MT][2]) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int mt = 0; mt < MT; mt++)
#pragma unroll
        for (int part = 0; part < 2; part++) {
            const uint32_t a = ((lds_words)(row0 + mt * 16 * 16))[part], b = ((lds_words)(row0 + mt * 16 * 16))[2 + part];
            s[mt][part] = pack_scale(a > b ? a : b);
        }
}
template <typename T, int MT, bool WHOLE>
__device__ __forceinline__ void finish_gated(const Epilogue& e, f32x4 (&acc)[MT][8], int64_t m, int64_t M, int64_t n, int64_t N, int g,
                                             const PackScale (*scales)[2]) {
    if (scales) {
        const int64_t G = (N + kPackGroup - 1) / kPackGroup;
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int64_t row = m + 16 * mt;
            if (row < M) {
#pragma unroll
                for (int part = 0; part < 2; part++) {
                    const PackScale s = scales[mt][part];
                    int8_t* codes = e.codes_out + (part * M + row) * N;
#pragma unroll
                    for (int t = 0; t < 2; t++) {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; i++) v[i] = acc[mt][part * 4 + 2 * t + (i >> 2)][i & 3];
                        if constexpr (WHOLE)
                            *(uint2*)(codes + n + 32 * t) = make_uint2(pack_codes4(v, s.up), pack_codes4(v + 4, s.up));
                        else if (n + 32 * t < N)
                            st_codes<8>(codes, n + 32 * t, N, v, s.up);
                    }
                    if (n % kPackGroup == 0) e.scales_out[(part * M + row) * G + n / kPackGroup] = s.step;  // (the first wave's g = 0)
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    with_act(e.act, [&](auto which) {
        constexpr int ACT = decltype(which)::value;
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int64_t row = m + 16 * mt;
            if (row >= M) continue;
#pragma unroll
            for (int t = 0; t < 2; t++) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] = act_value<ACT, kFast<T>>(acc[mt][2 * t + (i >> 2)][i & 3]) * acc[mt][4 + 2 * t + (i >> 2)][i & 3];
                if (WHOLE || n + 32 * t < N) st8<T, WHOLE>((T*)e.out + row * N, n + 32 * t, N, v);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    });
}

// Sums over the 16 lanes of a row of lanes of 16 values each: lane r is left with the sum of value r.  Each step hands on the half
// of the values that the other lane of a pair goes on with.
__device__ __forceinline__ float sums_by_lane(float (&v)[16], int r) {
    const auto halve = [&](auto which) {
        constexpr int bit = decltype(which)::value;  // value i stays with the lanes whose bit is i's
        const bool up = r & bit;
#pragma unroll
        for (int i = 0; i < bit; i++) {
            const float keep = up ? v[i + bit] : v[i], give = up ? v[i] : v[i + bit];
            float got;
            if constexpr (bit == 8) got = dpp_f32<0x128>(give);       // row_ror 8
            else if constexpr (bit == 4) got = __shfl_xor(give, 4, kWave);
            else if constexpr (bit == 2) got = dpp_f32<0x4E>(give);   // quad_perm [2, 3, 0, 1]
            else got = dpp_f32<0xB1>(give);                           // quad_perm [1, 0, 3, 2]
            v[i] = keep + got;
        }
    };
    halve(std::integral_constant<int, 8>()), halve(std::integral_constant<int, 4>());
    halve(std::integral_constant<int, 2>()), halve(std::integral_constant<int, 1>());
    return v[0];
}
// The gate's gradients, of rows of at least eight columns: lane (r, g) as in finish_rows; sums: this wave's row of col_sums.  Two pairs
// of tiles at a time for all rows, so that the sums over rows are 32 registers, a row's codes under way while the one before it is
// worked on.  Nothing is stored before the last codes have come: loads and stores complete in the order of their issue, and a load
// behind stores would be waited for as long as those (us, 65536 x 1024 over 256 bfloat16 without sums: 163, now 136; without loads 102,
// without stores 93).  What is stored waits in the sums' registers, both gradients of an entry in one where they are bfloat16.
// ALIGNED: rows are whole groups of eight columns.  Otherwise the codes of a row's last group come with those before them, from its last
// eight (us, 16384 x 4097 over 1024 bfloat16: 380 with loads and stores entry by entry there, 310 so).
template <typename T, int ACT, int MT, bool ALIGNED>
__device__ __forceinline__ void finish_gate_grad(const Epilogue& e, f32x4 (&acc)[MT][8], int64_t m, int64_t M, int64_t n, int64_t N, int r, float* sums) {
    const int64_t G = (N + kPackGroup - 1) / kPackGroup, group = n / kPackGroup;
    float steps[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const int64_t row = m + 16 * mt < M ? m + 16 * mt : M - 1;
        steps[mt][0] = e.scales_in[row * G + group], steps[mt][1] = e.scales_in[(M + row) * G + group];
    }
    f32x4 second[sizeof(T) == 4 ? MT : 1][8];  // float: the value's gradients
    uint2 held[2][2][2];
    // from where a lane's eight codes come (columns behind the last: from any eight of the row)
    const auto from = [&](int64_t c) { return c + 8 <= N ? c : ALIGNED ? 0 : N - 8; };
    const auto request = [&](int at, uint2(&to)[2][2]) {  // at: half * MT + row
        const int64_t row = m + 16 * (at % MT) < M ? m + 16 * (at % MT) : M - 1;
        const int8_t *gate = e.codes_in + row * N, *value = gate + M * N;
#pragma unroll
        for (int t = 0; t < 2; t++) {
            const int64_t c = from(n + 64 * (at / MT) + 32 * t);
            if constexpr (ALIGNED) {
                to[t][0] = *(const uint2*)(gate + c), to[t][1] = *(const uint2*)(value + c);
            } else {
                const Codes8 a = *(const Codes8*)(gate + c), b = *(const Codes8*)(value + c);
                to[t][0] = make_uint2(a.w[0], a.w[1]), to[t][1] = make_uint2(b.w[0], b.w[1]);
            }
        }
    };
    request(0, held[0]);
#pragma unroll
    for (int half = 0; half < 2; half++) {
        float s[2][16];
#pragma unroll
        for (int i = 0; i < 32; i++) s[i / 16][i % 16] = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int step = half * MT + mt;
            if (step + 1 < 2 * MT) request(step + 1, held[(step + 1) & 1]);
#pragma unroll
            for (int t = 0; t < 2; t++) {
                if (m + 16 * mt < M) {
                    uint2 a = held[step & 1][t][0], b = held[step & 1][t][1];
                    if constexpr (!ALIGNED) {
                        const int64_t c = n + 64 * half + 32 * t;
                        const int by = (int)(c - from(c)) * 8 & 63;
                        const uint64_t x = (((uint64_t)a.y << 32) | a.x) >> by, y = (((uint64_t)b.y << 32) | b.x) >> by;
                        a = make_uint2((uint32_t)x, (uint32_t)(x >> 32)), b = make_uint2((uint32_t)y, (uint32_t)(y >> 32));
                    }
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const int nt = 4 * half + 2 * t + (i >> 2);
                        const float d = acc[mt][nt][i & 3];
                        const float gate = code_value(i < 4 ? a.x : a.y, i % 4) * steps[mt][0], value = code_value(i < 4 ? b.x : b.y, i % 4) * steps[mt][1];
                        float u, du;
                        act_both<ACT, kFast<T>>(gate, u, du);
                        float dg = d * value * du, dv = d * u;
                        s[t][i] += dg, s[t][8 + i] += dv;
                        // (here and now: left to the compiler, it is done where it is stored, from all it takes)
                        if constexpr (sizeof(T) == 2) {
                            uint32_t both = pack_bf16(dg, dv);
                            asm volatile("" : "+v"(both));
                            acc[mt][nt][i & 3] = __uint_as_float(both);
                        } else {
                            asm volatile("" : "+v"(dg), "+v"(dv));
                            acc[mt][nt][i & 3] = dg, second[mt][nt][i & 3] = dv;
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (sums) {
#pragma unroll
            for (int t = 0; t < 2; t++) {
                const float total = sums_by_lane(s[t], r);
                const int64_t c = n + 64 * half + 32 * t + (r & 7);
                if (c < N) sums[(r >> 3) * N + c] = total;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int mt = 0; mt < MT; mt++) {
        const int64_t row = m + 16 * mt;
        if (sizeof(T) == 2 && row >= M) continue;
        T* out = (T*)e.out + row * 2 * N + n;
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const int64_t left = N - (n + 32 * t);  // columns from this lane's first on
            if (left <= 0) continue;
            if constexpr (sizeof(T) == 2) {
                Group16<T> gate, value;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t lo = __float_as_uint(acc[mt][2 * t + (i >> 1)][2 * (i & 1)]), hi = __float_as_uint(acc[mt][2 * t + (i >> 1)][2 * (i & 1) + 1]);
                    gate.w[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u), value.w[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
                }
                if (ALIGNED) {
                    *(uint4*)(out + 32 * t) = make_uint4(gate.w[0], gate.w[1], gate.w[2], gate.w[3]);
                    *(uint4*)(out + N + 32 * t) = make_uint4(value.w[0], value.w[1], value.w[2], value.w[3]);
                } else if (left >= 8) {
                    *(Group16<T>*)(out + 32 * t) = gate, *(Group16<T>*)(out + N + 32 * t) = value;
                } else {
#pragma unroll
                    for (int i = 0; i < 7; i++)
                        if (i < left) out[32 * t + i] = (T)(gate.w[i / 2] >> 16 * (i % 2)), out[N + 32 * t + i] = (T)(value.w[i / 2] >> 16 * (i % 2));
                }
            } else {
                const auto store = [&](T* to, const f32x4& lo, const f32x4& hi) {
                    if (ALIGNED || left >= 8) {
                        st_float_rows((float*)to, 2 * N, M - (row - r), r, lo, hi);
                    } else if (row < M) {
                        const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                        st_entries<T, 8>(to, 0, left, v);
                    }
                };
                store(out + 32 * t, acc[mt][2 * t], acc[mt][2 * t + 1]);
                store(out + N + 32 * t, second[mt][2 * t], second[mt][2 * t + 1]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Workgroups stay for all of their tiles: a tile's first loads are under way while the one before it is finished and stored.
// ACT, ALIGNED: of the gate's gradients (one kernel for all activations leaves the compiler no registers); ACT < 0, for those: the joining
// kernel works them out.
template <typename E, typename T, int KIND, int TM, int TN, int WM, int ACT = -1, bool ALIGNED = true>
__global__ __launch_bounds__((TM / WM) * (TN / 128) * 64, 2) void k_gemm(const GemmArgs a) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass does not know all of the builtins, and would leave out the kernel's stub)
    constexpr bool GATED = KIND == kGated, FORWARD = KIND == kForward || GATED, PT = !FORWARD, QT = KIND == kWeightGrad;
    constexpr int WN = 128, W = (TM / WM) * (TN / WN), MT = WM / 16, NT = WN / 16;
    constexpr int kStep = kStepBytes / (int)sizeof(E);
    constexpr int kBuf = (TM + TN) * kStepBytes;
    // columns of out a tile, and a wave: gated, half of them, since a wave's 128 are 64 of the gate and the same 64 of the value
    constexpr int TO = GATED ? TN / 2 : TN, WO = GATED ? WN / 2 : WN;
    // what a tile's end reads from LDS, for two tiles in turn: the bias, then the scales of p's rows and of q's (8-bit operands)
    constexpr int kEnd = 1024 * (sizeof(E) == 1 ? 3 : 1);
    constexpr bool kExchange = GATED && TO == kPackGroup && sizeof(E) > 1;  // (narrower tiles: the joining kernel packs)
    __shared__ __attribute__((aligned(1024))) char lds_mem[2 * kBuf + 2 * kEnd + (kExchange ? TM * 16 : 0)];
    const lds_char lds = (lds_char)lds_mem, lds_bias = lds + 2 * kBuf;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (TN / WN), wn = wave % (TN / WN);

    // Workgroups go to the eight XCDs in turn; each XCD takes a run of neighbouring tiles, eight columns of them at a time, so
    // that what its L2 holds of either operand serves many of them.  With shares of k the run goes through the tiles of a share and
    // then of the next one: an XCD reads its share of k and not all of it.
    const uint32_t tm = (uint32_t)((a.m + TM - 1) / TM), tn = (uint32_t)((a.n + TO - 1) / TO), tiles = tm * tn;
    const uint32_t xcd = blockIdx.x & 7, all = tiles * (uint32_t)a.splits, share = all / 8, more = all % 8;
    uint32_t stride = (gridDim.x - xcd + 7) / 8, end = (xcd + 1) * share + (xcd + 1 < more ? xcd + 1 : more);
    uint32_t t = xcd * share + (xcd < more ? xcd : more) + blockIdx.x / 8, share_of_k = 0;
    if (t >= end) return;
    if (a.splits > 1) share_of_k = t / tiles, t -= share_of_k * tiles, end = t + 1, stride = 1;  // (a tile each)
    const auto place = [&](uint32_t tile, uint32_t& m0, uint32_t& n0) { tile_place(tile, tm, tn, m0, n0); };

    // (a weight gradient's p in two terms: the shares of the second one stand behind the first's)
    const uint32_t term = KIND == kWeightGrad && a.splits > a.k_shares ? share_of_k / (uint32_t)a.k_shares : 0;
    const void* const p = KIND == kWeightGrad ? (const char*)a.p + term * a.p_bytes : a.p;
    const int64_t k0 = (int64_t)(share_of_k - term * (uint32_t)a.k_shares) * a.k_split, k_all = a.k - k0 < a.k_split ? a.k - k0 : a.k_split;
    Stage<E, PT, true, TN, W> sp;
    Stage<E, QT, false, TM, W> sq;
    Fragments<E, PT, true, TN> fp;
    Fragments<E, QT, false, TM> fq;
    const auto addresses = [&](int of_lane) {
        sp.init(a.ldp, wave, of_lane);
        sq.init(a.ldq, wave, of_lane);
        fp.init(wn * NT, of_lane);
        fq.init(wm * MT, of_lane);
    };
    addresses(lane);
    constexpr int kAll = MT * NT, kLoads = decltype(sp)::kLoads;
    static_assert(kLoads == 4 && decltype(sq)::kLoads == 4, "");

    // The row of p at which a tile's rows in LDS would begin for those that this wave brings: gated, 64 rows of the gate and the same
    // 64 of the value in turn, a wave's 32 of one or the other.
    const auto first_p = [&](uint32_t tile) {
        const int64_t n0 = (int64_t)tile * TO;
        return GATED ? ((wave >> 1) & 1) * a.n + n0 + (wave >> 2) * 64 + (wave & 1) * 32 - wave * 32 : n0;
    };
    // The next step to be requested, of this tile or of the next one (behind the last tile: of that one again, not used).
    const int steps = (int)((k_all + kStep - 1) / kStep), tail = (int)(k_all - (int64_t)(steps - 1) * kStep);
    uint32_t tile_m, tile_n;
    place(t, tile_m, tile_n);
    int ahead = steps;
    sp.tile(p, a.p_bytes, first_p(tile_n), k0, sp.base, sp.left);
    sq.tile(a.q, a.q_bytes, (int64_t)tile_m * TM, k0, sq.base, sq.left);
    const char *next_p, *next_q;
    int64_t next_p_left, next_q_left;
    const auto look_ahead = [&](uint32_t next) {
        uint32_t next_m, next_n;
        place(next < end ? next : t, next_m, next_n);
        sp.tile(p, a.p_bytes, first_p(next_n), k0, next_p, next_p_left);
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
    for (;; t += stride, odd ^= kEnd) {
        const int64_t m0 = (int64_t)tile_m * TM, n0 = (int64_t)tile_n * TO;
        // The addresses are made anew for every tile, from a lane number that the compiler takes for another one: kept over a
        // tile's end they would not fit the registers, and their way back from memory would wait for that tile's stores.
        int lane_again = lane;
        asm volatile("" : "+v"(lane_again));
        addresses(lane_again);
        look_ahead(t + (steps > 1 ? 1 : 2) * stride);  // (tiles of one step: the next one's is requested already)
        // the tile's bias into LDS, for its end (without one, and with shares of k, which the joining kernel finishes: zeros)
        if (KIND == kForward && wave == 0) {
            const int64_t there = a.e.bias && !a.parts ? (a.n - n0) * 4 : 0;
            auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.e.bias + n0), 0, there < TN * 4 ? (uint32_t)there : TN * 4, 0x00027000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds_bias + odd), 16, lane_again * 16, 0, 0, 0);
        }
        if constexpr (GATED) {  // (the value's bias and scales start on any float's boundary: a float a lane, a wave 64 rows of p)
            if (wave < TN / 64) {
                const int64_t from = n0 + (wave >> 1) * 64, rest = a.n - from, at = (wave & 1) * a.n + from;
                const uint32_t there = a.parts || rest <= 0 ? 0 : rest < 64 ? (uint32_t)rest * 4 : 256;
                auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.e.bias + at), 0, a.e.bias ? there : 0, 0x00027000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds_bias + odd + wave * 256), 4, lane_again * 4, 0, 0, 0);
                if constexpr (sizeof(E) == 1) {
                    rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.e.col_scales + at), 0, there, 0x00027000);
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds_bias + odd + 1024 + wave * 256), 4, lane_again * 4, 0, 0, 0);
                }
            }
        }
        if constexpr (sizeof(E) == 1) {
            if (!GATED && wave == 1) {
                const int64_t there = a.parts ? 0 : (a.n - n0) * 4;
                auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.e.col_scales + n0), 0, there < TN * 4 ? (uint32_t)there : TN * 4, 0x00027000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds_bias + odd + 1024), 16, lane_again * 16, 0, 0, 0);
            }
            if (wave == W - 1) {
                const int64_t there = a.parts ? 0 : (a.m - m0) * 4;
                auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.e.row_scales + m0), 0, there < TM * 4 ? (uint32_t)there : TM * 4, 0x00027000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void)(lds_bias + odd + 2048), 16, lane_again * 16, 0, 0, 0);
            }
        }
        Sums<E> sums[MT][NT];
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
            for (int nt = 0; nt < NT; nt++) sums[mt][nt] = Sums<E>{0, 0, 0, 0};
        // A step's second half is read while the first is multiplied, and the next step's first half while the second half's last
        // rows are: the wait for the next step's loads, and for the waves that still read this one's, stands before those rows, and
        // the loads of the step after it follow, one by one between the products.
        const auto multiply_rows = [&](const f32x4(&pf)[NT], const f32x4(&qf)[MT], int from, int to) {  // products from .. to - 1
#pragma unroll
            for (int i = from; i < to; i++) sums[i / NT][i % NT] = multiply<E>(pf[i % NT], qf[i / NT], sums[i / NT][i % NT]);
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
        const int64_t nw = n0 + wn * WO, nl = nw + 8 * g;  // the wave's first column; this lane's of pair t: nl + 32 t (gated: t & 1)
        if (KIND == kWeightGrad && a.tiled) {  // 1 KB a store of a wave (us, 1024 x 4096 over 16384 rows: 158 with pieces of 16 bytes of rows, 140 so)
            float* part = (float*)a.parts + (((int64_t)share_of_k * tiles + t) * (TM * TN) + wave * (WM * WN)) + lane_end * 4;
#pragma unroll
            for (int i = 0; i < MT * NT; i++) *(Sums<E>*)(part + i * 256) = sums[i / NT][i % NT];
        } else if (a.parts) {  // the sums as they are (of a share of k, say): a kernel of its own goes on with them
            const int64_t width = GATED ? 2 * a.n : a.n;
#pragma unroll
            for (int mt = 0; mt < MT; mt++) {
                const int64_t m = m0 + wm * WM + mt * 16 + r;
                if (m >= a.m) continue;
                float* part = (float*)a.parts + ((int64_t)share_of_k * a.m + m) * width;
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    const int64_t n = nl + ((nt >> 1) & (GATED ? 1 : 3)) * 32 + 4 * (nt & 1);
                    const f32x4 b = __builtin_bit_cast(f32x4, sums[mt][nt]);
                    const float v[4] = {b[0], b[1], b[2], b[3]};
                    if (n < a.n) st_group_to(part + (GATED && nt >= 4 ? a.n : 0), n, a.n, v);
                }
            }
        } else {
            f32x4 acc[MT][NT];
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                f32x4 b = f32x4{0.f, 0.f, 0.f, 0.f}, by = b;
                const int column = (wn * WN + 8 * g + (nt >> 1) * 32 + 4 * (nt & 1)) * 4;
                if constexpr (FORWARD) b = *(__attribute__((address_space(3))) f32x4*)(lds_bias + odd + column);
                if constexpr (sizeof(E) == 1) by = *(__attribute__((address_space(3))) f32x4*)(lds_bias + odd + 1024 + column);
#pragma unroll
                for (int mt = 0; mt < MT; mt++) {
                    if constexpr (sizeof(E) == 1) {  // (the sum of integers rounds once to 32 bits, from 2^24 on; so do both products)
                        const float scale = *(__attribute__((address_space(3))) float*)(lds_bias + odd + 2048 + (wm * WM + mt * 16 + r) * 4);
#pragma unroll
                        for (int i = 0; i < 4; i++) acc[mt][nt][i] = fmaf((float)sums[mt][nt][i], scale * by[i], b[i]);
                    } else {
                        acc[mt][nt] = sums[mt][nt];
                        if constexpr (FORWARD) acc[mt][nt] += b;
                    }
                }
            }
            const int64_t m = m0 + wm * WM + r;
            if constexpr (GATED) {
                PackScale scales[MT][2];
                const bool pack = kExchange && a.e.codes_out;
                if constexpr (kExchange) {
                    if (pack) {
                        const lds_char row0 = lds_bias + 2 * kEnd + (wm * WM + r) * 16;
                        if (nw + WO <= a.n) gated_top<MT, true>(acc, nl, a.n, row0, wn, g);
                        else gated_top<MT, false>(acc, nl, a.n, row0, wn, g);
                        gated_scales<MT>(row0, scales);
                    }
                }
                if (nw + WO <= a.n && a.n % 8 == 0)
                    finish_gated<T, MT, true>(a.e, acc, m, a.m, nl, a.n, g, pack ? scales : nullptr);
                else if (nw < a.n)
                    finish_gated<T, MT, false>(a.e, acc, m, a.m, nl, a.n, g, pack ? scales : nullptr);
            } else if constexpr (KIND == kGatedGrad) {
                float* col_sums = a.e.col_sums ? a.e.col_sums + ((int64_t)tile_m * (TM / WM) + wm) * 2 * a.n : nullptr;
                if constexpr (ACT >= 0) {
                    if (nw < a.n) finish_gate_grad<T, ACT, MT, ALIGNED>(a.e, acc, m, a.m, nl, a.n, r, col_sums);
                }
            } else {
                constexpr bool kI8 = sizeof(E) == 1;
                if (nw + WN <= a.n && a.n % 8 == 0)
                    finish_rows<T, KIND, kI8, MT, true>(a.e, acc, m, a.m, nl, a.n, g);
                else if (kI8 && nw < a.n && a.n % 8 == 0)
                    finish_rows<T, KIND, kI8, MT, true, kI8>(a.e, acc, m, a.m, nl, a.n, g);
                else if (kI8 && nw + WN <= a.n)
                    finish_rows<T, KIND, kI8, MT, true, false, !kI8>(a.e, acc, m, a.m, nl, a.n, g);
                else if (nw < a.n)
                    finish_rows<T, KIND, kI8, MT, false>(a.e, acc, m, a.m, nl, a.n, g);
            }
        }
        if (t + stride >= end) break;
        place(t + stride, tile_m, tile_n);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loads ahead: no wave ends while LDS is still written for it
#endif
}

template <typename E, typename T, int KIND, int TM, int TN, int WM, int ACT = -1, bool ALIGNED = true>
cat_status launch_gemm_tiles(const GemmArgs& a, hipStream_t st) {
    constexpr int TO = KIND == kGated ? TN / 2 : TN;
    const int64_t tiles = ((a.m + TM - 1) / TM) * ((a.n + TO - 1) / TO);
    if (tiles * a.splits >= (1ll << 31)) return set_error(CAT_ERR_UNSUPPORTED, "product of %lld x %lld entries has too many tiles", (long long)a.m, (long long)a.n);
    // as many workgroups as the card holds at a time (256 CUs, by LDS one large tile's or two small ones' each)
    const int64_t most = 256 * (TM == 256 ? 1 : 2);
    hipLaunchKernelGGL((k_gemm<E, T, KIND, TM, TN, WM, ACT, ALIGNED>), dim3((unsigned)(a.splits > 1 ? tiles * a.splits : tiles < most ? tiles : most)), dim3((TM / WM) * (TN / 128) * 64), 0, st, a);
    CAT_LAUNCH_CHECK("k_gemm");
    return CAT_OK;
}

// the gate's gradients: a kernel for each activation and for either alignment of rows, or the sums alone
template <typename T, int EDGE, int WM, bool ALIGNED>
cat_status launch_gate_grad(const GemmArgs& a, hipStream_t st) {
    switch (a.e.act) {
        case CAT_ACT_NONE: return launch_gemm_tiles<T, T, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_NONE, ALIGNED>(a, st);
        case CAT_ACT_RELU: return launch_gemm_tiles<T, T, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_RELU, ALIGNED>(a, st);
        case CAT_ACT_GELU: return launch_gemm_tiles<T, T, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_GELU, ALIGNED>(a, st);
        case CAT_ACT_GELU_TANH: return launch_gemm_tiles<T, T, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_GELU_TANH, ALIGNED>(a, st);
        default: return launch_gemm_tiles<T, T, kGatedGrad, EDGE, EDGE, WM, CAT_ACT_SILU, ALIGNED>(a, st);
    }
}
template <typename T, int EDGE, int WM>
cat_status launch_gate_grad(const GemmArgs& a, hipStream_t st) {
    if (a.parts) return launch_gemm_tiles<T, T, kGatedGrad, EDGE, EDGE, WM>(a, st);
    return a.n % 8 ? launch_gate_grad<T, EDGE, WM, false>(a, st) : launch_gate_grad<T, EDGE, WM, true>(a, st);
}

}  // namespace cat
