// product_tile.h -- the MFMA tile shared by the experts' product and its gradients.
//
// A workgroup computes a TI x TJ tile of C[j][i] = sum_c A[i][c] B[j][c].  i is the index
// that is contiguous in C: a lane of the 32x32 matrix instruction holds four consecutive i of
// one j at a time, so results leave in vectors.  Both operands go from memory to LDS without
// passing registers (16 bytes per lane, in buffer loads whose range check gives zeros past the
// last row), 128 bytes of the contraction (64 bf16 or 128 e4m3 values) per step: whole cache
// lines.  (Measured with the loads alone, 256 x 256 tiles of 16-bit rows out of L2: 128-byte
// pieces 24.6 TB/s over the chip, 64-byte pieces 15.0, from which the product cannot pass
// 1100 TFLOP/s.)  A step is multiplied in two halves, and the fragments of a half are read
// from LDS while the half before it is multiplied.
//
// An operand comes in one of two forms:
//   rows along c      [index][c], c contiguous: LDS rows of 128 bytes, whose 16-byte chunks are
//                     exchanged within the row by the row's number, so that the 16 rows that
//                     a fragment reads at once lie in different banks;
//   rows across c     [c][index], index contiguous (bf16): LDS rows of T indexes, read by the
//                     transposing LDS load; their 32-byte chunks are exchanged likewise.
#pragma once

#include "layer.h"
#include "wave.h"

#include "ep_layer.h"

#include <type_traits>

namespace ep {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

#define EP_LDS __attribute__((address_space(3)))

constexpr int kStepBytes = 128;  // bytes of the contraction per step, rows along c
constexpr int kStepRows = 64;   // rows of the contraction per step, rows across c
constexpr uint32_t kNowhere = 0x80000000u;  // an offset past every buffer's range

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const char *base, uint32_t bytes) {
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    const uint64_t u = ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32) |
                       (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a);
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(u), 0,
                                             (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t offset, char EP_LDS *dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (void EP_LDS *)dst, 16, (int)offset, 0, 0, 0);
}

// 1 KiB loads of a T-index operand per wave and step.  An operand with fewer of them than
// there are waves is loaded by several waves alike, so that every wave counts the same.
template <int T, int W>
constexpr int loads_per_wave() {
    static_assert(T / 8 % W == 0 || W % (T / 8) == 0, "every wave loads as much");
    return T / 8 > W ? T / 8 / W : 1;
}

// An operand with rows along c: T rows, loaded by W waves.
template <int T, int W>
struct AlongC {
    static constexpr int kLoads = loads_per_wave<T, W>();
    static constexpr bool kChained = false;
    const char *base;
    uint32_t left;    // bytes from base to the end of the operand
    int32_t bytes;    // bytes of the contraction left
    uint32_t offset[kLoads];

    // The chunk that a row's chunk number `p` holds.
    __device__ __forceinline__ static int swizzle(int row, int p) { return p ^ ((row >> 1) & 7); }
    __device__ __forceinline__ static int load_number(int wave, int q) { return (wave * kLoads + q) % (T / 8); }

    // row_offset(r): the byte offset from base of tile row r, or kNowhere.
    template <typename F>
    __device__ __forceinline__ void init(const char *b, uint32_t size, int32_t contraction_bytes, int wave, int lane,
                                         F row_offset) {
        base = b;
        left = size;
        bytes = contraction_bytes;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int row = load_number(wave, q) * 8 + lane / 8;
            offset[q] = row_offset(row) + swizzle(row, lane % 8) * 16;
        }
    }
    __device__ __forceinline__ void skip(int32_t steps) {
        base += (int64_t)steps * kStepBytes;
        left -= (uint32_t)(steps * kStepBytes);
        bytes -= steps * kStepBytes;
    }
    // A step's loads: begin (zeros where it is not live), the kLoads loads, end.
    __amdgpu_buffer_rsrc_t range;
    __device__ __forceinline__ void begin(bool live) { range = buffer_of(base, live ? left : 0); }
    __device__ __forceinline__ void load(int q, char EP_LDS *lds, int wave, int lane) {
        // the last step may be shorter: zeros past the contraction's end
        const int row = load_number(wave, q) * 8 + lane / 8;
        load_to_lds(range, swizzle(row, lane % 8) * 16 < bytes ? offset[q] : kNowhere, lds + load_number(wave, q) * 1024);
    }
    __device__ __forceinline__ void end() {
        base += kStepBytes;
        left -= kStepBytes;
        bytes -= kStepBytes;
    }
    // Fragment k of a wave whose first index is index0, quarter h (0..3) of the step: the 16
    // bytes of row index0 + 32 k + lane % 32 that lane group lane / 32 takes.  The places
    // within the fragment are the same for every k.
    uint32_t at[4];
    __device__ __forceinline__ void aim(int index0, int lane) {
#pragma unroll
        for (int h = 0; h < 4; ++h)
            at[h] = (uint32_t)((index0 + lane % 32) * 128 + swizzle(lane % 32, h * 2 + lane / 32) * 16);
    }
    __device__ __forceinline__ i32x4 read(const char EP_LDS *lds, int k, int h) const {
        return *reinterpret_cast<const i32x4 EP_LDS *>(lds + at[h] + k * 32 * 128);
    }
};

// The transposing LDS load.  The restricted pointer, once inlined, gives the load alias information, as a
// plain load's type does; without any the compiler waits before it for every load into LDS, also those
// that have one and a half steps to land.  (8192 rows of two 4096 x 4096 experts: dx 282 us instead of 249,
// dw 232 instead of 218.)
__device__ __forceinline__ s16x4 read_transposed(const s16x4 EP_LDS *__restrict__ p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<s16x4 EP_LDS *>(p));
}

// A bf16 operand with rows across c: T indexes per row, loaded by W waves.
template <int T, int W, int FRAGMENTS>
struct AcrossC {
    static constexpr int kLoads = loads_per_wave<T, W>();
    static constexpr bool kChained = false;
    static constexpr int kChunks = T / 16;  // 32-byte chunks of a row
    const char *base;
    int64_t stride;  // bytes of a row
    int64_t rows;    // rows of the contraction left
    uint32_t offset[kLoads];

    // What a row's chunk numbers are exchanged with.  It stays within the row's chunks: 4, 8 or
    // 16 of them, or 12, where only neighbouring pairs change places.
    static_assert(kChunks == 4 || kChunks == 8 || kChunks == 12 || kChunks == 16, "");
    __device__ __forceinline__ static int key(int row) {
        return kChunks % 8 ? (row >> 1 & 1) << 1 : kChunks == 8 ? (row & 3) << 1 : (row & 3) << 1 | (row >> 3 & 1) << 3;
    }
    __device__ __forceinline__ static int load_number(int wave, int q) { return (wave * kLoads + q) % (T / 8); }

    __device__ __forceinline__ void init(const char *b, int64_t row_bytes, int64_t n, int64_t index0, int wave, int lane) {
        base = b;
        stride = row_bytes;
        rows = n;
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            offset[q] = (uint32_t)(row_of(q, wave, lane) * stride) + column_of(q, (uint32_t)index0, wave, lane);
    }
    // Load q of a step: the row of the step that this lane brings, and its byte within the row.
    __device__ __forceinline__ static int row_of(int q, int wave, int lane) {
        return (load_number(wave, q) * 1024 + lane * 16) / (2 * T);
    }
    __device__ __forceinline__ static uint32_t column_of(int q, uint32_t index0, int wave, int lane) {
        const int p = load_number(wave, q) * 1024 + lane * 16;
        const int row = p / (2 * T), chunk = p % (2 * T) / 32, half = p / 16 % 2;
        return index0 * 2 + (uint32_t)((chunk ^ key(row)) * 32 + half * 16);
    }
    __device__ __forceinline__ void skip(int32_t steps) {
        base += (int64_t)steps * kStepRows * stride;
        rows -= (int64_t)steps * kStepRows;
    }
    __amdgpu_buffer_rsrc_t range;
    __device__ __forceinline__ void begin(bool live) {
        const int64_t n = !live ? 0 : rows < kStepRows ? rows : kStepRows;
        range = buffer_of(base, (uint32_t)(n * stride));
    }
    __device__ __forceinline__ void load(int q, char EP_LDS *lds, int wave, int) {
        load_to_lds(range, offset[q], lds + load_number(wave, q) * 1024);
    }
    __device__ __forceinline__ void end() {
        base += kStepRows * stride;
        rows -= kStepRows;
    }
    // As AlongC's, by the transposing load: it gives a lane four rows of one column, the sixteen
    // lanes of a group addressing those rows in 8-byte pieces.  The key looks at the bits 0, 1
    // and 3 of the row, which the quarter (16 rows) and the second four rows leave alone.
    uint32_t at[FRAGMENTS];
    __device__ __forceinline__ void aim(int index0, int lane) {
        const int q = lane % 16, row = lane / 32 * 8 + q / 4;
#pragma unroll
        for (int k = 0; k < FRAGMENTS; ++k)
            at[k] = (uint32_t)(row * (2 * T) + (((index0 + 32 * k) / 16 + lane / 16 % 2) ^ key(row)) * 32 + q % 4 * 8);
    }
    __device__ __forceinline__ i32x4 read(const char EP_LDS *lds, int k, int h) const {
        const char EP_LDS *p = lds + at[k] + h * 16 * (2 * T);
        const s16x4 a = read_transposed((const s16x4 EP_LDS *)p);
        const s16x4 b = read_transposed((const s16x4 EP_LDS *)(p + 4 * (2 * T)));
        return __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// TI x TJ tile, WI x WJ waves of FI x FJ fragments each, STAGES steps in LDS.
template <int TI, int TJ, int WI, int WJ, int STAGES>
struct TileShape {
    static constexpr int kI = TI, kJ = TJ, kWavesI = WI, kWavesJ = WJ, kWaves = WI * WJ, kThreads = kWaves * 64;
    static constexpr int FI = TI / WI / 32, FJ = TJ / WJ / 32, kStages = STAGES;
    static constexpr int kStageBytes = (TI + TJ) * kStepBytes;
    static_assert(FI * WI * 32 == TI && FJ * WJ * 32 == TJ && STAGES >= 2, "");
};

// What is multiplied: bf16 values; e4m3 values by the 8-bit matrix instruction; or e4m3 values
// widened to bf16, which holds each of them exactly.
enum class Mul { kBf16, kF8, kF8Wide };

__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Half a step's fragments of one wave: 32 bytes per lane and 32 indexes.
template <class S>
struct Fragments {
    i32x4 a[S::FI][2], b[S::FJ][2];
};

// Reads number `r` of the 2 (FI + FJ) fragments of a half.
template <class S, class OpA, class OpB>
__device__ __forceinline__ void read_fragment(Fragments<S> &f, int r, const OpA &a, const OpB &b, const char EP_LDS *stage,
                                              int half) {
    const int h = r / (S::FI + S::FJ), k = r % (S::FI + S::FJ);
    if (k < S::FI)
        f.a[k][h] = a.read(stage, k, 2 * half + h);
    else
        f.b[k - S::FI][h] = b.read(stage + S::kI * kStepBytes, k - S::FI, 2 * half + h);
}

// Multiplies a half: kMuls matrix instructions, after each of which `behind(m)` runs.  The
// compiler keeps that order: left to itself it puts the LDS reads and loads that belong
// between them behind all of them, and the wave waits.
template <class S, Mul M>
constexpr int muls() {
    return S::FI * S::FJ * (M == Mul::kF8 ? 1 : M == Mul::kBf16 ? 2 : 4);
}
template <class S, Mul M, typename F>
__device__ __forceinline__ void multiply(const Fragments<S> &f, f32x16 (&acc)[S::FI][S::FJ], F behind) {
    if constexpr (M == Mul::kF8) {
#pragma unroll
        for (int i = 0; i < S::FI; ++i)
#pragma unroll
            for (int j = 0; j < S::FJ; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                    __builtin_shufflevector(f.a[i][0], f.a[i][1], 0, 1, 2, 3, 4, 5, 6, 7),
                    __builtin_shufflevector(f.b[j][0], f.b[j][1], 0, 1, 2, 3, 4, 5, 6, 7), acc[i][j], 0, 0, 0, 0x7f7f7f7f,
                    0, 0x7f7f7f7f);
                behind(i * S::FJ + j);
                __builtin_amdgcn_sched_barrier(0);
            }
    } else {
        constexpr int kParts = M == Mul::kF8Wide ? 2 : 1;  // matrix instructions per 16 bytes
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                bf16x8 a[S::FI], b[S::FJ];
#pragma unroll
                for (int i = 0; i < S::FI; ++i)
                    a[i] = M == Mul::kF8Wide ? widen(f.a[i][h][2 * p], f.a[i][h][2 * p + 1])
                                             : __builtin_bit_cast(bf16x8, f.a[i][h]);
#pragma unroll
                for (int j = 0; j < S::FJ; ++j)
                    b[j] = M == Mul::kF8Wide ? widen(f.b[j][h][2 * p], f.b[j][h][2 * p + 1])
                                             : __builtin_bit_cast(bf16x8, f.b[j][h]);
#pragma unroll
                for (int i = 0; i < S::FI; ++i)
#pragma unroll
                    for (int j = 0; j < S::FJ; ++j) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
                        behind(((h * kParts + p) * S::FI + i) * S::FJ + j);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
    }
}

// Waits until at most VM of this wave's loads are in flight, with LDS also until its LDS reads
// are done, and then until every wave of the workgroup has come this far.
template <int VM, bool LDS>
__device__ __forceinline__ void wait_and_meet() {
    static_assert(VM < 64, "");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((VM & 15) | 7 << 4 | (LDS ? 0 : 15) << 8 | VM >> 4 << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
constexpr int kAnyLoads = 63;  // no wait for loads

// An operand may be chained (kChained: adapter_tile.h): its contraction goes on into a second part of
// another form behind the `first` steps left of the plain one, and both operands of a tile are.
// The steps that load the plain part have a loop of their own, without the second one's registers.
template <bool PLAIN, class Op>
__device__ __forceinline__ void begin_loads(Op &o, bool live) {
    if constexpr (PLAIN && Op::kChained)
        o.First::begin(live);
    else
        o.begin(live);
}
template <bool PLAIN, class Op>
__device__ __forceinline__ void end_loads(Op &o) {
    if constexpr (PLAIN && Op::kChained) {
        o.First::end();
        --o.first;
    } else {
        o.end();
    }
}

// Runs `steps` steps of the contraction into acc.  Step t's place in LDS is t % STAGES.
//
// A wave enters step t with its first half in registers.  Between the matrix instructions of
// the step it
//   - reads the second half, early;
//   - after a barrier (every wave has read the whole step) loads step t + STAGES into the
//     place of step t, spread over half a step;
//   - late, after a barrier (every wave's part of step t + 1 has landed), reads the first half
//     of step t + 1.
// So with two stages a load has one and a half steps to land.  Loads past the last step bring
// zeros, so that the count of loads in flight is the same in every step.
template <class S, Mul M, class OpA, class OpB>
__device__ __forceinline__ void tile_product(OpA &a, OpB &b, int32_t steps, char EP_LDS *lds, int wave, int lane,
                                             f32x16 (&acc)[S::FI][S::FJ]) {
    constexpr int kLoads = OpA::kLoads + OpB::kLoads, kReads = 2 * (S::FI + S::FJ), kMuls = muls<S, M>();
    constexpr int kReadSlots = kMuls * 3 / 8 > 0 ? kMuls * 3 / 8 : 1;  // matrix instructions that a half's reads stand behind
    constexpr int kFree = kMuls / 2;                // behind this one the step's place is free
    constexpr int kLanded = 2 * kMuls - kReadSlots;  // behind this one the next step is there
    if (steps <= 0)
        return;
    a.aim(wave % S::kWavesI * S::FI * 32, lane);
    b.aim(wave / S::kWavesI * S::FJ * 32, lane);
    const auto load = [&](int q, char EP_LDS *stage) {
        if (q < OpA::kLoads)
            a.load(q, stage, wave, lane);
        else
            b.load(q - OpA::kLoads, stage + S::kI * kStepBytes, wave, lane);
    };
#pragma unroll
    for (int s = 0; s < S::kStages; ++s) {
        a.begin(s < steps);
        b.begin(s < steps);
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            load(q, lds + s * S::kStageBytes);
        a.end();
        b.end();
    }
    Fragments<S> first, second;
    wait_and_meet<(S::kStages - 1) * kLoads, false>();
#pragma unroll
    for (int r = 0; r < kReads; ++r)
        read_fragment<S>(first, r, a, b, lds, 0);
    int place = 0;
    // Step t; PLAIN: the loads it issues are of operands in their plain form.
    const auto step = [&](int32_t t, auto plain) {
        constexpr bool PLAIN = decltype(plain)::value;
        char EP_LDS *here = lds + place * S::kStageBytes;
        place = place + 1 == S::kStages ? 0 : place + 1;
        const char EP_LDS *next = lds + place * S::kStageBytes;
        begin_loads<PLAIN>(a, t + S::kStages < steps);
        begin_loads<PLAIN>(b, t + S::kStages < steps);
        const auto behind = [&](int m) {
#pragma unroll
            for (int r = 0; r < kReads; ++r)
                if (r * kReadSlots / kReads == m)
                    read_fragment<S>(second, r, a, b, here, 1);
            if (m == kFree)
                wait_and_meet<kAnyLoads, true>();
#pragma unroll
            for (int q = 0; q < kLoads; ++q)
                if (kFree + q * kMuls / kLoads == m)
                    load(q, here);
            if (m == kLanded)
                wait_and_meet<(S::kStages - 1) * kLoads, false>();
#pragma unroll
            for (int r = 0; r < kReads; ++r)
                if (kLanded + r * kReadSlots / kReads == m)
                    read_fragment<S>(first, r, a, b, next, 0);
        };
        multiply<S, M>(first, acc, behind);
        multiply<S, M>(second, acc, [&](int m) { behind(kMuls + m); });
        end_loads<PLAIN>(a);
        end_loads<PLAIN>(b);
    };
    int32_t t = 0;
    if constexpr (OpA::kChained)  // as long as both operands' loads are of their first part
        for (; t < steps && a.first > 0; ++t)
            step(t, std::true_type{});
    for (; t < steps; ++t)
        step(t, std::integral_constant<bool, !OpA::kChained>{});
    // every load has landed and every read is done before the kernel uses the LDS again
    wait_and_meet<0, true>();
}

// Hands the tile out in rows: result(row, col, v, f) gets the PER neighbouring sums C[row][col..]
// of tile row `row` from a lane whose neighbours get the columns beside them, so that results
// leave in whole cache lines.  (The accumulators themselves hold four columns of 32 rows per
// instruction.)  A wave turns its own 32 rows at a time over in its own piece of LDS; a lane
// always gets the same columns, first_col(...) + 0 .. PER-1.  What a row needs from memory
// besides, f = fetch(row), is on its way four turns earlier (rows past the wave's own may be
// fetched in vain).
template <class S, int PER>
__device__ __forceinline__ int first_col(int wave, int lane) {
    return wave % S::kWavesI * S::FI * 32 + lane % (S::FI * 32 / PER) * PER;
}
template <class S, int PER, typename G, typename F>
__device__ __forceinline__ void tile_rows_out(const f32x16 (&acc)[S::FI][S::FJ], char EP_LDS *lds, int wave, int lane, G fetch,
                                              F result) {
    constexpr int kCols = S::FI * 32, kStride = kCols + 4;    // floats of a row, and with the padding
    constexpr int kLanes = kCols / PER, kRows = 64 / kLanes;  // lanes of a row, rows at a time
    constexpr int kTurns = 32 / kRows, kAhead = 4;
    static_assert(S::kWaves * 32 * kStride * 4 <= S::kStages * S::kStageBytes, "");
    float EP_LDS *own = reinterpret_cast<float EP_LDS *>(lds) + wave * 32 * kStride;
    const float EP_LDS *from = own + lane / kLanes * kStride + lane % kLanes * PER;
    int row = wave / S::kWavesI * S::FJ * 32 + lane / kLanes;
    decltype(fetch(0)) got[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        got[i] = fetch(row + i * kRows);
#pragma unroll
    for (int j = 0; j < S::FJ; ++j) {
#pragma unroll
        for (int i = 0; i < S::FI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4 EP_LDS *>(own + lane % 32 * kStride + i * 32 + q * 8 + lane / 32 * 4) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __builtin_amdgcn_wave_barrier();
        // not unrolled: the epilogue's code, once per turn, would not stay in the instruction cache
#pragma unroll 1
        for (int r = 0; r < kTurns; ++r) {
            float v[PER];
#pragma unroll
            for (int q = 0; q < PER; q += 4) {
                const f32x4 x = *reinterpret_cast<const f32x4 EP_LDS *>(from + r * kRows * kStride + q);
                v[q] = x[0], v[q + 1] = x[1], v[q + 2] = x[2], v[q + 3] = x[3];
            }
            const auto now = got[0];
#pragma unroll
            for (int i = 0; i + 1 < kAhead; ++i)
                got[i] = got[i + 1];
            got[kAhead - 1] = fetch(row + kAhead * kRows);
            result(row, first_col<S, PER>(wave, lane), v, now);
            row += kRows;
        }
        __builtin_amdgcn_wave_barrier();
    }
}
struct Nothing {};
template <class S, typename F>
__device__ __forceinline__ void tile_results(const f32x16 (&acc)[S::FI][S::FJ], char EP_LDS *lds, int wave, int lane, F result) {
    tile_rows_out<S, 8>(
        acc, lds, wave, lane, [](int) { return Nothing{}; },
        [&](int row, int col, float *v, Nothing) { result(row, col, v); });
}

// ---- which rows a tile has --------------------------------------------------------
struct RowTile {
    int32_t e;     // expert, -1: no such tile
    int64_t row0;  // first row
    int32_t n;     // rows of the expert from row0 on, at most `per`
};

__device__ __forceinline__ int64_t clamp_row(int64_t r, int64_t rows) { return r < 0 ? 0 : r > rows ? rows : r; }

// The rows [begin, end) of expert e.
__device__ __forceinline__ void expert_rows(const int32_t *offsets, int64_t rows, int e, int64_t &begin, int64_t &end) {
    begin = offsets ? clamp_row(offsets[e], rows) : 0;
    end = offsets ? clamp_row(offsets[e + 1], rows) : rows;
    if (end < begin)
        end = begin;
}

// Row tiles in all: every expert's rows in tiles of `per`.  The same in every lane.
__device__ __forceinline__ int32_t count_row_tiles(const int32_t *offsets, int64_t rows, int E, int per, int lane) {
    int32_t total = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        int32_t n = 0;
        if (e0 + lane < E) {
            int64_t b, t;
            expert_rows(offsets, rows, e0 + lane, b, t);
            n = (int32_t)((uint32_t)(t - b + per - 1) / (uint32_t)per);
        }
        total += __builtin_amdgcn_readlane(wave_inclusive_scan(n), 63);
    }
    return total;
}

// Row tile number idx, expert after expert.
__device__ __forceinline__ RowTile find_row_tile(const int32_t *offsets, int64_t rows, int E, int per, int32_t idx, int lane) {
    int32_t before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        int64_t b = 0, t = 0;
        if (e0 + lane < E)
            expert_rows(offsets, rows, e0 + lane, b, t);
        const int32_t n = (int32_t)((uint32_t)(t - b + per - 1) / (uint32_t)per);
        const int32_t incl = wave_inclusive_scan(n);
        const uint64_t past = __ballot(before + incl > idx);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int32_t tile = idx - before - (__builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(n, at));
            const int64_t begin = (int64_t)__builtin_amdgcn_readlane((int32_t)b, at);  // rows < 2^31
            const int64_t end = (int64_t)__builtin_amdgcn_readlane((int32_t)t, at);
            const int64_t row0 = begin + (int64_t)tile * per;
            const int64_t left = end - row0;
            if (left <= 0)  // more tiles than 32 bits count: only where offsets decrease
                return {-1, 0, 0};
            return {e0 + at, row0, (int32_t)(left < per ? left : per)};
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    return {-1, 0, 0};
}

// ---- order of the tiles -----------------------------------------------------------
// Workgroup b of a grid of at least total + 8 takes tile number: workgroups go to the eight
// XCDs in turn, and each XCD (its own L2) gets one contiguous range of the tiles.  -1: none.
__device__ __forceinline__ int64_t tile_of_block(int64_t b, int64_t total) {
    const int64_t per = (total + 7) / 8;
    const int64_t t = (b % 8) * per + b / 8;
    return b / 8 < per && t < total ? t : -1;
}

// Within a range: kBand row tiles at a time against every column tile, so that tiles running
// at once share rows and columns in L2.
constexpr int kBand = 4;
__device__ __forceinline__ void tile_order(int64_t t, int32_t row_tiles, int32_t col_tiles, int32_t &row, int32_t &col) {
    const int64_t band = t / ((int64_t)kBand * col_tiles);
    const int32_t in = (int32_t)(t - band * kBand * col_tiles);
    const int32_t first = (int32_t)band * kBand;
    const int32_t h = row_tiles - first < kBand ? row_tiles - first : kBand;
    row = first + in % h;
    col = in / h;
}

constexpr int64_t kMostTiles = 1 << 30;  // of a grid (launch_traced refuses the ones too large for their workgroups)
// The most row tiles that any counts give: every expert that has rows may begin one more.
inline int64_t row_tiles_most(int64_t rows, int32_t E, int per) {
    const int64_t some = std::min<int64_t>(E, rows);
    return some + (rows - some) / per;
}

// The two large tiles, one workgroup of 8 waves per compute unit each.  A tile of Broad takes
// 0.78 of the time of one of Large (measured), a little more than its share; it wins where Large
// leaves a last turn of the chip nearly empty (8192 rows of two 4096 x 4096 experts: 528 tiles of
// Large in three turns 306 us, 699 of Broad in three turns 266 us).
typedef TileShape<256, 256, 4, 2, 2> Large;
typedef TileShape<256, 192, 4, 2, 2> Broad;
inline bool broad_wins(double tiles_large, double tiles_broad) {
    const auto turns = [](double tiles) { return (double)(int64_t)((tiles + kCus - 1) / kCus); };
    return turns(tiles_broad) * 0.78 < turns(tiles_large);
}
// Row tiles to expect: half a tile more than the rows fill for every expert, one at least.
inline double row_tiles_likely(int64_t rows, int32_t E, int per) {
    return E == 1 ? (double)((rows + per - 1) / per)
                  : std::max((double)std::min<int64_t>(E, rows), (double)rows / per + 0.5 * E);
}
inline bool broad_rows(int64_t rows, int32_t E, int64_t cols) {
    return broad_wins(row_tiles_likely(rows, E, Large::kJ) * cols, row_tiles_likely(rows, E, Broad::kJ) * cols);
}

// Small tiles, for sizes with fewer large tiles than compute units.
typedef TileShape<128, 128, 2, 2, 2> Medium;  // two workgroups per compute unit (64 KiB of LDS)
typedef TileShape<64, 64, 2, 2, 4> Small;     // two (64 KiB)
typedef TileShape<128, 32, 4, 1, 4> Tiny;     // two (80 KiB)
// What a step takes, in us, measured.  Small tiles: with a workgroup per compute unit (`less`) and
// with two, the most there are (`full`).  Large ones: with next to no compute unit busy and with
// all, in between by the share that is.
struct StepCost {
    bool two;
    double less, full;
};
constexpr StepCost kLargeCost{false, 1.10, 1.85}, kBroadCost{false, 0.86, 1.44}, kMediumCost{true, 0.55, 0.90},
    kSmallCost{true, 0.28, 0.43}, kTinyCost{true, 0.30, 0.50};
// Estimated us of `tiles` tiles whose contraction is cut into `parts` of `steps` steps: the
// turns of the workgroups, and for more than one part a second kernel and the fp32 sums
// written and read again (6 MB a us: most of them stay in the memory-side cache).  The longest tile
// has `longest` times as many steps as the mean one.
inline double estimate(StepCost cost, double tiles, int32_t parts, int32_t steps, int64_t outputs, double longest = 1.0) {
    const double groups = tiles * parts;
    double turns;
    if (cost.two) {
        turns = groups <= kCus ? cost.less * longest : cost.full * std::max(std::ceil(groups / (2 * kCus)), longest);
    } else {
        const double whole = std::floor(groups / kCus), rest = groups / kCus - whole;
        turns = whole * cost.full + (rest > 0 ? cost.less + rest * (cost.full - cost.less) : 0.0);
        turns = whole < 1 ? turns * longest : std::max(turns, cost.full * longest);
    }
    return turns * steps + (parts > 1 ? 3.0 + (double)parts * (double)outputs * 8 / 6e6 : 0.0);
}
constexpr int32_t kSplitSteps = 4;  // fewest steps of a part

// Activations, and their derivatives.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + quick_exp(-z)); }
// The normal distribution function from e = exp(-z^2 / 2).  Its tail is e G(|z|), G(x) = erfc(x / sqrt 2)
// exp(x^2 / 2) / 2, a smooth function of t = 1 / (1 + 0.3 x) that vanishes with t: t times a polynomial,
// fitted to G / t for x up to 14.5 by least squares whose weights were raised where the relative error was
// largest, until that was even (1.7e-7).  So the tail keeps its digits however small it is: with
// the arithmetic in fp32 it is within 16 2^-24 of itself, plus what e is off (1.2 z^2 2^-24).  The library's
// erf takes three times as long, which made the gradient of the gelu's product wait for it
// (62 us for 8192 x 4096 values, 49 with this one and four rows on their way at a time).
__device__ __forceinline__ float normal_cdf(float z, float e) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(z), 1.f));
    float p = fmaf(0.0354237221f, t, -0.156158388f);
    p = fmaf(p, t, 0.204556704f);
    p = fmaf(p, t, -0.0520339459f);
    p = fmaf(p, t, 0.127691746f);
    p = fmaf(p, t, 0.100175954f);
    p = fmaf(p, t, 0.120712139f);
    p = fmaf(p, t, 0.119632006f);
    const float tail = p * t * e;
    return z < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float silu_grad(float z) {
    const float s = sigmoid(z);
    return s * (1.f + z * (1.f - s));
}
// Eight values at a time: one branch on the activation for all of them.
template <typename F>
__device__ __forceinline__ void each8(float *v, F f) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
        v[q] = f(v[q]);
}
__device__ __forceinline__ void activate8(float *z, int act) {
    if (act == EP_ACT_RELU)
        each8(z, [](float v) { return v < 0.f ? 0.f : v; });  // a NaN stays one
    else if (act == EP_ACT_SILU)
        each8(z, [](float v) { return v * sigmoid(v); });
    else if (act == EP_ACT_GELU)
        each8(z, [](float v) { return v * normal_cdf(v, quick_exp(-0.5f * v * v)); });
}
__device__ __forceinline__ void activation_grad8(float *z, int act) {
    if (act == EP_ACT_RELU)
        each8(z, [](float v) { return v > 0.f ? 1.f : v != v ? v : 0.f; });
    else if (act == EP_ACT_SILU)
        each8(z, silu_grad);
    else if (act == EP_ACT_GELU)
        each8(z, [](float v) {
            const float e = quick_exp(-0.5f * v * v);
            return normal_cdf(v, e) + v * e * 0.3989422804014327f;
        });
    else
        each8(z, [](float) { return 1.f; });
}

}  // namespace ep
