// product_tile.h -- the MFMA tile shared by the experts' product and its gradients.
//
// A workgroup computes a TI x TJ tile of C[j][i] = sum_c A[i][c] B[j][c].  i is the index
// that is contiguous in C: a lane of the 16x16 matrix instruction holds four consecutive i of
// one j, so results leave in vectors.  Both operands go from memory to LDS without passing
// registers (16 bytes per lane, in buffer loads whose range check gives zeros past the last
// row), 128 bytes of the contraction (64 bf16 or 128 e4m3 values) per step.
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

namespace ep {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

#define EP_LDS __attribute__((address_space(3)))

constexpr int kStepBytes = 128;     // bytes of the contraction per step, rows along c
constexpr int kStepRows = 64;       // rows of the contraction per step, rows across c
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

// An operand with rows along c: T rows, loaded by W waves.
template <int T, int W>
struct AlongC {
    static constexpr int kLoads = T / 8 / W;  // 1 KiB loads per wave and step
    static_assert(T % (8 * W) == 0, "");
    const char *base;
    uint32_t left;        // bytes from base to the end of the operand
    uint32_t offset[kLoads];
    int32_t tail;         // bytes of the contraction in the last step (1..128)

    // The chunk that a row's chunk number `p` holds.
    __device__ __forceinline__ static int swizzle(int row, int p) { return p ^ ((row >> 1) & 7); }

    // row_offset(r): the byte offset from base of tile row r, or kNowhere.
    template <typename F>
    __device__ __forceinline__ void init(const char *b, uint32_t bytes, int32_t contraction_bytes, int wave, int lane,
                                         F row_offset) {
        base = b;
        left = bytes;
        tail = (contraction_bytes - 1) % kStepBytes + 1;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int row = (wave * kLoads + q) * 8 + lane / 8;
            offset[q] = row_offset(row) + swizzle(row, lane % 8) * 16;
        }
    }
    __device__ __forceinline__ void skip(int64_t steps) {
        base += steps * kStepBytes;
        left -= (uint32_t)(steps * kStepBytes);
    }
    __device__ __forceinline__ void load(char EP_LDS *lds, int wave, int lane, bool last) {
        const __amdgpu_buffer_rsrc_t r = buffer_of(base, left);
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            uint32_t o = offset[q];
            if (last) {
                const int row = (wave * kLoads + q) * 8 + lane / 8;
                o = swizzle(row, lane % 8) * 16 < tail ? o : kNowhere;
            }
            load_to_lds(r, o, lds + (wave * kLoads + q) * 1024);
        }
        base += kStepBytes;
        left -= kStepBytes;
    }
    // The 16 bytes of fragment row `row0 + lane % 16` that half h (0, 1) of the step gives
    // lane group lane / 16.
    __device__ __forceinline__ static i32x4 read(const char EP_LDS *lds, int row0, int h, int lane) {
        const int row = row0 + lane % 16;
        return *reinterpret_cast<const i32x4 EP_LDS *>(lds + row * 128 + swizzle(row, h * 4 + lane / 16) * 16);
    }
};

// A bf16 operand with rows across c: T indexes per row, loaded by W waves.
template <int T, int W>
struct AcrossC {
    static constexpr int kLoads = T / 8 / W;
    static constexpr int kChunks = T / 16;  // 32-byte chunks of a row
    static_assert(T % (8 * W) == 0, "");
    const char *base;
    int64_t stride;  // bytes of a row
    int64_t rows;    // rows of the contraction left
    uint32_t offset[kLoads];

    __device__ __forceinline__ static int key(int row) { return ((row & 3) | ((row >> 3) & 3) << 2) & (kChunks - 1); }

    __device__ __forceinline__ void init(const char *b, int64_t row_bytes, int64_t n, int64_t index0, int wave, int lane) {
        base = b;
        stride = row_bytes;
        rows = n;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int p = (wave * kLoads + q) * 1024 + lane * 16;
            const int row = p / (2 * T), chunk = p % (2 * T) / 32, half = p / 16 % 2;
            offset[q] = (uint32_t)(row * stride + index0 * 2 + (chunk ^ key(row)) * 32 + half * 16);
        }
    }
    __device__ __forceinline__ void load(char EP_LDS *lds, int wave, int, bool) {
        const int64_t n = rows < kStepRows ? rows : kStepRows;
        const __amdgpu_buffer_rsrc_t r = buffer_of(base, (uint32_t)(n * stride));
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            load_to_lds(r, offset[q], lds + (wave * kLoads + q) * 1024);
        base += kStepRows * stride;
        rows -= kStepRows;
    }
    // As AlongC::read for the indexes row0 + lane % 16: the transposing load gives a lane four
    // rows of one column, the sixteen lanes of a group addressing those rows in 8-byte pieces.
    __device__ __forceinline__ static i32x4 read(const char EP_LDS *lds, int index0, int h, int lane) {
        const int g = lane / 16, q = lane % 16;
        const int row = h * 32 + g * 8 + q / 4;
        const char EP_LDS *p = lds + row * (2 * T) + ((index0 / 16) ^ key(row)) * 32 + q % 4 * 8;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 EP_LDS *)p);
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 EP_LDS *)(p + 4 * (2 * T)));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// TI x TJ tile, WI x WJ waves of FI x FJ fragments each.
template <int TI, int TJ, int WI, int WJ>
struct TileShape {
    static constexpr int kI = TI, kJ = TJ, kWavesI = WI, kWavesJ = WJ, kWaves = WI * WJ, kThreads = kWaves * 64;
    static constexpr int FI = TI / WI / 16, FJ = TJ / WJ / 16;
    static constexpr int kStageBytes = (TI + TJ) * kStepBytes;
};

// What is multiplied: bf16 values; e4m3 values by the 8-bit matrix instruction; or e4m3 values
// widened to bf16, which holds each of them exactly.
enum class Mul { kBf16, kF8, kF8Wide };

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Runs `steps` steps of the contraction into acc.  Two LDS stages: a step's loads are issued
// before the step before it is multiplied.
template <class S, Mul M, class OpA, class OpB>
__device__ __forceinline__ void tile_product(OpA &a, OpB &b, int64_t steps, int64_t steps_to_end, char EP_LDS *lds,
                                             int wave, int lane, f32x4 (&acc)[S::FI][S::FJ]) {
    const int wi = wave % S::kWavesI, wj = wave / S::kWavesI;
    const int i0 = wi * S::FI * 16, j0 = wj * S::FJ * 16;
    if (steps <= 0)
        return;
    a.load(lds, wave, lane, steps_to_end == 1);
    b.load(lds + S::kI * kStepBytes, wave, lane, steps_to_end == 1);
    for (int64_t s = 0; s < steps; ++s) {
        // this wave's loads of the step have landed, and after the barrier every wave's; the
        // other stage has been read by every wave
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        char EP_LDS *cur = lds + (s & 1) * S::kStageBytes;
        if (s + 1 < steps) {
            char EP_LDS *next = lds + ((s + 1) & 1) * S::kStageBytes;
            a.load(next, wave, lane, s + 2 == steps_to_end);
            b.load(next + S::kI * kStepBytes, wave, lane, s + 2 == steps_to_end);
        }
        const char EP_LDS *la = cur, *lb = cur + S::kI * kStepBytes;
        if constexpr (M == Mul::kF8) {
            i32x8 fa[S::FI], fb[S::FJ];
#pragma unroll
            for (int f = 0; f < S::FI; ++f)
                fa[f] = __builtin_shufflevector(OpA::read(la, i0 + f * 16, 0, lane), OpA::read(la, i0 + f * 16, 1, lane),
                                                0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int f = 0; f < S::FJ; ++f)
                fb[f] = __builtin_shufflevector(OpB::read(lb, j0 + f * 16, 0, lane), OpB::read(lb, j0 + f * 16, 1, lane),
                                                0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int i = 0; i < S::FI; ++i)
#pragma unroll
                for (int j = 0; j < S::FJ; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i], fb[j], acc[i][j], 0, 0, 0,
                                                                                0x7f7f7f7f, 0, 0x7f7f7f7f);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                i32x4 fa[S::FI], fb[S::FJ];
#pragma unroll
                for (int f = 0; f < S::FI; ++f)
                    fa[f] = OpA::read(la, i0 + f * 16, h, lane);
#pragma unroll
                for (int f = 0; f < S::FJ; ++f)
                    fb[f] = OpB::read(lb, j0 + f * 16, h, lane);
                constexpr int kParts = M == Mul::kF8Wide ? 2 : 1;  // matrix instructions per 16 bytes
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    bf16x8 va[S::FI], vb[S::FJ];
#pragma unroll
                    for (int f = 0; f < S::FI; ++f)
                        va[f] = M == Mul::kF8Wide ? widen(fa[f][2 * p], fa[f][2 * p + 1]) : __builtin_bit_cast(bf16x8, fa[f]);
#pragma unroll
                    for (int f = 0; f < S::FJ; ++f)
                        vb[f] = M == Mul::kF8Wide ? widen(fb[f][2 * p], fb[f][2 * p + 1]) : __builtin_bit_cast(bf16x8, fb[f]);
#pragma unroll
                    for (int i = 0; i < S::FI; ++i)
#pragma unroll
                        for (int j = 0; j < S::FJ; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[i], vb[j], acc[i][j], 0, 0, 0);
                }
            }
        }
        // every LDS read of this stage is done before the barrier that lets it be overwritten
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// ---- which rows a tile has --------------------------------------------------------
struct RowTile {
    int32_t e;     // expert, -1: no such tile
    int64_t row0;  // first row
    int32_t n;     // rows of the expert from row0 on, at most `per`
    int64_t tiles; // row tiles in all
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
            n = (int32_t)((t - b + per - 1) / per);
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
        const int32_t n = (int32_t)((t - b + per - 1) / per);
        const int32_t incl = wave_inclusive_scan(n);
        const uint64_t past = __ballot(before + incl > idx);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int32_t tile = idx - before - (__builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(n, at));
            const int64_t begin = (int64_t)__builtin_amdgcn_readlane((int32_t)b, at);  // rows < 2^31
            const int64_t end = (int64_t)__builtin_amdgcn_readlane((int32_t)t, at);
            const int64_t row0 = begin + (int64_t)tile * per;
            const int64_t left = end - row0;
            return {e0 + at, row0, (int32_t)(left < per ? left : per), 0};
        }
        before += __builtin_amdgcn_readlane(incl, 63);
    }
    return {-1, 0, 0, 0};
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
inline int64_t row_tiles_most(int64_t rows, int32_t E, int per) { return rows / per + std::min<int64_t>(E, rows); }

// Activation of one value, and its derivative.
__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
__device__ __forceinline__ float activation(float z, int act) {
    switch (act) {
    case 1: return z < 0.f ? 0.f : z;  // a NaN stays one
    case 2: return z * sigmoid(z);
    case 3: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    default: return z;
    }
}
__device__ __forceinline__ float activation_grad(float z, int act) {
    switch (act) {
    case 1: return z > 0.f ? 1.f : z != z ? z : 0.f;
    case 2: {
        const float s = sigmoid(z);
        return s * (1.f + z * (1.f - s));
    }
    case 3:
        return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.3989422804014327f;
    default: return 1.f;
    }
}

}  // namespace ep
