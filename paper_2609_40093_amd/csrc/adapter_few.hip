// adapter_few.hip -- the adapters' product for few rows (a decode step), in two kernels:
//   the first  makes parts of x W^T (tiles of product_tile.h, rows as they come) and parts of
//              x[order] a_a^T, side by side in one launch, since neither needs the other;
//   the second adds the parts up, in order, makes two bf16 values of each low-rank one (adapter_low.hip),
//              adds their products with b and runs the epilogue.
// Bound by the latencies of dependent loads and by the bytes of W, a and b: 64 rows of 7168 by 2048, 32 adapters of
// 16 ranks (38 MB) 10.6 and 8.5 us; 256 rows 7168 x 4096, 64 adapters of 32 ranks, without W (52 MB) 11.1 and 9.3.
//
// The low-rank parts: a workgroup takes 16 rows of one adapter, 16 ranks and a part of the contraction
// short enough for every load of its four waves to be on its way at once.  The second kernel: a wave
// takes 16 rows in the adapters' order, whoever's, and 32 columns (gated: 16 and their ups): it
// multiplies all 16 rows with the b of each adapter among them and keeps the rows that have it, so an
// adapter's infinities and NaN reach no other rows.
#include "adapter_tile.h"
#include "product_finish.h"
#include "product_plan.h"

namespace ep {
namespace {

constexpr int kRows = 16, kRanks = 16, kAhead = 6;  // kAhead: 64-value pieces of the contraction of a wave
constexpr int kPiece = 64, kPartPieces = 4 * kAhead;
constexpr int kPartsAhead = 8;  // parts of a sum on their way at once

// What the two kernels share.
struct FewArgs {
    ProductArgs p;
    const int32_t *order, *offsets;
    int32_t A, R;
    const uint16_t *a, *b;
    const float *scale;
    uint16_t *low;     // may be null
    float *low_parts;  // [low_count][rows][R] in the adapters' order
    int32_t low_count, low_tiles, rank_tiles;
    int32_t parts, row_tiles, col_tiles;  // of x W^T: a.p.partial [parts][rows][Nw]; parts 0: no W
};

__device__ __forceinline__ void low_part(const FewArgs &f, int32_t block, f32x4 EP_LDS *sums, int lane, int wave) {
    const int32_t tile = block % f.low_tiles, rest = block / f.low_tiles;
    const int rank0 = rest % f.rank_tiles * kRanks, part = rest / f.rank_tiles;
    const RowTile rt = find_row_tile(f.offsets, f.p.rows, f.A, kRows, tile, lane);
    if (rt.e < 0)
        return;
    const int K = f.p.K, g = lane / 16;  // g: which 16 bytes of a fragment's 64 this lane takes
    const int rank = rank0 + lane % 16;
    const bool has_a = rank < f.R;
    const uint16_t *ar = f.a + ((int64_t)rt.e * f.R + (has_a ? rank : 0)) * K;
    const int32_t r = lane % 16 < rt.n ? row_at(f.order, f.p.rows, rt.row0 + lane % 16) : -1;
    const uint16_t *xr = static_cast<const uint16_t *>(f.p.x) + (r >= 0 ? (int64_t)r * K : 0);
    const int32_t k0 = (part * kPartPieces + wave) * kPiece + g * 8;
    u32x4 av[kAhead][2], xv[kAhead][2];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t k = k0 + u * 4 * kPiece + h * 32;
            av[u][h] = u32x4{0, 0, 0, 0};
            if (k < K && has_a)
                av[u][h] = *reinterpret_cast<const u32x4 *>(ar + k);
        }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t k = k0 + u * 4 * kPiece + h * 32;
            xv[u][h] = u32x4{0, 0, 0, 0};
            if (k < K && r >= 0)
                xv[u][h] = *reinterpret_cast<const u32x4 *>(xr + k);
        }
    f32x4 acc = {};
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av[u][h]),
                                                          __builtin_bit_cast(bf16x8, xv[u][h]), acc, 0, 0, 0);
    sums[wave * 64 + lane] = acc;
    __syncthreads();
    if (wave > 0)
        return;
    const f32x4 s = (sums[lane] + sums[64 + lane]) + (sums[128 + lane] + sums[192 + lane]);
    const int q = rank0 + g * 4, row = lane % 16;  // a lane holds four ranks of one row
    if (row < rt.n && q < f.R)
        *reinterpret_cast<f32x4 *>(f.low_parts + ((int64_t)part * f.p.rows + rt.row0 + row) * f.R + q) = s;
}

// The low-rank parts alone, with next to no LDS: all workgroups at once.
__global__ __launch_bounds__(256) void adapter_few_low_kernel(FewArgs f) {
    __shared__ f32x4 sums[256];
    low_part(f, (int32_t)blockIdx.x, (f32x4 EP_LDS *)sums, threadIdx.x & 63, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
}

template <class S, bool GATED>
__global__ __launch_bounds__(S::kThreads) void adapter_few_kernel(FewArgs f) {
    static_assert(S::kThreads == 256, "");
    __shared__ __attribute__((aligned(1024))) char lds[S::kStages * S::kStageBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t low_blocks = f.low_tiles * f.rank_tiles * f.low_count;
    if ((int32_t)blockIdx.x < low_blocks)
        return low_part(f, (int32_t)blockIdx.x, (f32x4 EP_LDS *)(char EP_LDS *)lds, lane, wave);
    const ProductArgs &a = f.p;
    const int64_t tiles = (int64_t)f.row_tiles * f.col_tiles;
    int64_t t = tile_of_block((int64_t)blockIdx.x - low_blocks, tiles * f.parts);
    if (t < 0)
        return;
    const int32_t part = (int32_t)(t / tiles);
    t -= part * tiles;
    int32_t tr, tc;
    tile_order(t, f.row_tiles, f.col_tiles, tr, tc);
    const int64_t r0 = (int64_t)tr * S::kJ;
    const int n_rows = a.rows - r0 < S::kJ ? (int)(a.rows - r0) : S::kJ;
    const int64_t kb = (int64_t)a.K * 2;
    const int32_t n0 = tc * (GATED ? S::kI / 2 : S::kI);
    AlongC<S::kI, S::kWaves> w;
    AlongC<S::kJ, S::kWaves> x;
    w.init(static_cast<const char *>(a.w), (uint32_t)(a.Nw * kb), (int32_t)kb, wave, lane, [&](int row) -> uint32_t {
        const int32_t n = GATED ? n0 + (row >> 4) * 8 + (row & 7) : n0 + row;
        return n < a.N ? (uint32_t)((n + (GATED && (row & 8) ? a.N : 0)) * kb) : kNowhere;
    });
    x.init(static_cast<const char *>(a.x) + r0 * kb, (uint32_t)(n_rows * kb), (int32_t)kb, wave, lane,
           [&](int row) -> uint32_t { return (uint32_t)(row * kb); });
    const int32_t all = (int32_t)((kb + kStepBytes - 1) / kStepBytes), per = (all + f.parts - 1) / f.parts;
    const int32_t first = part * per, steps = all - first < per ? all - first : per;  // 0 or less: none
    w.skip(first);
    x.skip(first);
    f32x16 acc[S::FI][S::FJ] = {};
    tile_product<S, Mul::kBf16>(w, x, steps, (char EP_LDS *)lds, wave, lane, acc);
    tile_results<S>(acc, (char EP_LDS *)lds, wave, lane, [&](int row, int col, const float *v) {
        const int32_t n = n0 + (GATED ? col / 16 * 8 : col);
        if (row >= n_rows || n >= a.N)
            return;
        f32x4 *dst = reinterpret_cast<f32x4 *>(a.partial + ((int64_t)part * a.rows + r0 + row) * a.Nw + n +
                                               (GATED && (col & 8) ? a.N : 0));
        dst[0] = f32x4{v[0], v[1], v[2], v[3]};
        dst[1] = f32x4{v[4], v[5], v[6], v[7]};
    });
}

__device__ __forceinline__ void unpack4(uint64_t v, float *f) {
    f[0] = bf16_lo((uint32_t)v);
    f[1] = bf16_hi((uint32_t)v);
    f[2] = bf16_lo((uint32_t)(v >> 32));
    f[3] = bf16_hi((uint32_t)(v >> 32));
}
__device__ __forceinline__ uint64_t pack4(const float *f) {
    return bf16_pair(f[0], f[1]) | (uint64_t)bf16_pair(f[2], f[3]) << 32;
}

// STEPS of 32 ranks.  The two fragments of a wave: 16 columns each, gated the gates' and the ups'.
template <int STEPS, bool GATED>
__global__ __launch_bounds__(64) void adapter_few_join_kernel(FewArgs f) {
    __shared__ Segment table[kRows];
    Segment EP_LDS *segments = (Segment EP_LDS *)table;
    const ProductArgs &a = f.p;
    const int lane = threadIdx.x & 63, g = lane / 16, j = lane % 16;
    const int64_t i0 = (int64_t)blockIdx.y * kRows;
    const int n_rows = a.rows - i0 < kRows ? (int)(a.rows - i0) : kRows;
    const int32_t r = j < n_rows ? row_at(f.order, a.rows, i0 + j) : -1;
    AdapterSide side{};
    side.offsets = f.offsets;
    side.A = f.A;
    const int count = __builtin_amdgcn_readfirstlane(find_segments<kRows>(side, a.rows, i0, n_rows, segments, lane));
    __syncthreads();
    // the columns: of this lane's weights (fragment u: one each), and of its results (four each)
    const int32_t n0 = (int32_t)blockIdx.x * (GATED ? 16 : 32);
    const auto row_of_b = [&](int u) { return n0 + j + (GATED ? 0 : u * 16); };

    // the results' parts and what the epilogue reads
    f32x4 acc[2] = {};
    int32_t n[2];
    bool mine[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        n[u] = n0 + g * 4 + (GATED ? 0 : u * 16);
        mine[u] = r >= 0 && n[u] < a.N;
    }
    const float *sums = a.partial + (int64_t)(r < 0 ? 0 : r) * a.Nw;
    for (int32_t p0 = 0; p0 < f.parts; p0 += kPartsAhead) {
        f32x4 v[kPartsAhead][2];
#pragma unroll
        for (int p = 0; p < kPartsAhead; ++p)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                v[p][u] = f32x4{};
                if (mine[u] && p0 + p < f.parts)
                    v[p][u] = *reinterpret_cast<const f32x4 *>(sums + (p0 + p) * a.rows * a.Nw + n[u] + (GATED && u ? a.N : 0));
            }
#pragma unroll
        for (int p = 0; p < kPartsAhead; ++p)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                acc[u] += v[p][u];
    }
    // this row's adapter, and its low-rank values
    int32_t e = -1;
    for (int s = 0; s < count; ++s) {
        const Segment t = segments[s];
        if (j >= (t[1] & 0xffff) && j < t[1] >> 16)
            e = t[0];
    }
    bf16x8 low[STEPS], rest[STEPS];
    const float scale = e >= 0 && f.scale ? f.scale[e] : 1.f;
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
        const int32_t rank = q * 32 + g * 8;
        f32x4 v[2] = {};
        for (int32_t p0 = 0; p0 < f.low_count; p0 += kPartsAhead) {
            f32x4 t[kPartsAhead][2];
#pragma unroll
            for (int p = 0; p < kPartsAhead; ++p) {
                t[p][0] = t[p][1] = f32x4{};
                if (e >= 0 && rank < f.R && p0 + p < f.low_count) {
                    const f32x4 *src =
                        reinterpret_cast<const f32x4 *>(f.low_parts + ((int64_t)(p0 + p) * a.rows + i0 + j) * f.R + rank);
                    t[p][0] = src[0];
                    t[p][1] = src[1];
                }
            }
#pragma unroll
            for (int p = 0; p < kPartsAhead; ++p) {
                v[0] += t[p][0];
                v[1] += t[p][1];
            }
        }
        u32x4 b, c, kept;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = v[i / 2][i % 2 * 2] * scale, hi = v[i / 2][i % 2 * 2 + 1] * scale;
            b[i] = first_pair(lo, hi);
            c[i] = rest_pair(lo, hi);
            kept[i] = bf16_pair(lo, hi);
        }
        low[q] = __builtin_bit_cast(bf16x8, b);
        rest[q] = __builtin_bit_cast(bf16x8, c);
        if (f.low && blockIdx.x == 0 && j < n_rows && rank < f.R)
            *reinterpret_cast<u32x4 *>(f.low + (i0 + j) * f.R + rank) = kept;
    }
    constexpr int kSegments = STEPS == 1 ? 8 : STEPS == 2 ? 4 : STEPS == 4 ? 2 : 1;  // whose weights are on their way at once
    for (int s0 = 0; s0 < count; s0 += kSegments) {
        u32x4 w[kSegments][2][STEPS];
        bool has[kSegments];
#pragma unroll
        for (int s = 0; s < kSegments; ++s) {
            const bool some = s0 + s < count;
            const Segment t = segments[some ? s0 + s : s0];
            has[s] = some && j >= (t[1] & 0xffff) && j < t[1] >> 16;
            const uint16_t *b = f.b + (int64_t)t[0] * a.Nw * f.R;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int q = 0; q < STEPS; ++q) {
                    const int32_t rank = q * 32 + g * 8;
                    w[s][u][q] = u32x4{0, 0, 0, 0};
                    if (some && row_of_b(u) < a.N && rank < f.R)
                        w[s][u][q] =
                            *reinterpret_cast<const u32x4 *>(b + (int64_t)(row_of_b(u) + (GATED && u ? a.N : 0)) * f.R + rank);
                }
        }
#pragma unroll
        for (int s = 0; s < kSegments; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x4 z = {};
#pragma unroll
                for (int q = 0; q < STEPS; ++q) {
                    const bf16x8 b = __builtin_bit_cast(bf16x8, w[s][u][q]);
                    z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, low[q], z, 0, 0, 0);
                    z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, rest[q], z, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[u][i] += has[s] ? z[i] : 0.f;
            }
    }
    float z[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        float bias[4] = {};
        if (a.bias && mine[u])
            unpack4(*reinterpret_cast<const uint64_t *>(static_cast<const uint16_t *>(a.bias) + n[u] + (GATED && u ? a.N : 0)), bias);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            z[u * 4 + i] = acc[u][i] + bias[i];
        if (a.pre && mine[u])
            *reinterpret_cast<uint64_t *>(static_cast<uint16_t *>(a.pre) + (int64_t)r * a.Nw + n[u] + (GATED && u ? a.N : 0)) =
                pack4(z + u * 4);
    }
    if (GATED) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            z[i] = z[i] * sigmoid(z[i]) * z[4 + i];
    } else {
        activate8(z, a.act);
    }
#pragma unroll
    for (int u = 0; u < (GATED ? 1 : 2); ++u) {
        if (!mine[u])
            continue;
        const int64_t at = (int64_t)r * a.N + n[u];
        if (a.residual) {
            float res[4];
            unpack4(*reinterpret_cast<const uint64_t *>(static_cast<const uint16_t *>(a.residual) + at), res);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                z[u * 4 + i] += res[i];
        }
        *reinterpret_cast<uint64_t *>(static_cast<uint16_t *>(a.y) + at) = pack4(z + u * 4);
    }
}

// The tile and the parts of x W^T, by the estimate of product_plan.h; one part leaves its sums too.
struct Base {
    Size size;
    int32_t row_tiles, col_tiles, parts;
};
Base plan_base(int64_t rows, int32_t K, int32_t N, bool gated) {
    const int32_t steps = (K + kStepRows - 1) / kStepRows;
    const int64_t outputs = rows * N * (gated ? 2 : 1);
    Base best{};
    double least = 0;
    for (Size size : {Size::kMedium, Size::kSmall, Size::kTiny}) {
        const int32_t row_tiles = (int32_t)((rows + tile_rows(size) - 1) / tile_rows(size));
        const int32_t col_tiles = (N + tile_cols(size, gated) - 1) / tile_cols(size, gated);
        const StepCost cost = size == Size::kMedium ? kMediumCost : size == Size::kSmall ? kSmallCost : kTinyCost;
        for (int32_t parts = 1; parts == 1 || steps / parts >= kSplitSteps; parts *= 2) {
            const double t = estimate(cost, (double)row_tiles * col_tiles, parts, (steps + parts - 1) / parts, outputs) +
                             (parts == 1 ? (double)outputs * 8 / 6e6 : 0.0);
            if (least == 0 || t < least) {
                least = t;
                best = {size, row_tiles, col_tiles, parts};
            }
        }
    }
    return best;
}

int32_t low_parts(int32_t K) { return (K + kPartPieces * kPiece - 1) / (kPartPieces * kPiece); }

template <class S, bool GATED>
hipError_t launch_first(const FewArgs &f, hipStream_t stream) {
    const int64_t blocks = (int64_t)f.low_tiles * f.rank_tiles * f.low_count;
    const int64_t tiles = (int64_t)f.row_tiles * f.col_tiles * f.parts + 8;
    if (blocks + tiles > kMostTiles)
        return hipErrorInvalidConfiguration;
    return launch_traced("adapter_few", adapter_few_kernel<S, GATED>, dim3((unsigned)(blocks + tiles)), S::kThreads, stream, f);
}

hipError_t launch_low(const FewArgs &f, hipStream_t stream) {
    const int64_t blocks = (int64_t)f.low_tiles * f.rank_tiles * f.low_count;
    if (blocks > kMostTiles)
        return hipErrorInvalidConfiguration;
    return launch_traced("adapter_few_low", adapter_few_low_kernel, dim3((unsigned)blocks), 256, stream, f);
}

template <bool GATED>
hipError_t launch_join(const FewArgs &f, hipStream_t stream) {
    const dim3 grid((unsigned)((f.p.N + (GATED ? 15 : 31)) / (GATED ? 16 : 32)), (unsigned)((f.p.rows + kRows - 1) / kRows));
#define EP_CALL(STEPS) \
    launch_traced("adapter_few_join", adapter_few_join_kernel<STEPS, GATED>, grid, 64, stream, f)
    return f.R <= 32 ? EP_CALL(1) : f.R <= 64 ? EP_CALL(2) : f.R <= 128 ? EP_CALL(4) : EP_CALL(8);
#undef EP_CALL
}

}  // namespace

// Few results, and few low-rank values: this way reads the rows once per 16 ranks, and the parts of their low-rank values once per
// 32 columns, half of that from the L2, at 5.5 TB/s; the pass of adapter_low.hip that it saves takes 3 us and 1.6 ns for each value of
// the contraction.  Measured, us, this way and by adapter_product.hip, with 8 adapters unless said:
//   16 ranks   449 rows 7168 x 1024 27 / 38, 1707 rows 53 / 58; 502 rows 7168 x 4096 51 / 59; 6828 rows 7168 x 64 49 / 43;
//              without W 873 rows 7168 x 4096 21 / 27, 2968 rows 7168 x 1024 25 / 27, 11875 rows 1024 x 64 14 / 16
//   64 ranks   449 rows 7168 x 1024 34 / 40, 1707 rows 74 / 69; without W 781 rows 7168 x 1024 24 / 25, 1875 rows 42 / 36,
//              7500 rows 7168 x 64 98 / 36; 700 adapters 300 rows 7168 x 2048 71 / 87
//   256 ranks  132 rows 7168 x 4096 54 / 55, 1796 rows 7168 x 64 124 / 49, 1707 rows 7168 x 1024 172 / 75;
//              without W 229 rows 7168 x 4096 43 / 47, 11875 rows 16384 x 64 1269 / 214
// Past the first limit the other way is the faster: 2965 rows 1664 x 1576, 16 ranks 47 / 38, 2400 rows 4096 x 1576 69 / 51;
// without W 9340 rows 4096 x 512, 16 ranks 35 / 34, 32 ranks 52 / 39.
bool adapter_few(int64_t rows, int32_t R, int32_t K, int32_t N, bool base, int32_t act) {
    const int64_t Nw = (act == EP_ACT_SWIGLU ? 2 : 1) * (int64_t)N;
    if (rows * (Nw + 256) > (base ? 2300000 : 4000000))
        return false;
    const int64_t rank_tiles = (R + kRanks - 1) / kRanks;
    return rows * (K * 2 * rank_tiles + (int64_t)low_parts(K) * R * 4 * Nw / 64) <= 16000000 + 9000 * (int64_t)K;
}

size_t adapter_few_bytes(int64_t rows, int32_t R, int32_t K, int32_t N, bool base, int32_t act) {
    const bool gated = act == EP_ACT_SWIGLU;
    const size_t low = (size_t)low_parts(K) * rows * R * sizeof(float);
    return low + (base ? (size_t)plan_base(rows, K, N, gated).parts * rows * N * (gated ? 2 : 1) * sizeof(float) : 0);
}

// rows > 0
hipError_t launch_adapter_few(const AdapterArgs &a, hipStream_t stream) {
    const bool gated = a.act == EP_ACT_SWIGLU;
    FewArgs f{};
    f.p.x = a.x;
    f.p.rows = a.rows;
    f.p.w = a.w;
    f.p.K = a.K;
    f.p.N = a.N;
    f.p.Nw = gated ? 2 * a.N : a.N;
    f.p.bias = a.bias;
    f.p.act = a.act;
    f.p.residual = a.residual;
    f.p.pre = a.pre;
    f.p.y = a.y;
    f.order = a.order;
    f.offsets = a.offsets;
    f.A = a.A;
    f.R = a.R;
    f.a = static_cast<const uint16_t *>(a.a);
    f.b = static_cast<const uint16_t *>(a.b);
    f.scale = a.scale;
    f.low = static_cast<uint16_t *>(a.low);
    f.low_count = low_parts(a.K);
    f.low_tiles = (int32_t)row_tiles_most(a.rows, a.A, kRows);
    f.rank_tiles = (a.R + kRanks - 1) / kRanks;
    f.low_parts = static_cast<float *>(a.workspace);
    f.p.partial = f.low_parts + (size_t)f.low_count * a.rows * a.R;
    Size size = Size::kSmall;
    if (a.w) {
        const Base base = plan_base(a.rows, a.K, a.N, gated);
        size = base.size;
        f.parts = base.parts;
        f.row_tiles = base.row_tiles;
        f.col_tiles = base.col_tiles;
    }
#define EP_CALL(S) (gated ? launch_first<S, true>(f, stream) : launch_first<S, false>(f, stream))
    const hipError_t e = !a.w ? launch_low(f, stream)
                         : size == Size::kMedium ? EP_CALL(Medium) : size == Size::kSmall ? EP_CALL(Small) : EP_CALL(Tiny);
#undef EP_CALL
    if (e != hipSuccess)
        return e;
    return gated ? launch_join<true>(f, stream) : launch_join<false>(f, stream);
}

}  // namespace ep
