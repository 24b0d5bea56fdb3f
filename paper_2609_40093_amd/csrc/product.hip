// product.hip -- the experts' matrix product over rows packed by expert:
//   z = x[r] W_e^T + bias_e;  y[r] = act(z) + residual[r]  for the rows r of expert e.
//
// Tiles of weight rows x packed rows on the matrix cores (product_tile.h).  A workgroup finds
// its expert and rows from the offsets in device memory, so the host never learns the counts:
// the grid covers the most tiles that any counts can give, and the rest end at once.  The
// gated product interleaves 8 gate rows with their 8 up rows of W, so that a lane holds a
// gate and its up value in neighbouring quads of its accumulators.
//
// Where the tiles are fewer than the compute units, the contraction is split as well: each
// part leaves its fp32 sums in the workspace, and a second kernel adds the parts in order and
// runs the epilogue.
//
// Bound by the weights' bytes for few rows per expert (2048 rows of 32 experts, K 7168, gated N
// 2048: 383 us, 1.93 GB, 5.0 TB/s), by the matrix cores and the LDS reads that feed them for many
// (32768 rows of the same from 8-bit rows: 957 us, 2010 TFLOP/s; 8192 x 8192 x 8192 in bf16 1210).
#include "product_finish.h"
#include "product_plan.h"

namespace ep {
namespace {

template <class S, Mul M, bool GATED>
__global__ __launch_bounds__(S::kThreads) void product_kernel(ProductArgs a, int32_t col_tiles, Split split) {
    constexpr bool F8 = M != Mul::kBf16;
    __shared__ __attribute__((aligned(1024))) char lds[S::kStages * S::kStageBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t row_tiles = count_row_tiles(a.offsets, a.rows, a.E, S::kJ, lane);
    const int64_t tiles = (int64_t)row_tiles * col_tiles;
    int64_t t = tile_of_block(blockIdx.x, tiles * split.parts);
    if (t < 0)
        return;
    const int32_t part = split.parts == 1 ? 0 : (int32_t)(t / tiles);
    t -= part * tiles;
    int32_t tr, tc;
    tile_order(t, row_tiles, col_tiles, tr, tc);
    const RowTile rt = find_row_tile(a.offsets, a.rows, a.E, S::kJ, tr, lane);
    if (rt.e < 0)
        return;
    const int64_t kb = (int64_t)a.K * (F8 ? 1 : 2), xs = F8 ? a.K + EP_ROWS8_EXTRA : kb;
    constexpr int kOut = GATED ? S::kI / 2 : S::kI;  // output columns of a tile
    const int32_t n0 = tc * kOut;
    AlongC<S::kI, S::kWaves> w;
    AlongC<S::kJ, S::kWaves> x;
    const char *wbase = static_cast<const char *>(a.w) + rt.e * (a.Nw * kb);
    w.init(wbase, (uint32_t)(a.Nw * kb), (int32_t)kb, wave, lane, [&](int row) -> uint32_t {
        const int32_t n = GATED ? n0 + (row >> 4) * 8 + (row & 7) : n0 + row;
        return n < a.N ? (uint32_t)((n + (GATED && (row & 8) ? a.N : 0)) * kb) : kNowhere;
    });
    x.init(static_cast<const char *>(a.x) + rt.row0 * xs, (uint32_t)(rt.n * xs), (int32_t)kb, wave, lane,
           [&](int row) -> uint32_t { return (uint32_t)(row * xs); });
    f32x16 acc[S::FI][S::FJ] = {};
    int32_t steps = (int32_t)((kb + kStepBytes - 1) / kStepBytes);
    if (split.parts > 1) {
        const int32_t first = part * split.steps;
        steps = steps - first < split.steps ? steps - first : split.steps;
        w.skip(first);
        x.skip(first);
    }
    tile_product<S, M>(w, x, steps, (char EP_LDS *)lds, wave, lane, acc);

    if (split.parts > 1) {
        tile_results<S>(acc, (char EP_LDS *)lds, wave, lane, [&](int row, int col, const float *v) {
            // gated: the ups' eight columns lie N behind the gates'
            const int32_t n = n0 + (GATED ? col / 16 * 8 : col);
            if (row >= rt.n || n >= a.N)
                return;
            f32x4 *dst = reinterpret_cast<f32x4 *>(a.partial + ((int64_t)part * a.rows + rt.row0 + row) * a.Nw + n +
                                                   (GATED && (col & 8) ? a.N : 0));
            dst[0] = f32x4{v[0], v[1], v[2], v[3]};
            dst[1] = f32x4{v[4], v[5], v[6], v[7]};
        });
        return;
    }
    // a lane's columns: eight results, gated from the eight gates and the eight ups behind them
    constexpr int kPer = GATED ? 16 : 8;
    const int32_t n = n0 + first_col<S, kPer>(wave, lane) / (kPer / 8);
    Columns<F8, GATED> columns;
    if (n < a.N)
        columns.load(a, rt.e, n);
    tile_rows_out<S, kPer>(
        acc, (char EP_LDS *)lds, wave, lane,
        [&](int row) {
            RowExtra<F8> x;
            if (row < rt.n && n < a.N)
                x.load(a, rt.row0 + row, n);
            return x;
        },
        [&](int row, int, float *v, const RowExtra<F8> &x) {
            if (row < rt.n && n < a.N)
                finish8<F8, GATED>(a, columns, x, rt.row0 + row, n, v, v + kPer / 2);
        });
}

// Adds the parts of a split contraction and runs the epilogue.  A wave takes 64 / LANES groups
// of eight neighbouring results; the LANES lanes of a group add every LANES-th part each, in
// order, and are added up in a fixed order.  (A split product has few tiles: 32 bits number its
// groups.)  LANES is 1 up to four parts, which a lane has on their way at once: with 8 lanes whatever
// the parts, a product of 8000 rows 1536 x 1536 in two parts took 120 us instead of 76.
template <bool F8, bool GATED, int LANES>
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a, Split split, FastDiv groups) {
    const int lane = threadIdx.x & 63, first = lane / (64 / LANES);
    const uint32_t at = (blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 / LANES) + lane % (64 / LANES);
    const uint32_t row = groups.div(at);
    const int64_t r = row;
    const int32_t n = (int32_t)(at - row * (uint32_t)(a.N / 8)) * 8;
    bool mine = r < a.rows;
    int32_t e = 0;
    if (mine && a.offsets) {  // the last expert that begins at or before r
        int32_t hi = a.E;
        while (hi - e > 1) {
            const int32_t mid = (e + hi) / 2;
            if (a.offsets[mid] <= r)
                e = mid;
            else
                hi = mid;
        }
        mine = r >= a.offsets[e] && r < a.offsets[e + 1];
    }
    float z[8] = {}, up[8] = {};
    if (mine) {
        constexpr int kAhead = 4;
        const int64_t part = a.rows * a.Nw;
        const float *src = a.partial + r * a.Nw + n;
        for (int32_t p0 = first; p0 < split.parts; p0 += LANES * kAhead) {
            f32x4 v[kAhead][GATED ? 4 : 2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int h = 0; h < (GATED ? 4 : 2); ++h) {
                    v[i][h] = f32x4{};
                    if (p0 + LANES * i < split.parts)
                        v[i][h] = *reinterpret_cast<const f32x4 *>(src + (p0 + LANES * i) * part + (h / 2) * a.N + (h & 1) * 4);
                }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    z[q] += v[i][q / 4][q % 4];
                    if (GATED)
                        up[q] += v[i][(GATED ? 2 : 0) + q / 4][q % 4];
                }
        }
    }
#pragma unroll
    for (int d = 64 / LANES; d < 64; d *= 2)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            z[q] += __shfl_xor(z[q], d);
            if (GATED)
                up[q] += __shfl_xor(up[q], d);
        }
    if (!mine || first != 0)
        return;
    Columns<F8, GATED> columns;
    columns.load(a, e, n);
    RowExtra<F8> x;
    x.load(a, r, n);
    finish8<F8, GATED>(a, columns, x, r, n, z, up);
}

template <class S, Mul M, bool GATED>
hipError_t launch_tiles(const ProductArgs &a, const Plan &p, hipStream_t stream) {
    if (p.tiles * p.split.parts > kMostTiles)
        return hipErrorInvalidConfiguration;
    const hipError_t e = launch_traced("expert_product", product_kernel<S, M, GATED>,
                                       dim3((unsigned)(p.tiles * p.split.parts + 8)), S::kThreads, stream, a, p.cols, p.split);
    if (e != hipSuccess || p.split.parts == 1)
        return e;
    const int64_t groups = a.rows * (a.N / 8);
#define EP_CALL(LANES)                                                                                                \
    launch_traced("expert_product_join", product_join_kernel<M != Mul::kBf16, GATED, LANES>,                          \
                  dim3((unsigned)((groups * LANES + 255) / 256)), 256, stream, a, p.split, fast_div((uint32_t)(a.N / 8)))
    return p.split.parts <= 4 ? EP_CALL(1) : EP_CALL(8);  // a lane has 4 parts on their way
#undef EP_CALL
}
// The 8-bit matrix instruction doubles the rate, but it lines its products up to the largest
// and drops what lies more than 13 bits below (measured: a sum of 7168 products of 8-bit rows
// is 1.5e-5 off by its 2-norm, of 64 products 1.3e-5; widened to bf16, 4e-7).  That is a hundredth of the bf16
// result's own rounding, so long sums that end in bf16 take it; fp32 results and short sums,
// which the memory bounds anyway, are multiplied as bf16.
constexpr int32_t kLongSum = 512;
template <class S>
hipError_t launch_shape(const ProductArgs &a, const Plan &p, hipStream_t stream) {
    const bool gated = a.act == EP_ACT_SWIGLU;
    if (!a.bits8)
        return gated ? launch_tiles<S, Mul::kBf16, true>(a, p, stream) : launch_tiles<S, Mul::kBf16, false>(a, p, stream);
    if (a.K >= kLongSum && !a.f32)
        return gated ? launch_tiles<S, Mul::kF8, true>(a, p, stream) : launch_tiles<S, Mul::kF8, false>(a, p, stream);
    return gated ? launch_tiles<S, Mul::kF8Wide, true>(a, p, stream) : launch_tiles<S, Mul::kF8Wide, false>(a, p, stream);
}

}  // namespace

size_t product_workspace_bytes(int64_t rows, int32_t E, int32_t K, int32_t N, bool bits8, int32_t act) {
    if (rows == 0)
        return 0;
    const bool gated = act == EP_ACT_SWIGLU;
    const Plan p = make_plan(rows, E, K, N, bits8, gated);
    return p.split.parts == 1 ? 0 : (size_t)p.split.parts * rows * N * (gated ? 2 : 1) * sizeof(float);
}

hipError_t launch_product(const ProductArgs &a, hipStream_t stream) {
    if (a.rows == 0)
        return hipSuccess;
    const Plan p = make_plan(a.rows, a.E, a.K, a.N, a.bits8, a.act == EP_ACT_SWIGLU);
    switch (p.size) {
    case Size::kLarge: return launch_shape<Large>(a, p, stream);
    case Size::kBroad: return launch_shape<Broad>(a, p, stream);
    case Size::kMedium: return launch_shape<Medium>(a, p, stream);
    case Size::kSmall: return launch_shape<Small>(a, p, stream);
    case Size::kWide: return launch_shape<Wide>(a, p, stream);
    case Size::kFew: return launch_shape<Few>(a, p, stream);
    default: return launch_shape<Tiny>(a, p, stream);
    }
}

}  // namespace ep
