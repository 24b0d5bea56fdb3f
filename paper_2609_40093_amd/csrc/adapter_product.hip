// adapter_product.hip -- a shared projection with the low-rank adapters of its rows:
//   z = x[r] W^T + low[r] b_a^T;  y[r] = act(z + bias) + residual[r],  a the adapter of row r.
//
// The low-rank values low = scale_a x a_a^T come from adapter_low.hip.  Rows go in the adapters'
// order: a tile gathers its rows of x through it and leaves its results through it.  The
// contraction over K goes on over the ranks of the adapters that the tile's rows have
// (adapter_tile.h), so the adapters cost the tile (segments * 2 R) / 64 steps, and y is written
// once.  Without W the contraction begins with the ranks.
//
// Bound by the matrix cores and the LDS reads that feed them, as the experts' product is: 16379 rows of 7168 by
// 2 x 2048, gated, 8 adapters of 64 ranks 787 us (1222 TFLOP/s without counting the ranks), 8192 rows 4096 x 4096, 16
// adapters of 16 ranks 240 (1145; the experts' product of one such expert 217).
#include "adapter_tile.h"
#include "product_finish.h"
#include "product_plan.h"

namespace ep {
namespace {

// The sums of place i (row r), columns n..n+7, of their own terms alone, if others of the tile, whose first
// place is i0, could have made them NaN.
__device__ __forceinline__ void redo8(const ProductArgs &a, const AdapterSide &s, int64_t i0, int tile_rows, int64_t i, int64_t r,
                                      int32_t n, float *z) {
    const int32_t e = adapter_of(s, a.rows, i);
    const auto broken = [&](int32_t other) {
        const u32x4 *b = reinterpret_cast<const u32x4 *>(s.weights + ((int64_t)other * a.Nw + n) * s.R);
#pragma unroll 1
        for (int32_t j = 0; j < s.R; ++j)  // eight columns of R / 8 vectors, one after the other
            if (any_not_finite(b[j]))
                return true;
        return false;
    };
    if (!others_broken(s, a.rows, i0, tile_rows, e, broken))
        return;
#pragma unroll 1
    for (int q = 0; q < 8; ++q) {
        float sum = 0.f;
        const auto dot8 = [&](const uint16_t *u, const uint16_t *v) {
            float f[8], g[8];
            unpack8(*reinterpret_cast<const u32x4 *>(u), f);
            unpack8(*reinterpret_cast<const u32x4 *>(v), g);
#pragma unroll
            for (int p = 0; p < 8; ++p)
                sum = fmaf(f[p], g[p], sum);
        };
        if (a.w)
#pragma unroll 1
            for (int32_t k = 0; k < a.K; k += 8)
                dot8(static_cast<const uint16_t *>(a.x) + r * a.K + k,
                     static_cast<const uint16_t *>(a.w) + (int64_t)(n + q) * a.K + k);
        if (e >= 0)
#pragma unroll 1
            for (int32_t j = 0; j < 2 * s.R; j += 8)
                dot8(s.low + i * s.width + s.value_at(j), s.weights + ((int64_t)e * a.Nw + n + q) * s.R + s.rank_of(j));
#pragma unroll
        for (int p = 0; p < 8; ++p)
            z[p] = p == q ? sum : z[p];
    }
}
template <bool GATED>
__device__ __forceinline__ void check8(const ProductArgs &a, const AdapterSide &s, int64_t i0, int tile_rows, int64_t i,
                                       int64_t r, int32_t n, float *z, float *up) {
    if (__builtin_expect(any_nan(z, 8) || (GATED && any_nan(up, 8)), false)) {
        redo8(a, s, i0, tile_rows, i, r, n, z);
        if (GATED)
            redo8(a, s, i0, tile_rows, i, r, n + a.N, up);
    }
}

// The weights' row of a tile's row, -1: none (gated: 8 gate rows beside their 8 up rows, as in the experts' product).
template <bool GATED>
struct WeightRow {
    static constexpr bool kLow = false, kSkips = false;
    int32_t n0, N;
    __device__ __forceinline__ int32_t operator()(int row) const {
        const int32_t n = GATED ? n0 + (row >> 4) * 8 + (row & 7) : n0 + row;
        return n < N ? n + (GATED && (row & 8) ? N : 0) : -1;
    }
};

template <class S, bool GATED>
__global__ __launch_bounds__(S::kThreads) void adapter_product_kernel(ProductArgs a, AdapterSide s, int32_t row_tiles,
                                                                      int32_t col_tiles, int32_t parts) {
    __shared__ __attribute__((aligned(1024))) char lds[TileLds<S>::kBytes];
    const TileLds<S> tile{(char EP_LDS *)lds};
    const int32_t EP_LDS *row_of = tile.row_of();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t tiles = (int64_t)row_tiles * col_tiles;
    int64_t t = tile_of_block(blockIdx.x, tiles * parts);
    if (t < 0)
        return;
    const int32_t part = parts == 1 ? 0 : (int32_t)(t / tiles);
    t -= part * tiles;
    int32_t tr, tc;
    tile_order(t, row_tiles, col_tiles, tr, tc);
    const int64_t i0 = (int64_t)tr * S::kJ;
    const int n_rows = a.rows - i0 < S::kJ ? (int)(a.rows - i0) : S::kJ;
    const int count = tile.fill(s, a.rows, i0, n_rows, wave, lane);

    const int64_t kb = (int64_t)a.K * 2;
    constexpr int kOut = GATED ? S::kI / 2 : S::kI;  // output columns of a tile
    const int32_t n0 = tc * kOut;
    const int32_t main = a.w ? (int32_t)((kb + kStepBytes - 1) / kStepBytes) : 0;
    const WeightRow<GATED> column{n0, a.N};
    ChainAlong<S::kI, S::kWaves, WeightRow<GATED>> w;
    ChainAlong<S::kJ, S::kWaves, LowRows<false>> x;
    w.init(static_cast<const char *>(a.w), (uint32_t)(a.Nw * kb), (int32_t)kb, wave, lane, [&](int row) -> uint32_t {
        const int32_t n = column(row);
        return n < 0 ? kNowhere : (uint32_t)(n * kb);
    });
    w.chain(main, s, tile.segments(), count, s.weights, (uint64_t)s.A * a.Nw * s.R * 2, a.Nw, column);
    // through an order from x's first row on (x is smaller than 2^31 bytes then)
    const char *xb = static_cast<const char *>(a.x);
    x.init(s.order ? xb : xb + i0 * kb, (uint32_t)((s.order ? a.rows : n_rows) * kb), (int32_t)kb, wave, lane,
           [&](int row) -> uint32_t {
               if (!s.order)
                   return (uint32_t)(row * kb);
               const int32_t r = row_of[row];
               return r < 0 ? kNowhere : (uint32_t)(r * kb);
           });
    x.chain(main, s, tile.segments(), count, s.low + i0 * s.width, (uint64_t)n_rows * s.width * 2, 0, LowRows<false>{});

    int32_t steps = main + (count * (int32_t)s.chunks.d + 7) / 8;
    if (parts > 1) {
        const int32_t per = (steps + parts - 1) / parts, first = part * per;
        steps = steps - first < per ? steps - first : per;
        w.skip(first);
        x.skip(first);
    }
    f32x16 acc[S::FI][S::FJ] = {};
    tile_product<S, Mul::kBf16>(w, x, steps, (char EP_LDS *)lds, wave, lane, acc);

    if (parts > 1) {
        tile_results<S>(acc, (char EP_LDS *)lds, wave, lane, [&](int row, int col, const float *v) {
            const int32_t n = n0 + (GATED ? col / 16 * 8 : col);
            if (row >= n_rows || n >= a.N)
                return;
            f32x4 *dst = reinterpret_cast<f32x4 *>(a.partial + ((int64_t)part * a.rows + i0 + row) * a.Nw + n +
                                                   (GATED && (col & 8) ? a.N : 0));
            dst[0] = f32x4{v[0], v[1], v[2], v[3]};
            dst[1] = f32x4{v[4], v[5], v[6], v[7]};
        });
        return;
    }
    constexpr int kPer = GATED ? 16 : 8;
    const int32_t n = n0 + first_col<S, kPer>(wave, lane) / (kPer / 8);
    Columns<false, GATED> columns;
    if (n < a.N)
        columns.load(a, 0, n);
    struct Row {
        int32_t r;
        RowExtra<false> x;
    };
    tile_rows_out<S, kPer>(
        acc, (char EP_LDS *)lds, wave, lane,
        [&](int row) {
            Row f;
            f.r = row < n_rows && n < a.N ? row_of[row] : -1;
            if (f.r >= 0)
                f.x.load(a, f.r, n);
            return f;
        },
        [&](int row, int, float *v, const Row &f) {
            if (f.r < 0)
                return;
            check8<GATED>(a, s, i0, S::kJ, i0 + row, f.r, n, v, v + kPer / 2);
            finish8<false, GATED>(a, columns, f.x, f.r, n, v, v + kPer / 2);
        });
}

// Adds the parts of a split contraction and runs the epilogue, as the experts' product does: LANES
// lanes add every LANES-th part of eight neighbouring results each, and are added up in a fixed order.
template <bool GATED, int LANES>
__global__ __launch_bounds__(256) void adapter_join_kernel(ProductArgs a, AdapterSide s, int32_t parts, int32_t tile_rows,
                                                          FastDiv groups) {
    const int lane = threadIdx.x & 63, first = lane / (64 / LANES);
    const uint32_t at = (blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 / LANES) + lane % (64 / LANES);
    const uint32_t row = groups.div(at);
    const int64_t i = row;
    const int32_t n = (int32_t)(at - row * groups.d) * 8;
    const int32_t r = i < a.rows ? row_at(s.order, a.rows, i) : -1;
    float z[8] = {}, up[8] = {};
    if (r >= 0) {
        constexpr int kAhead = 4;
        const int64_t part = a.rows * a.Nw;
        const float *src = a.partial + i * a.Nw + n;
        for (int32_t p0 = first; p0 < parts; p0 += LANES * kAhead) {
            f32x4 v[kAhead][GATED ? 4 : 2];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int h = 0; h < (GATED ? 4 : 2); ++h) {
                    v[u][h] = f32x4{};
                    if (p0 + LANES * u < parts)
                        v[u][h] = *reinterpret_cast<const f32x4 *>(src + (p0 + LANES * u) * part + (h / 2) * a.N + (h & 1) * 4);
                }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    z[q] += v[u][q / 4][q % 4];
                    if (GATED)
                        up[q] += v[u][(GATED ? 2 : 0) + q / 4][q % 4];
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
    if (r < 0 || first != 0)
        return;
    check8<GATED>(a, s, i - i % tile_rows, tile_rows, i, r, n, z, up);
    Columns<false, GATED> columns;
    columns.load(a, 0, n);
    RowExtra<false> x;
    x.load(a, r, n);
    finish8<false, GATED>(a, columns, x, r, n, z, up);
}

Plan adapter_plan(int64_t rows, int32_t A, int32_t R, int32_t K, int32_t N, bool base, bool gated) {
    return make_plan(rows, 1, base ? K : 0, N, false, gated, [&](int per) { return adapter_steps(rows, A, R, per); });
}

template <class S, bool GATED>
hipError_t launch_tiles(const ProductArgs &a, const AdapterSide &s, const Plan &p, hipStream_t stream) {
    if (p.tiles * p.split.parts > kMostTiles)
        return hipErrorInvalidConfiguration;
    const hipError_t e = launch_traced("adapter_product", adapter_product_kernel<S, GATED>,
                                       dim3((unsigned)(p.tiles * p.split.parts + 8)), S::kThreads, stream, a, s,
                                       (int32_t)(p.tiles / p.cols), p.cols, p.split.parts);
    if (e != hipSuccess || p.split.parts == 1)
        return e;
    const int64_t groups = a.rows * (a.N / 8);
#define EP_CALL(LANES)                                                                                                     \
    launch_traced("adapter_product_join", adapter_join_kernel<GATED, LANES>, dim3((unsigned)((groups * LANES + 255) / 256)), \
                  256, stream, a, s, p.split.parts, S::kJ, fast_div((uint32_t)(a.N / 8)))
    return p.split.parts <= 4 ? EP_CALL(1) : EP_CALL(8);  // a lane has 4 parts on their way
#undef EP_CALL
}
template <class S>
hipError_t launch_shape(const ProductArgs &a, const AdapterSide &s, const Plan &p, hipStream_t stream) {
    return a.act == EP_ACT_SWIGLU ? launch_tiles<S, true>(a, s, p, stream) : launch_tiles<S, false>(a, s, p, stream);
}

// The split low-rank values, then the parts' sums.
size_t split_bytes(int64_t rows, int32_t R) { return ((size_t)rows * split_width(R) * 2 + 255) & ~(size_t)255; }

}  // namespace

size_t adapter_product_workspace_bytes(int64_t rows, int32_t A, int32_t R, int32_t K, int32_t N, bool base, int32_t act) {
    if (rows == 0)
        return 0;
    if (adapter_few(rows, R, K, N, base, act))
        return adapter_few_bytes(rows, R, K, N, base, act);
    const bool gated = act == EP_ACT_SWIGLU;
    const Plan p = adapter_plan(rows, A, R, K, N, base, gated);
    return split_bytes(rows, R) +
           (p.split.parts == 1 ? 0 : (size_t)p.split.parts * rows * N * (gated ? 2 : 1) * sizeof(float));
}

hipError_t launch_adapter_product(const AdapterArgs &a, hipStream_t stream) {
    if (a.rows == 0)
        return hipSuccess;
    if (adapter_few(a.rows, a.R, a.K, a.N, a.w != nullptr, a.act))
        return launch_adapter_few(a, stream);
    const bool gated = a.act == EP_ACT_SWIGLU;
    ProductArgs p{};
    p.x = a.x;
    p.rows = a.rows;
    p.E = 1;
    p.w = a.w;
    p.K = a.K;
    p.N = a.N;
    p.Nw = gated ? 2 * a.N : a.N;
    p.bias = a.bias;
    p.act = a.act;
    p.residual = a.residual;
    p.pre = a.pre;
    p.y = a.y;
    p.partial = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + split_bytes(a.rows, a.R));
    const int32_t width = split_width(a.R), log = split_log(a.R);
    const hipError_t e = launch_adapter_low(
        {a.x, a.rows, a.order, a.offsets, a.A, a.R, a.K, a.a, false, a.scale, a.low, a.workspace, width, log}, stream);
    if (e != hipSuccess)
        return e;
    const AdapterSide s = adapter_side(a.order, a.offsets, a.A, a.R, a.workspace, width, log, a.b);
    const Plan plan = adapter_plan(a.rows, a.A, a.R, a.K, a.N, a.w != nullptr, gated);
    switch (plan.size) {
    case Size::kLarge: return launch_shape<Large>(p, s, plan, stream);
    case Size::kBroad: return launch_shape<Broad>(p, s, plan, stream);
    case Size::kMedium: return launch_shape<Medium>(p, s, plan, stream);
    case Size::kSmall: return launch_shape<Small>(p, s, plan, stream);
    case Size::kWide: return launch_shape<Wide>(p, s, plan, stream);
    case Size::kFew: return launch_shape<Few>(p, s, plan, stream);
    default: return launch_shape<TinyRows>(p, s, plan, stream);
    }
}

}  // namespace ep
