// adapter_grad.hip -- gradients of the adapters' product y = act(x W^T + low b_a^T + bias) + residual, W held:
//   dz = d_y act'(pre);  v = scale_a dz b_a;  dx = dz W + v a_a;  da_a = v^T x;  db_a = dz^T low.
//
// v is made as low is (adapter_low.hip).  dx has the product's form: the contraction over W's rows goes on
// over the ranks of the tile's adapters (adapter_tile.h).  da and db are contractions over an
// adapter's rows, of a long side (x, dz) that is read once and a short one (v, low): bound by the long
// side's bytes, so the rows are shared out over workgroups until there is one for every compute unit,
// and a second kernel adds their fp32 sums in order.  Rows go in the adapters' order, and every kernel
// gathers its rows of x and d_y through it; only with an activation dz is kept, in that order.
//
// dz is rounded to bf16 between the kernels, v to two bf16 values: the products multiply bf16.
//
// 8192 rows 4096 x 4096, one adapter of 64 ranks: v 24 us, dx 237 (1160 TFLOP/s), da and db 28 (4.7 TB/s) and their join
// 5.  5003 rows 2888 x 1448 through silu, 15 adapters of 24 ranks: dz 10, v 9, dx 56, da and db 22.
#include "adapter_tile.h"
#include "product_plan.h"

namespace ep {
namespace {

// dz[i] = d_y[r] act'(pre[r]), r = order[i]: eight values per thread.  Without an activation (pre null)
// it gathers rows.
template <bool GATED>
__global__ __launch_bounds__(256) void adapter_dz_kernel(const int32_t *order, int64_t rows, int32_t N, int32_t act,
                                                         const uint16_t *pre, const uint16_t *d_y, uint16_t *dz) {
    constexpr int kParts = GATED ? 2 : 1;
    const int64_t Nw = (int64_t)N * kParts;
    for (int64_t i = blockIdx.y; i < rows; i += gridDim.y) {
        const int32_t n = ((int32_t)blockIdx.x * 256 + (int32_t)threadIdx.x) * 8;
        const int32_t r = row_at(order, rows, i);
        if (n >= N)
            continue;
        float d[8] = {}, z[kParts][8] = {}, o[kParts][8];
        if (r >= 0) {
            unpack8(*reinterpret_cast<const u32x4 *>(d_y + r * (int64_t)N + n), d);
#pragma unroll
            for (int p = 0; p < kParts; ++p)
                if (pre)
                    unpack8(*reinterpret_cast<const u32x4 *>(pre + r * Nw + p * N + n), z[p]);
        }
        if (GATED) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float s = sigmoid(z[0][q]);
                o[0][q] = d[q] * z[kParts - 1][q] * s * (1.f + z[0][q] * (1.f - s));
                o[kParts - 1][q] = d[q] * z[0][q] * s;
            }
        } else {
            if (pre)
                activation_grad8(z[0], act);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                o[0][q] = pre ? d[q] * z[0][q] : d[q];
        }
#pragma unroll
        for (int p = 0; p < kParts; ++p)
            *reinterpret_cast<u32x4 *>(dz + i * Nw + p * N + n) = pack8(o[p]);
    }
}

struct DxArgs {
    int64_t rows;
    int32_t K, Nw;
    const uint16_t *w, *dz;
    const int32_t *dz_order;  // dz's rows; null: they are in the adapters' order
    uint16_t *dx;
    float *partial;  // parts > 1: [parts][rows][K], in the adapters' order
    int32_t row_tiles, col_tiles, parts, tile_rows;
};

// The sums of place i, columns k..k+7, of their own terms alone, if others of the tile, whose first place is
// i0, could have made them NaN.
__device__ __forceinline__ void redo8(const DxArgs &a, const AdapterSide &s, int64_t i0, int tile_rows, int64_t i, int32_t k,
                                      float *z) {
    const int32_t e = adapter_of(s, a.rows, i), r = row_at(a.dz_order, a.rows, i);
    const auto broken = [&](int32_t other) {
        const uint16_t *w = s.weights + (int64_t)other * s.R * a.K + k;
#pragma unroll 1
        for (int32_t j = 0; j < s.R; ++j, w += a.K)
            if (any_not_finite(*reinterpret_cast<const u32x4 *>(w)))
                return true;
        return false;
    };
    if (!others_broken(s, a.rows, i0, tile_rows, e, broken))
        return;
#pragma unroll
    for (int q = 0; q < 8; ++q)
        z[q] = 0.f;
    const auto add = [&](uint16_t f, const uint16_t *row) {
        float g[8];
        unpack8(*reinterpret_cast<const u32x4 *>(row + k), g);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            z[q] = fmaf(__uint_as_float((uint32_t)f << 16), g[q], z[q]);
    };
    if (a.w)
#pragma unroll 1
        for (int32_t n = 0; n < a.Nw; ++n)
            add(a.dz[(int64_t)r * a.Nw + n], a.w + (int64_t)n * a.K);
    if (e >= 0)
#pragma unroll 1
        for (int32_t j = 0; j < 2 * s.R; ++j)
            add(s.low[i * s.width + s.value_at(j)], s.weights + ((int64_t)e * s.R + s.rank_of(j)) * a.K);
}

// dx[order[i]][k] = sum_n dz[i][n] w[n][k] + sum_j v[i][j] a_e[j][k]: i = k across the contraction, j = rows.
template <class S>
__global__ __launch_bounds__(S::kThreads) void adapter_dx_kernel(DxArgs a, AdapterSide s) {
    __shared__ __attribute__((aligned(1024))) char lds[TileLds<S>::kBytes];
    const TileLds<S> tile{(char EP_LDS *)lds};
    const int32_t EP_LDS *row_of = tile.row_of();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t tiles = (int64_t)a.row_tiles * a.col_tiles;
    int64_t t = tile_of_block(blockIdx.x, tiles * a.parts);
    if (t < 0)
        return;
    const int32_t part = a.parts == 1 ? 0 : (int32_t)(t / tiles);
    t -= part * tiles;
    int32_t tr, tc;
    tile_order(t, a.row_tiles, a.col_tiles, tr, tc);
    const int64_t i0 = (int64_t)tr * S::kJ;
    const int n_rows = a.rows - i0 < S::kJ ? (int)(a.rows - i0) : S::kJ;
    const int count = tile.fill(s, a.rows, i0, n_rows, wave, lane);
    const int32_t k0 = tc * S::kI;
    const int32_t main = a.w ? (a.Nw + kStepRows - 1) / kStepRows : 0;
    ChainAcross<S::kI, S::kWaves, S::FI> w;
    ChainAlong<S::kJ, S::kWaves, LowRows<true>> z;
    w.init(reinterpret_cast<const char *>(a.w), (int64_t)a.K * 2, a.Nw, k0, wave, lane);
    w.chain(main, s, tile.segments(), count, (uint64_t)s.A * s.R * a.K * 2, k0);
    const int64_t zs = (int64_t)a.Nw * 2;
    const char *zb = reinterpret_cast<const char *>(a.dz);
    z.init(a.dz_order ? zb : zb + i0 * zs, (uint32_t)((a.dz_order ? a.rows : n_rows) * zs), (int32_t)zs, wave, lane,
           [&](int row) -> uint32_t {
               const int32_t r = a.dz_order ? row_of[row] : row;
               return r < 0 ? kNowhere : (uint32_t)(r * zs);
           });
    z.chain(main, s, tile.segments(), count, s.low + i0 * s.width, (uint64_t)n_rows * s.width * 2, 0, LowRows<true>{});
    int32_t steps = main + (count * (int32_t)s.chunks.d + 7) / 8;
    if (a.parts > 1) {
        const int32_t per = (steps + a.parts - 1) / a.parts, first = part * per;
        steps = steps - first < per ? steps - first : per;  // 0 or less: none
        w.skip(first);
        z.skip(first);
    }
    f32x16 acc[S::FI][S::FJ] = {};
    tile_product<S, Mul::kBf16>(w, z, steps, (char EP_LDS *)lds, wave, lane, acc);
    if (a.parts > 1) {
        tile_results<S>(acc, (char EP_LDS *)lds, wave, lane, [&](int row, int col, const float *v) {
            if (row >= n_rows || k0 + col >= a.K)
                return;
            f32x4 *dst = reinterpret_cast<f32x4 *>(a.partial + ((int64_t)part * a.rows + i0 + row) * a.K + k0 + col);
            dst[0] = f32x4{v[0], v[1], v[2], v[3]};
            dst[1] = f32x4{v[4], v[5], v[6], v[7]};
        });
        return;
    }
    const int32_t k = k0 + first_col<S, 8>(wave, lane);
    tile_rows_out<S, 8>(
        acc, (char EP_LDS *)lds, wave, lane,
        [&](int row) -> int32_t { return row < n_rows && k < a.K ? row_of[row] : -1; },
        [&](int row, int, float *v, int32_t r) {
            if (r < 0)
                return;
            if (__builtin_expect(any_nan(v, 8), false))
                redo8(a, s, i0, S::kJ, i0 + row, k, v);
            *reinterpret_cast<u32x4 *>(a.dx + (int64_t)r * a.K + k) = pack8(v);
        });
}

// dx from its parts, added in order: eight values per thread.
__global__ __launch_bounds__(256) void adapter_dx_join_kernel(DxArgs a, AdapterSide s, FastDiv groups) {
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = groups.div(at);
    const int64_t i = row;
    const int32_t k = (int32_t)(at - row * groups.d) * 8;
    const int32_t r = i < a.rows ? row_at(s.order, a.rows, i) : -1;
    if (r < 0)
        return;
    float z[8] = {};
    const float *src = a.partial + i * a.K + k;
    constexpr int kAhead = 4;
    for (int32_t p0 = 0; p0 < a.parts; p0 += kAhead) {
        f32x4 v[kAhead][2];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v[u][h] = f32x4{};
                if (p0 + u < a.parts)
                    v[u][h] = *reinterpret_cast<const f32x4 *>(src + (p0 + u) * a.rows * a.K + h * 4);
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int q = 0; q < 8; ++q)
                z[q] += v[u][q / 4][q % 4];
    }
    if (__builtin_expect(any_nan(z, 8), false))
        redo8(a, s, i - i % a.tile_rows, a.tile_rows, i, k, z);
    *reinterpret_cast<u32x4 *>(a.dx + (int64_t)r * a.K + k) = pack8(z);
}

// The tile of dx and the parts of its contraction, by the estimate of the time.
// The large tiles' costs are the experts' gradient's; those of the small ones were fitted to 40 sizes in every tile and
// 1 to 8 parts: the choice takes 1.03 of the best one's time in the mean (114 rows of 25 adapters 4608 x 1576 13 us
// instead of 19, 427 rows of 3 2048 x 1536 16 instead of 21).
enum class DxSize { kLarge, kBroad, kMedium, kSmall, kTiny };
struct DxTile {
    DxSize size;
    int i, j;
    StepCost cost;
};
constexpr DxTile kDxTiles[] = {{DxSize::kLarge, Large::kI, Large::kJ, kGradTiles[0].cost},
                               {DxSize::kBroad, Broad::kI, Broad::kJ, kGradTiles[1].cost},
                               {DxSize::kMedium, Medium::kI, Medium::kJ, kGradTiles[2].cost},
                               {DxSize::kSmall, Small::kI, Small::kJ, {true, 0.40, 0.65}},
                               {DxSize::kTiny, TinyRows::kI, TinyRows::kJ, {true, 0.42, 0.60}}};
struct DxPlan {
    DxSize size;
    int32_t row_tiles, col_tiles, parts, tile_rows;
};
DxPlan plan_adapter_dx(int64_t rows, int32_t A, int32_t R, int32_t K, int32_t main) {
    DxPlan best{};
    double least = 0;
    for (const DxTile &g : kDxTiles) {
        const int32_t steps = main + adapter_steps(rows, A, R, g.j);
        const int32_t row_tiles = (int32_t)((rows + g.j - 1) / g.j), col_tiles = (K + g.i - 1) / g.i;
        for (int32_t parts = 1; parts == 1 || steps / parts >= kSplitSteps; parts *= 2) {
            const double t = estimate(g.cost, (double)row_tiles * col_tiles, parts, (steps + parts - 1) / parts, rows * K);
            if (least == 0 || t < least) {
                least = t;
                best = {g.size, row_tiles, col_tiles, parts, g.j};
            }
        }
    }
    return best;
}
int32_t main_steps(bool base, int32_t Nw) { return base ? (Nw + kStepRows - 1) / kStepRows : 0; }

template <class S>
hipError_t launch_dx(const DxArgs &a, const AdapterSide &s, hipStream_t stream) {
    const int64_t tiles = (int64_t)a.row_tiles * a.col_tiles * a.parts;
    if (tiles > kMostTiles)
        return hipErrorInvalidConfiguration;
    const hipError_t e =
        launch_traced("adapter_dx", adapter_dx_kernel<S>, dim3((unsigned)(tiles + 8)), S::kThreads, stream, a, s);
    if (e != hipSuccess || a.parts == 1)
        return e;
    const int64_t groups = a.rows * (a.K / 8);
    return launch_traced("adapter_dx_join", adapter_dx_join_kernel, dim3((unsigned)((groups + 255) / 256)), 256, stream, a, s,
                         fast_div((uint32_t)(a.K / 8)));
}

// ---- da and db -----------------------------------------------------------------------
// Rows across the contraction, gathered through an order.  The next step's entries of the order are on
// their way while a step's rows are loaded.
template <int T, int W, int FRAGMENTS>
struct GatherAcross : AcrossC<T, W, FRAGMENTS> {
    typedef AcrossC<T, W, FRAGMENTS> First;
    using First::kLoads;
    __amdgpu_buffer_rsrc_t order;
    int32_t place, last;  // of the order, from its first entry on: the next step's first, and the end
    const char *all;
    uint32_t size, column;  // bytes of all rows; the tile's first column
    int32_t total;
    int32_t next[kLoads];

    // Places begin .. end - 1 of the n rows, from step `first` on.  (As the rows are smaller than 2^31 bytes, and
    // eight values or more each, the order is smaller than 2^29.)
    __device__ __forceinline__ void start(const int32_t *o, const char *rows, int64_t n, int64_t row_bytes, int64_t begin,
                                          int64_t end, int32_t index0, int32_t first, int wave, int lane) {
        First::init(rows, row_bytes, 0, index0, wave, lane);
        order = buffer_of(reinterpret_cast<const char *>(o + begin), (uint32_t)(end - begin) * 4);
        all = rows;
        size = (uint32_t)(n * row_bytes);
        column = (uint32_t)index0;
        total = (int32_t)n;
        place = first * kStepRows;
        last = (int32_t)(end - begin);
        fetch(wave, lane);
    }
    __device__ __forceinline__ void fetch(int wave, int lane) {
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            next[q] = __builtin_amdgcn_raw_buffer_load_b32(order, (place + First::row_of(q, wave, lane)) * 4, 0, 0);
        place += kStepRows;
    }
    __device__ __forceinline__ void begin(bool live) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        First::range = buffer_of(all, live ? size : 0);
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            First::offset[q] = place - kStepRows + First::row_of(q, wave, lane) < last && (uint32_t)next[q] < (uint32_t)total
                                   ? (uint32_t)next[q] * (uint32_t)First::stride + First::column_of(q, column, wave, lane)
                                   : kNowhere;
        fetch(wave, lane);
    }
    __device__ __forceinline__ void end() {}
};

struct WeightArgs {
    const int32_t *order, *offsets;  // order: of the long rows alone; null: they are in the adapters' order
    int64_t rows;
    int32_t A, R, L, width;
    const uint16_t *side, *low;  // [rows][L]; [rows][width]: v in two values (da) or low (db)
    uint16_t *out;               // da [A][R][L], db [A][L][R]
    float *partial;              // parts > 1: [parts] of the same
    int32_t tiles, groups, parts;  // along L, of the ranks, of an adapter's rows
    int32_t blocks;              // workgroups, a multiple of 8; 0: not wanted
};

// da: i = the long side's columns, j = a block of v's ranks, the first values and then the second, which are
// added up at the end.  db: i = ranks, j = the long side's columns.
template <class S, bool DA, bool GATHERED>
__device__ __forceinline__ void weight_tile(const WeightArgs &a, int32_t block, char EP_LDS *lds, int lane, int wave) {
    int64_t t = tile_of_block(block, (int64_t)a.A * a.parts * a.groups * a.tiles);
    if (t < 0)
        return;
    const int32_t tile = (int32_t)(t % a.tiles);
    t /= a.tiles;
    const int32_t group = (int32_t)(t % a.groups);
    t /= a.groups;
    const int32_t part = (int32_t)(t % a.parts), e = (int32_t)(t / a.parts);
    int64_t b, end;
    expert_rows(a.offsets, a.rows, e, b, end);
    const int32_t all = (int32_t)((end - b + kStepRows - 1) / kStepRows), per = (all + a.parts - 1) / a.parts;
    const int32_t first = part * per, steps = all - first < per ? all - first : per;  // 0 or less: none
    constexpr int kLong = DA ? S::kI : S::kJ, kShort = DA ? S::kJ : S::kI;
    const int32_t l0 = tile * kLong;
    std::conditional_t<GATHERED, GatherAcross<kLong, S::kWaves, DA ? S::FI : S::FJ>,
                       AcrossC<kLong, S::kWaves, DA ? S::FI : S::FJ>>
        x;
    AcrossC<kShort, S::kWaves, DA ? S::FJ : S::FI> v;
    if constexpr (GATHERED) {
        x.start(a.order, reinterpret_cast<const char *>(a.side), a.rows, (int64_t)a.L * 2, b, end, l0, first, wave, lane);
    } else {
        x.init(reinterpret_cast<const char *>(a.side + b * a.L), (int64_t)a.L * 2, end - b, l0, wave, lane);
        x.skip(first);
    }
    v.init(reinterpret_cast<const char *>(a.low + b * a.width), (int64_t)a.width * 2, end - b, group * kShort, wave, lane);
    v.skip(first);
    f32x16 acc[S::FI][S::FJ] = {};
    // where eight results go: in the weights, counted in values
    const auto put = [&](int64_t at, const float *o) {
        if (a.parts == 1) {
            *reinterpret_cast<u32x4 *>(a.out + at) = pack8(o);
        } else {
            f32x4 *dst = reinterpret_cast<f32x4 *>(a.partial + (int64_t)part * a.A * a.R * a.L + at);
            dst[0] = f32x4{o[0], o[1], o[2], o[3]};
            dst[1] = f32x4{o[4], o[5], o[6], o[7]};
        }
    };
    if constexpr (DA) {
        tile_product<S, Mul::kBf16>(x, v, steps, lds, wave, lane, acc);
        typedef TileShape<S::kI, S::kJ / 2, S::kWavesI, S::kWavesJ, S::kStages> Half;
        static_assert(S::kWavesJ == 1, "both values of a rank are one wave's");
        f32x16 sum[Half::FI][Half::FJ];
#pragma unroll
        for (int i = 0; i < Half::FI; ++i)
#pragma unroll
            for (int j = 0; j < Half::FJ; ++j)
                sum[i][j] = acc[i][j] + acc[i][j + Half::FJ];
        tile_results<Half>(sum, lds, wave, lane, [&](int row, int col, const float *o) {
            const int32_t rank = group * (kShort / 2) + row, l = l0 + col;
            if (rank < a.R && l < a.L)
                put(((int64_t)e * a.R + rank) * a.L + l, o);
        });
    } else {
        tile_product<S, Mul::kBf16>(v, x, steps, lds, wave, lane, acc);
        tile_results<S>(acc, lds, wave, lane, [&](int row, int col, const float *o) {
            const int32_t rank = group * kShort + col, l = l0 + row;
            if (rank < a.R && l < a.L)
                put(((int64_t)e * a.L + l) * a.R + rank, o);
        });
    }
}

template <class S, bool DA>
__device__ __forceinline__ void any_weight_tile(const WeightArgs &a, int32_t block, char EP_LDS *lds, int lane, int wave) {
    if (a.order)
        weight_tile<S, DA, true>(a, block, lds, lane, wave);
    else
        weight_tile<S, DA, false>(a, block, lds, lane, wave);
}

// Both in one launch: neither fills the chip for long, and they do not need each other.
template <class SA, class SB>
__global__ __launch_bounds__(SA::kThreads) void adapter_weights_kernel(WeightArgs da, WeightArgs db) {
    static_assert(SA::kThreads == SB::kThreads, "");
    constexpr int kA = SA::kStages * SA::kStageBytes, kB = SB::kStages * SB::kStageBytes;
    __shared__ __attribute__((aligned(1024))) char lds[kA > kB ? kA : kB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int32_t)blockIdx.x < da.blocks)
        any_weight_tile<SA, true>(da, (int32_t)blockIdx.x, (char EP_LDS *)lds, lane, wave);
    else
        any_weight_tile<SB, false>(db, (int32_t)blockIdx.x - da.blocks, (char EP_LDS *)lds, lane, wave);
}

// The parts added up in order: eight values per thread, da's and then db's.
struct JoinArgs {
    const float *partial;
    int32_t parts;  // 1: nothing to do
    int64_t groups;
    uint16_t *out;
};
__global__ __launch_bounds__(256) void adapter_weights_join_kernel(JoinArgs da, JoinArgs db) {
    int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const bool second = i >= da.groups;
    i -= second ? da.groups : 0;
    const float *partial = second ? db.partial : da.partial;
    const int32_t parts = second ? db.parts : da.parts;
    const int64_t groups = second ? db.groups : da.groups;
    if (i >= groups)
        return;
    float s[8] = {};
    const f32x4 *src = reinterpret_cast<const f32x4 *>(partial) + i * 2;
    constexpr int kAhead = 4;
    for (int32_t p0 = 0; p0 < parts; p0 += kAhead) {
        f32x4 v[kAhead][2];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v[u][h] = f32x4{};
                if (p0 + u < parts)
                    v[u][h] = src[(p0 + u) * groups * 2 + h];
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int q = 0; q < 8; ++q)
                s[q] += v[u][q / 4][q % 4];
    }
    reinterpret_cast<u32x4 *>(second ? db.out : da.out)[i] = pack8(s);
}

// 32 and 64 ranks of da, 64 of db.  Two stages (48, 64 and 48 KiB of LDS), so that three workgroups or two fit a compute
// unit: 1103 rows of 47 adapters 14 us, 18 with three stages; 6744 rows of 49 22, 25.
typedef TileShape<128, 64, 4, 1, 2> Da32;
typedef TileShape<128, 128, 4, 1, 2> Da64;
typedef TileShape<64, 128, 2, 2, 2> Db64;

// Tiles along the long side (x for da, dz for db) and of the ranks, and the parts of the rows, until each of the two
// products has a tile per compute unit (8192 rows, 4096 x 4096, 64 ranks, from the memory-side cache: 24 us and 4 for the
// parts' sums; two tiles each 29 and 6).  A long adapter among short ones has no more parts than they have (6855 rows of 9
// adapters, 2888 x 1448, 16 ranks: 14 us, 39 with four fifths of the rows one adapter's): pieces of so many rows instead would
// need the kernel that joins them in every call, 4 us.
struct WeightPlan {
    int32_t tiles, groups, parts;
    WeightPlan(int64_t rows, int32_t A, int32_t R, int32_t L, bool da) {
        const int32_t ranks = da ? 1 << split_log(R) : Db64::kI;
        tiles = (L + 127) / 128;
        groups = (R + ranks - 1) / ranks;
        const int64_t steps = (rows / A + kStepRows - 1) / kStepRows;  // of an adapter, to expect
        parts = 1;
        while ((int64_t)A * tiles * groups * parts < kCus && steps / (parts * 2) >= kSplitSteps)
            parts *= 2;
    }
    size_t bytes(int32_t A, int32_t R, int32_t L) const { return parts > 1 ? (size_t)parts * A * R * L * 4 : 0; }
};

void set_plan(WeightArgs &a, const WeightPlan &p) {
    a.tiles = p.tiles;
    a.groups = p.groups;
    a.parts = p.parts;
    a.blocks = (int32_t)(((int64_t)a.A * p.tiles * p.groups * p.parts + 15) / 8 * 8);
}
JoinArgs join_args(const WeightArgs &a) {
    return {a.partial, a.parts, a.blocks && a.parts > 1 ? (int64_t)a.A * a.R * a.L / 8 : 0, a.out};
}

hipError_t launch_weights(const WeightArgs &da, const WeightArgs &db, int32_t log, hipStream_t stream) {
    const dim3 grid((unsigned)(da.blocks + db.blocks));
    const hipError_t e =
        log == 5 ? launch_traced("adapter_weights", adapter_weights_kernel<Da32, Db64>, grid, Db64::kThreads, stream, da, db)
                 : launch_traced("adapter_weights", adapter_weights_kernel<Da64, Db64>, grid, Db64::kThreads, stream, da, db);
    const JoinArgs ja = join_args(da), jb = join_args(db);
    if (e != hipSuccess || ja.groups + jb.groups == 0)
        return e;
    return launch_traced("adapter_weights_join", adapter_weights_join_kernel,
                         dim3((unsigned)((ja.groups + jb.groups + 255) / 256)), 256, stream, ja, jb);
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Rows that are gathered through an order are addressed in 31 bits; larger arrays are copied in order.
bool too_far(int64_t rows, int64_t length) { return rows * length * 2 > INT32_MAX; }

// v [rows][split_width], dz [rows][Nw] (with an activation, or out of a gather's reach), x's rows [rows][K] (out
// of its reach), and the parts of dx, of da and of db.
struct Workspace {
    size_t dz = 0, x = 0, dx_sums = 0, da_sums = 0, db_sums = 0, bytes = 0;
    bool own_dz, own_x;
    Workspace(int64_t rows, int32_t A, int32_t R, int32_t K, int32_t N, int32_t act, bool base, bool order, bool dx, bool da,
              bool db) {
        const int64_t Nw = act == EP_ACT_SWIGLU ? 2 * (int64_t)N : N;
        own_dz = (dx || da || db) && rows > 0 && (act != EP_ACT_NONE || (order && too_far(rows, Nw)));
        own_x = da && order && too_far(rows, K);
        dz = dx || da ? align256((size_t)rows * split_width(R) * 2) : 0;
        x = dz + (own_dz ? align256((size_t)(rows * Nw * 2)) : 0);
        dx_sums = x + (own_x ? align256((size_t)rows * K * 2) : 0);
        const int32_t parts = dx && rows > 0 ? plan_adapter_dx(rows, A, R, K, main_steps(base, (int32_t)Nw)).parts : 1;
        da_sums = dx_sums + (parts > 1 ? align256((size_t)parts * rows * K * 4) : 0);
        db_sums = da_sums + (da ? align256(WeightPlan(rows, A, R, K, true).bytes(A, R, K)) : 0);
        bytes = db_sums + (db ? WeightPlan(rows, A, R, (int32_t)Nw, false).bytes(A, R, (int32_t)Nw) : 0);
    }
};

}  // namespace

size_t adapter_grad_workspace_bytes(int64_t rows, int32_t A, int32_t R, int32_t K, int32_t N, int32_t act, bool base, bool order,
                                    bool dx, bool da, bool db) {
    return Workspace(rows, A, R, K, N, act, base, order, dx, da, db).bytes;
}

hipError_t launch_adapter_grad(const AdapterGradArgs &a, hipStream_t stream) {
    const bool gated = a.act == EP_ACT_SWIGLU, activated = a.act != EP_ACT_NONE;
    const int32_t Nw = gated ? 2 * a.N : a.N;
    const Workspace ws(a.rows, a.A, a.R, a.K, a.N, a.act, a.w != nullptr, a.order != nullptr, a.dx, a.da, a.db);
    char *base = static_cast<char *>(a.workspace);
    uint16_t *v = reinterpret_cast<uint16_t *>(base);
    const uint16_t *dz = static_cast<const uint16_t *>(a.d_y), *x = static_cast<const uint16_t *>(a.x);
    const int32_t *dz_order = a.order, *x_order = a.order;
    const auto in_order = [&](const uint16_t *pre, const uint16_t *rows, int32_t N, bool two, uint16_t *to) {
        const dim3 grid((unsigned)((N / 8 + 255) / 256), (unsigned)std::min<int64_t>(a.rows, 1 << 15));
#define EP_CALL(GATED)                                                                                                 \
    launch_traced("adapter_dz", adapter_dz_kernel<GATED>, grid, 256, stream, a.order, a.rows, N, a.act, pre, rows, to)
        return two ? EP_CALL(true) : EP_CALL(false);
#undef EP_CALL
    };
    hipError_t e = hipSuccess;
    if (ws.own_dz) {
        uint16_t *to = reinterpret_cast<uint16_t *>(base + ws.dz);
        e = in_order(activated ? static_cast<const uint16_t *>(a.pre) : nullptr, dz, a.N, gated, to);
        if (e != hipSuccess)
            return e;
        dz = to;
        dz_order = nullptr;
    }
    if (ws.own_x) {
        uint16_t *to = reinterpret_cast<uint16_t *>(base + ws.x);
        e = in_order(nullptr, x, a.K, false, to);
        if (e != hipSuccess)
            return e;
        x = to;
        x_order = nullptr;
    }
    const int32_t width = split_width(a.R), log = split_log(a.R);
    if (a.dx || a.da) {
        e = launch_adapter_low({dz, a.rows, dz_order, a.offsets, a.A, a.R, Nw, a.b, true, a.scale, nullptr, v, width, log}, stream);
        if (e != hipSuccess)
            return e;
    }
    if (a.rows > 0 && a.dx) {
        const DxPlan plan = plan_adapter_dx(a.rows, a.A, a.R, a.K, main_steps(a.w != nullptr, Nw));
        const DxArgs d{a.rows, a.K, Nw, static_cast<const uint16_t *>(a.w), dz, dz_order, static_cast<uint16_t *>(a.dx),
                       reinterpret_cast<float *>(base + ws.dx_sums), plan.row_tiles, plan.col_tiles, plan.parts, plan.tile_rows};
        const AdapterSide s = adapter_side(a.order, a.offsets, a.A, a.R, v, width, log, a.a);
        e = plan.size == DxSize::kLarge    ? launch_dx<Large>(d, s, stream)
            : plan.size == DxSize::kBroad  ? launch_dx<Broad>(d, s, stream)
            : plan.size == DxSize::kMedium ? launch_dx<Medium>(d, s, stream)
            : plan.size == DxSize::kSmall  ? launch_dx<Small>(d, s, stream)
                                           : launch_dx<TinyRows>(d, s, stream);
        if (e != hipSuccess)
            return e;
    }
    WeightArgs da{}, db{};
    if (a.da) {
        da = {x_order, a.offsets, a.rows, a.A, a.R, a.K, width, x, v, static_cast<uint16_t *>(a.da),
              reinterpret_cast<float *>(base + ws.da_sums), 0, 0, 0, 0};
        set_plan(da, WeightPlan(a.rows, a.A, a.R, a.K, true));
    }
    if (a.db) {
        db = {dz_order, a.offsets, a.rows, a.A, a.R, Nw, a.R, dz, static_cast<const uint16_t *>(a.low),
              static_cast<uint16_t *>(a.db), reinterpret_cast<float *>(base + ws.db_sums), 0, 0, 0, 0};
        set_plan(db, WeightPlan(a.rows, a.A, a.R, Nw, false));
    }
    return da.blocks + db.blocks ? launch_weights(da, db, log, stream) : e;
}

}  // namespace ep
