// product_grad.hip -- gradients of the experts' product y = act(x W_e^T + b_e):
//   dz = d_y act'(pre);  dx = dz W_e;  dw_e = dz^T x;  db_e = column sums of dz.
//
// Three kernels: dz and the bias's column sums element by element (HBM-bound; left out where
// dz is d_y itself and no bias is wanted), then two matrix products on the tile of
// product_tile.h.  Neither needs a transposed copy: W in dx, and dz and x in dw, are read
// across the contraction by the transposing LDS load.
//
// 8192 rows of two 4096 x 4096 experts through gelu, with a bias: dz 49 us, dbias 5, dx 270 (1020
// TFLOP/s), dw 234 (1180), one after the other in a call.  dx is the slower since the two experts' rows
// fill no whole number of tiles nor of the chip's turns; both products are bound by the matrix cores
// and the LDS reads that feed them.
//
// dz is rounded to bf16 between the kernels, though it is nobody's result: both products multiply
// bf16, and dz in more bits would double its traffic and their matrix instructions.  It takes
// the gradients' error from 0.0017 of their 2-norm (their own rounding) to 0.0023.
#include "product_tile.h"

namespace ep {
namespace {

constexpr int kDzCols = 512;  // columns of one dz tile: 64 lanes of 8
// Rows of one dz tile, one expert's: 4 waves of 16 rows (the longer tiles leave fewer sums for the
// bias), or of 4 where that gives fewer than two workgroups per compute unit.  Measured, us: 4725
// rows of 352 15.8 / 8.7, 7574 rows of 512 gated 19.9 / 11.7.
int dz_rows(int64_t rows, int32_t E, int32_t N) {
    return row_tiles_most(rows, E, 64) * ((N + kDzCols - 1) / kDzCols) < 2 * kCus ? 16 : 64;
}

// dz (null: not stored) and the column sums of each row tile (partial, null: not wanted).
template <bool GATED>
__global__ __launch_bounds__(256) void product_dz_kernel(const int32_t *offsets, int64_t rows, int32_t E, int per, int32_t N,
                                                         int32_t act, const uint16_t *pre, const uint16_t *d_y,
                                                         uint16_t *dz, float *partial) {
    constexpr int kParts = GATED ? 2 : 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const RowTile rt = find_row_tile(offsets, rows, E, per, (int32_t)blockIdx.x, lane);
    if (rt.e < 0)
        return;
    const int32_t Nw = N * kParts;
    const int32_t n = (int32_t)blockIdx.y * kDzCols + lane * 8;
    float sum[kParts][8] = {};
    if (n < N) {
        // kAhead rows on their way at a time
        constexpr int kAhead = GATED ? 2 : 4;
        for (int i0 = wave; i0 < rt.n; i0 += 4 * kAhead) {
            u32x4 dv[kAhead], zv[kAhead][kParts];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t r = rt.row0 + (i0 + 4 * u < rt.n ? i0 + 4 * u : i0);
                dv[u] = *reinterpret_cast<const u32x4 *>(d_y + r * N + n);
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
                    zv[u][p] = u32x4{0, 0, 0, 0};
                    if (pre)
                        zv[u][p] = *reinterpret_cast<const u32x4 *>(pre + r * Nw + p * N + n);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (i0 + 4 * u >= rt.n)
                    break;
                const int64_t r = rt.row0 + i0 + 4 * u;
                float d[8], z[kParts][8], o[kParts][8];
                unpack8(dv[u], d);
#pragma unroll
                for (int p = 0; p < kParts; ++p)
                    unpack8(zv[u][p], z[p]);
                if (GATED) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float s = sigmoid(z[0][q]);
                        o[0][q] = d[q] * z[kParts - 1][q] * s * (1.f + z[0][q] * (1.f - s));
                        o[kParts - 1][q] = d[q] * z[0][q] * s;
                    }
                } else if (pre) {
                    activation_grad8(z[0], act);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        o[0][q] = d[q] * z[0][q];
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        o[0][q] = d[q];
                }
#pragma unroll
                for (int p = 0; p < kParts; ++p) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        sum[p][q] += o[p][q];
                    if (dz)
                        *reinterpret_cast<u32x4 *>(dz + r * Nw + p * N + n) = pack8(o[p]);
                }
            }
        }
    }
    if (!partial)
        return;
    __shared__ float part[4][64][9];
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 8; ++q)
            part[wave][lane][q] = sum[p][q];
        __syncthreads();
        if (wave == 0 && n < N)
#pragma unroll
            for (int q = 0; q < 8; ++q)
                partial[(int64_t)blockIdx.x * Nw + p * N + n + q] =
                    part[0][lane][q] + part[1][lane][q] + part[2][lane][q] + part[3][lane][q];
    }
}

// dbias[e][n] = sum over the expert's row tiles, of which `partial` holds `most` (offsets that
// decrease would make more).
__global__ __launch_bounds__(1024) void product_dbias_kernel(const int32_t *offsets, int64_t rows, int32_t E, int per, int32_t Nw,
                                                             const float *partial, int64_t most, float *dbias) {
    const int e = blockIdx.y;
    const int64_t first = clamp_row(count_row_tiles(offsets, rows, e, per, threadIdx.x & 63), most);
    int64_t b, t;
    expert_rows(offsets, rows, e, b, t);
    const int64_t n = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const float s = column_sum(partial, first, clamp_row(first + (t - b + per - 1) / per, most), Nw, n);
    if (threadIdx.x < 32 && n < Nw)
        dbias[(int64_t)e * Nw + n] = s;
}

struct GradTileArgs {
    const int32_t *offsets;
    int64_t rows;
    int32_t E, K, Nw;
    const uint16_t *x, *w, *dz;
    uint16_t *out;
    float *partial;  // dw in parts: [parts][E][Nw][K]
    int32_t parts;
};

// dx[r][k] = sum_n dz[r][n] W_e[n][k]: i = k across the contraction, j = rows along it.
template <class S>
__global__ __launch_bounds__(S::kThreads) void product_dx_kernel(GradTileArgs a, int32_t col_tiles) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kStages * S::kStageBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t row_tiles = count_row_tiles(a.offsets, a.rows, a.E, S::kJ, lane);
    const int64_t t = tile_of_block(blockIdx.x, (int64_t)row_tiles * col_tiles);
    if (t < 0)
        return;
    int32_t tr, tc;
    tile_order(t, row_tiles, col_tiles, tr, tc);
    const RowTile rt = find_row_tile(a.offsets, a.rows, a.E, S::kJ, tr, lane);
    if (rt.e < 0)
        return;
    const int32_t k0 = tc * S::kI;
    AcrossC<S::kI, S::kWaves, S::FI> w;
    AlongC<S::kJ, S::kWaves> z;
    w.init(reinterpret_cast<const char *>(a.w + (int64_t)rt.e * a.Nw * a.K), (int64_t)a.K * 2, a.Nw, k0, wave, lane);
    const int64_t zs = (int64_t)a.Nw * 2;
    z.init(reinterpret_cast<const char *>(a.dz) + rt.row0 * zs, (uint32_t)(rt.n * zs), (int32_t)zs, wave, lane,
           [&](int row) -> uint32_t { return (uint32_t)(row * zs); });
    f32x16 acc[S::FI][S::FJ] = {};
    tile_product<S, Mul::kBf16>(w, z, (a.Nw + kStepRows - 1) / kStepRows, (char EP_LDS *)lds, wave, lane, acc);
    tile_results<S>(acc, (char EP_LDS *)lds, wave, lane, [&](int row, int col, const float *v) {
        if (row < rt.n && k0 + col < a.K)
            *reinterpret_cast<u32x4 *>(a.out + (rt.row0 + row) * a.K + k0 + col) = pack8(v);
    });
}

// dw_e[n][k] = sum_r dz[r][n] x[r][k]: both operands across the contraction.
template <class S>
__global__ __launch_bounds__(S::kThreads) void product_dw_kernel(GradTileArgs a, int32_t n_tiles, int32_t k_tiles) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kStages * S::kStageBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Every XCD takes a contiguous eighth of each expert's tiles, expert after expert: an expert's
    // tiles cost as many steps as it has rows.  (With a contiguous eighth of all tiles, 8192 rows
    // split 1520 / 6672 over two 4096 x 4096 experts took 347 us, split evenly 244.)
    const int64_t per_expert = (int64_t)n_tiles * k_tiles, per_xcd = (per_expert + 7) / 8;
    const int64_t turn = blockIdx.x / 8;
    const int32_t part = (int32_t)(turn / per_xcd % a.parts);
    const int e = (int)(turn / per_xcd / a.parts);
    const int64_t t = blockIdx.x % 8 * per_xcd + turn % per_xcd;
    if (t >= per_expert)
        return;
    int32_t tn, tk;
    tile_order(t, n_tiles, k_tiles, tn, tk);
    int64_t b, end;
    expert_rows(a.offsets, a.rows, e, b, end);
    const int32_t k0 = tk * S::kI, n0 = tn * S::kJ;
    AcrossC<S::kI, S::kWaves, S::FI> x;
    AcrossC<S::kJ, S::kWaves, S::FJ> z;
    x.init(reinterpret_cast<const char *>(a.x + b * a.K), (int64_t)a.K * 2, end - b, k0, wave, lane);
    z.init(reinterpret_cast<const char *>(a.dz + b * a.Nw), (int64_t)a.Nw * 2, end - b, n0, wave, lane);
    f32x16 acc[S::FI][S::FJ] = {};
    const int32_t all = (int32_t)((end - b + kStepRows - 1) / kStepRows), per = (all + a.parts - 1) / a.parts;
    const int32_t first = part * per, steps = all - first < per ? all - first : per;  // of this part; 0 or less: none
    x.skip(first);
    z.skip(first);
    tile_product<S, Mul::kBf16>(x, z, steps, (char EP_LDS *)lds, wave, lane, acc);
    tile_results<S>(acc, (char EP_LDS *)lds, wave, lane, [&](int row, int col, const float *v) {
        if (n0 + row >= a.Nw || k0 + col >= a.K)
            return;
        if (a.parts == 1) {
            *reinterpret_cast<u32x4 *>(a.out + ((int64_t)e * a.Nw + n0 + row) * a.K + k0 + col) = pack8(v);
        } else {
            f32x4 *dst = reinterpret_cast<f32x4 *>(a.partial + (((int64_t)part * a.E + e) * a.Nw + n0 + row) * a.K + k0 + col);
            dst[0] = f32x4{v[0], v[1], v[2], v[3]};
            dst[1] = f32x4{v[4], v[5], v[6], v[7]};
        }
    });
}

// dw from its parts, added in order: eight values per thread.
__global__ __launch_bounds__(256) void product_dw_join_kernel(const float *partial, int32_t parts, int64_t groups,
                                                              uint16_t *dw) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
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
    reinterpret_cast<u32x4 *>(dw)[i] = pack8(s);
}

template <class S>
hipError_t launch_dx(const GradTileArgs &a, hipStream_t stream) {
    const int32_t cols = (a.K + S::kI - 1) / S::kI;
    const int64_t tiles = row_tiles_most(a.rows, a.E, S::kJ) * cols;
    if (tiles > kMostTiles)
        return hipErrorInvalidConfiguration;
    return launch_traced("expert_product_dx", product_dx_kernel<S>, dim3((unsigned)(tiles + 8)), S::kThreads, stream, a,
                         cols);
}
template <class S>
hipError_t launch_dw(const GradTileArgs &a, hipStream_t stream) {
    const int32_t kt = (a.K + S::kI - 1) / S::kI, nt = (a.Nw + S::kJ - 1) / S::kJ;
    const int64_t groups = ((int64_t)kt * nt + 7) / 8 * 8 * a.E * a.parts;
    if (groups > kMostTiles)
        return hipErrorInvalidConfiguration;
    return launch_traced("expert_product_dw", product_dw_kernel<S>, dim3((unsigned)groups), S::kThreads, stream, a, nt, kt);
}

enum class GradSize { kLarge, kBroad, kMedium, kSmall };
struct GradTile {
    GradSize size;
    int i, j;
    StepCost cost;
};
// An operand read across the contraction makes a step longer, the smaller the tile the more.
constexpr GradTile kGradTiles[] = {{GradSize::kLarge, Large::kI, Large::kJ, {false, 1.15, 1.90}},
                                   {GradSize::kBroad, Broad::kI, Broad::kJ, {false, 1.00, 1.48}},
                                   {GradSize::kMedium, Medium::kI, Medium::kJ, {true, 0.75, 1.10}},
                                   {GradSize::kSmall, Small::kI, Small::kJ, {true, 0.50, 0.65}}};

// The tile of dx: the large ones where the experts fill them and there is one for every compute
// unit, else by the estimate of the time.  Measured, us: 300 rows 2048 x 2048, a call's dx and dw,
// 28 with Medium alone, 21; dx of 4096 rows of four 2048 x 1408 experts 33 with Broad, 46 with
// Medium; of 574 rows of eight 3168 x 3056 experts 58 with Medium, 88 with Small.
GradSize plan_dx(int64_t rows, int32_t E, int32_t K, int32_t Nw) {
    const int64_t large = (K + Large::kI - 1) / Large::kI;
    if (rows / E >= 160 && row_tiles_most(rows, E, Large::kJ) * large >= kCus)
        return broad_rows(rows, E, large) ? GradSize::kBroad : GradSize::kLarge;
    const int32_t steps = (Nw + kStepRows - 1) / kStepRows;
    GradSize best = GradSize::kMedium;
    double least = 0;
    for (const GradTile &g : kGradTiles) {
        const double t = estimate(g.cost, row_tiles_likely(rows, E, g.j) * ((K + g.i - 1) / g.i), 1, steps, 0);
        if (least == 0 || t < least) {
            least = t;
            best = g.size;
        }
    }
    return best;
}

// The tile and the parts of dw, from the rows per expert to expect: by the estimate where the large
// tiles are fewer than the compute units.  The expert with the most rows has the longest tiles: of
// E experts about the fourth root of E times the mean's (routing with a normal bias of 0.5 or a
// Zipf one of 0.7 gives 1.2 to 1.3 at 2 experts, 2.1 to 3.2 at 16).
struct DwPlan {
    GradSize size;
    int32_t parts;
};
DwPlan plan_dw(int64_t rows, int32_t E, int32_t K, int64_t Nw) {
    const auto tiles = [&](int i, int j) { return (double)E * ((K + i - 1) / i) * ((Nw + j - 1) / j); };
    const double large = tiles(Large::kI, Large::kJ);
    if (large >= kCus)
        return {broad_wins(large, tiles(Broad::kI, Broad::kJ)) ? GradSize::kBroad : GradSize::kLarge, 1};
    const int32_t steps = (int32_t)std::max<int64_t>(1, (rows / E + kStepRows - 1) / kStepRows);
    DwPlan best{GradSize::kMedium, 1};
    double least = 0;
    for (const GradTile &g : kGradTiles)
        for (int32_t parts = 1; parts == 1 || steps / parts >= kSplitSteps; parts *= 2) {
            const double t = estimate(g.cost, tiles(g.i, g.j), parts, (steps + parts - 1) / parts, E * Nw * K,
                                      std::sqrt(std::sqrt((double)E)));
            if (least == 0 || t < least) {
                least = t;
                best = {g.size, parts};
            }
        }
    return best;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// dz [rows][Nw] bf16 (with an activation, for the products), then the bias's partial sums [row tiles][Nw]
// fp32, then dw's parts [parts][E][Nw][K] fp32 (more than one).
struct GradWorkspace {
    size_t bias = 0, parts = 0, bytes = 0;  // offsets, and the size
    GradWorkspace(int64_t rows, int32_t E, int32_t K, int32_t N, int64_t Nw, bool with_dz, bool with_bias, int32_t dw_parts) {
        bias = with_dz ? align256((size_t)(rows * Nw * 2)) : 0;
        parts = bias + (with_bias ? align256((size_t)(row_tiles_most(rows, E, dz_rows(rows, E, N)) * Nw * 4)) : 0);
        bytes = parts + (dw_parts > 1 ? (size_t)dw_parts * E * Nw * K * 4 : 0);
    }
};

}  // namespace

size_t product_grad_workspace_bytes(int64_t rows, int32_t E, int32_t K, int32_t N, int32_t act, bool dx, bool dw, bool bias) {
    const int64_t Nw = act == EP_ACT_SWIGLU ? 2 * (int64_t)N : N;
    return GradWorkspace(rows, E, K, N, Nw, act != EP_ACT_NONE && (dx || dw), bias, dw ? plan_dw(rows, E, K, Nw).parts : 1).bytes;
}

hipError_t launch_product_grad(const ProductGradArgs &a, hipStream_t stream) {
    const bool activated = a.act != EP_ACT_NONE, with_dz = activated && (a.dx || a.dw);
    uint16_t *own_dz = with_dz ? static_cast<uint16_t *>(a.workspace) : nullptr;
    const DwPlan dw = a.dw ? plan_dw(a.rows, a.E, a.K, a.Nw) : DwPlan{GradSize::kMedium, 1};
    const GradWorkspace ws(a.rows, a.E, a.K, a.N, a.Nw, with_dz, a.dbias != nullptr, dw.parts);
    const int per = dz_rows(a.rows, a.E, a.N);
    float *partial = nullptr;
    if (a.dbias)
        partial = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + ws.bias);
    if (a.rows > 0 && (own_dz || partial)) {
        const dim3 grid((unsigned)row_tiles_most(a.rows, a.E, per), (unsigned)((a.N + kDzCols - 1) / kDzCols));
#define EP_CALL(GATED)                                                                                              \
    launch_traced("expert_product_dz", product_dz_kernel<GATED>, grid, 256, stream, a.offsets, a.rows, a.E, per, a.N, a.act, \
                  (const uint16_t *)(activated ? a.pre : nullptr), (const uint16_t *)a.d_y, own_dz, partial)
        const hipError_t e = a.act == EP_ACT_SWIGLU ? EP_CALL(true) : EP_CALL(false);
#undef EP_CALL
        if (e != hipSuccess)
            return e;
    }
    if (a.dbias) {
        const hipError_t e = launch_traced("expert_product_dbias", product_dbias_kernel,
                                           dim3((unsigned)((a.Nw + 31) / 32), (unsigned)a.E), 1024, stream, a.offsets,
                                           a.rows, a.E, per, a.Nw, (const float *)partial, row_tiles_most(a.rows, a.E, per),
                                           a.dbias);
        if (e != hipSuccess)
            return e;
    }
    GradTileArgs g{a.offsets, a.rows, a.E, a.K, a.Nw, (const uint16_t *)a.x, (const uint16_t *)a.w,
                   own_dz ? own_dz : (const uint16_t *)a.d_y, nullptr, nullptr, 1};
    if (a.dx && a.rows > 0) {
        g.out = static_cast<uint16_t *>(a.dx);
        const GradSize size = plan_dx(a.rows, a.E, a.K, a.Nw);
        const hipError_t e = size == GradSize::kLarge    ? launch_dx<Large>(g, stream)
                             : size == GradSize::kBroad  ? launch_dx<Broad>(g, stream)
                             : size == GradSize::kMedium ? launch_dx<Medium>(g, stream)
                                                         : launch_dx<Small>(g, stream);
        if (e != hipSuccess)
            return e;
    }
    if (a.dw) {
        g.out = static_cast<uint16_t *>(a.dw);
        g.parts = dw.parts;
        g.partial = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + ws.parts);
        const hipError_t e = dw.size == GradSize::kLarge    ? launch_dw<Large>(g, stream)
                             : dw.size == GradSize::kBroad  ? launch_dw<Broad>(g, stream)
                             : dw.size == GradSize::kMedium ? launch_dw<Medium>(g, stream)
                                                          : launch_dw<Small>(g, stream);
        if (e != hipSuccess || dw.parts == 1)
            return e;
        const int64_t groups = (int64_t)a.E * a.Nw * a.K / 8;
        return launch_traced("expert_product_dw_join", product_dw_join_kernel, dim3((unsigned)((groups + 255) / 256)), 256,
                             stream, (const float *)g.partial, dw.parts, groups, g.out);
    }
    return hipSuccess;
}

}  // namespace ep
