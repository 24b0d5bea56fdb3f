// adapter_grad.hip -- gradients of the adapters' product y = act(x W^T + low b_a^T + bias) + residual, W held:
//   dz = d_y act'(pre);  v = scale_a dz b_a;  dx = dz W + v a_a;  da_a = v^T x;  db_a = dz^T low.
//
// v is made as low is (adapter_low.hip), from b transposed.  dx has the product's form: the contraction
// over W's rows goes on over the ranks of the tile's adapters (adapter_tile.h).  da and db are
// contractions over an adapter's rows (product_grad.hip).  Rows go in the adapters' order; where they
// come in another one, or there is an activation, dz is kept in that order, and so are x's rows for da.
//
// v and dz are rounded to bf16 between the kernels: the products multiply bf16.
#include "adapter_tile.h"
#include "product_plan.h"

namespace ep {
namespace {

// b [A][N][R] into [A][R][N]: 64 columns n and 64 ranks at a time.
__global__ __launch_bounds__(256) void adapter_turn_kernel(const uint16_t *b, int32_t N, int32_t R, uint16_t *turned) {
    __shared__ uint16_t part[64][72];
    const int32_t n0 = (int32_t)blockIdx.x * 64, r0 = (int32_t)blockIdx.y * 64;
    const int64_t base = (int64_t)blockIdx.z * N * R;
    const int width = R - r0 < 64 ? R - r0 : 64, vecs = width / 8;
    for (int i = threadIdx.x; i < 64 * vecs; i += 256) {
        const int n = i / vecs, v = i % vecs;
        if (n0 + n < N)
            *reinterpret_cast<u32x4 *>(&part[n][v * 8]) =
                *reinterpret_cast<const u32x4 *>(b + base + (int64_t)(n0 + n) * R + r0 + v * 8);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < width * 8; i += 256) {
        const int r = i / 8, n = i % 8 * 8;
        if (n0 + n >= N)
            continue;
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
            o[q] = part[n + 2 * q][r] | (uint32_t)part[n + 2 * q + 1][r] << 16;
        *reinterpret_cast<u32x4 *>(turned + base + (int64_t)(r0 + r) * N + n0 + n) = u32x4{o[0], o[1], o[2], o[3]};
    }
}

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
    uint16_t *dx;
};

// The sums of place i, columns k..k+7, of their own terms alone.
__device__ __forceinline__ void redo8(const DxArgs &a, const AdapterSide &s, int64_t i, int32_t k, float *z) {
    const int32_t e = adapter_of(s, a.rows, i);
#pragma unroll
    for (int q = 0; q < 8; ++q)
        z[q] = 0.f;
    const auto add = [&](const uint16_t *u, const uint16_t *v, int32_t length) {
#pragma unroll 1
        for (int32_t n = 0; n < length; ++n) {
            float g[8];
            unpack8(*reinterpret_cast<const u32x4 *>(v + (int64_t)n * a.K + k), g);
            const float f = __uint_as_float((uint32_t)u[n] << 16);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                z[q] = fmaf(f, g[q], z[q]);
        }
    };
    if (a.w)
        add(a.dz + i * a.Nw, a.w, a.Nw);
    if (e >= 0)
        add(s.low + i * s.R, s.weights + (int64_t)e * s.R * a.K, s.R);
}

// dx[order[i]][k] = sum_n dz[i][n] w[n][k] + sum_j v[i][j] a_e[j][k]: i = k across the contraction, j = rows.
template <class S>
__global__ __launch_bounds__(S::kThreads) void adapter_dx_kernel(DxArgs a, AdapterSide s, int32_t row_tiles, int32_t col_tiles) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kStages * S::kStageBytes];
    __shared__ Segment table[S::kJ];
    Segment EP_LDS *segments = (Segment EP_LDS *)table;
    __shared__ int32_t found;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = tile_of_block(blockIdx.x, (int64_t)row_tiles * col_tiles);
    if (t < 0)
        return;
    int32_t tr, tc;
    tile_order(t, row_tiles, col_tiles, tr, tc);
    const int64_t i0 = (int64_t)tr * S::kJ;
    const int n_rows = a.rows - i0 < S::kJ ? (int)(a.rows - i0) : S::kJ;
    if (wave == 0) {
        const int n = find_segments<S::kJ>(s, a.rows, i0, n_rows, segments, lane);
        if (lane == 0)
            found = n;
    }
    __syncthreads();
    const int count = __builtin_amdgcn_readfirstlane(found);
    const int32_t k0 = tc * S::kI;
    const int32_t main = a.w ? (a.Nw + kStepRows - 1) / kStepRows : 0;
    ChainAcross<S::kI, S::kWaves, S::FI> w;
    ChainAlong<S::kJ, S::kWaves, true> z;
    w.init(reinterpret_cast<const char *>(a.w), (int64_t)a.K * 2, a.Nw, k0, wave, lane);
    w.chain(main, s, segments, count, (uint64_t)s.A * s.R * a.K * 2);
    const int64_t zs = (int64_t)a.Nw * 2;
    z.init(reinterpret_cast<const char *>(a.dz) + i0 * zs, (uint32_t)(n_rows * zs), (int32_t)zs, wave, lane,
           [&](int row) -> uint32_t { return (uint32_t)(row * zs); });
    z.chain(main, s, segments, count, s.low + i0 * s.R, (uint64_t)n_rows * s.R * 2, 0, wave, lane, [](int row) { return row; });
    f32x16 acc[S::FI][S::FJ] = {};
    tile_product<S, Mul::kBf16>(w, z, main + (count * (s.R / 8) + 7) / 8, (char EP_LDS *)lds, wave, lane, acc);
    const int32_t k = k0 + first_col<S, 8>(wave, lane);
    tile_rows_out<S, 8>(
        acc, (char EP_LDS *)lds, wave, lane,
        [&](int row) -> int32_t { return row < n_rows && k < a.K ? row_at(s.order, a.rows, i0 + row) : -1; },
        [&](int row, int, float *v, int32_t r) {
            if (r < 0)
                return;
            if (__builtin_expect(any_nan(v, 8), false))
                redo8(a, s, i0 + row, k, v);
            *reinterpret_cast<u32x4 *>(a.dx + (int64_t)r * a.K + k) = pack8(v);
        });
}

template <class S>
hipError_t launch_dx(const DxArgs &a, const AdapterSide &s, hipStream_t stream) {
    const int32_t cols = (a.K + S::kI - 1) / S::kI;
    const int64_t row_tiles = (a.rows + S::kJ - 1) / S::kJ;
    if (row_tiles * cols > kMostTiles)
        return hipErrorInvalidConfiguration;
    return launch_traced("adapter_dx", adapter_dx_kernel<S>, dim3((unsigned)(row_tiles * cols + 8)), S::kThreads, stream, a, s,
                         (int32_t)row_tiles, cols);
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// v [rows][R], b turned [A][R][Nw], dz [rows][Nw] and x's rows [rows][K] in the adapters' order, and the
// workspace of da's and db's contractions.
struct Workspace {
    size_t turned = 0, dz = 0, x = 0, sums = 0, bytes = 0;
    Workspace(int64_t rows, int32_t A, int32_t R, int32_t K, int32_t N, int32_t act, bool order, bool dx, bool da, bool db) {
        const int64_t Nw = act == EP_ACT_SWIGLU ? 2 * (int64_t)N : N;
        const bool v = dx || da;
        turned = v ? align256((size_t)rows * R * 2) : 0;
        dz = turned + (v ? align256((size_t)A * R * Nw * 2) : 0);
        x = dz + (order || act != EP_ACT_NONE ? align256((size_t)(rows * Nw * 2)) : 0);
        sums = x + (order && da ? align256((size_t)rows * K * 2) : 0);
        const size_t sa = da ? product_grad_workspace_bytes(rows, A, K, R, EP_ACT_NONE, false, true, false) : 0;
        const size_t sb = db ? product_grad_workspace_bytes(rows, A, R, (int32_t)Nw, EP_ACT_NONE, false, true, false) : 0;
        bytes = sums + std::max(sa, sb);
    }
};

}  // namespace

size_t adapter_grad_workspace_bytes(int64_t rows, int32_t A, int32_t R, int32_t K, int32_t N, int32_t act, bool order, bool dx,
                                    bool da, bool db) {
    return Workspace(rows, A, R, K, N, act, order, dx, da, db).bytes;
}

hipError_t launch_adapter_grad(const AdapterGradArgs &a, hipStream_t stream) {
    const bool gated = a.act == EP_ACT_SWIGLU, activated = a.act != EP_ACT_NONE;
    const int32_t Nw = gated ? 2 * a.N : a.N;
    const Workspace ws(a.rows, a.A, a.R, a.K, a.N, a.act, a.order != nullptr, a.dx, a.da, a.db);
    char *base = static_cast<char *>(a.workspace);
    uint16_t *v = reinterpret_cast<uint16_t *>(base), *turned = reinterpret_cast<uint16_t *>(base + ws.turned);
    const uint16_t *dz = static_cast<const uint16_t *>(a.d_y), *x = static_cast<const uint16_t *>(a.x);
    const auto gather = [&](const uint16_t *pre, const uint16_t *rows, int32_t N, bool two, uint16_t *to) {
        const dim3 grid((unsigned)((N / 8 + 255) / 256), (unsigned)std::min<int64_t>(a.rows, 1 << 15));
#define EP_CALL(GATED)                                                                                                 \
    launch_traced("adapter_dz", adapter_dz_kernel<GATED>, grid, 256, stream, a.order, a.rows, N, a.act, pre, rows, to)
        return two ? EP_CALL(true) : EP_CALL(false);
#undef EP_CALL
    };
    hipError_t e = hipSuccess;
    if (a.rows > 0 && (a.order || activated)) {
        uint16_t *to = reinterpret_cast<uint16_t *>(base + ws.dz);
        e = gather(activated ? static_cast<const uint16_t *>(a.pre) : nullptr, dz, a.N, gated, to);
        if (e != hipSuccess)
            return e;
        dz = to;
    }
    if (a.rows > 0 && (a.dx || a.da)) {
        e = launch_traced("adapter_turn", adapter_turn_kernel,
                          dim3((unsigned)((Nw + 63) / 64), (unsigned)((a.R + 63) / 64), (unsigned)a.A), 256, stream,
                          (const uint16_t *)a.b, Nw, a.R, turned);
        if (e != hipSuccess)
            return e;
        e = launch_adapter_low({dz, a.rows, nullptr, a.offsets, a.A, a.R, Nw, turned, a.scale, v}, stream);
        if (e != hipSuccess)
            return e;
    }
    if (a.rows > 0 && a.dx) {
        const DxArgs d{a.rows, a.K, Nw, static_cast<const uint16_t *>(a.w), dz, static_cast<uint16_t *>(a.dx)};
        const AdapterSide s{a.order, a.offsets, a.A, a.R, v, static_cast<const uint16_t *>(a.a), fast_div((uint32_t)a.R),
                            fast_div((uint32_t)(a.R / 8))};
        const GradSize size = plan_dx(a.rows, 1, a.K, a.w ? Nw : a.R);
        e = size == GradSize::kLarge    ? launch_dx<Large>(d, s, stream)
            : size == GradSize::kBroad  ? launch_dx<Broad>(d, s, stream)
            : size == GradSize::kMedium ? launch_dx<Medium>(d, s, stream)
                                        : launch_dx<Small>(d, s, stream);
        if (e != hipSuccess)
            return e;
    }
    ProductGradArgs p{};
    p.rows = a.rows;
    p.offsets = a.offsets;
    p.E = a.A;
    p.act = EP_ACT_NONE;
    p.workspace = base + ws.sums;
    if (a.da) {
        if (a.rows > 0 && a.order) {
            uint16_t *to = reinterpret_cast<uint16_t *>(base + ws.x);
            e = gather(nullptr, x, a.K, false, to);
            if (e != hipSuccess)
                return e;
            x = to;
        }
        p.x = x;
        p.d_y = v;
        p.K = a.K;
        p.N = p.Nw = a.R;
        p.dw = a.da;
        e = launch_product_grad(p, stream);
        if (e != hipSuccess)
            return e;
    }
    if (a.db) {
        p.x = a.low;
        p.d_y = dz;
        p.K = a.R;
        p.N = p.Nw = Nw;
        p.dw = a.db;
        e = launch_product_grad(p, stream);
    }
    return e;
}

}  // namespace ep
