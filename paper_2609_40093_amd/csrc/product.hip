// product.hip -- the experts' matrix product over rows packed by expert:
//   z = x[r] W_e^T + bias_e;  y[r] = act(z) + residual[r]  for the rows r of expert e.
//
// Tiles of weight rows x packed rows on the matrix cores (product_tile.h).  A workgroup finds
// its expert and rows from the offsets in device memory, so the host never learns the counts:
// the grid covers the most tiles that any counts can give, and the rest end at once.  The
// gated product interleaves 16 gate rows with their 16 up rows of W, so that a lane holds a
// gate and its up value in neighbouring accumulators.
#include "product_tile.h"

namespace ep {
namespace {

struct Epilogue {
    const float *w_scale;    // of the expert, [Nw], or null
    const uint16_t *bias;    // of the expert, [Nw], or null
};

// Four neighbouring outputs n..n+3 of row r from their sums z (gated: the gates' zg too).
__device__ __forceinline__ f32x4 scaled(f32x4 z, int32_t col, const Epilogue &ep, float x_scale) {
    if (ep.w_scale) {
        const f32x4 s = *reinterpret_cast<const f32x4 *>(ep.w_scale + col);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            z[q] *= x_scale * s[q];
    }
    if (ep.bias) {
        const uint2 b = *reinterpret_cast<const uint2 *>(ep.bias + col);
        z[0] += bf16_lo(b.x);
        z[1] += bf16_hi(b.x);
        z[2] += bf16_lo(b.y);
        z[3] += bf16_hi(b.y);
    }
    return z;
}
__device__ __forceinline__ void store_bf16x4(void *base, int64_t at, f32x4 v) {
    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(base) + at) = uint2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
}
template <bool GATED>
__device__ __forceinline__ void finish4(const ProductArgs &a, const Epilogue &ep, int64_t r, int32_t n, float x_scale,
                                        f32x4 z, f32x4 up) {
    z = scaled(z, n, ep, x_scale);
    if (GATED)
        up = scaled(up, a.N + n, ep, x_scale);
    if (a.pre) {
        store_bf16x4(a.pre, r * a.Nw + n, z);
        if (GATED)
            store_bf16x4(a.pre, r * a.Nw + a.N + n, up);
    }
    f32x4 y;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        y[q] = GATED ? activation(z[q], EP_ACT_SILU) * up[q] : activation(z[q], a.act);
    if (a.residual) {
        const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(a.residual) + r * a.N + n);
        y[0] += bf16_lo(v.x);
        y[1] += bf16_hi(v.x);
        y[2] += bf16_lo(v.y);
        y[3] += bf16_hi(v.y);
    }
    if (a.f32)
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + r * a.N + n) = y;
    else
        store_bf16x4(a.y, r * a.N + n, y);
}

template <class S, Mul M, bool GATED>
__global__ __launch_bounds__(S::kThreads) void product_kernel(ProductArgs a, int32_t col_tiles) {
    constexpr bool F8 = M != Mul::kBf16;
    __shared__ __attribute__((aligned(1024))) char lds[2 * S::kStageBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t row_tiles = count_row_tiles(a.offsets, a.rows, a.E, S::kJ, lane);
    const int64_t t = tile_of_block(blockIdx.x, (int64_t)row_tiles * col_tiles);
    if (t < 0)
        return;
    int32_t tr, tc;
    tile_order(t, row_tiles, col_tiles, tr, tc);
    const RowTile rt = find_row_tile(a.offsets, a.rows, a.E, S::kJ, tr, lane);
    const int64_t kb = (int64_t)a.K * (F8 ? 1 : 2), xs = F8 ? a.K + EP_ROWS8_EXTRA : kb;
    constexpr int kOut = GATED ? S::kI / 2 : S::kI;  // output columns of a tile
    const int32_t n0 = tc * kOut;
    AlongC<S::kI, S::kWaves> w;
    AlongC<S::kJ, S::kWaves> x;
    const char *wbase = static_cast<const char *>(a.w) + rt.e * (a.Nw * kb);
    w.init(wbase, (uint32_t)(a.Nw * kb), (int32_t)kb, wave, lane, [&](int row) -> uint32_t {
        const int32_t n = GATED ? n0 + (row >> 5) * 16 + (row & 15) : n0 + row;
        return n < a.N ? (uint32_t)((n + (GATED && (row & 16) ? a.N : 0)) * kb) : kNowhere;
    });
    x.init(static_cast<const char *>(a.x) + rt.row0 * xs, (uint32_t)(rt.n * xs), (int32_t)kb, wave, lane,
           [&](int row) -> uint32_t { return (uint32_t)(row * xs); });
    f32x4 acc[S::FI][S::FJ] = {};
    const int64_t steps = (kb + kStepBytes - 1) / kStepBytes;
    tile_product<S, M>(w, x, steps, steps, (char EP_LDS *)lds, wave, lane, acc);

    const Epilogue ep{a.w_scale ? a.w_scale + (int64_t)rt.e * a.Nw : nullptr,
                      a.bias ? static_cast<const uint16_t *>(a.bias) + (int64_t)rt.e * a.Nw : nullptr};
    const int wi = wave % S::kWavesI, wj = wave / S::kWavesI;
#pragma unroll
    for (int j = 0; j < S::FJ; ++j) {
        const int row = (wj * S::FJ + j) * 16 + lane % 16;
        if (row >= rt.n)
            continue;
        const int64_t r = rt.row0 + row;
        float x_scale = 1.f;
        if (F8)
            x_scale = *reinterpret_cast<const float *>(static_cast<const char *>(a.x) + r * xs + a.K);
#pragma unroll
        for (int i = 0; i < S::FI; i += GATED ? 2 : 1) {
            const int frag = wi * S::FI + i;
            const int32_t n = n0 + (GATED ? frag / 2 : frag) * 16 + lane / 16 * 4;
            if (n < a.N)
                finish4<GATED>(a, ep, r, n, x_scale, acc[i][j], GATED ? acc[i + 1][j] : f32x4{});
        }
    }
}

typedef TileShape<256, 256, 4, 2> Large;
typedef TileShape<128, 128, 2, 2> Medium;

template <class S, Mul M, bool GATED>
hipError_t launch_tiles(const ProductArgs &a, hipStream_t stream) {
    constexpr int kOut = GATED ? S::kI / 2 : S::kI;
    const int32_t cols = (a.N + kOut - 1) / kOut;
    const int64_t tiles = row_tiles_most(a.rows, a.E, S::kJ) * cols;
    if (tiles > kMostTiles)
        return hipErrorInvalidConfiguration;
    return launch_traced("expert_product", product_kernel<S, M, GATED>, dim3((unsigned)(tiles + 8)), S::kThreads, stream,
                         a, cols);
}
// The 8-bit matrix instruction doubles the rate, but it lines its products up to the largest
// and drops what lies more than 13 bits below (measured: a sum of 7168 products of 8-bit rows
// is 1.5e-5 off by its 2-norm, of 64 products 1.3e-5; widened to bf16, 4e-7).  That is a hundredth of the bf16
// result's own rounding, so long sums that end in bf16 take it; fp32 results and short sums,
// which the memory bounds anyway, are multiplied as bf16.
constexpr int32_t kLongSum = 512;
Mul multiplication(const ProductArgs &a) {
    return !a.bits8 ? Mul::kBf16 : a.K >= kLongSum && !a.f32 ? Mul::kF8 : Mul::kF8Wide;
}
template <class S>
hipError_t launch_shape(const ProductArgs &a, hipStream_t stream) {
    const bool gated = a.act == EP_ACT_SWIGLU;
    switch (multiplication(a)) {
    case Mul::kBf16:
        return gated ? launch_tiles<S, Mul::kBf16, true>(a, stream) : launch_tiles<S, Mul::kBf16, false>(a, stream);
    case Mul::kF8:
        return gated ? launch_tiles<S, Mul::kF8, true>(a, stream) : launch_tiles<S, Mul::kF8, false>(a, stream);
    default:
        return gated ? launch_tiles<S, Mul::kF8Wide, true>(a, stream) : launch_tiles<S, Mul::kF8Wide, false>(a, stream);
    }
}

}  // namespace

size_t product_workspace_bytes(int64_t, int32_t, int32_t, int32_t, bool, int32_t) { return 0; }

hipError_t launch_product(const ProductArgs &a, hipStream_t stream) {
    if (a.rows == 0)
        return hipSuccess;
    return a.rows / a.E >= 192 ? launch_shape<Large>(a, stream) : launch_shape<Medium>(a, stream);
}

}  // namespace ep
