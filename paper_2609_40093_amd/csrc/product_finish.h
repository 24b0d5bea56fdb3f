// product_finish.h -- the epilogue of a product: eight neighbouring results of a row from their sums,
// with scales, bias, activation and residual (the experts' product and the adapters').
#pragma once

#include "product_tile.h"

namespace ep {

// What eight neighbouring results n..n+7 of every row of expert e share: the scales and the
// bias of their weight rows (gated: the gates' rows, then the ups').
template <bool F8, bool GATED>
struct Columns {
    float scale[GATED ? 2 : 1][F8 ? 8 : 1], bias[GATED ? 2 : 1][8];
    __device__ __forceinline__ void load(const ProductArgs &a, int64_t e, int32_t n) {
#pragma unroll
        for (int p = 0; p < (GATED ? 2 : 1); ++p) {
            const int64_t at = e * a.Nw + p * a.N + n;
            if constexpr (F8)
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    scale[p][q] = a.w_scale[at + q];
#pragma unroll
            for (int q = 0; q < 8; ++q)
                bias[p][q] = 0.f;
            if (a.bias)
                unpack8(*reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.bias) + at), bias[p]);
        }
    }
    __device__ __forceinline__ void apply(int p, float x_scale, float *z) const {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            z[q] = F8 ? fmaf(z[q], x_scale * scale[p][F8 ? q : 0], bias[p][q]) : z[q] + bias[p][q];
    }
};
// What a row brings besides: its eight residuals and its scale.
template <bool F8>
struct RowExtra {
    u32x4 residual;
    float scale;
    __device__ __forceinline__ void load(const ProductArgs &a, int64_t r, int32_t n) {
        residual = u32x4{0, 0, 0, 0};
        if (a.residual)
            residual = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(a.residual) + r * a.N + n);
        scale = 1.f;
        if (F8)
            scale = *reinterpret_cast<const float *>(static_cast<const char *>(a.x) + r * (a.K + EP_ROWS8_EXTRA) + a.K);
    }
};
// The results n..n+7 of row r from their sums (gated: z the gates', up the ups').
template <bool F8, bool GATED>
__device__ __forceinline__ void finish8(const ProductArgs &a, const Columns<F8, GATED> &c, const RowExtra<F8> &x, int64_t r,
                                        int32_t n, float *z, float *up) {
    c.apply(0, x.scale, z);
    if constexpr (GATED)
        c.apply(1, x.scale, up);
    if (a.pre) {
        uint16_t *pre = static_cast<uint16_t *>(a.pre) + r * a.Nw + n;
        *reinterpret_cast<u32x4 *>(pre) = pack8(z);
        if (GATED)
            *reinterpret_cast<u32x4 *>(pre + a.N) = pack8(up);
    }
    if (GATED) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            z[q] = z[q] * sigmoid(z[q]) * up[q];
    } else {
        activate8(z, a.act);
    }
    if (a.residual) {
        float res[8];
        unpack8(x.residual, res);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            z[q] += res[q];
    }
    if (a.f32) {
        f32x4 *dst = reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + r * a.N + n);
        dst[0] = f32x4{z[0], z[1], z[2], z[3]};
        dst[1] = f32x4{z[4], z[5], z[6], z[7]};
    } else {
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.y) + r * a.N + n) = pack8(z);
    }
}

}  // namespace ep
