// adapter_low.hip -- the low-rank values of the adapters' rows: low[i] = scale_a x[order[i]] a_a^T, rounded
// to bf16 (the products that read them multiply bf16).  Rows without an adapter get zeros.  Its second
// use is the gradient's v = scale_a dz b_a, from b transposed.
//
// Bound by the rows' bytes, or for few rows by the adapters'.  A workgroup takes the rows of one
// adapter, 16 or 32 at a time, and up to 64 ranks; its waves share out the contraction, 64 values
// (whole cache lines) at a time, straight from memory into the operands of 16x16 matrix
// instructions, and are added up through LDS in a fixed order.
#include "adapter_tile.h"

namespace ep {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// FQ fragments of 16 ranks, FR of 16 rows.
template <int FQ, int FR, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void adapter_low_kernel(LowArgs a) {
    constexpr int kRows = FR * 16, kRanks = FQ * 16;
    __shared__ f32x4 sums[WAVES][FQ * FR][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rank0 = (int)blockIdx.y * kRanks;
    const RowTile rt = find_row_tile(a.offsets, a.rows, a.A, kRows, (int32_t)blockIdx.x, lane);
    uint16_t *low = static_cast<uint16_t *>(a.low);
    if (rt.e < 0) {  // rows without an adapter: before the first one's and behind the last one's
        if (!a.offsets)
            return;
        const int64_t z = (int64_t)blockIdx.x - count_row_tiles(a.offsets, a.rows, a.A, kRows, lane);
        const int64_t before = clamp_row(a.offsets[0], a.rows), behind = clamp_row(a.offsets[a.A], a.rows);
        const int width = a.R - rank0 < kRanks ? a.R - rank0 : kRanks;
        for (int i = threadIdx.x; i < kRows * (width / 8); i += WAVES * 64) {
            const int64_t p = z * kRows + i / (width / 8);
            const int64_t row = p < before ? p : behind + (p - before);
            if (z >= 0 && row < a.rows)
                *reinterpret_cast<u32x4 *>(low + row * a.R + rank0 + i % (width / 8) * 8) = u32x4{0, 0, 0, 0};
        }
        return;
    }
    const int g = lane / 16;  // which 16 bytes of a fragment's 64 this lane takes
    const uint16_t *xr[FR], *ar[FQ];
    bool has_x[FR], has_a[FQ];
#pragma unroll
    for (int f = 0; f < FR; ++f) {
        const int row = f * 16 + lane % 16;
        const int32_t r = row < rt.n ? row_at(a.order, a.rows, rt.row0 + row) : -1;
        has_x[f] = r >= 0;
        xr[f] = static_cast<const uint16_t *>(a.x) + (has_x[f] ? (int64_t)r * a.K : 0);
    }
#pragma unroll
    for (int f = 0; f < FQ; ++f) {
        const int rank = rank0 + f * 16 + lane % 16;
        has_a[f] = rank < a.R;
        ar[f] = static_cast<const uint16_t *>(a.weights) + ((int64_t)rt.e * a.R + (has_a[f] ? rank : 0)) * a.K;
    }
    f32x4 acc[FQ][FR] = {};
    constexpr int kAhead = 2;
    for (int32_t k0 = wave * 64; k0 < a.K; k0 += WAVES * 64 * kAhead) {
        u32x4 xv[kAhead][2][FR], av[kAhead][2][FQ];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int32_t k = k0 + u * WAVES * 64 + h * 32 + g * 8;
                const bool in = k < a.K;
#pragma unroll
                for (int f = 0; f < FR; ++f) {
                    xv[u][h][f] = u32x4{0, 0, 0, 0};
                    if (in && has_x[f])
                        xv[u][h][f] = *reinterpret_cast<const u32x4 *>(xr[f] + k);
                }
#pragma unroll
                for (int f = 0; f < FQ; ++f) {
                    av[u][h][f] = u32x4{0, 0, 0, 0};
                    if (in && has_a[f])
                        av[u][h][f] = *reinterpret_cast<const u32x4 *>(ar[f] + k);
                }
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < FQ; ++q)
#pragma unroll
                    for (int f = 0; f < FR; ++f)
                        acc[q][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av[u][h][q]),
                                                                            __builtin_bit_cast(bf16x8, xv[u][h][f]),
                                                                            acc[q][f], 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < FQ; ++q)
#pragma unroll
        for (int f = 0; f < FR; ++f)
            sums[wave][q * FR + f][lane] = acc[q][f];
    __syncthreads();
    const float scale = a.scale ? a.scale[rt.e] : 1.f;
    for (int i = threadIdx.x; i < FQ * FR * 64; i += WAVES * 64) {
        const int at = i / 64, l = i % 64;  // a lane holds four ranks of one row
        f32x4 s = sums[0][at][l];
#pragma unroll
        for (int v = 1; v < WAVES; ++v)
            s += sums[v][at][l];
        const int rank = rank0 + at / FR * 16 + l / 16 * 4, row = at % FR * 16 + l % 16;
        if (row < rt.n && rank < a.R)
            *reinterpret_cast<uint64_t *>(low + (rt.row0 + row) * a.R + rank) =
                bf16_pair(s[0] * scale, s[1] * scale) | (uint64_t)bf16_pair(s[2] * scale, s[3] * scale) << 32;
    }
}

template <int FQ, int FR, int WAVES>
hipError_t launch_shape(const LowArgs &a, hipStream_t stream) {
    // every row is one of an adapter or one of none: two tiles more than an adapter more would give
    const int64_t tiles = row_tiles_most(a.rows, a.A + 2, FR * 16);
    return launch_traced("adapter_low", adapter_low_kernel<FQ, FR, WAVES>,
                         dim3((unsigned)tiles, (unsigned)((a.R + FQ * 16 - 1) / (FQ * 16))), WAVES * 64, stream, a);
}

}  // namespace

hipError_t launch_adapter_low(const LowArgs &a, hipStream_t stream) {
    if (a.rows == 0)
        return hipSuccess;
    const bool few = a.rows / a.A < 24 || a.rows < 2048;
    if (a.R <= 16)
        return few ? launch_shape<1, 1, 16>(a, stream) : launch_shape<1, 2, 8>(a, stream);
    if (a.R <= 32)
        return few ? launch_shape<2, 1, 16>(a, stream) : launch_shape<2, 2, 8>(a, stream);
    return few ? launch_shape<4, 1, 16>(a, stream) : launch_shape<4, 2, 8>(a, stream);
}

}  // namespace ep
