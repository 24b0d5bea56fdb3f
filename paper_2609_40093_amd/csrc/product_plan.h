// product_plan.h -- choice of a product's tile and of the parts its contraction is cut into, from the
// sizes the host knows (the experts' product and its gradient, the adapters' product and its gradient).
#pragma once

#include "product_tile.h"

namespace ep {

// The rest of a call's arguments that the two kernels share.
struct Split {
    int32_t parts;  // of the contraction; 1: the tile kernel runs the epilogue
    int32_t steps;  // of one part
};

// Besides the sizes of product_tile.h, for many experts of few rows:
typedef TileShape<256, 128, 4, 2, 2> Wide;   // one workgroup per compute unit (96 KiB of LDS)
typedef TileShape<256, 64, 4, 2, 3> Few;     // one (120 KiB)

// ---- choice of the tile and of the split, from the sizes the host knows ----------------
// By the mean rows per expert.  Measured, us (bf16 gated, 32 experts, K 7168, N 2048; then 128
// experts, K 2048, N 768), Large / Wide / Few / Medium:
//   mean  24  363 / 338 / 398 / 355    178 / 180 / 180 / 162
//   mean  64  389 / 427 / 394 / 421    183 / 195 / 203 / 187
//   mean  96  507 / 431 / 534 / 464    218 / 194 / 221 / 207
//   mean 160  538 / 548 / 738 / 600    248 / 246 / 287 / 250
//   mean 256  609 / 721 / 991 / 820
// Below 80 rows the weights' bytes bound it, and what differs is how evenly the tiles fill the
// compute units.  With less than 16 rows Tiny gains up to a tenth on Medium (16 experts, K 4096,
// N 1536, mean 8: 84 / 93).
//
// Where that tile gives fewer tiles than compute units (the dense products of a decode step,
// few experts), the tiles and the parts of the contraction are weighed by an estimate of the time
// (product_tile.h).  Measured, us, estimate's choice against the larger tile split to
// fill the chip: 256 rows K 7168 N 256 12 / 15, 500 rows 4096 x 4096 30 / 40, 256 rows 2048 x 2048
// 12 / 22; against the small tiles alone: 3190 rows of 15 experts 4176 x 1984 120 / 193.
enum class Size { kLarge, kBroad, kWide, kFew, kMedium, kSmall, kTiny };
inline Size tile_size(int64_t rows, int32_t E) {
    const int64_t mean = rows / E;
    return mean >= 160 ? Size::kLarge : mean >= 80 ? Size::kWide : mean >= 40 ? Size::kFew : mean >= 16 ? Size::kMedium : Size::kTiny;
}
inline int tile_rows(Size s) {
    switch (s) {
    case Size::kLarge: return Large::kJ;
    case Size::kBroad: return Broad::kJ;
    case Size::kWide: return Wide::kJ;
    case Size::kFew: return Few::kJ;
    case Size::kMedium: return Medium::kJ;
    case Size::kSmall: return Small::kJ;
    default: return Tiny::kJ;
    }
}
inline int tile_cols(Size s, bool gated) {
    return (s < Size::kMedium ? Large::kI : s == Size::kSmall ? Small::kI : Medium::kI) / (gated ? 2 : 1);
}

struct Plan {
    Size size;
    int64_t tiles;  // at most
    int32_t cols;
    Split split;
};
// more(per): steps that the contraction of a tile of `per` rows has besides.
template <typename F>
inline Plan make_plan(int64_t rows, int32_t E, int32_t K, int32_t N, bool bits8, bool gated, F more) {
    const int32_t own = (int32_t)(((int64_t)K * (bits8 ? 1 : 2) + kStepBytes - 1) / kStepBytes);
    const auto plan = [&](Size size, int32_t parts) {
        Plan p;
        const int32_t steps = own + more(tile_rows(size));
        p.size = size;
        p.cols = (N + tile_cols(size, gated) - 1) / tile_cols(size, gated);
        p.tiles = row_tiles_most(rows, E, tile_rows(size)) * p.cols;
        p.split.steps = (steps + parts - 1) / parts;
        p.split.parts = (steps + p.split.steps - 1) / p.split.steps;
        return p;
    };
    Plan best = plan(tile_size(rows, E), 1);
    if (best.size == Size::kLarge && broad_rows(rows, E, best.cols))
        best = plan(Size::kBroad, 1);
    if (best.tiles >= kCus)
        return best;
    double least = 0;
    bool any = false;
    for (Size size : {Size::kLarge, Size::kBroad, Size::kMedium, Size::kSmall, Size::kTiny})
        for (int32_t parts = 1; parts == 1 || (own + more(tile_rows(size))) / parts >= kSplitSteps; parts *= 2) {
            const Plan p = plan(size, parts);
            const StepCost cost = size == Size::kLarge    ? kLargeCost
                                  : size == Size::kBroad  ? kBroadCost
                                  : size == Size::kMedium ? kMediumCost
                                  : size == Size::kSmall  ? kSmallCost
                                                          : kTinyCost;
            const double t = estimate(cost, row_tiles_likely(rows, E, tile_rows(size)) * p.cols, p.split.parts, p.split.steps,
                                      rows * N * (gated ? 2 : 1));
            if (!any || t < least) {
                any = true;
                least = t;
                best = p;
            }
        }
    return best;
}
inline Plan make_plan(int64_t rows, int32_t E, int32_t K, int32_t N, bool bits8, bool gated) {
    return make_plan(rows, E, K, N, bits8, gated, [](int) { return 0; });
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
inline GradSize plan_dx(int64_t rows, int32_t E, int32_t K, int32_t Nw) {
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

}  // namespace ep
