// adapter_tile.h -- operands of the MFMA tile (product_tile.h) whose contraction goes on into a second
// part: the low-rank terms of the adapters whose rows a tile holds.
//
// Rows are taken in the adapters' order (row i of the order is row order[i] of x and y), so the rows
// that an adapter has in a tile are a segment of it.  The second part is as long as the segments'
// ranks together: its places are (segment, rank), rank fastest; where low is kept as two values each, a segment has the
// ranks twice.  The row operand holds zeros at the
// places of the segments that a row is not in, and the column operand the weights of the place's
// adapter, so one accumulator adds up both parts; 64 places are one step whoever's they are: four
// adapters of rank 8 cost what one of rank 32 costs.
//
// Zeros times another adapter's infinities or NaN are NaN, which the epilogues look for (redo below).
#pragma once

#include "product_tile.h"

namespace ep {

// An adapter's rows [lo, hi) in a tile: the adapter, and lo | hi << 16.
typedef int32_t Segment __attribute__((ext_vector_type(2)));

struct AdapterSide {
    const int32_t *order;    // null: the rows come in the adapters' order
    const int32_t *offsets;  // null: one adapter with every row
    int32_t A, R;
    const uint16_t *low;     // LowArgs's split [rows][width], in the adapters' order
    const uint16_t *weights; // b [A][Nw][R] of the product, a [A][R][K] of its gradient
    int32_t width, log;
    FastDiv places, chunks;  // by a segment's 2 R places, and by an eighth of them

    // A segment's places are its ranks with the first values, then its ranks with the second.  The rank of
    // place j, and where the value lies in a row of low.
    __device__ __forceinline__ int32_t rank_of(int32_t j) const { return j >= R ? j - R : j; }
    __device__ __forceinline__ int32_t value_at(int32_t j) const {
        const int32_t rank = rank_of(j);
        return rank + (((rank >> log) + (j >= R ? 1 : 0)) << log);
    }
};
inline AdapterSide adapter_side(const int32_t *order, const int32_t *offsets, int32_t A, int32_t R, const void *low,
                                int32_t width, int32_t log, const void *weights) {
    return {order, offsets, A, R, static_cast<const uint16_t *>(low), static_cast<const uint16_t *>(weights), width, log,
            fast_div((uint32_t)R * 2), fast_div((uint32_t)R / 4)};
}
// Steps that the adapters add to a tile of `per` rows: its segments to expect.
inline int32_t adapter_steps(int64_t rows, int32_t A, int32_t R, int per) {
    const int64_t some = std::min<int64_t>(std::min<int64_t>(A, per), (int64_t)A * per / std::max<int64_t>(rows, 1) + 1);
    return (int32_t)((some * 2 * R + kStepRows - 1) / kStepRows);
}
// Tiny (product_tile.h) with a stage less, so that two workgroups and their tables fit a compute unit.
typedef TileShape<128, 32, 4, 1, 3> TinyRows;

// A low-rank value v as the sum of two bf16 values: the largest one that lies before v on the way from zero, and the rest
// of v, which the caller rounds.  Their sum is v itself where bf16 holds v, else within 2^-16 of it, or 2^-133, bf16's
// smallest number.  Both have v's sign, and neither is zero where |v| is above 2^-133: so with an infinite
// weight w the products' first w + rest w is v w.  (Rounding the first to nearest would be within 2^-17, but leaves a rest that
// is zero or of the other sign, and infinite weights NaN.)
// Zeros, infinities and NaN are both values.  (Told by their bits: v may be a product, and v - v contracted with it.)
__device__ __forceinline__ bool splits(float v) {
    return v != 0.f && (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u;
}
__device__ __forceinline__ float first_of(float v) {
    return splits(v) ? __uint_as_float((__float_as_uint(v) - 1u) & 0xffff0000u) : v;
}
__device__ __forceinline__ float rest_of(float v) {
    return splits(v) ? copysignf(fmaxf(fabsf(v - first_of(v)), 0x1p-133f), v) : v;
}
__device__ __forceinline__ uint32_t first_pair(float lo, float hi) { return bf16_pair(first_of(lo), first_of(hi)); }
__device__ __forceinline__ uint32_t rest_pair(float lo, float hi) { return bf16_pair(rest_of(lo), rest_of(hi)); }
// The layout of split: blocks of 32 ranks (up to 32 ranks) or 64, the first values of a block, then the second.
inline int32_t split_log(int32_t R) { return R <= 32 ? 5 : 6; }
inline int32_t split_width(int32_t R) {
    const int32_t block = 1 << split_log(R);
    return (R + block - 1) / block * block * 2;
}

// The segments of rows i0 .. i0 + n - 1, in the adapters' order; at most PER (more only where offsets
// decrease).  One wave calls it.
template <int PER>
__device__ __forceinline__ int find_segments(const AdapterSide &s, int64_t rows, int64_t i0, int n, Segment EP_LDS *out,
                                             int lane) {
    int count = 0;
    for (int a0 = 0; a0 < s.A; a0 += 64) {
        int64_t b = 0, t = 0;
        if (a0 + lane < s.A)
            expert_rows(s.offsets, rows, a0 + lane, b, t);
        const int64_t lo = b > i0 ? b - i0 : 0, hi = t < i0 + n ? t - i0 : n;
        const bool here = lo < hi;
        const uint64_t m = __ballot(here);
        const int at = count + lanes_below(m);
        if (here && at < PER)
            out[at] = Segment{a0 + lane, (int32_t)(lo | hi << 16)};
        count += __builtin_popcountll(m);
    }
    return count < PER ? count : PER;
}
// The row that place i of the order stands for, -1: none.
__device__ __forceinline__ int32_t row_at(const int32_t *order, int64_t rows, int64_t i) {
    if (!order)
        return (int32_t)i;
    const int32_t r = order[i];
    return r >= 0 && r < rows ? r : -1;
}

// LDS of a tile with chained operands, in one array: the stages, the segments, each row's place in memory
// and the number of segments.  (With several __shared__ variables the compiler tells their accesses apart, and then
// waits for every load into LDS before it reads there: the loads of a step no longer run under the step
// before, and 16379 rows of 7168 by 4096 take 871 us instead of 772.)
template <class S>
struct TileLds {
    static constexpr int kTable = S::kStages * S::kStageBytes, kRows = kTable + S::kJ * 8, kFound = kRows + S::kJ * 4;
    static constexpr int kBytes = kFound + 16;
    char EP_LDS *stages;
    __device__ __forceinline__ Segment EP_LDS *segments() const { return (Segment EP_LDS *)(stages + kTable); }
    __device__ __forceinline__ int32_t EP_LDS *row_of() const { return (int32_t EP_LDS *)(stages + kRows); }
    // Fills the tables for rows i0 .. i0 + n - 1 and gives the number of segments.
    __device__ __forceinline__ int fill(const AdapterSide &s, int64_t rows, int64_t i0, int n, int wave, int lane) const {
        for (int j = threadIdx.x; j < S::kJ; j += S::kThreads)
            row_of()[j] = j < n ? row_at(s.order, rows, i0 + j) : -1;
        int32_t EP_LDS *found = (int32_t EP_LDS *)(stages + kFound);
        if (wave == 0) {
            const int count = find_segments<S::kJ>(s, rows, i0, n, segments(), lane);
            if (lane == 0)
                *found = count;
        }
        __syncthreads();
        return __builtin_amdgcn_readfirstlane(*found);
    }
};

// This lane's number, in the large tiles unknown to the compiler anew in every step: what the second part's steps make
// of it is not kept in registers through the first part's, where those tiles have none to spare.
template <int T>
__device__ __forceinline__ int lane_of_step() {
    int lane = threadIdx.x & 63;
    if (T >= 256)
        asm volatile("" : "+v"(lane));
    return lane;
}

// Rows along the contraction (AlongC), then the second part: the rows' low-rank values (Index: LowRows), else
// the weights b of each column, whose row Index gives for a tile's row (-1: none).  The second
// part's offsets take the place of the first one's, which are not needed any more.
// SKIPS: branches round places that none of a wave's lanes has, where the gradient's tiles gain from them (762 rows of 21
// adapters 36 us, 37.5 without); the product's do without (7393 rows of 62 adapters, 64 ranks 117 us, 129 with them).
template <bool SKIPS>
struct LowRows {
    static constexpr bool kLow = true, kSkips = SKIPS;
};
template <int T, int W, typename Index>
struct ChainAlong : AlongC<T, W> {
    typedef AlongC<T, W> First;
    using First::kLoads;
    static constexpr bool kChained = true;
    static constexpr bool LOW = Index::kLow;
    int32_t first;        // steps of the first part left
    int32_t chunk, most;  // 16-byte chunks of the second part: the next step's first, and all
    const Segment EP_LDS *segments;
    const AdapterSide *side;
    const char *base2;
    uint32_t size2;
    uint32_t adapter_rows;  // of the weights
    Index index;

    // steps: of the first part.  base, size: of the second one's array.
    __device__ __forceinline__ void chain(int32_t steps, const AdapterSide &s, const Segment EP_LDS *at, int count,
                                          const void *base, uint64_t size, int64_t rows, Index index_of) {
        first = steps;
        chunk = 0;
        most = count * (int32_t)s.chunks.d;
        segments = at;
        side = &s;
        base2 = static_cast<const char *>(base);
        size2 = (uint32_t)size;
        adapter_rows = (uint32_t)rows;
        index = index_of;
    }
    __device__ __forceinline__ void skip(int32_t steps) {
        const int32_t n = steps < first ? steps : first;
        if (n > 0)
            First::skip(n);
        first -= n;
        chunk += (steps - n) * 8;
    }
    __device__ __forceinline__ void begin(bool live) {
        if (first > 0) {
            First::begin(live);
            return;
        }
        const int lane = lane_of_step<T>(), wave = threadIdx.x >> 6;
        First::range = buffer_of(base2, live ? size2 : 0);
        First::bytes = kStepBytes;  // every chunk of the step is looked up
        if constexpr (Index::kSkips) {
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const int row = First::load_number(wave, q) * 8 + lane / 8;
                const int32_t c = chunk + First::swizzle(row, lane % 8);
                uint32_t o = kNowhere;
                if (live && c < most) {
                    const uint32_t at = side->chunks.div((uint32_t)c), in = (uint32_t)c - at * side->chunks.d;
                    const Segment s = segments[at];
                    if (row >= (s[1] & 0xffff) && row < s[1] >> 16)
                        o = (uint32_t)(row * side->width + side->value_at((int32_t)in * 8)) * 2;
                }
                First::offset[q] = o;
            }
            return;
        }
        // A lane's rows are of two kinds, by which chunk they bring: rows of even and of odd load numbers.
        bool has[2];
        Segment of[2];
        uint32_t place[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t c = chunk + First::swizzle(h * 8 + lane / 8, lane % 8);
            has[h] = live && c < most;
            const uint32_t at = has[h] ? side->chunks.div((uint32_t)c) : 0;
            of[h] = segments[at];
            place[h] = ((uint32_t)c - at * side->chunks.d) * 8;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            place[h] = (LOW ? (uint32_t)side->value_at((int32_t)place[h])
                            : (uint32_t)of[h][0] * adapter_rows * (uint32_t)side->R + (uint32_t)side->rank_of((int32_t)place[h])) *
                       2;
        const uint32_t row_bytes = (uint32_t)(LOW ? side->width : side->R) * 2;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int number = First::load_number(wave, q), row = number * 8 + lane / 8;
            const bool odd = number & 1;
            const int32_t rows = odd ? of[1][1] : of[0][1];
            bool here = odd ? has[1] : has[0];
            int32_t n = row;
            if constexpr (LOW) {
                here = here && row >= (rows & 0xffff) && row < rows >> 16;
            } else {
                n = index(row);
                here = here && n >= 0;
            }
            First::offset[q] = here ? (uint32_t)n * row_bytes + (odd ? place[1] : place[0]) : kNowhere;
        }
    }
    __device__ __forceinline__ void end() {
        if (first > 0) {
            First::end();
            --first;
        } else {
            chunk += 8;
        }
    }
};

// Rows across the contraction (AcrossC), then the second part: the rows of a, [A][R][K].
template <int T, int W, int FRAGMENTS>
struct ChainAcross : AcrossC<T, W, FRAGMENTS> {
    typedef AcrossC<T, W, FRAGMENTS> First;
    using First::kLoads;
    static constexpr bool kChained = true;
    int32_t first;        // steps of the first part left
    int32_t place, most;  // places of the second part: the next step's first, and all
    const Segment EP_LDS *segments;
    const AdapterSide *side;
    uint32_t size2, column;  // column: the tile's first

    __device__ __forceinline__ void chain(int32_t steps, const AdapterSide &s, const Segment EP_LDS *at, int count, uint64_t size,
                                          int32_t index0) {
        first = steps;
        place = 0;
        most = count * (int32_t)s.places.d;
        segments = at;
        side = &s;
        size2 = (uint32_t)size;
        column = (uint32_t)index0;
    }
    __device__ __forceinline__ void skip(int32_t steps) {
        const int32_t n = steps < first ? steps : first;
        if (n > 0)
            First::skip(n);
        first -= n;
        place += (steps - n) * kStepRows;
    }
    __device__ __forceinline__ void begin(bool live) {
        if (first > 0) {
            First::begin(live);
            return;
        }
        const int lane = lane_of_step<T>(), wave = threadIdx.x >> 6;
        First::range = buffer_of(reinterpret_cast<const char *>(side->weights), live ? size2 : 0);
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int row = First::row_of(q, wave, lane);
            const int32_t p = place + row;
            uint32_t o = kNowhere;
            if (live && p < most) {
                const uint32_t at = side->places.div((uint32_t)p);
                const uint32_t rank = (uint32_t)side->rank_of((int32_t)((uint32_t)p - at * side->places.d));
                o = ((uint32_t)segments[at][0] * (uint32_t)side->R + rank) * (uint32_t)First::stride +
                    First::column_of(q, column, wave, lane);
            }
            First::offset[q] = o;
        }
    }
    __device__ __forceinline__ void end() {
        if (first > 0) {
            First::end();
            --first;
        } else {
            place += kStepRows;
        }
    }
};

// ---- results that are NaN ------------------------------------------------------------
// A tile adds zeros times the weights of the other adapters in it, which is NaN where those are
// infinite or NaN.  Where results come out NaN and another adapter of the tile has such weights, they are summed again
// of their own terms alone, one after the other.  (That is slow, so rows that are NaN by themselves, as a padded
// batch may have them, are not: with 4096 such rows among 8192 of 4096 x 4096 the product took 36 ms, now 266 us.)
__device__ __forceinline__ bool any_nan(const float *v, int n) {
    float s = 0.f;
    for (int i = 0; i < n; ++i)
        s += v[i];
    return s != s;
}
// Whether one of eight bf16 values is infinite or NaN.
__device__ __forceinline__ bool any_not_finite(u32x4 v) {
    bool any = false;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        any = any || (v[q] & 0x7f80u) == 0x7f80u || (v[q] & 0x7f800000u) == 0x7f800000u;
    return any;
}
// The last adapter that begins at place i of the order or before, else the first.
__device__ __forceinline__ int32_t last_before(const AdapterSide &s, int64_t rows, int64_t i) {
    int32_t a = 0, hi = s.A;
    while (hi - a > 1) {
        const int32_t mid = (a + hi) / 2;
        if (clamp_row(s.offsets[mid], rows) <= i)
            a = mid;
        else
            hi = mid;
    }
    return a;
}
// Whether an adapter with rows among places i0 .. i0 + n - 1, but not e, is broken(a).
template <typename F>
__device__ __forceinline__ bool others_broken(const AdapterSide &s, int64_t rows, int64_t i0, int n, int32_t e, F broken) {
    if (!s.offsets)
        return false;
#pragma unroll 1
    for (int32_t a = last_before(s, rows, i0); a < s.A; ++a) {
        const int64_t begin = clamp_row(s.offsets[a], rows), end = clamp_row(s.offsets[a + 1], rows);
        if (begin >= i0 + n)
            break;
        if (a != e && end > begin && end > i0 && broken(a))
            return true;
    }
    return false;
}
// The adapter that row i of the order has, -1: none.
__device__ __forceinline__ int32_t adapter_of(const AdapterSide &s, int64_t rows, int64_t i) {
    if (!s.offsets)
        return 0;
    const int32_t a = last_before(s, rows, i);
    return i >= clamp_row(s.offsets[a], rows) && i < clamp_row(s.offsets[a + 1], rows) ? a : -1;
}

}  // namespace ep
