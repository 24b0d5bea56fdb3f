// adapter_tile.h -- operands of the MFMA tile (product_tile.h) whose contraction goes on into a second
// part: the low-rank terms of the adapters whose rows a tile holds.
//
// Rows are taken in the adapters' order (row i of the order is row order[i] of x and y), so the rows
// that an adapter has in a tile are a segment of it.  The second part is as long as the segments'
// ranks together: its places are (segment, rank), rank fastest.  The row operand holds zeros at the
// places of the segments that a row is not in, and the column operand the weights of the place's
// adapter, so one accumulator adds up both parts; 64 places are one step whoever's they are: four
// adapters of rank 16 cost what one of rank 64 costs.  (A step per adapter would take 64 steps
// more for 64 rows with an adapter each; of rank 16 it is 16.)
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
    const uint16_t *low;     // [rows][R], in the adapters' order
    const uint16_t *weights; // b [A][Nw][R] of the product, a [A][R][K] of its gradient
    FastDiv places, chunks;  // by R and R / 8
};

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

// Rows along the contraction (AlongC), then the second part: LOW: the rows' low-rank values, else the
// weights b of each column.
template <int T, int W, bool LOW>
struct ChainAlong : AlongC<T, W> {
    typedef AlongC<T, W> First;
    using First::kLoads;
    int32_t first;        // steps of the first part left
    int32_t chunk, most;  // 16-byte chunks of the second part: the next step's first, and all
    const Segment EP_LDS *segments;
    FastDiv per;          // chunks of a segment
    const char *base2;
    uint32_t size2;
    uint32_t row_bytes;   // of a row of the second part
    uint32_t adapter_bytes;
    uint32_t now[kLoads];
    int32_t index[kLoads];  // LOW: the tile's row; else the weights' row, -1: none

    template <typename F>
    __device__ __forceinline__ void chain(int32_t steps, const AdapterSide &s, const Segment EP_LDS *at, int count, const void *base,
                                          uint64_t size, int64_t adapter_rows, int wave, int lane, F index_of) {
        first = steps;
        chunk = 0;
        most = count * (s.R / 8);
        segments = at;
        per = s.chunks;
        base2 = static_cast<const char *>(base);
        size2 = (uint32_t)size;
        row_bytes = (uint32_t)s.R * 2;
        adapter_bytes = (uint32_t)(adapter_rows * row_bytes);
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            index[q] = index_of(First::load_number(wave, q) * 8 + lane / 8);
    }
    __device__ __forceinline__ void skip(int32_t steps) {
        const int32_t n = steps < first ? steps : first;
        if (n > 0)
            First::skip(n);
        first -= n;
        chunk += (steps - n) * 8;
    }
    __device__ __forceinline__ void begin(bool live) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (first > 0) {
            First::begin(live);
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const int row = First::load_number(wave, q) * 8 + lane / 8;
                now[q] = First::swizzle(row, lane % 8) * 16 < First::bytes ? First::offset[q] : kNowhere;
            }
            return;
        }
        First::range = buffer_of(base2, live ? size2 : 0);
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int row = First::load_number(wave, q) * 8 + lane / 8;
            const int32_t c = chunk + First::swizzle(row, lane % 8);
            now[q] = kNowhere;
            if (live && c < most) {
                const uint32_t at = per.div((uint32_t)c), in = (uint32_t)c - at * per.d;
                const Segment s = segments[at];
                if (LOW ? index[q] >= (s[1] & 0xffff) && index[q] < s[1] >> 16 : index[q] >= 0)
                    now[q] = (LOW ? 0u : (uint32_t)s[0] * adapter_bytes) + (uint32_t)index[q] * row_bytes + in * 16;
            }
        }
    }
    __device__ __forceinline__ void load(int q, char EP_LDS *lds, int wave, int) {
        load_to_lds(First::range, now[q], lds + First::load_number(wave, q) * 1024);
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
    int32_t first;        // steps of the first part left
    int32_t place, most;  // places of the second part: the next step's first, and all
    const Segment EP_LDS *segments;
    FastDiv per;          // places of a segment
    const char *base2;
    uint32_t size2;
    uint32_t now[kLoads];

    __device__ __forceinline__ void chain(int32_t steps, const AdapterSide &s, const Segment EP_LDS *at, int count, uint64_t size) {
        first = steps;
        place = 0;
        most = count * s.R;
        segments = at;
        per = s.places;
        base2 = reinterpret_cast<const char *>(s.weights);
        size2 = (uint32_t)size;
    }
    __device__ __forceinline__ void begin(bool live) {
        if (first > 0) {
            First::begin(live);
#pragma unroll
            for (int q = 0; q < kLoads; ++q)
                now[q] = First::offset[q];
            return;
        }
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        First::range = buffer_of(base2, live ? size2 : 0);
        const uint32_t row_bytes = (uint32_t)First::stride;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int row = (First::load_number(wave, q) * 1024 + lane * 16) / (2 * T);
            const int32_t p = place + row;
            now[q] = kNowhere;
            if (live && p < most) {
                const uint32_t at = per.div((uint32_t)p), in = (uint32_t)p - at * per.d;
                now[q] = ((uint32_t)segments[at][0] * per.d + in) * row_bytes + (First::offset[q] - (uint32_t)row * row_bytes);
            }
        }
    }
    __device__ __forceinline__ void load(int q, char EP_LDS *lds, int wave, int) {
        load_to_lds(First::range, now[q], lds + First::load_number(wave, q) * 1024);
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
// infinite or NaN.  Results that come out NaN are therefore summed again of their own terms alone,
// one after the other: slow, for broken weights and for rows that are NaN anyway.
__device__ __forceinline__ bool any_nan(const float *v, int n) {
    float s = 0.f;
    for (int i = 0; i < n; ++i)
        s += v[i];
    return s != s;
}
// The adapter that row i of the order has, -1: none.
__device__ __forceinline__ int32_t adapter_of(const AdapterSide &s, int64_t rows, int64_t i) {
    if (!s.offsets)
        return 0;
    int32_t a = 0, hi = s.A;
    while (hi - a > 1) {
        const int32_t mid = (a + hi) / 2;
        if (clamp_row(s.offsets[mid], rows) <= i)
            a = mid;
        else
            hi = mid;
    }
    return i >= clamp_row(s.offsets[a], rows) && i < clamp_row(s.offsets[a + 1], rows) ? a : -1;
}

}  // namespace ep
