// adapter_rows.hip -- the rows of a batch sorted by their adapter, stably: order[i] the i-th row, offsets[a]
// where adapter a's rows begin.  Rows of no adapter (an id outside [0, A)) come last.
//
// A counting sort in one workgroup of 16 waves.  Each wave takes a stretch of the rows and a counter
// per adapter of its own in LDS: it counts its rows 64 at a time (lanes of one adapter find each
// other by ballots, the first adds their number), the counters become the places where each wave's
// rows of each adapter begin, and the wave goes over its rows again.  Latency-bound, and made once for
// all the projections of a batch: 64 rows of 32 adapters take 2.9 us, 6136 of 20 take 8, 14368 of 14 take 17,
// 131072 of 64 take 147 (one workgroup, so the time goes with the rows).
#include "layer.h"
#include "wave.h"

#include "ep_layer.h"

namespace ep {
namespace {

constexpr int kWaves = 16;

template <int BITS>
__global__ __launch_bounds__(kWaves * 64) void adapter_rows_kernel(const int32_t *row_adapter, int64_t rows, int32_t A,
                                                                   int32_t *order, int32_t *offsets) {
    constexpr int kBins = 1 << BITS;
    __shared__ int32_t at[kWaves][kBins];
    __shared__ int32_t wave_total[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int i = threadIdx.x; i < kWaves * kBins; i += kWaves * 64)
        (&at[0][0])[i] = 0;
    __syncthreads();
    const int64_t per = ((rows + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int64_t begin = per * wave < rows ? per * wave : rows, end = begin + per < rows ? begin + per : rows;
    const auto id_of = [&](int64_t r) -> int32_t {
        if (r >= end)
            return A;
        const int32_t e = row_adapter[r];
        return e >= 0 && e < A ? e : A;
    };
    int32_t next = id_of(begin + lane);
    for (int64_t r = begin; r < end; r += 64) {
        const int32_t e = next;
        next = id_of(r + 64 + lane);
        const bool valid = r + lane < end;
        const uint64_t same = match_bits<BITS>(e, valid);
        if (valid && lanes_below(same) == 0)
            at[wave][e] += __builtin_popcountll(same);
    }
    __syncthreads();
    // where the rows of each wave and adapter begin: adapters first, then waves
    int32_t carry = 0;
    for (int b0 = 0; b0 <= A; b0 += kWaves * 64) {
        const int b = b0 + (int)threadIdx.x;
        int32_t n[kWaves], total = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            n[w] = b <= A ? at[w][b] : 0;
            total += n[w];
        }
        const int32_t incl = wave_inclusive_scan(total);
        if (lane == 63)
            wave_total[wave] = incl;
        __syncthreads();
        int32_t first = carry + incl - total;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave)
                first += wave_total[w];
            carry += wave_total[w];
        }
        if (b <= A) {
            offsets[b] = first;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                at[w][b] = first;
                first += n[w];
            }
        }
        __syncthreads();
    }
    next = id_of(begin + lane);
    for (int64_t r = begin; r < end; r += 64) {
        const int32_t e = next;
        next = id_of(r + 64 + lane);
        const bool valid = r + lane < end;
        const uint64_t same = match_bits<BITS>(e, valid);
        if (valid) {
            const int below = lanes_below(same);
            const int32_t first = at[wave][e];
            order[first + below] = (int32_t)(r + lane);
            if (below == 0)
                at[wave][e] = first + __builtin_popcountll(same);
        }
    }
}

}  // namespace

hipError_t launch_adapter_rows(const int32_t *row_adapter, int64_t rows, int32_t A, int32_t *order, int32_t *offsets,
                               hipStream_t stream) {
#define EP_CALL(BITS)                                                                                                  \
    launch_traced("adapter_rows", adapter_rows_kernel<BITS>, dim3(1), kWaves * 64, stream, row_adapter, rows, A, order, \
                  offsets)
    return A < 16 ? EP_CALL(4) : A < 64 ? EP_CALL(6) : A < 256 ? EP_CALL(8) : EP_CALL(11);
#undef EP_CALL
}

}  // namespace ep
