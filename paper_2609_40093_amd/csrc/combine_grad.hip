// combine_grad.hip -- gradient of the gate-weighted combine out[t] = sum_j w[t,j] y[p(t,j)]:
//   dy[p(t,j)] = w[t,j] d_out[t],  d_w[t,j] = <d_out[t], y[p(t,j)]>.
// HBM-bound: reads every row of y and of d_out once, writes every row of dy (8192 tokens, top-8,
// rows of 2048: 571 MB in 103 us, 5.5 TB/s).  One wave per slot; the k waves of a token are
// neighbours, so that d_out's row comes from HBM once and from L2 after that.  The dot product is
// summed in fp32 per lane and then over the wave.
#include "layer.h"

namespace ep {
namespace {

template <bool DY, bool DW>
__global__ __launch_bounds__(256) void combine_grad_kernel(const u32x4 *d_out, const u32x4 *y, int64_t max_rows,
                                                           const int32_t *slot_pos, const float *topk_w,
                                                           uint32_t slots, FastDiv k_div, int32_t vecs, u32x4 *dy,
                                                           float *d_w) {
    const int lane = threadIdx.x & 63;
    const uint32_t first = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    for (int64_t s = first; s < slots; s += (int64_t)gridDim.x * 4) {
        const uint32_t slot = (uint32_t)s;
        const int64_t pos = slot_pos[slot];
        if (pos < 0 || pos >= max_rows) {
            if (DW && lane == 0)
                d_w[slot] = 0.f;
            continue;
        }
        const u32x4 *d = d_out + (int64_t)k_div.div(slot) * vecs;
        const u32x4 *yr = y + pos * vecs;
        u32x4 *o = dy + pos * vecs;
        const float w = topk_w[slot];
        float dot = 0.f;
        constexpr int kUnroll = 4;
        for (int i0 = lane; i0 < vecs; i0 += 64 * kUnroll) {
            u32x4 dv[kUnroll], yv[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = i0 + u * 64;
                dv[u] = yv[u] = u32x4{0, 0, 0, 0};
                if (i < vecs) {
                    dv[u] = d[i];
                    if (DW)
                        yv[u] = __builtin_nontemporal_load(yr + i);
                }
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = i0 + u * 64;
                float f[8], g[8];
                unpack8(dv[u], f);
                if (DW) {
                    unpack8(yv[u], g);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        dot = fmaf(f[q], g[q], dot);
                }
                if (DY) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        f[q] *= w;
                    if (i < vecs)
                        __builtin_nontemporal_store(pack8(f), o + i);
                }
            }
        }
        if (DW) {
            dot = wave_sum(dot);
            if (lane == 0)
                d_w[slot] = dot;
        }
    }
}

}  // namespace

hipError_t launch_combine_grad(const void *d_out, const void *y, int64_t max_rows, const int32_t *slot_pos,
                               const float *topk_w, int64_t T, int32_t H, int32_t k, void *dy, float *d_topk_w,
                               hipStream_t stream) {
    const int64_t slots = T * k;
    if (slots == 0 || (!dy && !d_topk_w))
        return hipSuccess;
    const dim3 grid((unsigned)std::min<int64_t>((slots + 3) / 4, 1 << 23));
#define EP_CALL(DY, DW)                                                                                           \
    launch_traced("combine_grad", combine_grad_kernel<DY, DW>, grid, 256, stream, (const u32x4 *)d_out,          \
                  (const u32x4 *)y, max_rows, slot_pos, topk_w, (uint32_t)slots, fast_div((uint32_t)k), H / 8, (u32x4 *)dy, \
                  d_topk_w)
    return dy && d_topk_w ? EP_CALL(true, true) : dy ? EP_CALL(true, false) : EP_CALL(false, true);
#undef EP_CALL
}

}  // namespace ep
