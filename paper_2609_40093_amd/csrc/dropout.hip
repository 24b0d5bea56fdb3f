// dropout.hip -- out = residual + dropout(x): eight values (16 bytes) per lane, the mask from dropout.h.
// HBM-bound: the 32-bit products of a mask hide behind the bytes.  32768 rows of 7168 into a residual: 1.4 GB in
// 219 us, 6.4 TB/s; 128 rows of 1024 3 us, which a launch and a load take.
#include "dropout.h"

namespace ep {
namespace {

constexpr int kAhead = 4;  // groups of a thread on their way at once

template <bool RESIDUAL, bool NT>
__global__ __launch_bounds__(256) void dropout_kernel(const u32x4 *x, const u32x4 *residual, int64_t groups, DropArgs d,
                                                      u32x4 *out) {
    DropKey key;
    key.load(d);
    const int64_t first = (int64_t)blockIdx.x * (256 * kAhead) + threadIdx.x;
    u32x4 xv[kAhead], rv[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int64_t i = first + u * 256;
        if (i < groups) {
            xv[u] = NT ? __builtin_nontemporal_load(x + i) : x[i];
            if (RESIDUAL)
                rv[u] = NT ? __builtin_nontemporal_load(residual + i) : residual[i];
        }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int64_t i = first + u * 256;
        if (i >= groups)
            break;
        float v[8];
        unpack8(xv[u], v);
        drop8(key, (uint64_t)i, d.cut, d.factor, v);
        if (RESIDUAL) {
            float r[8];
            unpack8(rv[u], r);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                v[q] += r[q];
        }
        const u32x4 o = pack8(v);
        if (NT)
            __builtin_nontemporal_store(o, out + i);
        else
            out[i] = o;
    }
}

}  // namespace

// A thread takes kAhead groups, those of a workgroup side by side.
hipError_t launch_dropout(const void *x, const void *residual, int64_t count, const DropArgs &d, void *out, hipStream_t stream) {
    const int64_t groups = count / 8;
    if (groups == 0)
        return hipSuccess;
    const int64_t blocks = (groups + 256 * kAhead - 1) / (256 * kAhead);
    const bool nt = count * (residual ? 6 : 4) >= kNormStreamBytes;
#define EP_CALL(R, NT)                                                                                                    \
    launch_traced("dropout", dropout_kernel<R, NT>, dim3((unsigned)blocks), 256, stream, (const u32x4 *)x,                \
                  (const u32x4 *)residual, groups, d, (u32x4 *)out)
    if (residual)
        return nt ? EP_CALL(true, true) : EP_CALL(true, false);
    return nt ? EP_CALL(false, true) : EP_CALL(false, false);
#undef EP_CALL
}

}  // namespace ep
