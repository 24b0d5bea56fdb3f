// layer.h -- declarations and device helpers shared by the layer operators (norm, router,
// experts' product, combine gradient).
#pragma once

#include "ep_internal.h"

#include <algorithm>
#include <cmath>
#include <utility>

namespace ep {

// ---- device helpers ---------------------------------------------------------------
__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
// Two floats rounded to nearest-even bf16 (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, b2));
}
__device__ __forceinline__ void unpack8(u32x4 v, float *f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo(v[i]);
        f[2 * i + 1] = bf16_hi(v[i]);
    }
}
__device__ __forceinline__ u32x4 pack8(const float *f) {
    return u32x4{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7])};
}

// Wave reductions by DPP (row shifts, then the two row broadcasts); every lane gets the result.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float(dpp_or_zero<CTRL, ROWS>(__float_as_uint(v)));
}
__device__ __forceinline__ float wave_sum(float v) {
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    v = dpp_add<0x143, 0xc>(v);
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = dpp_or_zero<CTRL, ROWS>(v);
    return o > v ? o : v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = dpp_max<0x111, 0xf>(v);
    v = dpp_max<0x112, 0xf>(v);
    v = dpp_max<0x114, 0xf>(v);
    v = dpp_max<0x118, 0xf>(v);
    v = dpp_max<0x142, 0xa>(v);
    v = dpp_max<0x143, 0xc>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Sum over rows [begin, end) of column h of an fp32 matrix, in a fixed order: workgroups of
// 1024 threads, 32 neighbouring columns (h = base + threadIdx.x % 32) by 32 rows at a time.
// The sum is valid in the first 32 threads.
__device__ __forceinline__ float column_sum(const float *matrix, int64_t begin, int64_t end, int64_t width, int64_t h) {
    __shared__ float part[32][33];
    const int c = threadIdx.x & 31, lane = threadIdx.x >> 5;
    float s = 0.f;
    if (h < width) {
        constexpr int kAhead = 8;
        for (int64_t r = begin + lane; r < end; r += 32 * kAhead) {
            float v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                v[i] = r + i * 32 < end ? matrix[(r + i * 32) * width + h] : 0.f;
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                s += v[i];
        }
    }
    part[lane][c] = s;
    __syncthreads();
    if (lane == 0) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i)
            s += part[i][c];
    }
    return s;
}

// exp by the hardware's base-2 exponential: z log2(e) is rounded once, and the constant in fp32 is 0.22
// 2^-24 off, so the result is within (1.25 |z| + 2) 2^-24 of itself.
__device__ __forceinline__ float quick_exp(float z) { return __builtin_amdgcn_exp2f(z * 1.44269504f); }

// ---- launches ---------------------------------------------------------------------
// One kernel launch, timed under `name` while tracing is on.  A grid of 2^32 threads or more
// along x is an error (the hardware counts them in 32 bits).
template <typename K, typename... A>
hipError_t launch_traced(const char *name, K kernel, dim3 grid, int threads, hipStream_t stream, A &&...args) {
    if ((uint64_t)grid.x * (uint64_t)threads > 0xffffffffull)
        return hipErrorInvalidConfiguration;
    (void)hipGetLastError();
    TraceSlot ts = trace_acquire();
    hipExtLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, ts.start, ts.stop, 0, std::forward<A>(args)...);
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess)
        trace_submit(name, ts);
    return err;
}

// Compute units; the kernels that loop over their work size their grids by it.
constexpr int64_t kCus = 256;

struct NormArgs {
    const u32x4 *x, *residual, *weight;  // residual, weight may be null
    u32x4 *total, *out;                  // may be null
    uint8_t *rows8;                      // may be null
    int64_t T;
    int32_t H;
    float eps;
};
hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t stream);

struct NormGradArgs {
    const u32x4 *total, *weight, *d_out, *d_total;  // weight, d_total may be null
    u32x4 *dx;
    float *d_weight;  // may be null
    float *partial;   // [rmsnorm_grad_groups][H], with d_weight
    int64_t T;
    int32_t H;
    float eps;
};
int64_t rmsnorm_grad_groups(int64_t T, int32_t H);
hipError_t launch_rmsnorm_grad(const NormGradArgs &a, hipStream_t stream);

struct RouteArgs {
    const void *logits;
    bool bf16;
    const uint8_t *mask;  // may be null
    int64_t T;
    int32_t E, k;
    bool normalize;
    float balance;
    int32_t *topk_idx;
    float *topk_w;
    int32_t *counts;  // null: no counts, sums and loss
    float *prob_sums, *loss;
    void *workspace;  // of route_workspace_bytes; per group: int32 counts, fp32 sums, E rounded up to 4 of each
};
size_t route_workspace_bytes(int64_t T, int32_t E);
hipError_t launch_route(const RouteArgs &a, hipStream_t stream);

struct RouteGradArgs {
    const void *logits;
    bool bf16;
    const uint8_t *mask;
    const int32_t *topk_idx, *counts;
    const float *d_topk_w, *d_loss;  // may be null
    int64_t T;
    int32_t E, k;
    bool normalize;
    float balance;
    void *d_logits;
};
hipError_t launch_route_grad(const RouteGradArgs &a, hipStream_t stream);

hipError_t launch_combine_grad(const void *d_out, const void *y, int64_t max_rows, const int32_t *slot_pos,
                               const float *topk_w, int64_t T, int32_t H, int32_t k, void *dy, float *d_topk_w,
                               hipStream_t stream);

struct ProductArgs {
    const void *x;
    bool bits8;
    int64_t rows;
    const int32_t *offsets;  // null: one expert with every row
    int32_t E;
    const void *w;
    const float *w_scale;
    int32_t K, N, Nw;
    const void *bias;
    int32_t act;
    const void *residual;
    void *pre, *y;
    bool f32;
    float *partial;  // workspace of product_workspace_bytes
};
size_t product_workspace_bytes(int64_t rows, int32_t E, int32_t K, int32_t N, bool bits8, int32_t act);
hipError_t launch_product(const ProductArgs &a, hipStream_t stream);

struct ProductGradArgs {
    const void *x;
    int64_t rows;
    const int32_t *offsets;
    int32_t E;
    const void *w;
    int32_t K, N, Nw;
    int32_t act;
    const void *pre, *d_y;
    void *dx, *dw;
    float *dbias;
    void *workspace;  // of product_grad_workspace_bytes
};
size_t product_grad_workspace_bytes(int64_t rows, int32_t E, int32_t K, int32_t N, int32_t act, bool dx, bool dw, bool bias);
hipError_t launch_product_grad(const ProductGradArgs &a, hipStream_t stream);

}  // namespace ep
