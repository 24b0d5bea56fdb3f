// norm.hip -- RMS norm of the residual stream, forward and backward.
//
//   forward   s = x + r;  y = s * rstd * w,  rstd = 1 / sqrt(mean(s^2) + eps)
//   backward  g = d_out * w;  n = s * rstd;  dx = rstd * (g - n mean(g n)) + d_total;
//             d_weight = sum over tokens of d_out * n
//   with dropout of x (dropout.h)  s = drop(x) + r, and x's gradient is drop(dx)
//
// Both are HBM-bound: every row is read once and held in registers between its reduction and
// its results.  The forward reduces sum(s^2) and max|s w| in the same step: the row's largest
// |y| is max|s w| rstd, so the 8-bit rows need no second reduction; the backward likewise reduces
// sum(s^2) and sum(g s) together.  Only rows whose sums leave fp32 are reduced again.  32768 rows of
// 7168 with a residual, the sum, bf16 and 8-bit rows: 2.1 GB in 376 us, 5.6 TB/s; the gradient of
// 5003 rows of 2888: 116 MB in 27 us, 4.3 TB/s; 256 rows of 7168 into 8-bit rows: 5 us, of which 2 are
// bytes.  With dropout the same forward takes 380 us, and the gradient of 32768 rows of 7168, with d_total, 2.35 GB,
// 453 us, 5.2 TB/s (with a row's mask made while its loads are on their way 457).
#include "dropout.h"

namespace ep {
namespace {

constexpr float kLeastMax = 0x1p-100f;  // a row's max|y| counts as at least this: its scale stays normal
constexpr float kF8Max = 448.f;

// Row geometry: WAVES waves hold one row, V vectors of 8 elements per lane; workgroups of
// 256 threads hold 4 / WAVES rows for WAVES < 4.
template <int WAVES>
constexpr int block_threads() {
    return WAVES < 4 ? 256 : WAVES * 64;
}

// 1 / sqrt(mean(s^2) + eps) of a row from ss = sum(s^2), as the factors of s f r: f a power of two.
// Where the squares leave fp32's range (values above 2^52, or below 2^-40 with next to no eps), the
// row's sum is taken again of its values times f, which puts every row of finite values within the
// range: the values of the first kind, below 2^128, come to less than 2^32, and those of the second,
// bf16's subnormals among them, to 2^-37 .. 2^56.  `again(f)` gives sum((f s)^2) over the row.  r alone
// stays a normal number, where f r need not.  The condition is the same in every lane of a row; f is 1
// in rows of ordinary values.
struct InverseRms {
    float f, r;
};
template <typename F>
__device__ __forceinline__ InverseRms inverse_rms(float ss, int H, float eps, F again) {
    const bool large = ss > 0x1p120f, small = ss < 0x1p-80f && eps < 0x1p-80f;
    if (__builtin_expect(large || small, false)) {
        const float f = large ? 0x1p-96f : 0x1p96f;
        return {f, 1.f / sqrtf(again(f) / (float)H + eps * f * f)};
    }
    return {1.f, 1.f / sqrtf(ss / (float)H + eps)};
}

// Sum over the waves of a row; every wave of the workgroup calls it.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float *slot, int tid) {
    v = wave_sum(v);
    if (WAVES > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            slot[tid / 64] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i)
            v += slot[i];
    }
    return v;
}

// The same of the largest.
template <int WAVES>
__device__ __forceinline__ uint32_t row_max(uint32_t v, float *slot, int tid) {
    v = wave_max(v);
    if (WAVES > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
            slot[tid / 64] = __uint_as_float(v);
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const uint32_t m = __float_as_uint(slot[i]);
            v = m > v ? m : v;
        }
    }
    return v;
}

template <typename T>
__device__ __forceinline__ T load_row(const T *p, bool nt) {
    return nt ? __builtin_nontemporal_load(p) : *p;
}
template <typename T>
__device__ __forceinline__ void store_row(T v, T *p, bool nt) {
    if (nt)
        __builtin_nontemporal_store(v, p);
    else
        *p = v;
}

template <int WAVES, int V, bool NT, bool DROP>
__global__ __launch_bounds__(block_threads<WAVES>()) void rmsnorm_kernel(NormArgs a) {
    constexpr int kRows = block_threads<WAVES>() / (WAVES * 64);
    const int tid = (int)threadIdx.x % (WAVES * 64), sub = (int)threadIdx.x / (WAVES * 64);
    const int vecs = a.H / 8;
    __shared__ float red[2][WAVES][2], redo[WAVES];
    u32x4 wv[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = v * (WAVES * 64) + tid;
        wv[v] = u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        if (a.weight && i < vecs)
            wv[v] = a.weight[i];
    }
    DropKey key;
    if (DROP)
        key.load(a.drop);
    int parity = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + sub; row < a.T; row += (int64_t)gridDim.x * kRows) {
        const int64_t base = row * vecs;
        float s[V][8];
        float ss = 0.f;
        uint32_t top = 0;  // bits of max|s w|: a NaN's are above every number's
        u32x4 xv[V], rv[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = v * (WAVES * 64) + tid;
            xv[v] = rv[v] = u32x4{0, 0, 0, 0};
            if (i < vecs) {
                xv[v] = load_row(a.x + base + i, NT);
                if (a.residual)
                    rv[v] = load_row(a.residual + base + i, NT);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            unpack8(xv[v], s[v]);
            if (DROP)
                drop8(key, (uint64_t)(base + v * (WAVES * 64) + tid), a.drop.cut, a.drop.factor, s[v]);
            if (a.residual) {
                float r[8];
                unpack8(rv[v], r);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    s[v][q] += r[q];
            }
            float w[8];
            unpack8(wv[v], w);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                ss = fmaf(s[v][q], s[v][q], ss);
                const uint32_t m = __float_as_uint(s[v][q] * w[q]) & 0x7fffffffu;
                top = m > top ? m : top;
            }
        }
        ss = wave_sum(ss);
        top = wave_max(top);
        if (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
                red[parity][tid / 64][0] = ss;
                red[parity][tid / 64][1] = __uint_as_float(top);
            }
            __syncthreads();
            ss = 0.f;
            top = 0;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                ss += red[parity][i][0];
                const uint32_t m = __float_as_uint(red[parity][i][1]);
                top = m > top ? m : top;
            }
            parity ^= 1;  // the next row writes the other half: one barrier per row
        }
        const InverseRms rms = inverse_rms(ss, a.H, a.eps, [&](float f) {
            float q2 = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    q2 = fmaf(s[v][q] * f, s[v][q] * f, q2);
            return row_sum<WAVES>(q2, redo, tid);
        });
        float most = __uint_as_float(top) * rms.r;
        // The largest |y| itself where s w may have left fp32 and y not.  (A product below fp32's normal
        // numbers lacks digits, which counts where 1 / rms brings it above kLeastMax.)
        if (__builtin_expect(a.rows8 && (rms.f != 1.f || top == 0x7f800000u || (top < 0x00800000u && rms.r > 0x1p26f)), false)) {
            top = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float w[8];
                unpack8(wv[v], w);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const uint32_t m = __float_as_uint(s[v][q] * rms.f * rms.r * w[q]) & 0x7fffffffu;
                    top = m > top ? m : top;
                }
            }
            most = __uint_as_float(row_max<WAVES>(top, redo, tid));
        }
        const float scale = (most < kLeastMax ? kLeastMax : most) / kF8Max;  // a NaN stays one
        const float inv = 1.f / scale;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = v * (WAVES * 64) + tid;
            if (i >= vecs)
                continue;
            if (a.total)
                store_row(pack8(s[v]), a.total + base + i, NT);
            float w[8], y[8];
            unpack8(wv[v], w);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                y[q] = s[v][q] * rms.f * rms.r * w[q];
            if (a.out)
                store_row(pack8(y), a.out + base + i, NT);
            if (a.rows8) {
                uint32_t b[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h] * inv, y[4 * h + 1] * inv, 0, false);
                    b[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2] * inv, y[4 * h + 3] * inv, p, true);
                }
                uint8_t *dst = a.rows8 + row * (a.H + 16);
                store_row((uint64_t)b[1] << 32 | b[0], reinterpret_cast<uint64_t *>(dst) + i, NT);
            }
        }
        if (a.rows8 && tid == 0)
            *reinterpret_cast<u32x4 *>(a.rows8 + row * (a.H + 16) + a.H) = u32x4{__float_as_uint(scale), 0, 0, 0};
    }
}

// The rows of a workgroup follow each other, with few workgroups, so that the partial weight
// gradients stay few.  The next row is on its way while one is reduced where a lane has two
// vectors of it (5003 rows of 2888: 28.9 / 27.5 us); with four, the registers this takes cost more than it gives
// (20000 rows of 7168: 196 / 215 us).
template <int WAVES, int V, bool NT, bool DROP>
__global__ __launch_bounds__(block_threads<WAVES>()) void rmsnorm_grad_kernel(NormGradArgs a) {
    constexpr int kRows = block_threads<WAVES>() / (WAVES * 64);
    const int tid = (int)threadIdx.x % (WAVES * 64), sub = (int)threadIdx.x / (WAVES * 64);
    const int vecs = a.H / 8;
    __shared__ float red[2][WAVES][2], redo[WAVES];
    u32x4 wv[V];
    float dw[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = v * (WAVES * 64) + tid;
        wv[v] = u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        if (a.weight && i < vecs)
            wv[v] = a.weight[i];
#pragma unroll
        for (int q = 0; q < 8; ++q)
            dw[v][q] = 0.f;
    }
    DropKey key;
    if (DROP)
        key.load(a.drop);
    int parity = 0;
    const int64_t stride = (int64_t)gridDim.x * kRows;
    u32x4 sn[V], dn[V], tn[V];
    const auto load = [&](int64_t row) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = v * (WAVES * 64) + tid;
            sn[v] = dn[v] = tn[v] = u32x4{0, 0, 0, 0};
            if (row < a.T && i < vecs) {
                sn[v] = load_row(a.total + row * vecs + i, NT);
                dn[v] = load_row(a.d_out + row * vecs + i, NT);
                if (a.d_total)
                    tn[v] = load_row(a.d_total + row * vecs + i, NT);
            }
        }
    };
    constexpr bool kNextRow = V <= 2 && WAVES <= 4;
    int64_t row = (int64_t)blockIdx.x * kRows + sub;
    if (kNextRow)
        load(row);
    for (; row < a.T; row += stride) {
        const int64_t base = row * vecs;
        u32x4 sv[V], dv[V], tv[V];
        if (!kNextRow)
            load(row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            sv[v] = sn[v];
            dv[v] = dn[v];
            tv[v] = tn[v];
        }
        if (kNextRow)
            load(row + stride);
        float ss = 0.f, gs = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float s[8], d[8], w[8];
            unpack8(sv[v], s);
            unpack8(dv[v], d);
            unpack8(wv[v], w);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                ss = fmaf(s[q], s[q], ss);
                gs = fmaf(d[q] * w[q], s[q], gs);
            }
        }
        ss = wave_sum(ss);
        gs = wave_sum(gs);
        if (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
                red[parity][tid / 64][0] = ss;
                red[parity][tid / 64][1] = gs;
            }
            __syncthreads();
            ss = gs = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                ss += red[parity][i][0];
                gs += red[parity][i][1];
            }
            parity ^= 1;
        }
        const InverseRms rms = inverse_rms(ss, a.H, a.eps, [&](float f) {
            float q2 = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s[8];
                unpack8(sv[v], s);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    q2 = fmaf(s[q] * f, s[q] * f, q2);
            }
            return row_sum<WAVES>(q2, redo, tid);
        });
        // sum(g n); from its own terms where those of sum(g s) may have left fp32 (what they lose below its
        // normal numbers counts where 1 / rms is large)
        float gn = gs * rms.r;
        if (__builtin_expect(rms.f != 1.f || !(fabsf(gs) < INFINITY) || (fabsf(gs) < 0x1p-100f && rms.r > 16.f), false)) {
            gn = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s[8], d[8], w[8];
                unpack8(sv[v], s);
                unpack8(dv[v], d);
                unpack8(wv[v], w);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    gn = fmaf(d[q] * w[q], s[q] * rms.f * rms.r, gn);
            }
            gn = row_sum<WAVES>(gn, redo, tid);
        }
        const float c = gn / (float)a.H;  // mean(g n)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = v * (WAVES * 64) + tid;
            if (i >= vecs)
                continue;
            float s[8], d[8], w[8], t[8];
            unpack8(sv[v], s);
            unpack8(dv[v], d);
            unpack8(wv[v], w);
            unpack8(tv[v], t);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float n = s[q] * rms.f * rms.r;
                dw[v][q] = fmaf(d[q], n, dw[v][q]);
                t[q] = fmaf(rms.r, (d[q] * w[q] - n * c) * rms.f, t[q]);
            }
            if (!DROP) {
                store_row(pack8(t), a.dx + base + i, NT);
                continue;
            }
            if (a.d_residual)
                store_row(pack8(t), a.d_residual + base + i, NT);
            if (a.dx) {
                drop8(key, (uint64_t)(base + i), a.drop.cut, a.drop.factor, t);
                store_row(pack8(t), a.dx + base + i, NT);
            }
        }
    }
    if (!a.d_weight)
        return;
    // one partial row per workgroup, added up in a fixed order
    float *dst = a.partial + (int64_t)blockIdx.x * a.H;
    if constexpr (kRows > 1) {
        __shared__ float fold[kRows][V * 64 * 8];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < 8; ++q)
                fold[sub][(v * 64 + tid) * 8 + q] = dw[v][q];
        __syncthreads();
        for (int h = threadIdx.x; h < a.H; h += block_threads<WAVES>())
            dst[h] = (fold[0][h] + fold[1][h]) + (fold[2][h] + fold[3][h]);
        return;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int i = v * (WAVES * 64) + tid;
        if (i < vecs) {
            reinterpret_cast<float4 *>(dst)[2 * i] = float4{dw[v][0], dw[v][1], dw[v][2], dw[v][3]};
            reinterpret_cast<float4 *>(dst)[2 * i + 1] = float4{dw[v][4], dw[v][5], dw[v][6], dw[v][7]};
        }
    }
}

// d_weight[h] = sum over the partial rows.
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float *partial, int64_t rows, int32_t H, float *out) {
    const int64_t h = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const float s = column_sum(partial, 0, rows, H, h);
    if (threadIdx.x < 32 && h < H)
        out[h] = s;
}

// Waves of a row and vectors per lane.
struct RowGeom {
    int waves, vecs;
};
RowGeom row_geometry(int32_t H) {
    if (H <= 2048)
        return {1, H <= 512 ? 1 : H <= 1024 ? 2 : 4};
    if (H <= 8192)
        return {4, H <= 4096 ? 2 : 4};
    return {16, H <= 16384 ? 2 : H <= 32768 ? 4 : 8};
}

#define EP_ROW_GEOMETRY(g, CALL)                                      \
    do {                                                              \
        if (g.waves == 1)                                             \
            return g.vecs == 1 ? CALL(1, 1) : g.vecs == 2 ? CALL(1, 2) : CALL(1, 4); \
        if (g.waves == 4)                                             \
            return g.vecs == 2 ? CALL(4, 2) : CALL(4, 4);             \
        return g.vecs == 2 ? CALL(16, 2) : g.vecs == 4 ? CALL(16, 4) : CALL(16, 8); \
    } while (0)

int64_t row_groups(int64_t T, int waves, int64_t most) {
    const int rows = waves < 4 ? 4 / waves : 1;
    return std::min<int64_t>((T + rows - 1) / rows, most);
}

hipError_t launch_grad_rows(const NormGradArgs &a, int64_t groups, hipStream_t stream) {
    const RowGeom g = row_geometry(a.H);
    const bool nt = a.T * a.H * (a.d_total ? 8 : 6) >= kNormStreamBytes, drop = a.drop.rng != nullptr;
#define EP_LAUNCH(W, V, NT, DROP)                                                                                  \
    launch_traced(DROP ? "dropout_rmsnorm_grad" : "rmsnorm_grad", rmsnorm_grad_kernel<W, V, NT, DROP>,             \
                  dim3((unsigned)groups), block_threads<W>(), stream, a)
#define EP_CALL(W, V)                                                                     \
    (drop ? (nt ? EP_LAUNCH(W, V, true, true) : EP_LAUNCH(W, V, false, true))             \
          : (nt ? EP_LAUNCH(W, V, true, false) : EP_LAUNCH(W, V, false, false)))
    EP_ROW_GEOMETRY(g, EP_CALL);
#undef EP_CALL
#undef EP_LAUNCH
}

}  // namespace

// A workgroup per row (or four short ones).  Rows past what the memory-side cache holds are
// loaded and stored non-temporally.  Measured at 32768 rows of 7168 with every output (2.1 GB), us:
// 32 workgroups per compute unit that loop over the rows 402, one per row 382, non-temporal 372; 8
// per compute unit 415.
hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t stream) {
    if (a.T == 0)
        return hipSuccess;
    const RowGeom g = row_geometry(a.H);
    const dim3 grid((unsigned)row_groups(a.T, g.waves, 1 << 21));
    const int64_t per = 2 + (a.residual ? 2 : 0) + (a.total ? 2 : 0) + (a.out ? 2 : 0) + (a.rows8 ? 1 : 0);
    const bool nt = a.T * a.H * per >= kNormStreamBytes, drop = a.drop.rng != nullptr;
#define EP_LAUNCH(W, V, NT, DROP)                                                                                    \
    launch_traced(DROP ? "dropout_rmsnorm" : "rmsnorm", rmsnorm_kernel<W, V, NT, DROP>, grid, block_threads<W>(), stream, a)
#define EP_CALL(W, V)                                                                     \
    (drop ? (nt ? EP_LAUNCH(W, V, true, true) : EP_LAUNCH(W, V, false, true))             \
          : (nt ? EP_LAUNCH(W, V, true, false) : EP_LAUNCH(W, V, false, false)))
    EP_ROW_GEOMETRY(g, EP_CALL);
#undef EP_CALL
#undef EP_LAUNCH
}

// Workgroups, and partial rows of the weight gradient.  Two per compute unit: with one, 5003 rows
// of 2888 take 37 us instead of 29, with four, 8192 rows of 2048 46 instead of 36 (their partials
// grow).
int64_t rmsnorm_grad_groups(int64_t T, int32_t H) { return row_groups(T, row_geometry(H).waves, kCus * 2); }

hipError_t launch_rmsnorm_grad(const NormGradArgs &a, hipStream_t stream) {
    const int64_t groups = a.T ? rmsnorm_grad_groups(a.T, a.H) : 0;
    if (a.T) {
        const hipError_t e = launch_grad_rows(a, groups, stream);
        if (e != hipSuccess || !a.d_weight)
            return e;
    }
    if (!a.d_weight)
        return hipSuccess;
    return launch_traced("rmsnorm_grad_weight", norm_weight_kernel, dim3((unsigned)((a.H + 31) / 32)), 1024, stream,
                         (const float *)a.partial, groups, a.H, a.d_weight);
}

}  // namespace ep
