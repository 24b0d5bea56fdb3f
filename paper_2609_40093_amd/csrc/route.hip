// route.hip -- the router behind its logits: softmax, top-k, gates, counts per expert and the
// balance loss, forward and backward.
//
//   p = softmax(z);  ids = the k largest logits;  gates = p at the ids, or their softmax
//   loss = balance E sum_e c_e / (N k) P_e / N,  c_e = slots of e,  P_e = sum_t p_te
//   d z_i = w_i (dw_i - sum_j w_j dw_j) on the chosen (normalized gates), or the same through
//           p (gates p), plus p_i (g_i - sum_e p_e g_e), g_e = d_loss balance E c_e / (N k N)
//
// A wave holds one token, lane l the NV experts [l NV, (l + 1) NV).  The k largest are picked
// one after the other: each lane's best key, the wave's best by DPP, and the lowest lane that
// has it gives its expert up (the lowest index among equals, since lanes hold ascending
// ranges).  Keys are the logits' bits in integer order, so the choice is exact.  Counts go to
// LDS integers; a lane keeps the probability sums of its own experts in registers over all
// its tokens, and they are added up in a fixed order: over the waves in LDS, over the
// workgroups by a second kernel, which also computes the loss.
#include "layer.h"

namespace ep {
namespace {

// Bits of a logit in integer order: a larger number has a larger key, +0 and -0 the same one,
// a NaN the key 1 (below -inf's), and 0 is left for experts that do not exist or are taken.
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    const uint32_t key = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return z != z ? 1u : key;
}
__device__ __forceinline__ float key_logit(uint32_t key) {
    return __uint_as_float((key >> 31) ? key ^ 0x80000000u : ~key);
}

// The logits of this lane's experts; -inf past the last expert.
template <int NV, typename L>
__device__ __forceinline__ void load_logits(const L *row, int e0, int E, float *z) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        z[i] = -__builtin_inff();
        if (e0 + i < E) {
            if constexpr (sizeof(L) == 2)
                z[i] = bf16_lo(row[e0 + i]);
            else
                z[i] = row[e0 + i];
        }
    }
}

// exp(z - top) with a row of -inf alone giving zeros.
__device__ __forceinline__ float exp_below(float z, float top) {
    return top == -__builtin_inff() ? 0.f : expf(z - top);
}

template <int NV>
constexpr int route_waves() {
    return NV <= 8 ? 16 : 4;
}

template <int NV, typename L>
__global__ __launch_bounds__(route_waves<NV>() * 64) void route_kernel(RouteArgs a) {
    constexpr int W = route_waves<NV>();
    __shared__ int counts[64 * NV];
    __shared__ float sums[W][64 * NV];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int e0 = lane * NV;
    for (int i = threadIdx.x; i < 64 * NV; i += W * 64)
        counts[i] = 0;
    __syncthreads();
    float psum[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        psum[i] = 0.f;
    for (int64_t t = (int64_t)blockIdx.x * W + wave; t < a.T; t += (int64_t)gridDim.x * W) {
        const bool live = !a.mask || a.mask[t];
        int32_t *ids = a.topk_idx + t * a.k;
        float *gates = a.topk_w + t * a.k;
        if (!live) {
            for (int j = lane; j < a.k; j += 64) {
                ids[j] = (int32_t)((t * a.k + j) % a.E);
                gates[j] = 0.f;
            }
            continue;
        }
        float z[NV];
        uint32_t key[NV];
        load_logits<NV>(static_cast<const L *>(a.logits) + t * a.E, e0, a.E, z);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            key[i] = e0 + i < a.E ? order_key(z[i]) : 0u;
        float top = 0.f, chosen_sum = 0.f, mine = 0.f;
        for (int j = 0; j < a.k; ++j) {
            uint32_t best = key[0];
            int at = 0;
#pragma unroll
            for (int i = 1; i < NV; ++i)
                if (key[i] > best) {
                    best = key[i];
                    at = i;
                }
            const uint32_t m = wave_max(best);
            const int owner = __builtin_ctzll(__ballot(best == m));
            const float zj = m == 1u ? __builtin_nanf("") : key_logit(m);
            if (j == 0)
                top = zj;
            chosen_sum += exp_below(zj, top);
            if (lane == owner) {
                ids[j] = e0 + at;
                if (a.counts)
                    atomicAdd(&counts[e0 + at], 1);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (lane == owner && i == at)
                    key[i] = 0;
            if (lane == (j & 63)) {
                if (a.k > 64)
                    gates[j] = zj;  // the same lane reads it back below
                else
                    mine = zj;
            }
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            z[i] = exp_below(z[i], top);
            sum += z[i];
        }
        sum = wave_sum(sum);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            psum[i] += z[i] * inv;
        const float scale = !a.normalize ? inv : chosen_sum == 0.f ? 0.f : 1.f / chosen_sum;
        for (int j = lane; j < a.k; j += 64)
            gates[j] = exp_below(a.k > 64 ? gates[j] : mine, top) * scale;
    }
    if (!a.counts)
        return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        sums[wave][e0 + i] = psum[i];
    __syncthreads();
    int32_t *group_counts = static_cast<int32_t *>(a.workspace) + (int64_t)blockIdx.x * 2 * a.E;
    float *group_sums = reinterpret_cast<float *>(group_counts + a.E);
    for (int e = threadIdx.x; e < a.E; e += W * 64) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w)
            s += sums[w][e];
        group_counts[e] = counts[e];
        group_sums[e] = s;
    }
}

// Counts and sums over the groups, then the loss.  One workgroup; L lanes share a column.
__global__ __launch_bounds__(1024) void route_finish_kernel(const int32_t *workspace, int64_t groups, int32_t E,
                                                            int32_t k, float balance, int32_t *counts,
                                                            float *prob_sums, float *loss) {
    __shared__ int part_n[1024];
    __shared__ float part_s[1024];
    __shared__ float wave_loss[16];
    __shared__ int wave_n[16];
    float dot = 0.f;
    int total = 0;
    const int cols = E < 1024 ? E : 1024;
    const int lanes = 1024 / cols, col = threadIdx.x % cols, part = threadIdx.x / cols;
    for (int base = 0; base < E; base += cols) {
        const int e = base + col;
        int n = 0;
        float s = 0.f;
        if (part < lanes && e < E)
            for (int64_t g = part; g < groups; g += lanes) {
                n += workspace[g * 2 * E + e];
                s += reinterpret_cast<const float *>(workspace)[g * 2 * E + E + e];
            }
        part_n[threadIdx.x] = n;
        part_s[threadIdx.x] = s;
        __syncthreads();
        if (part == 0 && e < E) {
            for (int p = 1; p < lanes; ++p) {
                n += part_n[p * cols + col];
                s += part_s[p * cols + col];
            }
            counts[e] = n;
            prob_sums[e] = s;
            dot = fmaf((float)n, s, dot);
            total += n;
        }
        __syncthreads();
    }
    dot = wave_sum(dot);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1)
        total += __shfl_xor(total, d);
    if ((threadIdx.x & 63) == 0) {
        wave_loss[threadIdx.x >> 6] = dot;
        wave_n[threadIdx.x >> 6] = total;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        dot = 0.f;
        total = 0;
        for (int w = 0; w < 16; ++w) {
            dot += wave_loss[w];
            total += wave_n[w];
        }
        const float n = (float)(total / k);
        *loss = total == 0 ? 0.f : balance * (float)E * dot / (n * (float)k * n);
    }
}

template <int NV, typename L>
__global__ __launch_bounds__(256) void route_grad_kernel(RouteGradArgs a) {
    __shared__ float chosen[4][64 * NV];  // per wave: the gates' gradient by expert, zero elsewhere
    __shared__ int wave_n[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int e0 = lane * NV;
    float g[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        g[i] = 0.f;
        chosen[wave][e0 + i] = 0.f;
    }
    if (a.d_loss) {
        int n = 0;
        for (int e = threadIdx.x; e < a.E; e += 256)
            n += a.counts[e];
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1)
            n += __shfl_xor(n, d);
        if (lane == 0)
            wave_n[wave] = n;
        __syncthreads();
        const int total = wave_n[0] + wave_n[1] + wave_n[2] + wave_n[3];
        const float tokens = (float)(total / a.k);
        const float c = total == 0 ? 0.f : *a.d_loss * a.balance * (float)a.E / (tokens * (float)a.k * tokens);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (e0 + i < a.E)
                g[i] = c * (float)a.counts[e0 + i];
    }
    for (int64_t t = (int64_t)blockIdx.x * 4 + wave; t < a.T; t += (int64_t)gridDim.x * 4) {
        const L *row = static_cast<const L *>(a.logits) + t * a.E;
        L *out = static_cast<L *>(a.d_logits) + t * a.E;
        const bool live = !a.mask || a.mask[t];
        float z[NV];
        load_logits<NV>(row, e0, a.E, z);
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t key = e0 + i < a.E ? order_key(z[i]) : 0u;
            best = key > best ? key : best;
        }
        const uint32_t m = wave_max(best);
        const float top = m == 1u ? __builtin_nanf("") : key_logit(m);
        float sum = 0.f, pg = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            z[i] = exp_below(z[i], top);
            sum += z[i];
        }
        sum = wave_sum(sum);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            z[i] *= inv;
            pg = fmaf(z[i], g[i], pg);
        }
        if (a.d_loss)
            pg = wave_sum(pg);
        if (a.d_topk_w && live) {
            // the chosen experts' exponentials; their sum normalizes the gates
            float es = 0.f, ed = 0.f;
            for (int j = lane; j < a.k; j += 64) {
                const int e = a.topk_idx[t * a.k + j];
                if (e < 0 || e >= a.E)
                    continue;
                float v;
                if constexpr (sizeof(L) == 2)
                    v = exp_below(bf16_lo(row[e]), top);
                else
                    v = exp_below(row[e], top);
                es += v;
                ed = fmaf(v, a.d_topk_w[t * a.k + j], ed);
            }
            es = wave_sum(es);
            ed = wave_sum(ed);
            const float scale = !a.normalize ? inv : es == 0.f ? 0.f : 1.f / es;
            const float mean = ed * scale;
            for (int j = lane; j < a.k; j += 64) {
                const int e = a.topk_idx[t * a.k + j];
                if (e < 0 || e >= a.E)
                    continue;
                float v;
                if constexpr (sizeof(L) == 2)
                    v = exp_below(bf16_lo(row[e]), top);
                else
                    v = exp_below(row[e], top);
                chosen[wave][e] = v * scale * (a.d_topk_w[t * a.k + j] - (a.normalize ? mean : 0.f));
            }
            if (!a.normalize)
                pg += mean;
            __builtin_amdgcn_wave_barrier();
        }
        float d[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            d[i] = fmaf(z[i], g[i] - pg, chosen[wave][e0 + i]);
            chosen[wave][e0 + i] = 0.f;
            if (!live)
                d[i] = 0.f;
            if (e0 + i < a.E) {
                if constexpr (sizeof(L) == 2)
                    out[e0 + i] = (uint16_t)bf16_pair(d[i], 0.f);
                else
                    out[e0 + i] = d[i];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <int NV, typename L>
hipError_t launch_one(const RouteArgs &a, hipStream_t stream) {
    constexpr int W = route_waves<NV>();
    return launch_traced("route", route_kernel<NV, L>, dim3((unsigned)route_groups(a.T, a.E)), W * 64, stream, a);
}
template <int NV, typename L>
hipError_t launch_one(const RouteGradArgs &a, hipStream_t stream) {
    const int64_t groups = std::min<int64_t>((a.T + 3) / 4, kCus * 8);
    return launch_traced("route_grad", route_grad_kernel<NV, L>, dim3((unsigned)groups), 256, stream, a);
}
template <typename L, typename A>
hipError_t launch_experts(const A &a, hipStream_t stream) {
    if (a.E <= 64)
        return launch_one<1, L>(a, stream);
    if (a.E <= 128)
        return launch_one<2, L>(a, stream);
    if (a.E <= 256)
        return launch_one<4, L>(a, stream);
    if (a.E <= 512)
        return launch_one<8, L>(a, stream);
    return a.E <= 1024 ? launch_one<16, L>(a, stream) : launch_one<32, L>(a, stream);
}

}  // namespace

int64_t route_groups(int64_t T, int32_t E) {
    const int waves = E <= 512 ? 16 : 4;
    return std::min<int64_t>((T + waves - 1) / waves, kCus);
}

hipError_t launch_route(const RouteArgs &a, hipStream_t stream) {
    if (a.T > 0) {
        const hipError_t e = a.bf16 ? launch_experts<uint16_t>(a, stream) : launch_experts<float>(a, stream);
        if (e != hipSuccess || !a.counts)
            return e;
    }
    if (!a.counts)
        return hipSuccess;
    return launch_traced("route_finish", route_finish_kernel, dim3(1), 1024, stream, (const int32_t *)a.workspace,
                         a.T ? route_groups(a.T, a.E) : (int64_t)0, a.E, a.k, a.balance, a.counts, a.prob_sums,
                         a.loss);
}

hipError_t launch_route_grad(const RouteGradArgs &a, hipStream_t stream) {
    if (a.T == 0)
        return hipSuccess;
    return a.bf16 ? launch_experts<uint16_t>(a, stream) : launch_experts<float>(a, stream);
}

}  // namespace ep
