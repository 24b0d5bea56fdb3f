// route.hip -- the router behind its logits: softmax, top-k, gates, counts per expert and the
// balance loss, forward and backward.
//
//   p = softmax(z);  ids = the k largest logits;  gates = p at the ids, or their softmax
//   loss = balance E sum_e c_e / (N k) P_e / N,  c_e = slots of e,  P_e = sum_t p_te
//   d z_i = w_i (dw_i - sum_j w_j dw_j) on the chosen (normalized gates), or the same through
//           p (gates p), plus p_i (g_i - sum_e p_e g_e), g_e = d_loss balance E c_e / (N k N)
//
// A wave holds one token, lane l the NV experts [l NV, (l + 1) NV).  Each lane sorts its few
// experts once; the k largest are then picked one after the other: the best of the lanes'
// heads by DPP, the lowest lane that has it (the lowest index among equals, since lanes hold
// ascending ranges), and that lane moves on to its next.  Keys are the logits' bits in integer
// order, so the choice is exact.  What a pick leaves to do (the gate's exponential, the count,
// the stores) waits for the last pick and is done by k lanes at once.  Lanes with more than 4
// experts search them at every pick instead of sorting.
//
// Counts go to LDS integers; a lane keeps the probability sums of its own experts in registers
// over all its tokens, and they are added up in a fixed order: over the waves in LDS, over the
// workgroups by a second kernel, which also computes the loss.
//
// Bound by its instructions: 32768 tokens of 256 experts, top-8, are 34 MB of logits, 6 us of HBM;
// the forward takes 28 us, its second kernel 5 to 7, the gradient 18 (67 MB, 12 us of HBM); bf16
// logits, half the bytes, gain less than 1 us in each.  256 tokens: 5.5 and 4.2 us, latency.
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

// A lane's experts.  Lane l has [l NV, (l + 1) NV), and loads and stores them as one vector; where
// the experts end within it (EVEN: in no lane), the vector is moved down to [E - NV, E), and its
// first ones, which the lane before has, do not count.  (E >= NV: a launch takes the smallest NV
// that holds E.)  Before the vectors were moved, lanes loaded and stored such experts one by one:
// 32768 tokens of 511 experts forward and backward 129 us, now 91.
template <int NV, bool EVEN>
struct Lane {
    int first, e0;  // first expert of its own; first of its vector
    bool some;      // it has one
    __device__ __forceinline__ Lane(int lane, int E)
        : first(lane * NV), e0(first < E - NV ? first : E - NV), some(first < E) {}
    __device__ __forceinline__ bool has(int i) const { return EVEN ? some : e0 + i >= first; }
};
// NV elements at any element's alignment
template <int NV, typename L>
struct __attribute__((packed, aligned(sizeof(L)))) Elements {
    L v[NV];
};

// The logits of the lane's experts; -inf for those that do not count.
template <int NV, bool EVEN, typename L>
__device__ __forceinline__ void load_logits(const L *row, const Lane<NV, EVEN> &l, float *z) {
    const Elements<NV, L> raw = *reinterpret_cast<const Elements<NV, L> *>(row + l.e0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float v;
        if constexpr (sizeof(L) == 2)
            v = bf16_lo(raw.v[i]);
        else
            v = raw.v[i];
        z[i] = l.has(i) ? v : -__builtin_inff();
    }
}
template <typename L>
__device__ __forceinline__ float one_logit(const L *row, int e) {
    if constexpr (sizeof(L) == 2)
        return bf16_lo(row[e]);
    else
        return row[e];
}

// exp(z - top) with a row of -inf alone giving zeros.
__device__ __forceinline__ float exp_below(float z, float top) {
    return top == -__builtin_inff() && z == z ? 0.f : quick_exp(z - top);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_fmax(float v) {
    const int o = __builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, ROWS, 0xf, false);
    return fmaxf(v, __int_as_float(o));
}
// Largest over the wave; NaN only where every lane has one.
__device__ __forceinline__ float wave_fmax(float v) {
    v = dpp_fmax<0x111, 0xf>(v);
    v = dpp_fmax<0x112, 0xf>(v);
    v = dpp_fmax<0x114, 0xf>(v);
    v = dpp_fmax<0x118, 0xf>(v);
    v = dpp_fmax<0x142, 0xa>(v);
    v = dpp_fmax<0x143, 0xc>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) {
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true);
}
__device__ __forceinline__ int wave_sum_int(int v) {
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    v = dpp_add<0x143, 0xc>(v);
    return __builtin_amdgcn_readlane(v, 63);
}
// A lane's experts for the picks: the best one's key and number.
template <int NV>
struct Heads {
    static constexpr bool kSorted = NV <= 4;
    uint32_t key[NV];
    int at[kSorted ? NV : 1];
    __device__ __forceinline__ void order(int i, int j) {  // key[i] >= key[j], the lower number first among equals
        const bool swap = key[j] > key[i];
        const uint32_t k = swap ? key[j] : key[i];
        const int n = swap ? at[j] : at[i];
        key[j] = swap ? key[i] : key[j];
        at[j] = swap ? at[i] : at[j];
        key[i] = k;
        at[i] = n;
    }
    __device__ __forceinline__ void prepare() {
        if constexpr (kSorted) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                at[i] = i;
            // neighbours only: a stable exchange sort keeps equals in their order
#pragma unroll
            for (int round = 0; round < NV; ++round)
#pragma unroll
                for (int i = round % 2; i + 1 < NV; i += 2)
                    order(i, i + 1);
        }
    }
    __device__ __forceinline__ uint32_t best(int &number) const {
        if constexpr (kSorted) {
            number = at[0];
            return key[0];
        } else {
            uint32_t b = key[0];
            number = 0;
#pragma unroll
            for (int i = 1; i < NV; ++i)
                if (key[i] > b) {
                    b = key[i];
                    number = i;
                }
            return b;
        }
    }
    __device__ __forceinline__ void take(bool mine, int number) {
        if constexpr (kSorted) {
#pragma unroll
            for (int i = 0; i + 1 < NV; ++i) {
                key[i] = mine ? key[i + 1] : key[i];
                at[i] = mine ? at[i + 1] : at[i];
            }
            key[NV - 1] = mine ? 0u : key[NV - 1];
        } else {
            const int gone = mine ? number : -1;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                key[i] = i == gone ? 0u : key[i];
        }
    }
};

// Experts of a group's counts, and of its sums, in the workspace: whole vectors.
__host__ __device__ constexpr int group_experts(int E) { return (E + 3) / 4 * 4; }

template <int NV>
constexpr int route_waves() {
    return NV <= 8 ? 16 : 4;
}

template <int NV, bool EVEN, typename L>
__global__ __launch_bounds__(route_waves<NV>() * 64) void route_kernel(RouteArgs a) {
    constexpr int W = route_waves<NV>();
    __shared__ int counts[64 * NV];
    __shared__ float sums[W][64 * NV];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Lane<NV, EVEN> own(lane, a.E);
    for (int i = threadIdx.x; i < 64 * NV; i += W * 64)
        counts[i] = 0;
    __syncthreads();
    float psum[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        psum[i] = 0.f;
    const int64_t stride = (int64_t)gridDim.x * W;
    int64_t t = (int64_t)blockIdx.x * W + wave;
    float ahead[NV];  // the next token's logits
    if (t < a.T)
        load_logits(static_cast<const L *>(a.logits) + t * a.E, own, ahead);
    for (; t < a.T; t += stride) {
        float z[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            z[i] = ahead[i];
        if (t + stride < a.T)
            load_logits(static_cast<const L *>(a.logits) + (t + stride) * a.E, own, ahead);
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
        Heads<NV> heads;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            heads.key[i] = own.has(i) ? order_key(z[i]) : 0u;
        heads.prepare();
        // 64 picks at a time: lane j holds pick j's key and expert
        float top = 0.f, chosen_sum = 0.f, gate = 0.f;
        for (int j0 = 0; j0 < a.k; j0 += 64) {
            const int picks = a.k - j0 < 64 ? a.k - j0 : 64;
            uint32_t key = 0;
            int expert = 0;
            for (int j = 0; j < picks; ++j) {
                int number;
                const uint32_t b = heads.best(number);
                const uint32_t m = wave_max(b);
                const int owner = __builtin_ctzll(__ballot(b == m));
                const int e = __builtin_amdgcn_readlane(own.e0 + number, owner);
                key = lane == j ? m : key;
                expert = lane == j ? e : expert;
                heads.take(lane == owner, number);
            }
            float zj = key == 1u ? __builtin_nanf("") : key_logit(key);
            if (j0 == 0)
                top = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(zj), 0));
            if (lane < picks) {
                zj = exp_below(zj, top);
                chosen_sum += zj;
                ids[j0 + lane] = expert;
                gate = zj;
                if (a.k > 64)
                    gates[j0 + lane] = zj;  // the same lane scales it below
                if (a.counts)
                    atomicAdd(&counts[expert], 1);
            }
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            z[i] = exp_below(z[i], top);
            sum += z[i];
        }
        sum = wave_sum(sum);
        chosen_sum = wave_sum(chosen_sum);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            psum[i] = fmaf(z[i], inv, psum[i]);
        const float scale = !a.normalize ? inv : chosen_sum == 0.f ? 0.f : 1.f / chosen_sum;
        if (a.k > 64)
            for (int j = lane; j < a.k; j += 64)
                gates[j] *= scale;
        else if (lane < a.k)
            gates[lane] = gate * scale;
    }
    if (!a.counts)
        return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (own.has(i))
            sums[wave][own.e0 + i] = psum[i];
    __syncthreads();
    const int half = group_experts(a.E);
    int32_t *group_counts = static_cast<int32_t *>(a.workspace) + (int64_t)blockIdx.x * 2 * half;
    float *group_sums = reinterpret_cast<float *>(group_counts + half);
    for (int e = threadIdx.x; e < a.E; e += W * 64) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w)
            s += sums[w][e];
        group_counts[e] = counts[e];
        group_sums[e] = s;
    }
}

// Counts and sums over the groups, then the loss: one workgroup.  A thread adds 4 neighbouring
// experts of every lanes-th group, kAhead groups on their way at a time; the buffer's range gives
// zeros past the last group.  2^shift threads lie side by side over the experts, and `lanes` of
// those rows of threads share the groups.  The code is kept short: it runs once, out of a cold
// instruction cache.
__global__ __launch_bounds__(1024) void route_finish_kernel(void *workspace, int32_t groups, int32_t E, int32_t shift,
                                                            int32_t lanes, int32_t k, float balance, int32_t *counts,
                                                            float *prob_sums, float *loss) {
    __shared__ u32x4 part_n[1024], part_s[1024];
    __shared__ float wave_loss[16];
    __shared__ int wave_n[16];
    constexpr int kAhead = 8;
    constexpr uint32_t kNowhere = 0x80000000u;
    const int cols = 1 << shift, col = threadIdx.x & (cols - 1), part = threadIdx.x >> shift;
    const uint32_t half = (uint32_t)group_experts(E) * 4, row = 2 * half;  // bytes of a group: counts, then sums
    const __amdgpu_buffer_rsrc_t table = __builtin_amdgcn_make_buffer_rsrc(workspace, 0, groups * (int32_t)row, 0x00020000);
    float dot = 0.f;
    int total = 0;
    for (int base = 0; base < E; base += cols * 4) {
        const int e = base + col * 4;
        uint32_t at = e < E && part < lanes ? part * row + e * 4 : kNowhere;
        u32x4 n = {0, 0, 0, 0};
        float s[4] = {};
        for (int g = 0; g < groups; g += lanes * kAhead) {
            u32x4 vn[kAhead], vs[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                vn[i] = __builtin_amdgcn_raw_buffer_load_b128(table, at, 0, 0);
                vs[i] = __builtin_amdgcn_raw_buffer_load_b128(table, at + half, 0, 0);
                at += lanes * row;
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                n += vn[i];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    s[q] += __uint_as_float(vs[i][q]);
            }
        }
        part_n[threadIdx.x] = n;
        part_s[threadIdx.x] = u32x4{__float_as_uint(s[0]), __float_as_uint(s[1]), __float_as_uint(s[2]), __float_as_uint(s[3])};
        __syncthreads();
        for (int c = threadIdx.x; c < cols * 4 && base + c < E; c += 1024) {
            int cn = 0;
            float cs = 0.f;
#pragma unroll 4
            for (int p = 0; p < lanes; ++p) {
                cn += reinterpret_cast<const int *>(part_n)[p * cols * 4 + c];
                cs += reinterpret_cast<const float *>(part_s)[p * cols * 4 + c];
            }
            counts[base + c] = cn;
            prob_sums[base + c] = cs;
            dot = fmaf((float)cn, cs, dot);
            total += cn;
        }
        __syncthreads();
    }
    dot = wave_sum(dot);
    total = wave_sum_int(total);
    if ((threadIdx.x & 63) == 0) {
        wave_loss[threadIdx.x >> 6] = dot;
        wave_n[threadIdx.x >> 6] = total;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        dot = wave_sum(threadIdx.x < 16 ? wave_loss[threadIdx.x & 15] : 0.f);
        total = wave_sum_int(threadIdx.x < 16 ? wave_n[threadIdx.x & 15] : 0);
        const float n = (float)(total / k);
        if (threadIdx.x == 0)
            *loss = total == 0 ? 0.f : balance * (float)E * dot / (n * (float)k * n);
    }
}

template <int NV, bool EVEN, typename L>
__global__ __launch_bounds__(256) void route_grad_kernel(RouteGradArgs a) {
    __shared__ float chosen[4][64 * NV];  // per wave: the gates' gradient by expert, zero elsewhere
    __shared__ long long wave_n[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Lane<NV, EVEN> own(lane, a.E);
    float g[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        g[i] = 0.f;
        chosen[wave][i * 64 + lane] = 0.f;
    }
    // an expert's place: its lane's element, lanes side by side, so that no banks conflict
    const auto place = [&](uint32_t e) {
        const Lane<NV, EVEN> l(e / NV, a.E);
        return (EVEN ? e % NV : e - l.e0) * 64 + e / NV;
    };
    if (a.d_loss) {
        long long n = 0;  // a group's counts may pass 32 bits together
        for (int e = threadIdx.x; e < a.E; e += 256)
            n += a.counts[e];
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1)
            n += __shfl_xor(n, d);
        if (lane == 0)
            wave_n[wave] = n;
        __syncthreads();
        const long long total = wave_n[0] + wave_n[1] + wave_n[2] + wave_n[3];
        const float tokens = (float)((double)total / a.k);
        const float c = total == 0 ? 0.f : *a.d_loss * a.balance * (float)a.E / (tokens * (float)a.k * tokens);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (own.has(i))
                g[i] = c * (float)a.counts[own.e0 + i];
    }
    // normalized gates alone do not look at the others' p: a NaN there is none of theirs
    const bool through_p = a.d_loss || !a.normalize;
    const int64_t stride = (int64_t)gridDim.x * 4;
    for (int64_t t = (int64_t)blockIdx.x * 4 + wave; t < a.T; t += stride) {
        const L *row = static_cast<const L *>(a.logits) + t * a.E;
        L *out = static_cast<L *>(a.d_logits) + t * a.E;
        const bool live = !a.mask || a.mask[t];
        float z[NV];
        load_logits(row, own, z);
        // the chosen experts: lane j (and j + 64, ...) takes the j-th
        int expert = -1;
        float zc = 0.f, dc = 0.f;
        if (a.d_topk_w && lane < a.k) {
            expert = a.topk_idx[t * a.k + lane];
            dc = a.d_topk_w[t * a.k + lane];
            expert = expert < a.E ? expert : -1;
            if (expert >= 0)
                zc = one_logit(row, expert);
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < NV; ++i)
            top = fmaxf(top, z[i]);
        top = wave_fmax(top);
        float sum = 0.f, pg = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            z[i] = exp_below(z[i], top);
            sum += z[i];
            pg = fmaf(z[i], g[i], pg);
        }
        sum = wave_sum(sum);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        pg = a.d_loss ? wave_sum(pg) * inv : 0.f;
        if (a.d_topk_w && live) {
            // the chosen experts' exponentials; their sum normalizes the gates
            const float v = expert >= 0 ? exp_below(zc, top) : 0.f;
            float es = v, ed = v * dc;
            for (int j = lane + 64; j < a.k; j += 64) {
                const int e = a.topk_idx[t * a.k + j];
                if (e < 0 || e >= a.E)
                    continue;
                const float u = exp_below(one_logit(row, e), top);
                es += u;
                ed = fmaf(u, a.d_topk_w[t * a.k + j], ed);
            }
            ed = wave_sum(ed);
            if (a.normalize)
                es = wave_sum(es);
            const float scale = !a.normalize ? inv : es == 0.f ? 0.f : 1.f / es;
            const float mean = ed * scale, less = a.normalize ? mean : 0.f;
            if (expert >= 0)
                chosen[wave][place(expert)] = v * scale * (dc - less);
            for (int j = lane + 64; j < a.k; j += 64) {
                const int e = a.topk_idx[t * a.k + j];
                if (e >= 0 && e < a.E)
                    chosen[wave][place(e)] = exp_below(one_logit(row, e), top) * scale * (a.d_topk_w[t * a.k + j] - less);
            }
            if (!a.normalize)
                pg += mean;
            __builtin_amdgcn_wave_barrier();
        }
        Elements<NV, L> vec;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const float c = chosen[wave][i * 64 + lane];
            const float d = !live ? 0.f : through_p ? fmaf(z[i] * inv, g[i] - pg, c) : c;
            chosen[wave][i * 64 + lane] = 0.f;
            if constexpr (sizeof(L) == 2)
                vec.v[i] = (L)bf16_pair(d, 0.f);
            else
                vec.v[i] = d;
        }
        if (EVEN ? own.some : own.e0 == own.first) {
            *reinterpret_cast<Elements<NV, L> *>(out + own.e0) = vec;
        } else if (!EVEN) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (own.has(i))
                    out[own.e0 + i] = vec.v[i];
        }
        __builtin_amdgcn_wave_barrier();
    }
}

int64_t route_groups(int64_t T, int32_t E) {
    const int waves = E <= 512 ? route_waves<8>() : route_waves<16>();
    return std::min<int64_t>((T + waves - 1) / waves, kCus);
}
template <int NV, bool EVEN, typename L>
hipError_t launch_lanes(const RouteArgs &a, hipStream_t stream) {
    constexpr int W = route_waves<NV>();
    return launch_traced("route", route_kernel<NV, EVEN, L>, dim3((unsigned)route_groups(a.T, a.E)), W * 64, stream, a);
}
template <int NV, bool EVEN, typename L>
hipError_t launch_lanes(const RouteGradArgs &a, hipStream_t stream) {
    const int64_t groups = std::min<int64_t>((a.T + 3) / 4, kCus * 8);
    return launch_traced("route_grad", route_grad_kernel<NV, EVEN, L>, dim3((unsigned)groups), 256, stream, a);
}
template <int NV, typename L, typename A>
hipError_t launch_one(const A &a, hipStream_t stream) {
    if constexpr (NV > 1)
        if (a.E % NV)
            return launch_lanes<NV, false, L>(a, stream);
    return launch_lanes<NV, true, L>(a, stream);
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

size_t route_workspace_bytes(int64_t T, int32_t E) { return (size_t)route_groups(T, E) * group_experts(E) * 8; }

hipError_t launch_route(const RouteArgs &a, hipStream_t stream) {
    if (a.T > 0) {
        const hipError_t e = a.bf16 ? launch_experts<uint16_t>(a, stream) : launch_experts<float>(a, stream);
        if (e != hipSuccess || !a.counts)
            return e;
    }
    if (!a.counts)
        return hipSuccess;
    const int64_t groups = a.T ? route_groups(a.T, a.E) : 0;
    int32_t shift = 0;
    while (shift < 10 && (4 << shift) < a.E)
        ++shift;
    // with 32 rows of threads every group is on its way at once
    return launch_traced("route_finish", route_finish_kernel, dim3(1), 1024, stream, a.workspace, (int32_t)groups, a.E, shift,
                         std::min(1024 >> shift, 32), a.k, a.balance, a.counts, a.prob_sums, a.loss);
}

hipError_t launch_route_grad(const RouteGradArgs &a, hipStream_t stream) {
    if (a.T == 0)
        return hipSuccess;
    return a.bf16 ? launch_experts<uint16_t>(a, stream) : launch_experts<float>(a, stream);
}

}  // namespace ep
