// adapter_low.hip -- the low-rank values of the adapters' rows:
//   scale_a x[order[i]] a_a^T of the forward, scale_a dz[order[i]] b_a of the gradient,
// as the sum of two bf16 values each for the products that read them, and for the forward also as the one
// bf16 value that a caller keeps.  Rows without an adapter get zeros.
//
// Bound by the rows' bytes, or for few rows by the adapters' (16379 rows of 7168, 64 ranks 65 us, 3.6 TB/s; 8192 rows of
// 4096, 16 ranks, a quarter of them without an adapter 18).  Many rows go through LDS, with more than
// 32 ranks and in the gradient through the MFMA tile (product_tile.h).  Few rows go straight from memory into the operands of
// 16x16 matrix instructions: the 16 waves of a workgroup share out the contraction, 64 values (whole
// cache lines) at a time with every load of a wave on its way at once, and are added up through LDS in
// a fixed order.
//
// The products multiply bf16, and in one bf16 value each the low-rank values lose as much as the results
// do: a gated product's error is 0.0025 of its 2-norm that way and 0.0017, its own rounding, with the
// rest of each value in a second one; da's 0.0029 and 0.0023.  It takes the ranks' part of the contractions
// twice, a step or two of a hundred.
#include "adapter_tile.h"

namespace ep {
namespace {

// The rows without an adapter: before the first one's rows and behind the last one's.
struct Others {
    int64_t before, behind, count;
    __device__ __forceinline__ explicit Others(const LowArgs &a) {
        before = a.offsets ? clamp_row(a.offsets[0], a.rows) : 0;
        behind = a.offsets ? clamp_row(a.offsets[a.A], a.rows) : a.rows;
        count = before + a.rows - behind;
    }
};
// Zeros for the `per` of them from number z on.
__device__ __forceinline__ void clear_rows(const LowArgs &a, const Others &o, int64_t z, int per, int threads) {
    const int vecs = a.width / 8;
    for (int i = threadIdx.x; i < per * vecs; i += threads) {
        const int64_t p = z + i / vecs;
        const int64_t row = p < o.before ? p : o.behind + (p - o.before);
        const int at = i % vecs * 8;
        if (z < 0 || row >= a.rows)
            continue;
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.split) + row * a.width + at) = u32x4{0, 0, 0, 0};
        if (a.low && at < a.R)
            *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.low) + row * a.R + at) = u32x4{0, 0, 0, 0};
    }
}
// The tile of `per` rows of one adapter, and of `cols` its column `col`, that the workgroup takes; e < 0: none.  Each
// XCD takes a contiguous eighth of the tiles, so that an adapter's weights stay in one or two of the eight L2s; the
// workgroups left over clear the rows without an adapter.  (Dealt out together with those, the adapters'
// tiles leave an XCD idle and come twice to compute units of others: 8192 rows of 4096, a quarter without, from the
// memory-side cache 21 us instead of 14.)
__device__ __forceinline__ RowTile low_tile(const LowArgs &a, int32_t per, int32_t cols, int32_t &col, int threads, int lane) {
    const int32_t block = (int32_t)blockIdx.x;
    const int32_t tiles = count_row_tiles(a.offsets, a.rows, a.A, per, lane) * cols;
    const int32_t t = (int32_t)tile_of_block(block, tiles);
    if (t >= 0) {
        col = t % cols;
        return find_row_tile(a.offsets, a.rows, a.A, per, t / cols, lane);
    }
    const int32_t spare = block - (tiles + 7) / 8 * 8;
    const Others o(a);
    if (spare >= 0 && spare < (o.count + per - 1) / per)
        clear_rows(a, o, (int64_t)spare * per, per, threads);
    return {-1, 0, 0};
}
// All tiles, the rows without an adapter being one more adapter's, in whole eighths.
dim3 low_grid(const LowArgs &a, int per, int cols) {
    return dim3((unsigned)((row_tiles_most(a.rows, a.A + 1, per) * cols + 7) / 8 * 8 + 8));
}

// N neighbouring values (4 or 8) from rank on of a row: N / 2 words per array.
template <int N>
__device__ __forceinline__ void put_values(const LowArgs &a, int64_t row, int rank, const float *v) {
    uint32_t first[N / 2], rest[N / 2], kept[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        first[i] = first_pair(v[2 * i], v[2 * i + 1]);
        rest[i] = rest_pair(v[2 * i], v[2 * i + 1]);
        kept[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    }
    typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
    const auto put = [](void *to, int64_t at, const uint32_t *w) {
        words o;
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            o[i] = w[i];
        *reinterpret_cast<words *>(static_cast<uint16_t *>(to) + at) = o;
    };
    const int64_t at = row * a.width + rank + (rank >> a.log << a.log);
    put(a.split, at, first);
    put(a.split, at + (1 << a.log), rest);
    if (a.low)
        put(a.low, row * a.R + rank, kept);
}

// ---- few rows ------------------------------------------------------------------------
constexpr int kFewWaves = 16, kFewRows = 16, kFewRanks = 16;

__global__ __launch_bounds__(kFewWaves * 64) void adapter_low_few_kernel(LowArgs a) {
    __shared__ f32x4 sums[kFewWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t col;
    const RowTile rt = low_tile(a, kFewRows, (a.R + kFewRanks - 1) / kFewRanks, col, kFewWaves * 64, lane);
    if (rt.e < 0)
        return;
    const int rank0 = col * kFewRanks;
    const int g = lane / 16;  // which 16 bytes of a fragment's 64 this lane takes
    const int rank = rank0 + lane % 16;
    const bool has_a = rank < a.R;
    const uint16_t *ar = static_cast<const uint16_t *>(a.weights) + ((int64_t)rt.e * a.R + (has_a ? rank : 0)) * a.K;
    const int32_t r = lane % 16 < rt.n ? row_at(a.order, a.rows, rt.row0 + lane % 16) : -1;
    const uint16_t *xr = static_cast<const uint16_t *>(a.x) + (r >= 0 ? (int64_t)r * a.K : 0);
    f32x4 acc = {};
    constexpr int kAhead = 4;
    for (int32_t k0 = wave * 64; k0 < a.K; k0 += kFewWaves * 64 * kAhead) {
        u32x4 xv[kAhead][2], av[kAhead][2];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int32_t k = k0 + u * kFewWaves * 64 + h * 32 + g * 8;
                av[u][h] = u32x4{0, 0, 0, 0};
                if (k < a.K && has_a)
                    av[u][h] = *reinterpret_cast<const u32x4 *>(ar + k);
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int32_t k = k0 + u * kFewWaves * 64 + h * 32 + g * 8;
                xv[u][h] = u32x4{0, 0, 0, 0};
                if (k < a.K && r >= 0)
                    xv[u][h] = *reinterpret_cast<const u32x4 *>(xr + k);
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av[u][h]),
                                                              __builtin_bit_cast(bf16x8, xv[u][h]), acc, 0, 0, 0);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (threadIdx.x >= 64)
        return;
    const float scale = a.scale ? a.scale[rt.e] : 1.f;
    f32x4 s = sums[0][lane];
#pragma unroll
    for (int v = 1; v < kFewWaves; ++v)
        s += sums[v][lane];
    const int q = rank0 + lane / 16 * 4, row = lane % 16;  // a lane holds four ranks of one row
    if (row < rt.n && q < a.R) {
        const float o[4] = {s[0] * scale, s[1] * scale, s[2] * scale, s[3] * scale};
        put_values<4>(a, rt.row0 + row, q, o);
    }
}

// ---- many rows, up to 32 ranks -----------------------------------------------------------
// A wave takes 32 rows of one adapter and every WAVES-th step of 64 values of the contraction; the waves
// of a workgroup are added up at the end.  The rows go to LDS (their fragments are whole cache lines
// there), the weights, which no other wave of the workgroup needs, into registers.  No wave waits for another:
// each has kDeep steps on their way, and as loads return in order, as many of the weights' as of the
// rows'.  (3440 rows of 6656, 8 ranks: 15 us, as a tile of product_tile.h 21 to 27.  With 64 ranks the
// weights' loads, which touch a cache line per rank, take longer than the tile's: 16379 rows of 7168 132 us, 103.)
constexpr int kDeep = 5, kDeepRows = 32;

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void adapter_low_rows_kernel(LowArgs a) {
    typedef AlongC<kDeepRows, 1> Rows;
    constexpr int kStage = kDeepRows * kStepBytes, kLoads = Rows::kLoads + 4;
    static_assert((kDeep - 1) * kLoads < 64 && 4096 <= kDeep * kStage, "");
    __shared__ __attribute__((aligned(1024))) char lds[WAVES * kDeep * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t col;
    const RowTile rt = low_tile(a, kDeepRows, 1, col, WAVES * 64, lane);
    if (rt.e < 0)
        return;
    const int64_t kb = (int64_t)a.K * 2;
    char EP_LDS *own = (char EP_LDS *)lds + wave * kDeep * kStage;
    const char *xb = static_cast<const char *>(a.x);
    Rows x;
    // through an order from x's first row on (x is smaller than 2^31 bytes then)
    x.init(a.order ? xb : xb + rt.row0 * kb, (uint32_t)((a.order ? a.rows : rt.n) * kb), (int32_t)kb, 0, lane,
           [&](int row) -> uint32_t {
               if (row >= rt.n)
                   return kNowhere;
               const int32_t r = a.order ? row_at(a.order, a.rows, rt.row0 + row) : row;
               return r < 0 ? kNowhere : (uint32_t)(r * kb);
           });
    x.aim(0, lane);
    const __amdgpu_buffer_rsrc_t weights =
        buffer_of(static_cast<const char *>(a.weights) + (int64_t)rt.e * a.R * kb, (uint32_t)(a.R * kb));
    const int32_t end = lane % 32 < a.R ? (int32_t)kb : 0;  // of this lane's rank
    const uint32_t at = (uint32_t)(lane % 32 * kb);
    const int32_t all = (a.K + kStepRows - 1) / kStepRows;
    const int32_t steps = all > wave ? (all - wave + WAVES - 1) / WAVES : 0;
    int32_t next = 0;  // the step whose loads are issued next
    int32_t byte = (wave * kStepRows + lane / 32 * 8) * 2;  // of the contraction
    if (wave > 0)
        x.skip(wave);
    u32x4 w[kDeep][4];
    const auto load = [&](int place) {
        const bool live = next < steps;
        x.begin(live);
#pragma unroll
        for (int q = 0; q < Rows::kLoads; ++q)
            x.load(q, own + place * kStage, 0, lane);
        x.skip(WAVES);
        const int32_t until = live ? end : 0;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const uint32_t o = byte + h * 32 < until ? at + (uint32_t)(byte + h * 32) : kNowhere;
            w[place][h] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(weights, (int)o, 0, 0));
        }
        byte += WAVES * kStepBytes;
        ++next;
        __builtin_amdgcn_sched_barrier(0);
    };
    f32x16 acc = {};
#pragma unroll
    for (int p = 0; p < kDeep - 1; ++p)
        load(p);
    for (int32_t t = 0; t < steps; t += kDeep) {
#pragma unroll
        for (int p = 0; p < kDeep; ++p) {
            load((p + kDeep - 1) % kDeep);
            asm volatile("" ::: "memory");
            constexpr int kFlying = (kDeep - 1) * kLoads;  // this step has landed, the others are on their way
            __builtin_amdgcn_s_waitcnt((kFlying & 15) | 7 << 4 | 15 << 8 | kFlying >> 4 << 14);
            asm volatile("" ::: "memory");
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const bf16x8 r = __builtin_bit_cast(bf16x8, x.read(own + p * kStage, 0, h));
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[p][h]), r, acc, 0, 0, 0);
            }
            // the fragments are read before the place is loaded again
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(15 | 7 << 4 | 0 << 8 | 3 << 14);
            asm volatile("" ::: "memory");
        }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0 | 7 << 4 | 0 << 8);  // loads past the end have landed, too
    asm volatile("" ::: "memory");
    // four neighbouring ranks of one row per lane and quarter
    f32x4 EP_LDS *sums = reinterpret_cast<f32x4 EP_LDS *>(own);
#pragma unroll
    for (int q = 0; q < 4; ++q)
        sums[q * 64 + lane] = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
    __syncthreads();
    const float scale = a.scale ? a.scale[rt.e] : 1.f;
    const f32x4 EP_LDS *first = (const f32x4 EP_LDS *)(char EP_LDS *)lds;
    for (int i = threadIdx.x; i < 256; i += WAVES * 64) {
        f32x4 s = first[i];
#pragma unroll
        for (int v = 1; v < WAVES; ++v)
            s += first[v * (kDeep * kStage / 16) + i];
        const int l = i % 64, row = l % 32, rank = i / 64 * 8 + l / 32 * 4;
        if (row >= rt.n || rank >= a.R)
            continue;
        const float o[4] = {s[0] * scale, s[1] * scale, s[2] * scale, s[3] * scale};
        put_values<4>(a, rt.row0 + row, rank, o);
    }
}

// As many waves per workgroup as fill the compute units' LDS: six per compute unit of 20 KiB each.
hipError_t launch_rows(const LowArgs &a, hipStream_t stream) {
    const dim3 grid = low_grid(a, kDeepRows, 1);
    const int64_t tiles = a.rows / kDeepRows + a.A;
#define EP_CALL(W) launch_traced("adapter_low", adapter_low_rows_kernel<W>, grid, W * 64, stream, a)
    return tiles <= kCus ? EP_CALL(6) : tiles <= 2 * kCus ? EP_CALL(3) : EP_CALL(2);
#undef EP_CALL
}

// ---- many rows, more ranks or weights across the contraction ------------------------------
// ACROSS: the weights are [A][K][R], else [A][R][K].
template <class S, bool ACROSS>
__global__ __launch_bounds__(S::kThreads) void adapter_low_kernel(LowArgs a, int32_t per) {
    constexpr int kBytes = S::kStages * S::kStageBytes;
    __shared__ __attribute__((aligned(1024))) char lds[kBytes + S::kJ * 4];  // one array: see TileLds
    int32_t EP_LDS *row_of = (int32_t EP_LDS *)((char EP_LDS *)lds + kBytes);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t col;
    const RowTile rt = low_tile(a, per, (a.R + S::kI - 1) / S::kI, col, S::kThreads, lane);
    if (rt.e < 0)
        return;
    const int rank0 = col * S::kI;
    for (int j = threadIdx.x; j < S::kJ; j += S::kThreads)
        row_of[j] = j < rt.n ? row_at(a.order, a.rows, rt.row0 + j) : -1;
    __syncthreads();
    const int64_t kb = (int64_t)a.K * 2;
    const char *weights = static_cast<const char *>(a.weights) + (int64_t)rt.e * a.R * kb;
    const char *xb = static_cast<const char *>(a.x);
    AlongC<S::kJ, S::kWaves> x;
    // through an order from x's first row on (x is smaller than 2^31 bytes then)
    x.init(a.order ? xb : xb + rt.row0 * kb, (uint32_t)((a.order ? a.rows : rt.n) * kb), (int32_t)kb, wave, lane,
           [&](int row) -> uint32_t {
               const int32_t r = a.order ? row_of[row] : row;
               return r < 0 ? kNowhere : (uint32_t)(r * kb);
           });
    f32x16 acc[S::FI][S::FJ] = {};
    const int32_t steps = (a.K + kStepRows - 1) / kStepRows;
    if constexpr (ACROSS) {
        AcrossC<S::kI, S::kWaves, S::FI> w;
        w.init(weights, (int64_t)a.R * 2, a.K, rank0, wave, lane);
        tile_product<S, Mul::kBf16>(w, x, steps, (char EP_LDS *)lds, wave, lane, acc);
    } else {
        AlongC<S::kI, S::kWaves> w;
        w.init(weights, (uint32_t)(a.R * kb), (int32_t)kb, wave, lane,
               [&](int row) -> uint32_t { return rank0 + row < a.R ? (uint32_t)((rank0 + row) * kb) : kNowhere; });
        tile_product<S, Mul::kBf16>(w, x, steps, (char EP_LDS *)lds, wave, lane, acc);
    }
    const float scale = a.scale ? a.scale[rt.e] : 1.f;
    tile_results<S>(acc, (char EP_LDS *)lds, wave, lane, [&](int row, int col, const float *v) {
        const int rank = rank0 + col;
        if (row >= rt.n || rank >= a.R)
            return;
        float o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
            o[q] = v[q] * scale;
        put_values<8>(a, rt.row0 + row, rank, o);
    });
}

// 64 ranks by `per` rows, as many as leave every compute unit a tile (and with more than 128 every one of them
// two, three and so on): a tile takes as long as its loads, and a compute unit that has one tile more than the others takes
// all that time more.  In the smallest shape that holds them, of which two workgroups fit a compute unit's LDS.
// (16379 rows of 7168, eight adapters, in tiles of 64 rows, which are 260: 127 us, 103 in tiles of 128.)
typedef TileShape<64, 32, 2, 1, 5> Low32;
typedef TileShape<64, 64, 2, 2, 3> Low64;
typedef TileShape<64, 128, 2, 4, 3> Low128;

int tile_rows(int64_t rows, int32_t A, int32_t cols) {
    const int64_t partly = A > 1 ? (int64_t)A * cols : 0;  // every adapter's last tile may be nearly empty
    const int64_t turns = (rows * cols / Low128::kJ + partly + kCus) / kCus;
    const int64_t whole = turns * kCus - partly;
    return std::clamp((int)((rows * cols + whole - 1) / whole + 7) / 8 * 8, Low32::kJ, Low128::kJ);
}

template <bool ACROSS>
hipError_t launch_tiles(const LowArgs &a, hipStream_t stream) {
    const int32_t cols = (a.R + 63) / 64;
    const int per = tile_rows(a.rows, a.A, cols);
    const dim3 grid = low_grid(a, per, cols);
#define EP_CALL(S) launch_traced("adapter_low", adapter_low_kernel<S, ACROSS>, grid, S::kThreads, stream, a, per)
    return per <= Low32::kJ ? EP_CALL(Low32) : per <= Low64::kJ ? EP_CALL(Low64) : EP_CALL(Low128);
#undef EP_CALL
}

}  // namespace

hipError_t launch_adapter_low(const LowArgs &a, hipStream_t stream) {
    if (a.rows == 0)
        return hipSuccess;
    if (a.across)
        return launch_tiles<true>(a, stream);
    const bool far = a.order && a.rows * a.K * 2 > INT32_MAX;  // rows that a tile cannot address
    // Few rows: at most a workgroup of theirs per compute unit.  Measured, us, that way and by tiles, of 512 and 5000
    // values a row: 3000 rows of 20 adapters, 16 ranks (198 workgroups) 4.2 10.7 / 6.8 14.0, 5000 (322) 6.4 19.8 / 6.9 14.8;
    // 450 rows, 64 ranks (152) 4.2 9.7 / 5.3 18.6, 2000 (540) 8.1 25.2 / 5.1 18.8; 1500 rows of 300, 64 ranks 28 61 / 9.8 65.
    const int32_t cols = (a.R + kFewRanks - 1) / kFewRanks;
    if (far || row_tiles_likely(a.rows, a.A, kFewRows) * cols <= kCus)
        return launch_traced("adapter_low", adapter_low_few_kernel, low_grid(a, kFewRows, cols), kFewWaves * 64, stream, a);
    return a.R <= 32 ? launch_rows(a, stream) : launch_tiles<false>(a, stream);
}

}  // namespace ep
