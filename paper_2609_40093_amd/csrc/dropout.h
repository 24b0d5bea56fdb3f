// dropout.h -- the mask of dropout from a counter-based generator: made where it is used, forward and
// backward, and never stored.
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel Random Numbers: As Easy as 1, 2, 3", 2011) on
// the counter (group, group >> 32, step, site) with the seed as key gives 128 bits for a group of
// eight neighbouring values, 16 for each: value i of the array is number i % 8 of group i / 8, and takes
// the low, then the high half of word (i % 8) / 2.  A value stays if its 16 bits are at least `cut`,
// so the share that is dropped is a multiple of 2^-16; the factor of the others is that share's own
// inverse, 65536 / (65536 - cut), and the mean is kept exactly.  (32 bits a value would need the generator
// twice, which at 20 multiplications of 32 bits each time would pass the time of the rows' bytes.)
#pragma once

#include "layer.h"

namespace ep {

struct DropKey {
    uint32_t k0, k1, step, site;
    __device__ __forceinline__ void load(const DropArgs &d) {
        const int64_t seed = d.rng[0];
        k0 = (uint32_t)seed;
        k1 = (uint32_t)((uint64_t)seed >> 32);
        step = (uint32_t)d.rng[1];
        site = d.site;
    }
};

// The 128 bits of a group.
__device__ __forceinline__ u32x4 philox(const DropKey &key, uint64_t group) {
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32), c2 = key.step, c3 = key.site;
    uint32_t k0 = key.k0, k1 = key.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)q;
        c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// A group's eight values: dropped ones are 0 whatever they were.
__device__ __forceinline__ void drop8(const DropKey &key, uint64_t group, uint32_t cut, float factor, float *v) {
    const u32x4 bits = philox(key, group);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (bits[i] & 0xffffu) >= cut ? v[2 * i] * factor : 0.f;
        v[2 * i + 1] = bits[i] >> 16 >= cut ? v[2 * i + 1] * factor : 0.f;
    }
}

}  // namespace ep
