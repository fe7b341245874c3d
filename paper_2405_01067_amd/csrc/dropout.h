// Dropout whose mask is a function of (seed, offset, place) and is never stored: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", 2011), a block of 128 bits for eight elements, 16 bits each.  Ten rounds are 20 products of 32 x 32 bits, at a quarter of the vector rate: with
// 32 bits per element the generator took longer than memory for a bf16 tensor.
#pragma once

#include <math.h>

#include "common.h"

namespace abt {

struct Drop {
    const uint64_t* state;        // device: seed, offset; NULL: nothing is dropped
    uint64_t site;
    uint32_t threshold;           // an element is kept where its 16 bits are this or more
    float scale;                  // of the kept ones
};
// p in [0, 1], checked by the caller; nothing is dropped for a p that rounds to 0
inline Drop drop_of(const abt_dropout* d) {
    if (!d) return Drop{nullptr, 0, 0, 1.0f};
    const uint32_t t = (uint32_t)llround(d->p * 65536.0);
    if (t == 0) return Drop{nullptr, 0, 0, 1.0f};
    return Drop{d->state, d->site, t, t >= 65536 ? 0.0f : (float)(65536.0 / (65536.0 - t))};
}

struct DropKey { uint32_t k0, k1, c2, c3; };
__device__ __forceinline__ DropKey drop_key(const Drop& d) {
    const uint64_t seed = gload(d.state), at = gload(d.state + 1) + d.site;
    return DropKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)at, (uint32_t)(at >> 32)};
}
// the 128 bits of elements 8 block .. 8 block + 7, 16 bits each in order
__device__ __forceinline__ u32x4 drop_bits(const DropKey& key, uint64_t block) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = key.c2, c3 = key.c3, k0 = key.k0, k1 = key.k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)0xD2511F53u * c0, q = (uint64_t)0xCD9E8D57u * c2;
        c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(q >> 32), c1, k0, 0x96);          // a ^ b ^ c
        c1 = (uint32_t)q;
        c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(p >> 32), c3, k1, 0x96);
        c3 = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}
__device__ __forceinline__ bool drop_keeps(const Drop& d, const u32x4& bits, int i) { return ((bits[i >> 1] >> (16 * (i & 1))) & 0xffffu) >= d.threshold; }
// eight elements from 8 block on: 0 where dropped, whatever is there
__device__ __forceinline__ void drop8(const Drop& d, const DropKey& key, uint64_t block, float* v) {
    const u32x4 bits = drop_bits(key, block);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = drop_keeps(d, bits, i) ? v[i] * d.scale : 0.0f;
}

hipError_t launch_dropout(const void* X, const void* residual, void* Y, int64_t count, const Drop& d, bool bf16, hipStream_t s);

}  // namespace abt
