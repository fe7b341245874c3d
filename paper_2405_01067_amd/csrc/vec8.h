// Eight consecutive values of bf16 or fp32, as they lie and as fp32.
#pragma once

#include "common.h"

namespace abt {

template <bool BF16>
struct Raw8 { uint32_t w[BF16 ? 4 : 8]; };

template <bool BF16>
__device__ __forceinline__ Raw8<BF16> raw8(const void* p, int64_t i) {
    Raw8<BF16> r;
#pragma unroll
    for (int h = 0; h < (BF16 ? 1 : 2); ++h) {
        const u32x4 v = gload(reinterpret_cast<const u32x4*>((const char*)p + i * (BF16 ? 2 : 4)) + h);
#pragma unroll
        for (int k = 0; k < 4; ++k) r.w[4 * h + k] = v[k];
    }
    return r;
}
template <bool BF16>
__device__ __forceinline__ void values(const Raw8<BF16>& r, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
        v[k] = BF16 ? __builtin_bit_cast(float, k & 1 ? r.w[k >> 1] & 0xffff0000u : r.w[k >> 1] << 16) : __builtin_bit_cast(float, r.w[k & (BF16 ? 3 : 7)]);
}
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t i, float (&v)[8]) { values<BF16>(raw8<BF16>(p, i), v); }
template <bool BF16>
__device__ __forceinline__ void store8(void* p, int64_t i, const float (&v)[8]) {
    if (BF16) {
        gstore(reinterpret_cast<u32x4*>((uint16_t*)p + i), u32x4{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])});
    } else {
        gstore(reinterpret_cast<f32x4*>((float*)p + i), f32x4{v[0], v[1], v[2], v[3]});
        gstore(reinterpret_cast<f32x4*>((float*)p + i + 4), f32x4{v[4], v[5], v[6], v[7]});
    }
}

}  // namespace abt
