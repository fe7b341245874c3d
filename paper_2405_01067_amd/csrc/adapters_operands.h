// Operands of the products with an adapter's factors.
#pragma once

#include "common.h"

namespace abt {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// The rows of other adapters enter an adapter's product as zeros, and zero times an infinity or NaN is NaN.  So is this sum of zero times each of
// eight bf16 values; else it is 0.
__device__ __forceinline__ float zero_times(u32x4 v) {
    const uint32_t a = v[0], b = v[1], c = v[2], d = v[3];
    const auto add = [](uint32_t two, float sum) { return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), bf16x2{0, 0}, sum, false); };
    return add(a, add(b, 0.0f)) + add(c, add(d, 0.0f));
}
__device__ __forceinline__ bool any_not_finite(float found) { return __ballot(found != 0.0f) != 0; }
// infinities and NaN as zeros
__device__ __forceinline__ u32x4 finite_of(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= ((v[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((v[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
    return v;
}

}  // namespace
}  // namespace abt
