// Operands of the products with an adapter's factors.
#pragma once

#include "common.h"

namespace abt {
namespace {

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
typedef __attribute__((ext_vector_type(8))) int i32x8;
__device__ __forceinline__ i32x8 pair(u32x4 a, u32x4 b) { return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]}; }
// Products of 8-bit floats are added eight at a time, each cut at 2^-13 of the largest of the eight (also by the other 8-bit forms; bf16 keeps fp32): up to 1.7e-5 of
// the sum of the sizes was measured, next to 6 % in either operand's rounding.  The results may only be used where all lanes go: the compiler
// moves these instructions, unlike those for bf16, into a branch that holds all its uses, where only that branch's lanes would get operands.
__device__ __forceinline__ f32x16 mfma_f8(u32x4 a0, u32x4 a1, u32x4 b0, u32x4 b1, f32x16 c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(pair(a0, a1), pair(b0, b1), c, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);       // scales of 2^0
}
__device__ __forceinline__ f32x4 mfma16_f8(u32x4 a0, u32x4 a1, u32x4 b0, u32x4 b1, f32x4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(pair(a0, a1), pair(b0, b1), c, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
}

// the first `valid` of eight bf16 values, zeros behind them (all of them from eight on, none below one)
__device__ __forceinline__ u32x4 first_of(u32x4 v, int valid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= valid >= 2 * i + 2 ? 0xffffffffu : valid == 2 * i + 1 ? 0xffffu : 0u;
    return v;
}

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
