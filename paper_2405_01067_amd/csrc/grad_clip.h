// What the two kernels share that use the global norm of the gradients: the norm from the partial sums, and the factor.
#pragma once

#include "common.h"

namespace abt {

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// N from the sums, by every work-group of 256 threads for itself (all of its threads call)
__device__ __forceinline__ double norm_of(const double* sums, int nsums) {
    __shared__ double part[4];
    double v = 0.0;
    for (int i = threadIdx.x; i < nsums; i += 256) v += gload(sums + i);
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return sqrt(part[0] + part[1] + part[2] + part[3]);
}

// As it is reported, in fp32: the caller has to see what happened.  (False for NaN too.)
__device__ __forceinline__ bool norm_finite(double N) { return (float)N <= 3.4028234663852886e38f; }
// The factor as a product: where fp32 would hold it with fewer bits (below 2^-126), `second` is a power of two, otherwise 1.
struct ClipFactor {
    float first, second;
    __device__ __forceinline__ float operator()(float g) const { return first * g * second; }
};
// A norm that is not finite scales nothing.
__device__ __forceinline__ ClipFactor clip_factor(double N, double max_norm) {
    const double c = N > max_norm && norm_finite(N) ? max_norm / N : 1.0;
    return c < 0x1p-126 ? ClipFactor{(float)(c * 0x1p126), 0x1p-126f} : ClipFactor{(float)c, 1.0f};
}

}  // namespace abt
