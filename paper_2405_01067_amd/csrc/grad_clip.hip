// Global norm of many gradient tensors, clipping by it, and the optimiser step on clipped gradients:
//     N = sqrt(sum over all tensors of g^2),   c = max_norm / N where N > max_norm, else 1,   g' = c g
// Two passes over the gradients, as c is known only after the first: one launch sums squares (256 work-groups at most, so that
// whoever needs N afterwards adds up one value per thread), the next takes the sums, forms c and scales, or runs the AdamW step on
// c g without writing c g.  Squares are added in fp64: no overflow or underflow of a square, and the rate of fp64 is far
// above that of the loads.  Every sum has a fixed order.  Both passes are bound by memory where there is much of it: 36 tensors of 19 M elements 25.2 us (76 MB, 3.0 TB/s, what the
// step before left in the last-level cache included); 6 tensors of 100 thousand elements 4.3 and 4.5 us, a load, the sum and a launch.
#include <climits>

#include "grad_clip.h"

namespace abt {
namespace {

constexpr int kSumThreads = 1024;
constexpr int kSumChunk = 16 * 1024;           // elements that a work-group takes at a time
constexpr int kThreads = 256;
constexpr int kChunk = kThreads * 16;

// The tensor that a chunk belongs to: the last one with first <= chunk (tensors without elements are not in the table).
__device__ __forceinline__ int tensor_of(const int* first, int n, int chunk) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

// 256 work-groups at most, work-group b takes chunks b, b + gridDim.x, ..: each thread sixteen elements of a chunk as whole 16-byte loads.
__global__ __launch_bounds__(kSumThreads) void sum_squares_kernel(const GradTable a, int chunks, double* sums) {
    double sum = 0.0;
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int ti = tensor_of(a.first, a.n, c);
        const int64_t base = (int64_t)(c - a.first[ti]) * kSumChunk, left = a.count[ti] - base;
        const int here = left < kSumChunk ? (int)left : kSumChunk;
        if ((a.bf16[ti >> 6] >> (ti & 63)) & 1) {
            const uint16_t* const g = static_cast<const uint16_t*>(a.grad[ti]) + base;
            u32x4 v[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = (i * kSumThreads + (int)threadIdx.x) * 8;
                v[i] = e + 8 <= here ? gload(reinterpret_cast<const u32x4*>(g + e)) : u32x4{0, 0, 0, 0};
                if (e < here && e + 8 > here)
                    for (int j = e; j < here; ++j) { const double x = bf16_value(gload(g + j)); sum += x * x; }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const double x = bf16_value(v[i][j] & 0xffffu), y = __builtin_bit_cast(float, v[i][j] & 0xffff0000u);
                    sum += x * x;
                    sum += y * y;
                }
        } else {
            const float* const g = static_cast<const float*>(a.grad[ti]) + base;
            f32x4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = (i * kSumThreads + (int)threadIdx.x) * 4;
                v[i] = e + 4 <= here ? gload(reinterpret_cast<const f32x4*>(g + e)) : f32x4{0, 0, 0, 0};
                if (e < here && e + 4 > here)
                    for (int j = e; j < here; ++j) { const double x = gload(g + j); sum += x * x; }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) { const double x = v[i][j]; sum += x * x; }
        }
    }
    __shared__ double part[kSumThreads / 64];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < kSumThreads / 64; ++i) s += part[i];
        sums[blockIdx.x] = s;
    }
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double* sums, int nsums, float* norm_out) {
    const double N = norm_of(sums, nsums);
    if (threadIdx.x == 0) *norm_out = (float)N;
}

// Loads are issued before the sums are looked at.
__global__ __launch_bounds__(kThreads) void clip_kernel(const GradTable a, const double* sums, int nsums, double max_norm, float* norm_out) {
    const int ti = tensor_of(a.first, a.n, blockIdx.x);
    const int64_t base = (int64_t)((int)blockIdx.x - a.first[ti]) * kChunk, left = a.count[ti] - base;
    const int here = left < kChunk ? (int)left : kChunk;
    if ((a.bf16[ti >> 6] >> (ti & 63)) & 1) {
        const uint16_t* const g = static_cast<const uint16_t*>(a.grad[ti]) + base;
        uint16_t* const o = static_cast<uint16_t*>(a.out[ti]) + base;
        u32x4 v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = (i * kThreads + (int)threadIdx.x) * 8;
            if (e + 8 <= here) v[i] = gload(reinterpret_cast<const u32x4*>(g + e));
        }
        const double N = norm_of(sums, nsums);
        const ClipFactor c = clip_factor(N, max_norm);
        if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)N;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = (i * kThreads + (int)threadIdx.x) * 8;
            if (e + 8 <= here) {
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = pack2_bf16(c(bf16_value(v[i][j] & 0xffffu)), c(__builtin_bit_cast(float, v[i][j] & 0xffff0000u)));
                gstore(reinterpret_cast<u32x4*>(o + e), w);
            } else {
                for (int j = e; j < here; ++j) gstore(o + j, (uint16_t)(pack2_bf16(c(bf16_value(gload(g + j))), 0.0f) & 0xffffu));
            }
        }
    } else {
        const float* const g = static_cast<const float*>(a.grad[ti]) + base;
        float* const o = static_cast<float*>(a.out[ti]) + base;
        f32x4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = (i * kThreads + (int)threadIdx.x) * 4;
            if (e + 4 <= here) v[i] = gload(reinterpret_cast<const f32x4*>(g + e));
        }
        const double N = norm_of(sums, nsums);
        const ClipFactor c = clip_factor(N, max_norm);
        if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)N;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = (i * kThreads + (int)threadIdx.x) * 4;
            if (e + 4 <= here) {
                gstore(reinterpret_cast<f32x4*>(o + e), f32x4{c(v[i][0]), c(v[i][1]), c(v[i][2]), c(v[i][3])});
            } else {
                for (int j = e; j < here; ++j) gstore(o + j, c(gload(g + j)));
            }
        }
    }
}

}  // namespace

int grad_sums_capacity(int n) { return 256 * (n < 1 ? 1 : (int)ceil_div(n, kGradMaxTensors) + 1); }

hipError_t launch_grad_sums(const GradTensor* t, int n, double* sums, int* nsums, hipStream_t s) {
    GradTables tables(t, n);
    GradTable a;
    int chunks, used = 0;
    const int room = grad_sums_capacity(n);
    while (tables.next(a, kSumChunk, INT_MAX - 256, chunks)) {
        const int blocks = chunks < 256 ? chunks : 256;
        if (used + blocks > room) return hipErrorInvalidValue;
        hipLaunchKernelGGL(sum_squares_kernel, dim3((unsigned)blocks), dim3(kSumThreads), 0, s, a, chunks, sums + used);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        used += blocks;
    }
    *nsums = used;
    return hipSuccess;
}

hipError_t launch_grad_norm(const double* sums, int nsums, float* norm_out, hipStream_t s) {
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, s, sums, nsums, norm_out);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const GradTensor* t, int n, const double* sums, int nsums, double max_norm, float* norm_out, hipStream_t s) {
    GradTables tables(t, n);
    GradTable a;
    int chunks;
    bool any = false;
    while (tables.next(a, kChunk, kGradMaxBlocks, chunks)) {
        hipLaunchKernelGGL(clip_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, s, a, sums, nsums, max_norm, any ? nullptr : norm_out);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        any = true;
    }
    if (!any && norm_out) return launch_grad_norm(sums, nsums, norm_out, s);
    return hipSuccess;
}

}  // namespace abt
