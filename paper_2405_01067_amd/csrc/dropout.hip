// Dropout by itself: Y = residual + drop(X), eight elements per thread and block of random bits.
// Bound by memory: 50432 x 768 in bf16 with a residual 35 us (6.6 TB/s, part of it from the last-level cache); the generator, 20 products of 16 cycles and 20 xors for 512 elements, takes
// some 12 us of the vector units beside it.
#include "dropout.h"
#include "vec8.h"

namespace abt {
namespace {

template <bool BF16>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
    return BF16 ? __builtin_bit_cast(float, (uint32_t)gload((const uint16_t*)p + i) << 16) : gload((const float*)p + i);
}

template <bool BF16>
__global__ __launch_bounds__(256) void dropout_kernel(const void* X, const void* R, void* Y, int64_t count, const Drop d) {
    const int64_t step = (int64_t)gridDim.x * 256;
    const DropKey key = d.state ? drop_key(d) : DropKey{0, 0, 0, 0};
    for (int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; 8 * b < count; b += step) {
        const int64_t i = 8 * b;
        float x[8], r[8];
        if (i + 8 <= count) {
            load8<BF16>(X, i, x);
            if (R) load8<BF16>(R, i, r);
            if (d.state) drop8(d, key, (uint64_t)b, x);
            if (R)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] += r[k];
            store8<BF16>(Y, i, x);
            continue;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {                     // the last elements
            x[k] = i + k < count ? load1<BF16>(X, i + k) : 0.0f;
            r[k] = R && i + k < count ? load1<BF16>(R, i + k) : 0.0f;
        }
        if (d.state) drop8(d, key, (uint64_t)b, x);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k < count) {
                const float v = R ? x[k] + r[k] : x[k];
                if (BF16) gstore((uint16_t*)Y + i + k, (uint16_t)pack2_bf16(v, 0.0f));
                else gstore((float*)Y + i + k, v);
            }
    }
}

}  // namespace

hipError_t launch_dropout(const void* X, const void* residual, void* Y, int64_t count, const Drop& d, bool bf16, hipStream_t s) {
    const int64_t blocks = ceil_div(count, 2048);
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
    if (bf16) hipLaunchKernelGGL((dropout_kernel<true>), grid, dim3(256), 0, s, X, residual, Y, count, d);
    else hipLaunchKernelGGL((dropout_kernel<false>), grid, dim3(256), 0, s, X, residual, Y, count, d);
    return hipGetLastError();
}

}  // namespace abt
