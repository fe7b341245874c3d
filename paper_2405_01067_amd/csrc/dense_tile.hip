// Y = residual + drop(act(X W^T + bias)) for many rows: tiles of the product whose epilogue runs in the accumulators.  The residual comes straight to LDS
// while activation and mask are computed, and results and the sum before the activation leave through LDS as whole rows.
// Where the tiles are few, work-groups share out the contraction too and a second launch adds their sums up and does the epilogue.
// Bound by what reaches a compute unit and by the matrix unit's clock under load: 8190 rows, 4096 x 4096, 233 us (1180 TFLOP/s; 1410 for the library's product alone); 12608 rows, 768 x 2304,
// dropout and residual 56 us (800 TFLOP/s; the library's product alone 57); 48 rows, 4096 x 4096, four pieces, 10 + 4 us.  The epilogue costs 15 us of vector work for 29 million gelus
// (12608 x 2304), which two work-groups per compute unit hide in part: hence the tiles' third cost.
#include <climits>

#include "dense_tile.h"
#include "vec8.h"

namespace abt {
namespace {

template <class L, int PER_CU>
__global__ __launch_bounds__(64 * L::NW, PER_CU * L::NW / 4) void dense_kernel(const DenseProduct g, const Order order) {
    extern __shared__ __align__(1024) unsigned char lds[];
    dense_tile<L, false>(g, order, xcd_order(blockIdx.x, gridDim.x), 0, lds);
}
template <class L, int PER_CU>
__global__ __launch_bounds__(64 * L::NW, PER_CU * L::NW / 4) void dense_parts_kernel(const DenseProduct g, const Order order) {
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tiles = order.row_tiles * order.col_tiles, w = xcd_order(blockIdx.x, gridDim.x);
    dense_tile<L, true>(g, order, w % tiles, w / tiles, lds);
}

// The epilogue of a product that lies in parts, eight columns of a row per thread
__global__ __launch_bounds__(256) void dense_join_kernel(const DenseProduct g, int pieces) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, size = g.M * g.Q;
    if (i >= size) return;
    const int c = (int)(i % g.Q);
    float v[8], more[8], bias[8];
    if (g.residual) load8<true>(g.residual, i, more);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = bias[k] = 0.0f;
    if (g.bias) load8<false>(g.bias, c, bias);
    for (int p = 0; p < pieces; p += 4) {                 // four pieces on their way at a time
        Raw8<false> x[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = raw8<false>(g.parts, (p + q < pieces ? p + q : p) * size + i);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float part[8];
            values<false>(x[q], part);
            if (p + q < pieces)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] += part[k];
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = v[k] * g.alpha + bias[k];
    if (g.Z) store8<true>(g.Z, i, v);
    with_activation(g.act, [&](auto act) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = activate<decltype(act)::value>(v[k]);
    });
    if (g.drop.state) drop8(g.drop, drop_key(g.drop), (uint64_t)i >> 3, v);
    if (g.residual)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += more[k];
    store8<true>(g.Y, i, v);
}

using T256x256 = Tile<256, 256, 2, 4, 1>;
using T192x256 = Tile<192, 256, 2, 4, 1>;
using T128x192 = Tile<128, 192, 2, 2, 1>;
using T128x128 = Tile<128, 128, 2, 4, 1>;
using T64x128 = Tile<64, 128, 2, 2, 1>;
using T64x64 = Tile<64, 64, 2, 2, 2>;

template <class L, int PER_CU>
hipError_t launch_tile(const DenseProduct& p, hipStream_t s) {
    static std::atomic<bool> attr_set{false};
    const hipError_t e = lds_allowed(reinterpret_cast<const void*>(&dense_kernel<L, PER_CU>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    const int64_t rt = ceil_div(p.M, L::TM), ct = ceil_div(p.Q, L::TN);
    if (rt * ct > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((dense_kernel<L, PER_CU>), dim3((unsigned)(rt * ct)), dim3(64 * L::NW), L::lds, s, p, Order{(int)rt, (int)ct});
    return hipGetLastError();
}
hipError_t launch_pieces(DenseProduct p, int pieces, hipStream_t s) {
    using L = T64x64;
    static std::atomic<bool> attr_set{false};
    hipError_t e = lds_allowed(reinterpret_cast<const void*>(&dense_parts_kernel<L, 3>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    const int slabs = (p.K + 63) / 64;
    p.piece = (slabs + pieces - 1) / pieces;
    pieces = (slabs + p.piece - 1) / p.piece;
    const int64_t rt = ceil_div(p.M, L::TM), ct = ceil_div(p.Q, L::TN), blocks = ceil_div(p.M * p.Q, 2048);
    if (rt * ct * pieces > INT_MAX || blocks > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((dense_parts_kernel<L, 3>), dim3((unsigned)(rt * ct * pieces)), dim3(64 * L::NW), L::lds, s, p, Order{(int)rt, (int)ct});
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(dense_join_kernel, dim3((unsigned)blocks), dim3(256), 0, s, p, pieces);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dense(const DenseProduct& p, hipStream_t s) {
    const DenseWay w = dense_way(p.M, p.Q, p.K, p.Z || p.residual || p.drop.state || p.act > ABT_ACT_RELU);
    if (w.pieces > 1) return launch_pieces(p, w.pieces, s);
    switch (w.tile) {
        case kDenseFew: return launch_dense_few(p, s);
        case 0: return launch_tile<T256x256, 1>(p, s);
        case 1: return launch_tile<T192x256, 1>(p, s);
        case 2: return launch_tile<T128x192, 2>(p, s);
        case 3: return launch_tile<T128x128, 2>(p, s);
        case 4: return launch_tile<T64x128, 3>(p, s);
        default: return launch_tile<T64x64, 3>(p, s);
    }
}

}  // namespace abt
