// Y = residual + drop(act(X W^T + bias)) for many rows: tiles of the product whose epilogue runs in the accumulators.  The residual comes straight to LDS
// while activation and mask are computed, and results and the sum before the activation leave through LDS as whole rows.
// Where the tiles are few, work-groups share out the contraction too and a second launch adds their sums up and does the epilogue.
// Bound by what reaches a compute unit and by the matrix unit's clock under load: 8190 rows, 4096 x 4096, 231 us (1190 TFLOP/s; 1410 for the library's product alone); 12608 rows, 768 x 2304,
// dropout and residual 55 us (810 TFLOP/s; the library's product alone 57); 48 rows, 4096 x 4096, four pieces, 10 + 3 us.  The epilogue costs 18 us of vector work for 29 million gelus
// (12608 x 2304), which two work-groups per compute unit hide in part: hence the tiles' third cost.
#include <climits>
#include <cmath>

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

// What a tile costs, us: a slab and the rest where a compute unit is shared by as many as fit and where one has it to itself, and an epilogue that does more than add
// the bias.  Fitted to launches of all of them at 78 shapes (1 to 50432 rows, 32 to 6144 columns and contractions), with a bias alone and with gelu and Z.  It puts
// the ways in an order and is no time of a launch; what it takes is 2 % slower than the fastest on average (17 % at worst: 48 x 4096 x 4096).  us, bias alone:
//                      256x256   192x256   128x192   128x128   64x128    64x64   64x64 in pieces    few rows
//   48 x 4096 x 4096      82.7      67.8      47.4      40.7     37.0     21.6          11.6 (4)      18.0
//   394 x 768 x 768       20.8      17.1      12.8       8.3      7.3      6.3           8.6 (2)
//   1379 x 2304 x 768     22.4      18.0      14.5      12.0     11.6     14.6          25.4 (2)
//   12608 x 768 x 2304    57.8      49.9      51.7      62.5     57.9     72.3
//   12608 x 2304 x 768    53.1      61.1      54.6      58.3     67.0     83.7
//   8190 x 4096 x 4096     224       263       262       268      340      418                              1230 TFLOP/s
// A slab costs what its bytes do: some 50 KB a us reach a compute unit, whatever the tile, the depth of the ring (up to eight slabs) or the number of waves; so large tiles
// win where they fill the chip.
struct TileCost { int tm, tn, per_cu; float slab, rest, alone_slab, alone_rest, more; };
constexpr TileCost kTiles[] = {{256, 256, 1, 0.99f, 6.24f, 1.24f, 5.74f, 9.5f},  {192, 256, 1, 1.07f, 4.76f, 1.07f, 4.76f, 7.2f}, {128, 192, 2, 0.79f, 2.74f, 0.68f, 4.88f, 4.1f},
                               {128, 128, 2, 0.51f, 3.07f, 0.68f, 3.07f, 2.4f}, {64, 128, 3, 0.35f, 1.37f, 0.53f, 2.77f, 1.5f},  {64, 64, 3, 0.25f, 0.89f, 0.28f, 3.02f, 0.6f}};
constexpr int kSmallest = 5, kFew = -1;
float tile_cost(const TileCost& t, int64_t M, int Q, int K, int pieces, bool more) {
    const float tiles = (float)(ceil_div(M, t.tm) * ceil_div(Q, t.tn) * pieces), slabs = (float)ceil_div(ceil_div(K, 64), pieces), e = more ? t.more : 0.0f;
    const float shared = ceilf(tiles / 256.0f) * (slabs * t.slab + t.rest + e), alone = ceilf(tiles / (256.0f * (float)t.per_cu)) * (slabs * t.alone_slab + t.alone_rest + e);
    return shared > alone ? shared : alone;
}
// Which tile, or kFew, and in how many pieces
struct Way { int tile, pieces; float cost; };
Way way_of(int64_t M, int Q, int K, bool more) {
    Way best{0, 1, tile_cost(kTiles[0], M, Q, K, 1, more)};
    auto offer = [&](int tile, int pieces, float cost) {
        if (cost < best.cost) best = Way{tile, pieces, cost};
    };
    for (int i = 1; i <= kSmallest; ++i) offer(i, 1, tile_cost(kTiles[i], M, Q, K, 1, more));
    // four slabs a piece or more; the join is a launch and its bytes
    for (int pieces : {2, 3, 4, 6, 8})
        if (4 * pieces <= (K + 63) / 64)
            offer(kSmallest, pieces, tile_cost(kTiles[kSmallest], M, Q, K, pieces, false) + 2.8f + 0.35e-6f * (float)M * (float)Q * (float)(8 * pieces + (more ? 4 : 2)));
    if (M <= 64) {                                        // bytes of a work-group at 35 KB a us
        const float rows = (float)(M <= 16 ? 16 : M <= 32 ? 32 : 64), blocks = (float)Q / 4096.0f;
        offer(kFew, 1, 2.8f + (16.0f + rows) * 2.0f * (float)K / 35e3f * (blocks < 1.0f ? 1.0f : blocks));
    }
    return best;
}

}  // namespace

size_t dense_part_bytes(int64_t M, int Q, int K) {
    const int a = way_of(M, Q, K, false).pieces, b = way_of(M, Q, K, true).pieces, pieces = a > b ? a : b;
    return pieces == 1 ? 0 : (size_t)pieces * (size_t)M * (size_t)Q * 4;
}
float dense_cost(int64_t M, int Q, int K) { return way_of(M, Q, K, false).cost; }
SmallCost dense_small_cost(int64_t M, int Q, int K) {
    const TileCost& t = kTiles[kSmallest];
    return SmallCost{tile_cost(t, M, Q, K, 1, false), (float)(ceil_div(M, t.tm) * ceil_div(Q, t.tn)) / 256.0f * ((float)((K + 63) / 64) * t.slab + t.rest)};
}
hipError_t launch_dense(const DenseProduct& p, hipStream_t s) {
    const Way w = way_of(p.M, p.Q, p.K, p.Z || p.residual || p.drop.state || p.act > ABT_ACT_RELU);
    if (w.pieces > 1) return launch_pieces(p, w.pieces, s);
    switch (w.tile) {
        case kFew: return launch_dense_few(p, s);
        case 0: return launch_tile<T256x256, 1>(p, s);
        case 1: return launch_tile<T192x256, 1>(p, s);
        case 2: return launch_tile<T128x192, 2>(p, s);
        case 3: return launch_tile<T128x128, 2>(p, s);
        case 4: return launch_tile<T64x128, 3>(p, s);
        default: return launch_tile<T64x64, 3>(p, s);
    }
}

}  // namespace abt
