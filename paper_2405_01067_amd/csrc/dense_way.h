// Which kernels a call of the dense layer takes: rules on sizes alone (plain C++, no device code).
#pragma once

#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "int_util.h"

namespace abt {

// What a tile costs, us: a slab and the rest where a compute unit is shared by as many as fit and where one has it to itself, and an epilogue that does more than add
// the bias.  Fitted to launches of all of them at 78 shapes (1 to 50432 rows, 32 to 6144 columns and contractions), with a bias alone and with gelu and Z (which then still took a second pass behind
// the three smallest tiles, too: 0.3 us of `more` at 1379 rows).  It puts
// the ways in an order and is no time of a launch; what it takes is 2 % slower than the fastest on average (17 % at worst: 48 x 4096 x 4096).  us, bias alone:
//                      256x256   192x256   128x192   128x128   64x128    64x64   64x64 in pieces    few rows
//   48 x 4096 x 4096      82.7      67.8      47.4      40.7     37.0     21.6          11.6 (4)      18.0
//   394 x 768 x 768       20.8      17.1      12.8       8.3      7.3      6.3           8.6 (2)
//   1379 x 2304 x 768     22.4      18.0      14.5      12.0     11.6     14.6          25.4 (2)
//   12608 x 768 x 2304    57.8      49.9      51.7      62.5     57.9     72.3
//   12608 x 2304 x 768    53.1      61.1      54.6      58.3     67.0     83.7
//   8190 x 4096 x 4096     224       263       262       268      340      418                              1230 TFLOP/s
// A slab costs what its bytes do: by these costs 50 to 70 KB a us for a compute unit, and times did not change with the depth of the ring (up to eight slabs) or the number of waves; so large
// tiles win where they fill the chip.
struct DenseTileCost { int tm, tn, per_cu; float slab, rest, alone_slab, alone_rest, more; };
constexpr DenseTileCost kDenseTiles[] = {{256, 256, 1, 0.99f, 6.24f, 1.24f, 5.74f, 9.5f},  {192, 256, 1, 1.07f, 4.76f, 1.07f, 4.76f, 7.2f}, {128, 192, 2, 0.79f, 2.74f, 0.68f, 4.88f, 4.1f},
                               {128, 128, 2, 0.51f, 3.07f, 0.68f, 3.07f, 2.4f}, {64, 128, 3, 0.35f, 1.37f, 0.53f, 2.77f, 1.5f},  {64, 64, 3, 0.25f, 0.89f, 0.28f, 3.02f, 0.6f}};
constexpr int kDenseSmallest = 5, kDenseFew = -1;
inline float dense_tile_cost(const DenseTileCost& t, int64_t M, int Q, int K, int pieces, bool more) {
    const float tiles = (float)(ceil_div(M, t.tm) * ceil_div(Q, t.tn) * pieces), slabs = (float)ceil_div(ceil_div(K, 64), pieces), e = more ? t.more : 0.0f;
    const float shared = ceilf(tiles / 256.0f) * (slabs * t.slab + t.rest + e), alone = ceilf(tiles / (256.0f * (float)t.per_cu)) * (slabs * t.alone_slab + t.alone_rest + e);
    return shared > alone ? shared : alone;
}
// Which tile, or kDenseFew, and in how many pieces
struct DenseWay { int tile, pieces; float cost; };
inline DenseWay dense_way(int64_t M, int Q, int K, bool more) {
    DenseWay best{0, 1, dense_tile_cost(kDenseTiles[0], M, Q, K, 1, more)};
    auto offer = [&](int tile, int pieces, float cost) {
        if (cost < best.cost) best = DenseWay{tile, pieces, cost};
    };
    for (int i = 1; i <= kDenseSmallest; ++i) offer(i, 1, dense_tile_cost(kDenseTiles[i], M, Q, K, 1, more));
    // four slabs a piece or more; the join is a launch and its bytes
    for (int pieces : {2, 3, 4, 6, 8})
        if (4 * pieces <= (K + 63) / 64)
            offer(kDenseSmallest, pieces, dense_tile_cost(kDenseTiles[kDenseSmallest], M, Q, K, pieces, false) + 2.8f + 0.35e-6f * (float)M * (float)Q * (float)(8 * pieces + (more ? 4 : 2)));
    if (M <= 64) {                                        // bytes of a work-group at 35 KB a us
        const float rows = (float)(M <= 16 ? 16 : M <= 32 ? 32 : 64), blocks = (float)Q / 4096.0f;
        offer(kDenseFew, 1, 2.8f + (16.0f + rows) * 2.0f * (float)K / 35e3f * (blocks < 1.0f ? 1.0f : blocks));
    }
    return best;
}
// workspace: as many floats as pieces times results
inline size_t dense_part_bytes(int64_t M, int Q, int K) {
    const int a = dense_way(M, Q, K, false).pieces, b = dense_way(M, Q, K, true).pieces, pieces = a > b ? a : b;
    return pieces == 1 ? 0 : (size_t)pieces * (size_t)M * (size_t)Q * 4;
}

struct GradOrder { int col_tiles, tiles, splits, slabs; };       // pieces of the rows and their length in slabs
// What a tile of dW costs, us, as kDenseTiles has it for the forward: a slab and what each value adds to it, the rest, the same where a work-group has the compute
// unit to itself, and the sum of the partials as a launch and per million of them.  Fitted to launches of all three in 1 to 32 pieces of the rows at 48 shapes with one to three values (24 to 12608
// rows, 32 to 5920 columns; 650 times); what the rule takes is 2 % slower than the fastest on average (26 % at worst: 1156 rows, 1200 x 480).  us (pieces), three values / one, with the sum of the pieces:
//                                   256                 128                 64
//   394 rows, 768 x 768          25.5 (3) / 20.4     17.0 (3) / 10.2      9.6 (1) / 7.2
//   2000 rows, 1024 x 1024       41.6 (7) / 33.4     29.6 (4) / 24.8     30.2 (2) / 28.9
//   11737 rows, 352 x 3112        113 (9) / 70        110 (6) / 58        140 (5) / 75
//   12608 rows, 2304 x 768        140 (9) / 76        168 (7) / 80        199 (4) / 161       1040 TFLOP/s (three products of 45 GFLOP)
//   4096 rows, 4096 x 4096        326 (1) / 141       411 (1) / 170       532 (1) / 347       1270 TFLOP/s
struct DenseGradCost { int t, per_cu; float slab, value, rest, alone_slab, alone_value, alone_rest, join, partial; };
constexpr DenseGradCost kDenseGrads[] = {{256, 1, 0.67f, 0.095f, 0.0f, 0.20f, 0.55f, 6.1f, 1.6f, 2.07f}, {128, 2, 0.04f, 0.216f, 1.0f, 0.23f, 0.185f, 4.1f, 1.8f, 2.15f},
                               {64, 3, 0.13f, 0.037f, 2.45f, 0.15f, 0.079f, 3.9f, 1.7f, 0.98f}};
struct GradWay { int tile; GradOrder order; float cost; };
inline GradOrder grad_order(int t, int64_t M, int m, int n, int64_t splits) {
    const int64_t slabs = ceil_div(M, 32), each = ceil_div(slabs, splits);
    return GradOrder{(int)ceil_div(n, t), (int)(ceil_div(m, t) * ceil_div(n, t)), (int)ceil_div(slabs, each), (int)each};
}
inline float grad_cost(const DenseGradCost& t, const GradOrder& o, int m, int n, int values) {
    const float groups = (float)o.tiles * (float)o.splits, slabs = (float)o.slabs, v = (float)values;
    const float shared = ceilf(groups / 256.0f) * (slabs * (t.slab + v * t.value) + t.rest);
    const float alone = ceilf(groups / (256.0f * (float)t.per_cu)) * (slabs * (t.alone_slab + v * t.alone_value) + t.alone_rest);
    return (shared > alone ? shared : alone) + (o.splits > 1 ? t.join + 1e-6f * t.partial * (float)o.splits * (float)m * (float)n : 0.0f);
}
inline GradWay grad_way(int64_t M, int m, int n, int values) {
    GradWay best{0, {}, 1e30f};
    for (int i = 0; i < 3; ++i)
        for (int64_t splits = 1; splits <= 32 && (splits == 1 || splits * 4 <= ceil_div(M, 32)); ++splits) {
            const GradOrder o = grad_order(kDenseGrads[i].t, M, m, n, splits);
            const float c = grad_cost(kDenseGrads[i], o, m, n, values);
            if (c < best.cost) best = GradWay{i, o, c};
        }
    return best;
}

// dX [M, n] by a contraction of K, dW [m, n] and dbias of few rows in one launch (dense_few_rows_kernel)?
// Together: the longest work-group, or what all of them keep the chip busy; apart: one after the other.  Of 26 shapes (8 to 4000 rows) with three values and with one, what this takes is the faster, or
// 2 % slower (14 % once: 64 rows, 4096 x 4096, one value).  us of the whole backward, together / apart, three values: 394 rows, 768 x 768 18.2 / 28.1; 1000 rows, 2304 x 768 44.9 / 59.2;
// 1500 rows, 512 x 512 33.4 / 29.4; 4000 rows, 256 x 256 69.3 / 27.0.
// (As if all three were wanted: what is not changes no sums.)
inline bool dense_together(int64_t M, int m, int n, int K, int values) {
    const DenseTileCost& t = kDenseTiles[kDenseSmallest];
    const float x = dense_tile_cost(t, M, n, K, 1, false), x_load = (float)(ceil_div(M, t.tm) * ceil_div(n, t.tn)) / 256.0f * ((float)((K + 63) / 64) * t.slab + t.rest);
    const DenseGradCost& u = kDenseGrads[2];
    const GradOrder o = grad_order(u.t, M, m, n, 1);
    const float w = grad_cost(u, o, m, n, values), longest = x > w ? x : w;
    const float load = x_load + (float)o.tiles / 256.0f * ((float)o.slabs * (u.slab + (float)values * u.value) + u.rest);
    const float apart = dense_way(M, n, K, false).cost + grad_way(M, m, n, values).cost + 1.7f;
    return longest < apart && 0.9f * load < apart;
}

}  // namespace abt
