// Tiles of X W^T whose slabs of 128 bytes of every row come straight to LDS, as adapters.hip and dense_tile.hip use them.
#pragma once

#include "common.h"

namespace abt {
namespace {

// WM x WN waves, each RB x CB blocks of 32 x 32.  Slabs are requested AHEAD of their turn.
template <int TM_, int TN_, int WM_, int WN_, int AHEAD_>
struct Tile {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, AHEAD = AHEAD_, NW = WM * WN;
    static constexpr int RB = TM / (32 * WM), CB = TN / (32 * WN);
    static constexpr int xpart = TM * 128, wpart = TN * 128, wbase = (AHEAD + 1) * xpart, ring = wbase + (AHEAD + 1) * wpart;
    static constexpr int NX = TM / 8 / NW, NF = TN / 8 / NW, NL = NX + NF;       // load instructions per wave and slab: eight rows each
    static constexpr int opitch = TN * 2 + 16;
    static constexpr int out = TM * opitch;
    static constexpr int lds = out > ring ? out : ring;
    static constexpr int behind = (AHEAD - 1) * NL;       // loads issued after the last one of a slab
    static_assert(NX * 8 * NW == TM && NF * 8 * NW == TN && RB * 32 * WM == TM && CB * 32 * WN == TN, "");
    static_assert(NW % 2 == 0 && AHEAD >= 1 && behind < 64 && lds <= 160 * 1024, "");
};

struct Order { int row_tiles, col_tiles; };

// Work-groups go round the XCDs: of `n` each XCD gets a contiguous eighth of what they stand for.
__device__ __forceinline__ int xcd_order(int block, int n) {
    const int xcd = block & 7, per = n >> 3, rem = n & 7;
    return xcd * per + (xcd < rem ? xcd : rem) + (block >> 3);
}
// Tiles in panels of four row tiles, down the panel first: the tiles that run at the same time on one XCD share rows of X and rows of W in its L2.
__device__ __forceinline__ void tile_at(const Order& o, int w, int& rt, int& ct) {
    const int panel = w / (4 * o.col_tiles), rows = o.row_tiles - 4 * panel < 4 ? o.row_tiles - 4 * panel : 4;
    const int at = w - panel * 4 * o.col_tiles;
    rt = 4 * panel + at % rows;
    ct = at / rows;
}
__device__ __forceinline__ void tile_of(const Order& o, int block, int& rt, int& ct) { tile_at(o, xcd_order(block, o.row_tiles * o.col_tiles), rt, ct); }

}  // namespace
}  // namespace abt
