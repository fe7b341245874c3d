// The products of a dense layer with adapters for many rows:
//     Y_i = W x_i + A_a T_i          T_i = B_a x_i          a = adapter of row i, T scaled where it is an operand
// Y: a tile of the dense product, then in the same accumulators the adapters that occur among its rows, one after the other, with the T of other
// adapters' rows as zeros.  Rows that lie together by adapter cost a tile one or two short passes; rows in any other order more of them.
// T: 32 rows against the B of all adapters among them, side by side as columns of one product; every row keeps those of its own.  (Of up to 1024 rows row by row.)
//
// A slab is 128 bytes of every row: 64 columns in bf16, 128 in 8 bits.  It comes straight to LDS, NS slots in a ring, one barrier per
// slab.  Both types read LDS alike: two 16-byte pieces are two bf16 operands of 32x32x16 or one 8-bit operand of 32x32x64, whose columns are taken in
// the same order on both sides.
#include <atomic>
#include <climits>

#include "adapters_grad.h"

namespace abt {
namespace {

// The smallest of the lanes' values, INT_MAX where none is left
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const int o = __shfl_xor(v, d);
        v = o < v ? o : v;
    }
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int rank_of(const AdapterProduct& g, int a) {
    const int k = g.ranks ? gload(g.ranks + a) : g.r;
    return k < 0 ? 0 : k > g.r ? g.r : k;
}

// ------------------------------------------------------------------------------------------ Y
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

// Tiles in panels of four row tiles, down the panel first; each XCD gets a contiguous eighth: the tiles that run at the same time on one
// XCD share rows of X and rows of W in its L2.
__device__ __forceinline__ void tile_of(const Order& o, int block, int& rt, int& ct) {
    const int nb = o.row_tiles * o.col_tiles, xcd = block & 7, i = block >> 3, per = nb >> 3, rem = nb & 7;
    const int w = xcd * per + (xcd < rem ? xcd : rem) + i;
    const int panel = w / (4 * o.col_tiles), rows = o.row_tiles - 4 * panel < 4 ? o.row_tiles - 4 * panel : 4;
    const int at = w - panel * 4 * o.col_tiles;
    rt = 4 * panel + at % rows;
    ct = at / rows;
}

template <class L, bool F8>
__device__ __forceinline__ void y_tile(const AdapterProduct& g, const Order& order, int block, unsigned char* lds) {
    constexpr int RB = L::RB, CB = L::CB, NW = L::NW;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lj = lane & 31, lh = lane >> 5;
    const int wr = wave / L::WN, wc = wave % L::WN;
    int rt, ct;
    tile_of(order, block, rt, ct);
    const int64_t row0 = (int64_t)rt * L::TM;
    const int col0 = ct * L::TN;
    const int rows = g.M - row0 < L::TM ? (int)(g.M - row0) : L::TM;
    const int cols = g.Q - col0 < L::TN ? g.Q - col0 : L::TN;

    // Load instruction j of a wave covers rows 8 (wave + NW j) .. + 7 of X, or of W: this lane's row among them and its chunk (NW is even, so the chunk
    // is the same for all j).  Rows past the last one read zeros, and so do chunks past the end of a row.
    const int lrow = 8 * wave + (lane >> 3);
    const int chunk = ((lane & 7) ^ ((lrow >> 1) & 7)) * 16;
    const int bytes = g.kmain * (F8 ? 1 : 2), nmain = (bytes + 127) / 128;
    const rsrc_t xres = make_rsrc((const char*)g.X + row0 * bytes, (int64_t)rows * bytes);
    const rsrc_t wres = make_rsrc((const char*)g.W + (int64_t)col0 * bytes, (int64_t)cols * bytes);
    int xslot = 0, wslot = L::wbase;                      // of the next parts to be requested
    auto offset = [&](int s) { return s * 128 + chunk < bytes ? lrow * bytes + s * 128 + chunk : kBufNowhere; };
    auto issue_x = [&](int s) {
        unsigned char* const dst = lds + xslot + wave * 1024;
        xslot = xslot == L::AHEAD * L::xpart ? 0 : xslot + L::xpart;
        const int off = offset(s), step = off == kBufNowhere ? 0 : 8 * NW * bytes;
#pragma unroll
        for (int j = 0; j < L::NX; ++j) load_lds16(xres, dst + j * (NW * 1024), off + j * step, 0);
    };
    auto issue_w = [&](int s) {
        unsigned char* const dst = lds + wslot + wave * 1024;
        wslot = wslot == L::wbase + L::AHEAD * L::wpart ? L::wbase : wslot + L::wpart;
        const int off = offset(s), step = off == kBufNowhere ? 0 : 8 * NW * bytes;
#pragma unroll
        for (int j = 0; j < L::NF; ++j) load_lds16(wres, dst + j * (NW * 1024), off + j * step, 0);
    };
#pragma unroll
    for (int s = 0; s < L::AHEAD; ++s)                    // in the order of the loop below
        if (s < nmain) {
            issue_w(s);
            issue_x(s);
        }

    // the adapters of this lane's rows
    int mine[RB];
#pragma unroll
    for (int a = 0; a < RB; ++a) {
        const int r = (wr * RB + a) * 32 + lj;
        const int id = gload(g.row_adapter + row0 + (r < rows ? r : 0));
        mine[a] = r < rows && id >= 0 && id < g.count ? id : -1;
    }

    f32x16 acc[RB][CB];
#pragma unroll
    for (int a = 0; a < RB; ++a)
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    const int frow = out_row(lj);
    const int xsw = (lj >> 1) & 7, fsw = (frow >> 1) & 7;
    const int xbase = (wr * RB * 32 + lj) * 128, fbase = (wc * CB * 32 + frow) * 128;
    struct Ops { u32x4 x[RB], f[CB]; };
    int xat = 0, wat = L::wbase;                          // the slab that is read
    auto read = [&](Ops& o, int j) {                      // chunk 2 j + lh of this lane's rows
        const unsigned char* const x = lds + xat + xbase + (((2 * j + lh) ^ xsw) * 16);
        const unsigned char* const f = lds + wat + fbase + (((2 * j + lh) ^ fsw) * 16);
#pragma unroll
        for (int b = 0; b < CB; ++b) o.f[b] = *reinterpret_cast<const u32x4*>(f + b * 4096);
#pragma unroll
        for (int a = 0; a < RB; ++a) o.x[a] = *reinterpret_cast<const u32x4*>(x + a * 4096);
    };
    auto mma = [&](const Ops& o) {
#pragma unroll
        for (int a = 0; a < RB; ++a)
#pragma unroll
            for (int b = 0; b < CB; ++b) acc[a][b] = mfma_bf16(o.f[b], o.x[a], acc[a][b]);
    };
    auto mma8 = [&](const Ops& o, const Ops& p) {
#pragma unroll
        for (int a = 0; a < RB; ++a)
#pragma unroll
            for (int b = 0; b < CB; ++b) acc[a][b] = mfma_f8(o.f[b], p.f[b], o.x[a], p.x[a], acc[a][b]);
    };
    // The adapters of this wave's rows, in ascending order.  Their operands come straight from memory, there is little of them: the first before the last slab, each
    // of the others behind the one before.
    struct Piece { int a, rank, k; };                     // sixteen columns from k on
    auto after = [&](int a) {
        int best = INT_MAX;
#pragma unroll
        for (int i = 0; i < RB; ++i) best = mine[i] > a && mine[i] < best ? mine[i] : best;
        return wave_min(best);
    };
    auto adapter = [&](int a) {                           // the next one that has a rank, from a on
        int rank = 0;
        while (a != INT_MAX && (rank = __builtin_amdgcn_readfirstlane(rank_of(g, a))) == 0) a = after(a);
        return Piece{a, rank, 0};
    };
    const rsrc_t eres = make_rsrc(g.E + row0 * g.e_pitch, (int64_t)rows * g.e_pitch * 2);
    const int eoff = ((wr * RB * 32 + lj) * g.e_pitch + 8 * lh) * 2, foff = ((wc * CB * 32 + frow) * g.ke + 8 * lh) * 2;
    Ops ahead;
    auto fetch = [&](const Piece& l) {
        const rsrc_t fres = make_rsrc(g.F + ((int64_t)l.a * g.Q + col0) * g.ke, (int64_t)cols * g.ke * 2);
        const bool there = l.k + 8 * lh < l.rank;
#pragma unroll
        for (int b = 0; b < CB; ++b) ahead.f[b] = buf_load16(fres, there ? foff + b * 64 * g.ke + 2 * l.k : kBufNowhere, 0);
#pragma unroll
        for (int i = 0; i < RB; ++i) ahead.x[i] = buf_load16(eres, there && mine[i] == l.a ? eoff + i * 64 * g.e_pitch + 2 * l.k : kBufNowhere, 0);
    };
    Piece piece = adapter(after(-1)), coming = piece.a == INT_MAX ? piece : adapter(after(piece.a));
    // Slab s has landed: loads come back in the order of issue.
    auto slab = [&](int s) {
        if (s + L::AHEAD > nmain) wait_newest<0>();
        else wait_newest<L::behind>();
        lds_barrier();
        // into the slots whose reads ended before this barrier
        if (s + L::AHEAD < nmain) {
            issue_w(s + L::AHEAD);
            issue_x(s + L::AHEAD);
        }
        if (s + 1 == nmain && piece.a != INT_MAX) fetch(piece);
    };
    auto next = [&]() {
        xat = xat == L::AHEAD * L::xpart ? 0 : xat + L::xpart;
        wat = wat == L::wbase + L::AHEAD * L::wpart ? L::wbase : wat + L::wpart;
    };
    Ops o[2];
    if constexpr (F8) {
        for (int s = 0; s < nmain; ++s) {
            slab(s);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                read(o[0], 2 * j);
                read(o[1], 2 * j + 1);
                mma8(o[0], o[1]);
                __builtin_amdgcn_sched_barrier(0);
            }
            next();
        }
        // the dense product's scales
        float xs[RB];
#pragma unroll
        for (int a = 0; a < RB; ++a) {
            const int r = (wr * RB + a) * 32 + lj;
            xs[a] = gload(g.x_scale + row0 + (r < rows ? r : 0));
        }
#pragma unroll
        for (int b = 0; b < CB; ++b) {
            const int c = (wc * CB + b) * 32 + 16 * lh;
#pragma unroll
            for (int h = 0; h < 2; ++h) {                 // eight columns, all there or none (m is a multiple of 8)
                f32x4 w[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
                if (c + 8 * h < cols)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int v = 0; v < 4; ++v) w[q][v] = gload(g.w_scale + col0 + c + 8 * h + 4 * q + v);
#pragma unroll
                for (int a = 0; a < RB; ++a)
#pragma unroll
                    for (int v = 0; v < 8; ++v) acc[a][b][8 * h + v] *= xs[a] * w[v >> 2][v & 3];
            }
        }
    } else {
        // the operands of a step are read while the products of the step before run, across the barrier too
#pragma unroll
        for (int a = 0; a < RB; ++a) o[1].x[a] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < CB; ++b) o[1].f[b] = u32x4{0, 0, 0, 0};
        for (int s = 0; s < nmain; ++s) {
            slab(s);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                read(o[j & 1], j);
                mma(o[(j + 1) & 1]);
#pragma unroll
                for (int i = 0; i < RB + CB; ++i) {       // a read behind every product
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            next();
        }
        mma(o[1]);
    }

    // What is left of the adapters.  Infinities and NaN in them are left out here, where the rows of other adapters are summed up too.  Looking for them
    // costs 0 to 1 % of a launch where rows lie in runs, 1 to 4 % in any order (12608 x 2304 x 768, r = 16: 0.6 and 2 us).
    bool poisoned = false;
    while (piece.a != INT_MAX) {
        const Piece now = piece;
        Ops m = ahead;
        piece.k += 16;
        if (piece.k >= piece.rank) piece = coming;
        if (piece.a != INT_MAX) fetch(piece);
        if (now.a != piece.a && piece.a != INT_MAX) coming = adapter(after(piece.a));
        if (now.rank - now.k < 16 && (now.rank & 7)) {    // columns past the rank are no part of the adapter, whatever they hold (T is zero there)
            const int valid = now.rank - now.k - 8 * lh;
            if (valid < 8)
#pragma unroll
                for (int b = 0; b < CB; ++b) m.f[b] = first_of(m.f[b], valid);
        }
        float bad = 0.0f;
#pragma unroll
        for (int b = 0; b < CB; ++b) bad += zero_times(m.f[b]);
        if (__builtin_expect(any_not_finite(bad), 0)) {
            poisoned = true;
#pragma unroll
            for (int b = 0; b < CB; ++b) m.f[b] = finite_of(m.f[b]);
        }
        mma(m);
    }

    // out through LDS as whole rows
    lds_barrier();                                        // every wave has read its last slab, and nothing is on its way to LDS
#pragma unroll
    for (int a = 0; a < RB; ++a)
#pragma unroll
        for (int b = 0; b < CB; ++b) {
            unsigned char* const d = lds + ((wr * RB + a) * 32 + lj) * L::opitch + ((wc * CB + b) * 32 + 16 * lh) * 2;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = pack2_bf16(acc[a][b][8 * h + 2 * i], acc[a][b][8 * h + 2 * i + 1]);
                *reinterpret_cast<u32x4*>(d + 16 * h) = v;
            }
        }
    // and come into the rows of their own adapter, in this wave's part of the tile
    if (__builtin_expect(poisoned, 0))
        for (piece = adapter(after(-1)); piece.a != INT_MAX; piece = adapter(after(piece.a)))
            for (; piece.k < piece.rank; piece.k += 16) {
                fetch(piece);
                const int valid = piece.rank - piece.k - 8 * lh;
                float bad = 0.0f;
#pragma unroll
                for (int b = 0; b < CB; ++b) {
                    if (valid < 8) ahead.f[b] = first_of(ahead.f[b], valid);
                    bad += zero_times(ahead.f[b]);
                    ahead.f[b] ^= finite_of(ahead.f[b]);
                }
                if (!any_not_finite(bad)) continue;
#pragma unroll
                for (int a = 0; a < RB; ++a)
#pragma unroll
                    for (int b = 0; b < CB; ++b) {
                        f32x16 sum;
#pragma unroll
                        for (int v = 0; v < 16; ++v) sum[v] = 0.0f;
                        sum = mfma_bf16(ahead.f[b], ahead.x[a], sum);
                        u32x4* const d = reinterpret_cast<u32x4*>(lds + ((wr * RB + a) * 32 + lj) * L::opitch + ((wc * CB + b) * 32 + 16 * lh) * 2);
                        if (mine[a] != piece.a) continue;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            u32x4 y = d[h];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                y[i] = pack2_bf16(__builtin_bit_cast(float, y[i] << 16) + sum[8 * h + 2 * i], __builtin_bit_cast(float, y[i] & 0xffff0000u) + sum[8 * h + 2 * i + 1]);
                            d[h] = y;
                        }
                    }
            }
    lds_barrier();
    constexpr int CPR = L::TN / 8;
    const rsrc_t yres = make_rsrc(g.Y + row0 * g.Q + col0, ((int64_t)(rows - 1) * g.Q + cols) * 2);
#pragma unroll
    for (int i = 0; i < L::TM * CPR / (64 * NW); ++i) {
        const int e = i * (64 * NW) + (int)threadIdx.x, r = e / CPR, c = e % CPR;
        buf_store16(*reinterpret_cast<const u32x4*>(lds + r * L::opitch + c * 16), yres, r < rows && c * 8 < cols ? (r * g.Q + c * 8) * 2 : kBufNowhere, 0);
    }
}

template <class L, bool F8>
__global__ __launch_bounds__(64 * L::NW) void adapters_y_kernel(const AdapterProduct g, const Order order) {
    extern __shared__ __align__(1024) unsigned char lds[];
    y_tile<L, F8>(g, order, blockIdx.x, lds);
}

template <class L, bool F8>
hipError_t launch_tile(const AdapterProduct& p, hipStream_t s) {
    static std::atomic<bool> attr_set{false};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&adapters_y_kernel<L, F8>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    const int64_t rt = ceil_div(p.M, L::TM), ct = ceil_div(p.Q, L::TN);
    if (rt * ct > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((adapters_y_kernel<L, F8>), dim3((unsigned)(rt * ct)), dim3(64 * L::NW), L::lds, s, p, Order{(int)rt, (int)ct});
    return hipGetLastError();
}

// The tiles.  Two or three work-groups of the smaller ones share a compute unit, and while one starts or stores the others compute.
using T256x256 = Tile<256, 256, 2, 4, 1>;
using T192x256 = Tile<192, 256, 2, 4, 1>;
using T128x192 = Tile<128, 192, 2, 2, 1>;
using T128x128 = Tile<128, 128, 2, 2, 1>;
using T64x128 = Tile<64, 128, 2, 2, 1>;
using T64x64 = Tile<64, 64, 2, 2, 2>;

// What a tile costs, us: a slab and the rest of a tile where the compute unit is shared by as many as fit, and where it has the unit to itself.  Fitted to
// launches of all six at 54 shapes (140 to 12608 rows, 768 to 4096 columns and contractions; r = 16, runs of 197 rows) and looked at at 49 others: what the rule takes
// is slower than the fastest by 1.0 and 1.3 % on average in bf16 (16 % at worst: 300 x 4096 x 1024), 0.1 and 0.6 % in 8 bits (11 % at worst: 900 x 3000 x 1200).  It puts
// tiles in an order and is no time of a launch: 42 for the largest tile at 12608 x 2304 x 768, 127 for the smallest.  The ends of the range, us:
//                      256x256   192x256   128x192   128x128   64x128    64x64
//   140 x 768 x 768       19.9      16.3      13.2      10.3      8.3      7.5
//   1379 x 2304 x 768     22.8      18.7      15.7      13.0     12.7     17.6
//   12608 x 768 x 2304    61.4      52.2      54.4      64.0     61.5     87.9
//   12608 x 2304 x 768    56.1      62.2      54.4      58.4     68.6     99.6
//   8190 x 4096 x 4096   223.5     242.9     262.0     248.1    316.4    419.7        1230 TFLOP/s
//     in 8 bits          130.9     145.3     203.1     135.5    169.1    217.6        2100 TFLOP/s
struct TileCost { int tm, tn, per_cu; float slab, rest, alone_slab, alone_rest; };
constexpr TileCost kTiles[2][6] = {                       // bf16; 8 bits, where 128 x 192 has registers for one work-group per compute unit only
    {{256, 256, 1, 1.27f, 5.86f, 1.27f, 5.86f}, {192, 256, 1, 0.94f, 6.01f, 0.94f, 6.01f}, {128, 192, 2, 0.55f, 2.79f, 0.61f, 5.85f},
     {128, 128, 2, 0.46f, 2.66f, 0.56f, 5.33f}, {64, 128, 3, 0.27f, 1.36f, 0.56f, 2.22f},  {64, 64, 3, 0.27f, 1.30f, 0.33f, 2.65f}},
    {{256, 256, 1, 1.38f, 7.61f, 1.38f, 7.61f}, {192, 256, 1, 1.18f, 6.65f, 1.18f, 6.65f}, {128, 192, 1, 0.88f, 7.95f, 0.88f, 7.95f},
     {128, 128, 2, 0.39f, 3.66f, 0.54f, 5.92f}, {64, 128, 3, 0.26f, 2.66f, 0.46f, 4.61f},  {64, 64, 3, 0.165f, 1.64f, 0.33f, 4.48f}}};
constexpr int kTile128x192 = 2, kTile64 = 5;
float tile_cost(int i, const AdapterProduct& p, bool fp8) {
    const TileCost& t = kTiles[fp8][i];
    const int64_t tiles = ceil_div(p.M, t.tm) * ceil_div(p.Q, t.tn);
    const float slabs = (float)ceil_div((int64_t)p.kmain * (fp8 ? 1 : 2), 128);
    const float shared = (float)ceil_div(tiles, 256) * (slabs * t.slab + t.rest), alone = (float)ceil_div(tiles, 256 * t.per_cu) * (slabs * t.alone_slab + t.alone_rest);
    return shared > alone ? shared : alone;
}
int best_tile(const AdapterProduct& p, bool fp8) {
    int best = 0;
    for (int i = 1; i <= kTile64; ++i)
        if (tile_cost(i, p, fp8) < tile_cost(best, p, fp8)) best = i;
    return best;
}
template <bool F8>
hipError_t launch_y(const AdapterProduct& p, hipStream_t s) {
    switch (best_tile(p, F8)) {
        case 0: return launch_tile<T256x256, F8>(p, s);
        case 1: return launch_tile<T192x256, F8>(p, s);
        case 2: return launch_tile<T128x192, F8>(p, s);
        case 3: return launch_tile<T128x128, F8>(p, s);
        case 4: return launch_tile<T64x128, F8>(p, s);
        default: return launch_tile<T64x64, F8>(p, s);
    }
}

// dX and the factor gradients in one launch, the tiles of dX first: of few rows neither fills the chip; of many one is bound by the matrix unit and the
// other by memory, and a work-group of each fits a compute unit beside the other.
// 12608 x 2304 x 768, r = 16: 61 us for both (dX alone 51, the gradients 24.5); 394 x 768 x 768, r = 8: 7.9.
template <class L, int VB>
__global__ __launch_bounds__(256, 2) void adapters_dx_grad_kernel(const AdapterProduct x, const Order order, const AdapterGrads g, const Side a, const Side b, int piece) {
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tiles = order.row_tiles * order.col_tiles, blocks = a.blocks + b.blocks, i = (int)blockIdx.x - tiles;
    if (i < 0) y_tile<L, false>(x, order, blockIdx.x, lds);
    else grad_block<VB>(g, a, b, i % blocks, piece, i / blocks, lds);
}
// piece = 0: whole adapters
template <class L, int VB>
hipError_t launch_dx_grads(const AdapterProduct* x, const AdapterGrads& g, int piece, hipStream_t s) {
    constexpr int lds = L::lds > Grad<VB>::lds ? L::lds : Grad<VB>::lds;
    static std::atomic<bool> attr_set{false};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&adapters_dx_grad_kernel<L, VB>), lds, attr_set);
    if (e != hipSuccess) return e;
    const int64_t pieces = piece ? ceil_div(g.M, piece) : g.count;
    Side a, b;
    grad_sides(g, pieces + g.count, a, b);
    const Order order{x ? (int)ceil_div(g.M, L::TM) : 0, x ? (int)ceil_div(x->Q, L::TN) : 0};
    const int64_t blocks = (int64_t)order.row_tiles * order.col_tiles + (a.blocks + b.blocks) * pieces;
    if (blocks > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((adapters_dx_grad_kernel<L, VB>), dim3((unsigned)blocks), dim3(256), lds, s, x ? *x : AdapterProduct{}, order, g, a, b, piece);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------ T
// 32 rows a work-group.  A slab is two parts of 64 columns; the four waves share out the four steps of a part and add their sums at the end, in order.  CB blocks of
// 32 columns hold 32 CB / r adapters; rows of more adapters than that take another pass over their x.
// PLANES: the backward's dT_i = A_a^T dY_i.  A lies with the contraction first, [m, r]: parts of 64 rows of the adapters' A, one behind the other as they lie
// in memory, read with the transposing load.
// Bound by memory where there are many rows and one adapter or two in 32 of them, otherwise by latency: 5 us for the first load, the sums and the launch, then
// 0.14 us (r = 16 or 32) to 0.22 us (112) a part of 64 columns while only one work-group shares the compute unit.  One part per slab, each read followed by its
// product, took 0.19 to 0.27 us.  us, T / dT: 12608 rows of 768 in runs of 64, r = 32: 12.2 / 14.0 (one part: 13.3 / 16.4), r = 128: 33.6 / 47.6 (36.4 /
// 59.2); 1379 x 768, r = 32, runs of 7: 12.7 / 16.0 (14.2 / 19.0); 8190 x 4096, r = 32, one adapter: 21.6 / 20.9, 3.1 TB/s (21.9 / 23.8).
template <int CB_, int NS_>
struct Low {
    static constexpr int CB = CB_, KS = 2, NS = NS_, TN = 32 * CB;          // KS: parts of 128 bytes a row
    static constexpr int xpart = 4096, part = xpart + TN * 128, slab = KS * part, NF = KS * CB, NL = KS + NF;
    static constexpr int sums = 3 * CB * 4096;
    static constexpr int ring = NS * slab > sums ? NS * slab : sums;
    static constexpr int lds = ring + 32 * 4 * 4;         // and the adapters, their ranks and scales, the rows' places among them
    static constexpr int per_cu = 2 * lds <= 160 * 1024 ? 2 : 1;
    static_assert((NS - 2) * NL < 64 && lds <= 160 * 1024, "");
};

// Columns k .. k + 7 of a row.  Three bf16 values that add up to the fp32 one (each takes eight bits of what the ones before left): the factor gradients
// are fp32 sums of exact products, as they would be of fp32 operands.
__device__ __forceinline__ void store_planes(uint16_t* to, int64_t row, int k, int r, const float (&u)[8]) {
    const int rp = plane_columns(r);
    u32x4 w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = u[2 * i], y = u[2 * i + 1];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const uint32_t t = pack2_bf16(x, y);
            w[q][i] = t;
            x -= __builtin_bit_cast(float, t << 16);
            y -= __builtin_bit_cast(float, t & 0xffff0000u);
        }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        uint16_t* const d = to + (row * 3 + q) * rp;
        gstore(reinterpret_cast<u32x4*>(d + k), w[q]);
        if (k + 8 == r)                                   // the columns that the gradients' blocks have beyond r
            for (int z = r; z < rp; z += 8) gstore(reinterpret_cast<u32x4*>(d + z), u32x4{0, 0, 0, 0});
    }
}

template <class L, bool PLANES>
__device__ __forceinline__ void t_tile(const AdapterProduct& g, int tile, unsigned char* lds) {
    constexpr int CB = L::CB, KS = L::KS, NS = L::NS;
    int* const list = reinterpret_cast<int*>(lds + L::ring);
    int* const ranks = list + 32;
    int* const place = ranks + 32;
    float* const scales = reinterpret_cast<float*>(place + 32);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lj = lane & 31, lh = lane >> 5;
    const int64_t row0 = (int64_t)tile * 32;
    const int rows = g.M - row0 < 32 ? (int)(g.M - row0) : 32;
    const int n = g.ke, r = g.r;

    const int slots = L::TN / r;
    const int lrow = lane >> 3;
    const int ns = (n * 2 + 128 * KS - 1) / (128 * KS);
    const int xrow = 8 * wave + lrow, xchunk = ((lane & 7) ^ ((xrow >> 1) & 7)) * 16;
    const rsrc_t xres = make_rsrc(g.E + row0 * g.e_pitch, (int64_t)rows * g.e_pitch * 2);
    int xslot = 0, xissued = 0;
    auto issue_x = [&]() {
        unsigned char* const dst = lds + xslot + wave * 1024;
        xslot = xslot == (NS - 1) * L::slab ? 0 : xslot + L::slab;
        const int x = xissued * KS * 128 + xchunk;
        ++xissued;
#pragma unroll
        for (int k = 0; k < KS; ++k) load_lds16(xres, dst + k * L::part, x + k * 128 < 2 * n ? xrow * g.e_pitch * 2 + x + k * 128 : kBufNowhere, 0);
    };
    while (xissued < NS - 1 && xissued < ns) issue_x();   // before anything is known of the adapters

    // which adapters the rows have, in ascending order, and which of them each row has
    int id = gload(g.row_adapter + row0 + (lj < rows ? lj : 0));
    id = lj < rows && id >= 0 && id < g.count ? id : -1;
    int count = 0, at = -1;
    for (int a = wave_min(id >= 0 ? id : INT_MAX); a != INT_MAX; a = wave_min(id > a ? id : INT_MAX)) {
        if (id == a) at = count;
        if (threadIdx.x == 0) list[count] = a;
        ++count;
    }
    if (threadIdx.x < 32) place[lj] = at;
    __syncthreads();
    int rank = 0;                                         // (what lies past a rank is read beside it and masked at the end)
    float my_scale = 1.0f;
    if ((int)threadIdx.x < count) {
        rank = rank_of(g, list[threadIdx.x]);
        if (g.scales) my_scale = gload(g.scales + list[threadIdx.x]);
    }

    const int frow = out_row(lj);
    const int xsw = (lj >> 1) & 7, fsw = (frow >> 1) & 7;
    const int xread = lj * 128 + (((2 * wave + lh) ^ xsw) * 16), fread = L::xpart + frow * 128 + (((2 * wave + lh) ^ fsw) * 16);
    // the transposing load: sixteen lanes read four rows of sixteen columns, four columns an address; this lane's row of the step and its four columns
    int kread[CB];
#pragma unroll
    for (int b = 0; b < CB; ++b) {
        const int c = 32 * b + out_row(16 * ((lane >> 4) & 1) + 4 * (lane & 3)), of = c / r < slots ? c / r : 0;      // (columns of no adapter: anything)
        kread[b] = L::xpart + of * 128 * r + (16 * wave + 8 * (lane >> 5) + ((lane & 15) >> 2)) * 2 * r + (c % r) * 2;
    }
    for (int first = 0; first == 0 || first < count; first += slots) {
        const int used = (count - first < slots ? count - first : slots) * r;      // columns of this pass
        // B: load instruction j covers eight columns, of one adapter (r is a multiple of 8): rows 8 (wave + 4 j) .. of the side-by-side B
        rsrc_t fres[CB];
        // A: this lane's 16 bytes of the first slab, and where in its adapter's they lie
        const uint16_t* apart[CB];
        int at_a[CB];
        if constexpr (PLANES) {
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                const int pos = 64 * (wave + 4 * j) + lane, p = pos / (8 * r);
                at_a[j] = (pos - p * 8 * r) * 8;
                apart[j] = p < slots && first + p < count ? g.F + (int64_t)list[first + p] * n * r + at_a[j] : nullptr;
            }
        } else {
#pragma unroll
            for (int j = 0; j < CB; ++j) {
                const int c = 8 * (wave + 4 * j), p = first + c / r, k = c % r;
                const bool have = c / r < slots && p < count;
                const int a = have ? __builtin_amdgcn_readfirstlane(list[p]) : 0;
                fres[j] = make_rsrc(g.F + ((int64_t)a * r + k) * n, have ? (int64_t)8 * n * 2 : 0);
            }
        }
        int fslot = 0, fissued = 0;
        auto issue_f = [&]() {
            unsigned char* const dst = lds + fslot + L::xpart + wave * 1024;
            fslot = fslot == (NS - 1) * L::slab ? 0 : fslot + L::slab;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                if constexpr (PLANES) {
                    const int64_t off = (int64_t)64 * r * (fissued * KS + k);
#pragma unroll
                    for (int j = 0; j < CB; ++j)
                        load_lds16_at(apart[j] && off + at_a[j] < (int64_t)n * r ? (const void*)(apart[j] + off) : (const void*)zero_line, dst + k * L::part + j * 4096);
                } else {
                    const int x = (fissued * KS + k) * 128 + xchunk;      // (the same chunk of eight rows further on)
#pragma unroll
                    for (int j = 0; j < CB; ++j) load_lds16(fres[j], dst + k * L::part + j * 4096, x < 2 * n ? lrow * n * 2 + x : kBufNowhere, 0);
                }
            }
            ++fissued;
        };
        if (first) {
            xslot = xissued = 0;
            while (xissued < NS - 1 && xissued < ns) issue_x();
        }
        while (fissued < NS - 1 && fissued < ns) issue_f();
        f32x16 acc[CB];
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[b][v] = 0.0f;
        int slot = 0;
        for (int s = 0; s < ns; ++s) {
            // Slab s has landed.  Behind its last load: F of NS - 2 slabs at least, and from slab NS - 2 on X of as many.
            if (s + NS - 1 > ns) wait_newest<0>();
            else if (s < NS - 2) wait_newest<(NS - 2) * L::NF>();
            else wait_newest<(NS - 2) * L::NL>();
            lds_barrier();
            if (xissued < ns) { issue_x(); issue_f(); }
            const unsigned char* const x = lds + slot;
            slot = slot == (NS - 1) * L::slab ? 0 : slot + L::slab;
            // all reads before the first product: a read's way is as long as a product
            u32x4 xo[KS], fo[KS][CB];
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                xo[k] = *reinterpret_cast<const u32x4*>(x + k * L::part + xread);
                if constexpr (!PLANES)
#pragma unroll
                    for (int b = 0; b < CB; ++b) fo[k][b] = *reinterpret_cast<const u32x4*>(x + k * L::part + fread + b * 4096);
            }
            if constexpr (PLANES) {
                const uint32_t base = lds_address(x);
#pragma unroll
                for (int b = 0; b < CB; b += 2)
                    read_tr4<L::part>(base + kread[b], base + kread[b] + 8 * r, base + kread[b + 1], base + kread[b + 1] + 8 * r, fo[0][b], fo[0][b + 1], fo[1][b], fo[1][b + 1]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int b = 0; b < CB; ++b) acc[b] = mfma_bf16(fo[k][b], xo[k], acc[b]);
        }
        // the waves' sums: blocks of 32 columns in turn, b by wave b % 4
        if (first == 0 && (int)threadIdx.x < count) {
            ranks[threadIdx.x] = rank;
            scales[threadIdx.x] = my_scale;
        }
        lds_barrier();
#pragma unroll
        for (int b = 0; b < CB; ++b)
            if (wave != b % 4) {
                unsigned char* const d = lds + ((wave > b % 4 ? wave - 1 : wave) * CB + b) * 4096 + lane * 16;
#pragma unroll
                for (int v = 0; v < 4; ++v) *reinterpret_cast<f32x4*>(d + v * 1024) = f32x4{acc[b][4 * v], acc[b][4 * v + 1], acc[b][4 * v + 2], acc[b][4 * v + 3]};
            }
        lds_barrier();
#pragma unroll
        for (int b = 0; b < CB; ++b) {
            if (wave != b % 4 || (32 * b >= used && 32 * b >= r)) continue;
#pragma unroll
            for (int w = 0; w < 3; ++w) {
                const unsigned char* const d = lds + (w * CB + b) * 4096 + lane * 16;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const f32x4 o = *reinterpret_cast<const f32x4*>(d + v * 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[b][4 * v + i] += o[i];
                }
            }
            if (lj >= rows) continue;
            const int64_t row = row0 + lj;
            const int p = place[lj];
            const float scale = p < 0 ? 1.0f : scales[p];
            const int mine = p < 0 ? 0 : ranks[p];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = 32 * b + 16 * lh + 8 * h, of = c / r, k = c % r;       // eight columns, those of this row's adapter?
                if (of >= slots || (p < 0 ? first != 0 || of != 0 : p - first != of)) continue;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = k + i < mine ? acc[b][8 * h + i] : 0.0f;
                if constexpr (!PLANES) {
                    if (g.T) {
                        gstore(reinterpret_cast<f32x4*>(g.T + row * r + k), f32x4{v[0], v[1], v[2], v[3]});
                        gstore(reinterpret_cast<f32x4*>(g.T + row * r + k + 4), f32x4{v[4], v[5], v[6], v[7]});
                    }
                    // T as an operand of the second product: one rounding to bf16, of the scaled value
                    if (g.Tb) {
                        u32x4 w;
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = pack2_bf16(k + 2 * i < mine ? scale * v[2 * i] : 0.0f, k + 2 * i + 1 < mine ? scale * v[2 * i + 1] : 0.0f);
                        gstore(reinterpret_cast<u32x4*>(g.Tb + row * r + k), w);
                    }
                } else {
                    float u[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] = k + i < mine ? scale * v[i] : 0.0f;
                    store_planes(g.dT_planes, row, k, r, u);
                    if (g.T_planes) {
                        const f32x4 t0 = gload(reinterpret_cast<const f32x4*>(g.T_in + row * r + k)), t1 = gload(reinterpret_cast<const f32x4*>(g.T_in + row * r + k + 4));
#pragma unroll
                        for (int i = 0; i < 8; ++i) u[i] = k + i < mine ? scale * (i < 4 ? t0[i & 3] : t1[i & 3]) : 0.0f;
                        store_planes(g.T_planes, row, k, r, u);
                    }
                }
            }
        }
        lds_barrier();                                    // the ring is free for another pass
    }
}

template <class L>
__global__ __launch_bounds__(256, 2) void adapters_t_kernel(const AdapterProduct g) {
    extern __shared__ __align__(1024) unsigned char lds[];
    t_tile<L, false>(g, blockIdx.x, lds);
}

// dT, and beside it what only later launches need.  (More than 256 registers only where one work-group fills the compute unit: T gains nothing by them.)
template <class L>
__global__ __launch_bounds__(256, L::per_cu) void adapters_dt_kernel(const AdapterProduct g, const AdapterPrep p, const PrepBlocks n, int tiles) {
    extern __shared__ __align__(1024) unsigned char lds[];
    const int i = blockIdx.x, t = i - n.list;             // lists, tiles of dT, transposes
    if (t >= 0 && t < tiles) t_tile<L, true>(g, t, lds);
    else prepare(p, n, t < 0 ? i : i - tiles, lds);
}

// dT of few rows, in whatever order: a work-group for a row and 32 columns of its A, whose threads share out A's rows, eight columns each.
// Bound by latency, then by reads of A from L2 (2 M m r bytes).  us, row by row / tiles of 32 rows, in runs of 100 and any order: 394 rows of 768, r = 8 6.2 / 9.2, 6.1 / 10.0;
// 394 of 4096, r = 32 15.0 / 20.3, 14.8 / 52.4; 1024 of 2304, r = 16 11.0 / 14.6, 12.4 / 27.0; 1024 of 4096, r = 128 81.5 / 86.6, 79.4 / 173; but 2048 of 1024, r = 128
// 44.3 / 31.3, 45.0 / 60.4.
constexpr int kDtRowLds = 256 * 32 + 256 * 4;
__device__ __forceinline__ void dt_of_row(const AdapterProduct& g, int64_t row, int k0, unsigned char* lds) {
    float* const parts = reinterpret_cast<float*>(lds);
    float* const sums = parts + 256 * 8;
    const int t = threadIdx.x, r = g.r, m = g.ke, cols = r - k0 < 32 ? r - k0 : 32, groups = cols / 8;
    const int cg = t % groups, each = 256 / groups, first = t / groups;       // (of three groups one thread is left over)
    const int a = __builtin_amdgcn_readfirstlane(gload(g.row_adapter + row));
    const bool have = a >= 0 && a < g.count;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    if (have && first < each) {
        const uint16_t* const y = g.E + row * g.e_pitch;
        const uint16_t* const A = g.F + (int64_t)a * m * r + k0 + 8 * cg;
        for (int j = first; j < m; j += 8 * each) {       // eight loads on their way at a time
            u32x4 v[8];
            uint32_t d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = j + i * each < m ? j + i * each : j;
                v[i] = gload(reinterpret_cast<const u32x4*>(A + (int64_t)at * r));
                d[i] = gload(y + at);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (j + i * each >= m) continue;
                const float x = __builtin_bit_cast(float, d[i] << 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t w = v[i][e];
                    sum[2 * e] += x * __builtin_bit_cast(float, w << 16);
                    sum[2 * e + 1] += x * __builtin_bit_cast(float, w & 0xffff0000u);
                }
            }
        }
    }
    *reinterpret_cast<f32x4*>(parts + 8 * t) = f32x4{sum[0], sum[1], sum[2], sum[3]};
    *reinterpret_cast<f32x4*>(parts + 8 * t + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
    __syncthreads();
    const int c = t % cols, many = 256 / cols, p = t / cols;      // a column's parts in `many` sums, then those
    float v = 0.0f;
    if (p < many)
        for (int q = p; q < each; q += many) v += parts[8 * (q * groups + c / 8) + c % 8];
    sums[t] = v;
    __syncthreads();
    if (t < cols) {
        v = 0.0f;
        for (int q = 0; q < many; ++q) v += sums[q * cols + t];
        parts[t] = v;
    }
    __syncthreads();
    if (t >= groups) return;
    const int k = k0 + 8 * t, mine = have ? rank_of(g, a) : 0;
    const float scale = have && g.scales ? gload(g.scales + a) : 1.0f;
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = k + i < mine ? scale * parts[8 * t + i] : 0.0f;
    store_planes(g.dT_planes, row, k, r, u);
    if (!g.T_planes) return;
    const f32x4 t0 = gload(reinterpret_cast<const f32x4*>(g.T_in + row * r + k)), t1 = gload(reinterpret_cast<const f32x4*>(g.T_in + row * r + k + 4));
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = k + i < mine ? scale * (i < 4 ? t0[i & 3] : t1[i & 3]) : 0.0f;
    store_planes(g.T_planes, row, k, r, u);
}
__global__ __launch_bounds__(256) void adapters_dt_rows_kernel(const AdapterProduct g, const AdapterPrep p, const PrepBlocks n, int rows) {
    __shared__ __align__(16) unsigned char lds[kDtRowLds > kPrepLds ? kDtRowLds : kPrepLds];
    const int i = blockIdx.x, t = i - n.list, per = (g.r + 31) / 32;          // lists, rows, transposes
    if (t >= 0 && t < rows) dt_of_row(g, t / per, t % per * 32, lds);
    else prepare(p, n, t < 0 ? i : i - rows, lds);
}

template <class L>
hipError_t launch_t(const AdapterProduct& p, hipStream_t s) {
    static std::atomic<bool> attr_set{false};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&adapters_t_kernel<L>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((adapters_t_kernel<L>), dim3((unsigned)ceil_div(p.M, 32)), dim3(256), L::lds, s, p);
    return hipGetLastError();
}
template <class L>
hipError_t launch_dt(const AdapterProduct& p, const AdapterPrep& prep, hipStream_t s) {
    static std::atomic<bool> attr_set{false};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&adapters_dt_kernel<L>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    static_assert(L::lds >= kPrepLds, "");
    const PrepBlocks n = prep_blocks(prep);
    const int64_t tiles = ceil_div(p.M, 32), blocks = tiles + n.all;
    if (blocks > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((adapters_dt_kernel<L>), dim3((unsigned)blocks), dim3(256), L::lds, s, p, prep, n, (int)tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adapters_y(const AdapterProduct& p, bool fp8, hipStream_t s) { return fp8 ? launch_y<true>(p, s) : launch_y<false>(p, s); }
// 64 columns for r <= 32: half the bytes of the adapters' side where 32 rows have one adapter or two.  us, T with one part a step, 64 / 128 columns: 12608 x 768, r = 32, runs of 64
// 13.0 / 16.2; 1379 x 768, runs of 200 6.9 / 8.4, of 7 14.0 / 13.7; 8190 x 4096, runs of 9 51.8 / 43.2.  For r > 64, 256 columns: 12608 x 768, r = 128
// 46.6 / 35.7 with 128.
hipError_t launch_adapters_t(const AdapterProduct& p, hipStream_t s) {
    if (p.M <= 1024 && p.M * p.r <= kAdapterRowsOfT) return launch_adapters_t_rows(p, s);
    return p.r <= 32 ? launch_t<Low<2, 3>>(p, s) : launch_t<Low<4, 3>>(p, s);
}
hipError_t launch_adapters_dt(const AdapterProduct& p, const AdapterPrep& prep, hipStream_t s) {
    if (p.M <= kAdapterFewGradRows) {
        const PrepBlocks n = prep_blocks(prep);
        const int rows = (int)(p.M * ceil_div(p.r, 32));
        hipLaunchKernelGGL(adapters_dt_rows_kernel, dim3((unsigned)(rows + n.all)), dim3(256), 0, s, p, prep, n, rows);
        return hipGetLastError();
    }
    return p.r <= 32 ? launch_dt<Low<2, 3>>(p, prep, s) : launch_dt<Low<4, 3>>(p, prep, s);
}

hipError_t launch_adapters_few_dx_grads(const AdapterProduct* x, const AdapterGrads& g, hipStream_t s) {
    if (g.M > kAdapterFewGradRows) return hipErrorInvalidValue;
    // dX has the smallest tile here, and from r = 33 on one work-group fills a compute unit: it goes alone where its best tile costs 16 less, or from 400 tiles on.  us,
    // together / apart, r = 16 (what the best tile costs less): 1024 x 2304 x 768 28.4 / 35.9 (0), 911 x 2304 x 2304 45.5 / 46.9 (11), 1024 x 1024 x 4096 38.6 / 37.1 (11), 700 x 4096 x
    // 4096 79.0 / 75.5 (18), 1024 x 4096 x 4096 91.8 / 83.0 (36), 1024 x 2048 x 8192 96.8 / 76.2 (45); r = 64 (tiles): 512 x 768 x 2304 30.9 / 34.6 (288), 700 x 768 x 2304 34.3 / 36.8
    // (396), 911 x 768 x 2304 42.8 / 42.3 (540), 512 x 4096 x 4096 101 / 86 (512), 1024 x 4096 x 4096 167 / 123 (1024); but 300 x 4096 x 4096 81.1 / 72.6 (320).
    if (x && (g.r > 32 ? ceil_div(x->M, T64x64::TM) * ceil_div(x->Q, T64x64::TN) > 400
                       : tile_cost(kTile64, *x, false) > tile_cost(best_tile(*x, false), *x, false) + 16.0f)) {
        const hipError_t e = launch_adapters_y(*x, false, s);
        if (e != hipSuccess) return e;
        x = nullptr;
    }
    switch (plane_columns(g.r)) {
        case 16: return launch_dx_grads<T64x64, 1>(x, g, 0, s);
        case 32: return launch_dx_grads<T64x64, 2>(x, g, 0, s);
        case 64: return launch_dx_grads<T64x64, 4>(x, g, 0, s);
        default: return launch_dx_grads<T64x64, 8>(x, g, 0, s);
    }
}

// Beside the gradients dX has one tile only, which may not be its best; the gradients' time (their bytes at 4 TB/s) is half hidden and a launch, 3.6 us, saved.
// (From r = 33 on the gradients fill a compute unit alone.)  us, beside / apart, r = 16, where the rule says beside: 1500 x 768 x 2304 30.4 / 34.9, 3000 x 2304 x 2304
// 66.0 / 65.8, 4096 x 2304 x 768 51.2 / 55.1, 12608 x 768 x 768 43.4 / 50.5, 12608 x 2304 x 768 77.6 / 89.0; apart: 1500 x 2304 x 768 50.4 / 45.5, 1500 x 4096 x 1024 74.4 / 60.8, 8190 x 4096 x 4096
// 316 / 305; but 1500 x 768 x 768 26.1 / 28.9 and 6000 x 1536 x 1024 49.4 / 55.9 (of 34 shapes near the limit 14 are 2 to 13 % faster beside).
bool adapters_dx_beside_grads(const AdapterProduct& x, const AdapterGrads& g) {
    const float grads = 2.0f * (float)g.M * (float)((g.dA ? g.m : 0) + (g.dB ? g.n : 0)) / 4e6f;
    return g.r <= 32 && tile_cost(kTile128x192, x, false) - tile_cost(best_tile(x, false), x, false) < 0.5f * grads + 3.6f;
}
hipError_t launch_adapters_dx_grad_pieces(const AdapterProduct& x, const AdapterGrads& g, int piece, hipStream_t s) {
    return g.r <= 16 ? launch_dx_grads<T128x192, 1>(&x, g, piece, s) : launch_dx_grads<T128x192, 2>(&x, g, piece, s);
}

}  // namespace abt
