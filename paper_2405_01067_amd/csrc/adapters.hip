// The products of a dense layer with adapters for many rows:
//     Y_i = W x_i + A_a T_i          T_i = B_a x_i          a = adapter of row i, T scaled where it is an operand
// One kernel makes all of them: a tile of the result sums over slabs of the contraction, first those of the dense product, then for
// every adapter that occurs among its rows those of the low-rank one, with the rows of other adapters read as zeros.  Rows that
// lie together by adapter therefore cost a tile one or two short passes, rows in any other order more passes, and the result is the same
// but for the order of its sums.  T alone is the case without a dense product.
//
// A slab is 128 bytes of every row: 64 columns in bf16, 128 in 8 bits.  It comes straight to LDS, NS slots in a ring, one barrier per
// slab; the operands of a step are read while the products of the step before run, across the barrier too.  Both types read LDS alike: two
// 16-byte pieces are two bf16 operands of 32x32x16 or one 8-bit operand of 32x32x64, whose columns are taken in the same order on both sides.
#include <atomic>
#include <climits>

#include "adapters.h"

namespace abt {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

__device__ __forceinline__ f32x16 mfma_f8(u32x4 a0, u32x4 a1, u32x4 b0, u32x4 b1, f32x16 c) {
    const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
    const i32x8 b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);       // scales of 2^0
}

// the first `valid` (less than eight, may be negative) of eight bf16 values, zeros behind them
__device__ __forceinline__ u32x4 first_of(u32x4 v, int valid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= valid >= 2 * i + 2 ? 0xffffffffu : valid == 2 * i + 1 ? 0xffffu : 0u;
    return v;
}

enum { kOutY, kOutT, kOutPlanes };

// WM x WN waves, each RB x CB blocks of 32 x 32
template <int TM_, int TN_, int WM_, int WN_, int NS_>
struct Tile {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, NS = NS_, NW = WM * WN;
    static constexpr int RB = TM / (32 * WM), CB = TN / (32 * WN);
    static constexpr int xpart = TM * 128, slab = (TM + TN) * 128;
    static constexpr int NX = TM / 8 / NW, NF = TN / 8 / NW, NL = NX + NF;       // load instructions per wave and slab: eight rows each
    static constexpr int IDS = (TM + 63) / 64;
    static constexpr int opitch = TN * 2 + 16;
    static constexpr int out = TM * opitch;
    static __host__ __device__ constexpr int lds(int kind) { return kind == kOutY && out > NS * slab ? out : NS * slab; }
    static_assert(NX * 8 * NW == TM && NF * 8 * NW == TN && RB * 32 * WM == TM && CB * 32 * WN == TN, "");
    static_assert(NW % 2 == 0 && (NS - 2) * NL < 64, "");
};

struct Order { int row_tiles, col_tiles; };

// Tiles in panels of four row tiles, down the panel first; each XCD gets a contiguous eighth: the tiles that run at the same time on one
// XCD share rows of X and rows of W in its L2.
__device__ __forceinline__ void tile_of(const Order& o, int& rt, int& ct) {
    const int nb = gridDim.x, xcd = blockIdx.x & 7, i = blockIdx.x >> 3, per = nb >> 3, rem = nb & 7;
    const int w = xcd * per + (xcd < rem ? xcd : rem) + i;
    const int panel = w / (4 * o.col_tiles), rows = o.row_tiles - 4 * panel < 4 ? o.row_tiles - 4 * panel : 4;
    const int at = w - panel * 4 * o.col_tiles;
    rt = 4 * panel + at % rows;
    ct = at / rows;
}

template <class L, bool F8, int OUT>
__global__ __launch_bounds__(64 * L::NW) void adapters_kernel(const AdapterProduct g, const Order order) {
    constexpr int RB = L::RB, CB = L::CB, NW = L::NW, NS = L::NS;
    constexpr int ES = F8 ? 1 : 2;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lj = lane & 31, lh = lane >> 5;
    const int wr = wave / L::WN, wc = wave % L::WN;
    int rt, ct;
    tile_of(order, rt, ct);
    const int64_t row0 = (int64_t)rt * L::TM;
    const int col0 = ct * L::TN;
    const int rows = g.M - row0 < L::TM ? (int)(g.M - row0) : L::TM;
    const int cols = g.Q - col0 < L::TN ? g.Q - col0 : L::TN;

    // ---- loads: instruction j of a wave covers rows 8 (wave + NW j) .. + 7 of X, or of W; this lane's row among them and its chunk
    const int lrow = 8 * wave + (lane >> 3);
    const int chunk = ((lane & 7) ^ ((lrow >> 1) & 7)) * 16;       // NW is even: the same for all j
    const int main_bytes = g.kmain * ES;
    const int nmain = OUT == kOutY ? (main_bytes + 127) / 128 : 0;
    const rsrc_t xres = OUT == kOutY ? make_rsrc((const char*)g.X + row0 * main_bytes, (int64_t)rows * main_bytes) : make_rsrc(nullptr, 0);
    const rsrc_t wres = OUT == kOutY ? make_rsrc((const char*)g.W + (int64_t)col0 * main_bytes, (int64_t)cols * main_bytes) : make_rsrc(nullptr, 0);
    int issue_slot = 0;
    auto issue_main = [&](int s) {
        unsigned char* const dst = lds + issue_slot + wave * 1024;
        issue_slot = issue_slot == (NS - 1) * L::slab ? 0 : issue_slot + L::slab;
        const int at = s * 128 + chunk;                   // chunks past the end of a row arrive as zeros
        const int off = at < main_bytes ? lrow * main_bytes + at : kBufNowhere;
        const int step = at < main_bytes ? 8 * NW * main_bytes : 0;
#pragma unroll
        for (int j = 0; j < L::NX; ++j) load_lds16(xres, dst + j * (NW * 1024), off + j * step, 0);
#pragma unroll
        for (int j = 0; j < L::NF; ++j) load_lds16(wres, dst + L::xpart + j * (NW * 1024), off + j * step, 0);
    };
    int issued = 0;                                       // slabs
    if constexpr (OUT == kOutY) {
        for (; issued < NS - 1 && issued < nmain; ++issued) issue_main(issued);
    }

    // ---- adapters of the rows: of all rows of the tile (to find the next one), and of the rows this lane loads
    const int K = g.count;
    int ids[L::IDS], lid[L::NX];
#pragma unroll
    for (int i = 0; i < L::IDS; ++i) {
        const int r = 64 * i + lane;
        const int a = r < rows ? gload(g.row_adapter + row0 + r) : -1;
        ids[i] = a >= 0 && a < K ? a : -1;
    }
#pragma unroll
    for (int j = 0; j < L::NX; ++j) {
        const int r = lrow + 8 * NW * j;
        lid[j] = r < rows ? gload(g.row_adapter + row0 + r) : -1;
    }
    auto after = [&](int a) {                             // the smallest adapter above a that has rows here; INT_MAX: none
        int best = INT_MAX;
#pragma unroll
        for (int i = 0; i < L::IDS; ++i) best = ids[i] > a && ids[i] < best ? ids[i] : best;
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const int o = __shfl_xor(best, d);
            best = o < best ? o : best;
        }
        return __builtin_amdgcn_readfirstlane(best);
    };
    auto rank_of = [&](int a) {
        if (a == INT_MAX) return 0;
        int k = g.ranks ? __builtin_amdgcn_readfirstlane(gload(g.ranks + a)) : g.r;
        return k < 0 ? 0 : k > g.r ? g.r : k;
    };
    // Y: the contraction is the rank; T and the planes: the rank counts columns
    auto length_of = [&](int rank) { return OUT == kOutY ? rank : rank > col0 ? g.ke : 0; };
    struct Walk { int a, rank, len, k; };                 // adapter, its rank, its contraction, the next column of it
    auto settle = [&](Walk& w) {                          // to an adapter with something left to contract
        while (w.a != INT_MAX && w.k >= w.len) {
            w.a = after(w.a);
            w.rank = rank_of(w.a);
            w.len = w.a == INT_MAX ? 0 : length_of(w.rank);
            w.k = 0;
        }
    };
    Walk in{-1, 0, 0, 0};
    settle(in);
    Walk out = in;
    const rsrc_t eres = make_rsrc(g.E + row0 * g.e_pitch, (int64_t)rows * g.e_pitch * 2);
    auto issue_low = [&]() {
        unsigned char* const dst = lds + issue_slot + wave * 1024;
        issue_slot = issue_slot == (NS - 1) * L::slab ? 0 : issue_slot + L::slab;
        const int frows = OUT == kOutY ? cols : (in.rank - col0 < cols ? in.rank - col0 : cols);
        const rsrc_t fres = make_rsrc(g.F + ((int64_t)in.a * g.Q + col0) * g.ke, (int64_t)frows * g.ke * 2);
        const int at = in.k * 2 + chunk;
        const bool ok = at < in.len * 2;
#pragma unroll
        for (int j = 0; j < L::NX; ++j)
            load_lds16(eres, dst + j * (NW * 1024), ok && lid[j] == in.a ? (lrow + 8 * NW * j) * g.e_pitch * 2 + at : kBufNowhere, 0);
#pragma unroll
        for (int j = 0; j < L::NF; ++j)
            load_lds16(fres, dst + L::xpart + j * (NW * 1024), ok ? (lrow + 8 * NW * j) * g.ke * 2 + at : kBufNowhere, 0);
        in.k += 64;
        settle(in);
    };
    auto issue = [&]() {                                  // the next slab, if there is one
        if (issued < nmain) issue_main(issued);
        else if (in.a != INT_MAX) issue_low();
        else return;
        ++issued;
    };
    while (issued < NS - 1 && in.a != INT_MAX) issue();

    // ---- products
    f32x16 acc[RB][CB];
#pragma unroll
    for (int a = 0; a < RB; ++a)
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    const int frow = out_row(lj);
    const int xsw = (lj >> 1) & 7, fsw = (frow >> 1) & 7;
    const int xbase = (wr * RB * 32 + lj) * 128, fbase = L::xpart + (wc * CB * 32 + frow) * 128;
    struct Ops { u32x4 x[RB], f[CB]; };
    auto read = [&](Ops& o, int slot, int j) {            // chunk 2 j + lh of this lane's rows
        const unsigned char* const x = lds + slot + xbase + (((2 * j + lh) ^ xsw) * 16);
        const unsigned char* const f = lds + slot + fbase + (((2 * j + lh) ^ fsw) * 16);
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
    int done = 0, slot = 0;                               // slabs consumed, the slot of the next
    // Slab `done` has landed: loads come back in the order of issue, and NS - 2 slabs at most were requested after it.
    auto next_slab = [&]() {
        const int behind = issued - done - 1;
        if (behind >= NS - 2) wait_newest<(NS - 2) * L::NL>();
        else if (NS > 3 && behind == NS - 3) wait_newest<(NS > 3 ? NS - 3 : 0) * L::NL>();
        else wait_newest<0>();
        lds_barrier();
        issue();                                          // into the slot whose reads ended before this barrier
        const int at = slot;
        slot = slot == (NS - 1) * L::slab ? 0 : slot + L::slab;
        ++done;
        return at;
    };
    if constexpr (OUT == kOutY) {
        Ops o[2];
        for (int s = 0; s < nmain; ++s) {
            const int at = next_slab();
            if constexpr (F8) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    read(o[0], at, 2 * j);
                    read(o[1], at, 2 * j + 1);
                    mma8(o[0], o[1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    read(o[j & 1], at, j);
                    mma(o[j & 1]);
                }
            }
        }
        if constexpr (F8) {                               // the dense product's scales
#pragma unroll
            for (int a = 0; a < RB; ++a) {
                const int r = (wr * RB + a) * 32 + lj;
                const float xs = r < rows ? gload(g.x_scale + row0 + r) : 0.0f;
#pragma unroll
                for (int b = 0; b < CB; ++b)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int c = (wc * CB + b) * 32 + 16 * lh + v;
                        acc[a][b][v] *= xs * (c < cols ? gload(g.w_scale + col0 + c) : 0.0f);
                    }
            }
        }
    }
    while (out.a != INT_MAX) {
        const int at = next_slab();
        const int left = out.len - out.k < 64 ? out.len - out.k : 64;
        const bool ragged = (left & 7) != 0;
        const int steps = (left + 15) / 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j >= steps) break;
            Ops o;
            read(o, at, j);
            if (ragged) {                                 // columns past the rank are no part of the adapter, whatever they hold
                const int valid = left - (2 * j + lh) * 8;
#pragma unroll
                for (int b = 0; b < CB; ++b)
                    if (valid < 8) o.f[b] = first_of(o.f[b], valid);
#pragma unroll
                for (int a = 0; a < RB; ++a)
                    if (valid < 8) o.x[a] = first_of(o.x[a], valid);
            }
            mma(o);
        }
        out.k += 64;
        settle(out);
    }

    // ---- out
    if constexpr (OUT == kOutY) {
        lds_barrier();                                    // every wave has read its last slab, and nothing is on its way to LDS
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
        lds_barrier();
        constexpr int CPR = L::TN / 8;
        const rsrc_t yres = make_rsrc(g.Y + row0 * g.Q + col0, ((int64_t)(rows - 1) * g.Q + cols) * 2);
#pragma unroll
        for (int i = 0; i < L::TM * CPR / (64 * NW); ++i) {
            const int e = i * (64 * NW) + (int)threadIdx.x, r = e / CPR, c = e % CPR;
            buf_store16(*reinterpret_cast<const u32x4*>(lds + r * L::opitch + c * 16), yres, r < rows && c * 8 < cols ? (r * g.Q + c * 8) * 2 : kBufNowhere, 0);
        }
    } else {
#pragma unroll
        for (int a = 0; a < RB; ++a) {
            const int r = (wr * RB + a) * 32 + lj;
            if (r >= rows) continue;
            const int64_t row = row0 + r;
            int id = gload(g.row_adapter + row);
            if (id < 0 || id >= K) id = -1;
            const float s = id < 0 ? 0.0f : g.scales ? gload(g.scales + id) : 1.0f;
            int rank = id < 0 ? 0 : g.ranks ? gload(g.ranks + id) : g.r;
            rank = rank > g.r ? g.r : rank;
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = col0 + (wc * CB + b) * 32 + 16 * lh + 8 * h;      // eight columns
                    if constexpr (OUT == kOutT) {
                        if (c >= g.r) continue;
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = c + i < rank ? acc[a][b][8 * h + i] : 0.0f;
                        if (g.T) {
                            gstore(reinterpret_cast<f32x4*>(g.T + row * g.r + c), f32x4{v[0], v[1], v[2], v[3]});
                            gstore(reinterpret_cast<f32x4*>(g.T + row * g.r + c + 4), f32x4{v[4], v[5], v[6], v[7]});
                        }
                        // T as an operand of the second product: one rounding to bf16, of the scaled value
                        if (g.Tb) {
                            u32x4 w;
#pragma unroll
                            for (int i = 0; i < 4; ++i) w[i] = pack2_bf16(c + 2 * i < rank ? s * v[2 * i] : 0.0f, c + 2 * i + 1 < rank ? s * v[2 * i + 1] : 0.0f);
                            gstore(reinterpret_cast<u32x4*>(g.Tb + row * g.r + c), w);
                        }
                    } else {
                        const int rp = plane_columns(g.r);
                        if (c >= rp) continue;
                        // Three bf16 values that add up to the fp32 one (each takes eight bits of what the ones before left): the factor gradients are
                        // fp32 sums of exact products, as they would be of fp32 operands.
                        auto planes = [&](uint16_t* to, const float (&v)[8]) {
                            u32x4 w[3];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float x = v[2 * i], y = v[2 * i + 1];
#pragma unroll
                                for (int p = 0; p < 3; ++p) {
                                    const uint32_t q = pack2_bf16(x, y);
                                    w[p][i] = q;
                                    x -= __builtin_bit_cast(float, q << 16);
                                    y -= __builtin_bit_cast(float, q & 0xffff0000u);
                                }
                            }
#pragma unroll
                            for (int p = 0; p < 3; ++p) gstore(reinterpret_cast<u32x4*>(to + (row * 3 + p) * rp + c), w[p]);
                        };
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = c + i < rank ? s * acc[a][b][8 * h + i] : 0.0f;
                        planes(g.dT_planes, v);
                        if (g.T_planes) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = c + i < rank ? s * gload(g.T_in + row * g.r + c + i) : 0.0f;
                            planes(g.T_planes, v);
                        }
                    }
                }
        }
    }
}

template <class L, bool F8, int OUT>
hipError_t launch_tile(const AdapterProduct& p, hipStream_t s) {
    const void* const fn = reinterpret_cast<const void*>(&adapters_kernel<L, F8, OUT>);
    static_assert(L::lds(OUT) <= 160 * 1024, "");
    static std::atomic<bool> attr_set{false};
    if (!attr_set.load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, L::lds(OUT));
        if (e != hipSuccess) return e;
        attr_set.store(true, std::memory_order_release);
    }
    const int64_t rt = ceil_div(p.M, L::TM), ct = ceil_div(OUT == kOutPlanes ? plane_columns(p.r) : p.Q, L::TN);
    if (rt * ct > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((adapters_kernel<L, F8, OUT>), dim3((unsigned)(rt * ct)), dim3(64 * L::NW), L::lds(OUT), s, p, Order{(int)rt, (int)ct});
    return hipGetLastError();
}

using T256 = Tile<256, 256, 2, 4, 2>;
using T128 = Tile<128, 128, 2, 2, 4>;
using T64 = Tile<64, 64, 2, 2, 6>;

template <bool F8>
hipError_t launch_y(const AdapterProduct& p, hipStream_t s) {
    const int64_t big = ceil_div(p.M, 256) * ceil_div(p.Q, 256), mid = ceil_div(p.M, 128) * ceil_div(p.Q, 128);
    if (big >= 192) return launch_tile<T256, F8, kOutY>(p, s);
    if (mid >= 192) return launch_tile<T128, F8, kOutY>(p, s);
    return launch_tile<T64, F8, kOutY>(p, s);
}

template <int OUT>
hipError_t launch_low(const AdapterProduct& p, hipStream_t s) {
    if (p.r <= 32) return launch_tile<Tile<64, 32, 2, 1, 8>, false, OUT>(p, s);
    if (p.r <= 64) return launch_tile<Tile<64, 64, 2, 2, 6>, false, OUT>(p, s);
    return launch_tile<Tile<64, 128, 2, 2, 5>, false, OUT>(p, s);
}

}  // namespace

hipError_t launch_adapters_y(const AdapterProduct& p, bool fp8, hipStream_t s) { return fp8 ? launch_y<true>(p, s) : launch_y<false>(p, s); }
hipError_t launch_adapters_t(const AdapterProduct& p, hipStream_t s) { return launch_low<kOutT>(p, s); }
hipError_t launch_adapters_planes(const AdapterProduct& p, hipStream_t s) { return launch_low<kOutPlanes>(p, s); }

}  // namespace abt
