// Gradients of the dense layer: what its products are made of, and dW = dZ^T X, a contraction over the rows.
// 12608 rows, 2304 x 768, gelu (three values): dZ 64 us, bound by memory (290 MB at 4.5 TB/s); dX 104 (dense_tile.hip, a contraction of twice 2304: 89 GFLOP at 850 TFLOP/s); dW 132 (134 GFLOP of three
// products at 1010 TFLOP/s); the sum of its nine pieces 14 (71 MB, 5 TB/s).  394 rows, 768 x 768, silu: dZ 7.5 us, everything else 11.2: latency.  (Medians under a profiler; the passes take 286 and 17.9.)
#include <climits>

#include "dense_tile.h"

namespace abt {
namespace {

// ------------------------------------------------------------------------------------------ dZ, W^T
constexpr int kSlopeCols = 512;                           // a wave has a row of them, eight a lane

__device__ __forceinline__ void unpack8(u32x4 w, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[2 * k] = __builtin_bit_cast(float, w[k] << 16);
        v[2 * k + 1] = __builtin_bit_cast(float, w[k] & 0xffff0000u);
    }
}

// The next part of eight values: the leading eight bits of what is left of each, which loses them.  Nothing is left of what is not finite (infinities and NaN are in the first part).
__device__ __forceinline__ u32x4 cut8(const float (&v)[8], float (&left)[8]) {
    uint32_t part[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t sign = __builtin_bit_cast(uint32_t, v[k]) & 0x80000000u, least = v[k] == 0.0f ? 0 : 0x10000u;
        const uint32_t size = __builtin_bit_cast(uint32_t, left[k]) & 0x7fff0000u;
        part[k] = (size > least ? size : least) | sign;
        left[k] = size < 0x7f800000u ? left[k] - __builtin_bit_cast(float, size | sign) : 0.0f;
    }
    u32x4 out;
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = part[2 * k] >> 16 | part[2 * k + 1];
    return out;
}

__device__ __forceinline__ void slope_piece(const DenseSlope& g, int piece, int col0, float (*sums)[kSlopeCols]) {
    constexpr int B = 4;                                  // rows of a wave on their way at a time
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = col0 + 8 * lane;
    const bool there = col < g.m;
    const int64_t first = (int64_t)piece * g.rows, last = first + g.rows < g.M ? first + g.rows : g.M;
    float total[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) total[k] = 0.0f;
    const DropKey key = g.drop.state ? drop_key(g.drop) : DropKey{0, 0, 0, 0};
    Drop drop = g.drop;
    if (!g.scaled) drop.scale = 1.0f;
    if (there)
        for (int64_t r = first + wave; r < last; r += 4 * B) {
            u32x4 dy[B], z[B];
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const int64_t at = (r + 4 * i < last ? r + 4 * i : r) * g.m + col;
                dy[i] = gload(reinterpret_cast<const u32x4*>(g.dY + at));
                if (g.Z) z[i] = gload(reinterpret_cast<const u32x4*>(g.Z + at));
            }
#pragma unroll
            for (int i = 0; i < B; ++i) {
                if (r + 4 * i >= last) break;
                const int64_t at = (r + 4 * i) * g.m + col;
                float v[8];
                unpack8(dy[i], v);
                if (g.Z) {
                    float zz[8];
                    unpack8(z[i], zz);
                    with_activation(g.act, [&](auto act) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] = through<decltype(act)::value>(zz[k], v[k]);
                    });
                }
                if (g.drop.state) drop8(drop, key, (uint64_t)at >> 3, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) total[k] += v[k];
                if (!g.value[0]) continue;
                float left[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) left[k] = v[k];
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    if (!g.value[q]) break;
                    const int64_t to = q < 2 ? (r + 4 * i) * pitch_of(g.values) * g.m + col : at;
                    gstore(reinterpret_cast<u32x4*>(g.value[q] + to), cut8(v, left));
                }
            }
        }
    if (!g.sums) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) sums[wave][8 * lane + k] = total[k];
    __syncthreads();
    for (int c = threadIdx.x; c < kSlopeCols && col0 + c < g.m; c += 256) gstore(g.sums + (int64_t)piece * g.m + col0 + c, (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]));
}

// 64 x 64 of W
__device__ __forceinline__ void transpose_block(const DenseSlope& g, int block, uint16_t (*tile)[72]) {
    const int cols = (g.n + 63) / 64, r0 = block / cols * 64, c0 = block % cols * 64;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int e = i * 256 + threadIdx.x, r = e >> 3, c = (e & 7) * 8;
        if (r0 + r < g.m && c0 + c < g.n) *reinterpret_cast<u32x4*>(&tile[r][c]) = gload(reinterpret_cast<const u32x4*>(g.W + (int64_t)(r0 + r) * g.n + c0 + c));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int e = i * 256 + threadIdx.x, c = e & 63, r = (e >> 6) * 8;    // column c of the tile, rows r .. r + 7
        if (c0 + c >= g.n || r0 + r >= g.m) continue;
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (uint32_t)tile[r + 2 * k][c] | (uint32_t)tile[r + 2 * k + 1][c] << 16;
        uint16_t* const to = g.Wt + (int64_t)(c0 + c) * pitch_of(g.values) * g.m + r0 + r;
        gstore(reinterpret_cast<u32x4*>(to), v);
        if (g.values > 1) gstore(reinterpret_cast<u32x4*>(to + g.m), v);
    }
}

__global__ __launch_bounds__(256) void dense_slope_kernel(const DenseSlope g, int pieces, int slabs) {
    __shared__ union { float sums[4][kSlopeCols]; uint16_t tile[64][72]; } lds;
    const int i = blockIdx.x, own = pieces * slabs;
    if (i < own) slope_piece(g, i / slabs, i % slabs * kSlopeCols, lds.sums);
    else transpose_block(g, i - own, lds.tile);
}

// ------------------------------------------------------------------------------------------ dW
// TP x TQ of dW by WP x WQ waves of RB x CB blocks of 32 x 32; a slab is 32 rows of X and of each of dZ's values as they lie, in two slots.  All are read with the
// transposing load: sixteen lanes ask for four rows of sixteen columns, and lane i gets the four of column i.  The slabs come through registers: beside loads that go straight to
// LDS the compiler lets the transposing load wait for all of them, and in inline asm, with a wait of its own, nothing runs beside it (256 x 256, two values, 12608 rows:
// 100 us against 96).
template <int TP_, int TQ_, int WP_, int WQ_, int VALUES_>
struct GradTile {
    static constexpr int TP = TP_, TQ = TQ_, WP = WP_, WQ = WQ_, VALUES = VALUES_, NW = WP * WQ;
    static constexpr int RB = TP / (32 * WP), CB = TQ / (32 * WQ);
    static constexpr int ppart = 32 * TP * 2, qpart = 32 * TQ * 2, xbase = VALUES * ppart, slab = xbase + qpart, lds = 2 * slab;
    static constexpr int NP = ppart / 1024 / NW, NQ = qpart / 1024 / NW;       // load instructions per wave and slab
    static_assert(NP * NW * 1024 == ppart && NQ * NW * 1024 == qpart && RB * 32 * WP == TP && CB * 32 * WQ == TQ && TP >= 64 && TQ >= 64 && lds <= 160 * 1024, "");
    // Chunk c of row r lies at c ^ turn(r): the four rows of 64 bytes that half a wave asks for fall on all banks.
    static __device__ __forceinline__ int turn(int width, int r) { return width == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2; }
};

typedef __attribute__((ext_vector_type(4))) short s16x4;
// sixteen rows of 32 columns, whose halves are `back` bytes apart
__device__ __forceinline__ u32x4 read_operand(const unsigned char* at, int back) {
    auto half = [](const unsigned char* p) {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(void*)p));
    };
    const u32x2 a = half(at), b = half(at + back);
    return u32x4{a[0], a[1], b[0], b[1]};
}

template <class L>
__device__ __forceinline__ void grad_tile(const DenseGrads& g, const GradOrder& o, int block, unsigned char* lds) {
    constexpr int RB = L::RB, CB = L::CB, NW = L::NW;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lj = lane & 31, lh = lane >> 5, li = lane & 15;
    const int wp = wave / L::WQ, wq = wave % L::WQ;
    const int split = block / o.tiles, tile = block % o.tiles;
    const int p0 = tile / o.col_tiles * L::TP, q0 = tile % o.col_tiles * L::TQ;
    const int pcols = g.m - p0 < L::TP ? g.m - p0 : L::TP, qcols = g.n - q0 < L::TQ ? g.n - q0 : L::TQ;
    const int64_t first = (int64_t)split * o.slabs * 32, last = first + (int64_t)o.slabs * 32 < g.M ? first + (int64_t)o.slabs * 32 : g.M;
    const int ns = (int)((last - first + 31) / 32);

    auto lane_offset = [&](int width, int pitch, int cols, int j) {
        const int pos = (j * NW + wave) * 64 + lane, r = pos / (width / 8), c = ((pos % (width / 8)) ^ L::turn(width, r)) * 8;
        return c < cols ? (r * pitch + c) * 2 : kBufNowhere;
    };
    constexpr int KINDS = L::VALUES == 1 ? 1 : 2;         // the first and second part have rows of their own pitch
    const int pitch[2] = {pitch_of(L::VALUES) * g.m, g.m};
    int poff[KINDS][L::NP], qoff[L::NQ];
#pragma unroll
    for (int k = 0; k < KINDS; ++k)
#pragma unroll
        for (int j = 0; j < L::NP; ++j) poff[k][j] = lane_offset(L::TP, pitch[k], pcols, j);
#pragma unroll
    for (int j = 0; j < L::NQ; ++j) qoff[j] = lane_offset(L::TQ, g.n, qcols, j);
    u32x4 pnext[L::VALUES][L::NP], qnext[L::NQ];          // the slab on its way
    auto request = [&](int s) {
        const int64_t row = first + (int64_t)s * 32;
        const int rows = last - row < 32 ? (int)(last - row) : 32;            // rows past the last one read zeros
        const int64_t qbytes = ((int64_t)(rows - 1) * g.n + qcols) * 2;
#pragma unroll
        for (int q = 0; q < L::VALUES; ++q) {
            const int k = q / 2;
            const rsrc_t res = make_rsrc(g.value[q] + row * pitch[k] + p0, ((int64_t)(rows - 1) * pitch[k] + pcols) * 2);
#pragma unroll
            for (int j = 0; j < L::NP; ++j) pnext[q][j] = buf_load16(res, poff[k][j], 0);
        }
        const rsrc_t res = make_rsrc(g.X + row * g.n + q0, qbytes);
#pragma unroll
        for (int j = 0; j < L::NQ; ++j) qnext[j] = buf_load16(res, qoff[j], 0);
    };
    auto keep = [&](int slot) {
        unsigned char* const dst = lds + slot * L::slab + (wave * 64 + lane) * 16;
#pragma unroll
        for (int q = 0; q < L::VALUES; ++q)
#pragma unroll
            for (int j = 0; j < L::NP; ++j) *reinterpret_cast<u32x4*>(dst + q * L::ppart + j * (NW * 1024)) = pnext[q][j];
#pragma unroll
        for (int j = 0; j < L::NQ; ++j) *reinterpret_cast<u32x4*>(dst + L::xbase + j * (NW * 1024)) = qnext[j];
    };
    request(0);

    f32x16 acc[RB][CB];
#pragma unroll
    for (int a = 0; a < RB; ++a)
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    // Rows 4 lh + li / 4 and 8 more of a step of sixteen; quad t of a block's columns, taken in the order of out_row on X's side, so that a lane's sums are
    // sixteen consecutive columns of a row of dW.
    const int t = 4 * ((lane >> 4) & 1) + (li & 3), tx = 4 * (t & 1) + (t >> 1), trow = 4 * lh + (li >> 2);
    int pat[RB], qat[CB];
#pragma unroll
    for (int a = 0; a < RB; ++a) pat[a] = trow * (L::TP * 2) + ((((wp * RB + a) * 4 + (t >> 1)) ^ L::turn(L::TP, trow)) * 16) + (t & 1) * 8;
#pragma unroll
    for (int b = 0; b < CB; ++b) qat[b] = L::xbase + trow * (L::TQ * 2) + ((((wq * CB + b) * 4 + (tx >> 1)) ^ L::turn(L::TQ, trow)) * 16) + (tx & 1) * 8;
    struct Ops { u32x4 x[CB], z[L::VALUES][RB]; };
    auto read = [&](Ops& o, const unsigned char* slab, int half) {
#pragma unroll
        for (int b = 0; b < CB; ++b) o.x[b] = read_operand(slab + qat[b] + half * (16 * L::TQ * 2), 8 * L::TQ * 2);
#pragma unroll
        for (int q = 0; q < L::VALUES; ++q)
#pragma unroll
            for (int a = 0; a < RB; ++a) o.z[q][a] = read_operand(slab + pat[a] + q * L::ppart + half * (16 * L::TP * 2), 8 * L::TP * 2);
    };
    auto mma = [&](const Ops& o) {
#pragma unroll
        for (int q = 0; q < L::VALUES; ++q)
#pragma unroll
            for (int a = 0; a < RB; ++a)
#pragma unroll
                for (int b = 0; b < CB; ++b) acc[a][b] = mfma_bf16(o.x[b], o.z[q][a], acc[a][b]);
    };
    // the operands of a step are read while the products of the step before run, across the barrier too
    Ops ops[2];
#pragma unroll
    for (int b = 0; b < CB; ++b) ops[1].x[b] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < L::VALUES; ++q)
#pragma unroll
        for (int a = 0; a < RB; ++a) ops[1].z[q][a] = u32x4{0, 0, 0, 0};
    keep(0);
    if (ns > 1) request(1);
    for (int s = 0; s < ns; ++s) {
        lds_barrier();
        if (s + 1 < ns) keep((s + 1) & 1);                // into the slot whose reads ended before this barrier
        if (s + 2 < ns) request(s + 2);
        const unsigned char* const slab = lds + (s & 1) * L::slab;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            read(ops[h], slab, h);
            mma(ops[1 - h]);
#pragma unroll
            for (int i = 0; i < 2 * (CB + L::VALUES * RB); ++i) {             // a read behind every product
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    mma(ops[1]);
    // row lj of a block of dZ's columns, columns 16 lh .. + 15 of one of X's
    const bool whole = o.splits == 1;
    float* const out = whole ? g.dW : g.partials + (int64_t)split * g.m * g.n;
#pragma unroll
    for (int a = 0; a < RB; ++a) {
        const int r = (wp * RB + a) * 32 + lj;
        if (r >= pcols) continue;
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = (wq * CB + b) * 32 + 16 * lh + 4 * q;
                if (c >= qcols) continue;
                f32x4 v;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = acc[a][b][4 * q + k] * g.alpha;
                f32x4* const d = reinterpret_cast<f32x4*>(out + (int64_t)(p0 + r) * g.n + q0 + c);
                if (whole && g.accumulate) v += gload(d);
                gstore(d, v);
            }
    }
}

// 32 columns of dbias from the sums of the pieces
__device__ __forceinline__ void bias_block(const DenseGrads& g, int block, float (*lds)[32]) {
    const int c = block * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    float s = 0.0f;
    if (c < g.m) {
        const float* const from = g.sums + c;
        for (int r = part; r < g.pieces; r += 64) {       // eight loads on their way at a time
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = gload(from + (int64_t)(r + 8 * k < g.pieces ? r + 8 * k : r) * g.m);
#pragma unroll
            for (int k = 0; k < 8; ++k) s += r + 8 * k < g.pieces ? v[k] : 0.0f;
        }
    }
    lds[part][threadIdx.x & 31] = s;
    __syncthreads();
    if (part || c >= g.m) return;
    for (int k = 1; k < 8; ++k) s += lds[k][threadIdx.x];
    s *= g.alpha;
    gstore(g.dbias + c, g.accumulate ? gload(g.dbias + c) + s : s);
}

template <class L, int PER_CU>
__global__ __launch_bounds__(64 * L::NW, PER_CU * L::NW / 4) void dense_grad_kernel(const DenseGrads g, const GradOrder o) {
    extern __shared__ __align__(1024) unsigned char lds[];
    grad_tile<L>(g, o, xcd_order(blockIdx.x, gridDim.x), lds);      // an XCD has few pieces of the rows and reads few of them
}

// dW (+)= the sum of the partials in order; behind those work-groups the ones of dbias
__global__ __launch_bounds__(256) void dense_sum_kernel(const DenseGrads g, int splits, int blocks) {
    __shared__ float lds[8][32];
    if ((int)blockIdx.x >= blocks) {
        bias_block(g, (int)blockIdx.x - blocks, lds);
        return;
    }
    const int64_t size = (int64_t)g.m * g.n, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= size) return;
    f32x4 v = {0, 0, 0, 0};
    for (int p = 0; p < splits; p += 4) {                 // four loads on their way at a time
        f32x4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = gload(reinterpret_cast<const f32x4*>(g.partials + (p + k < splits ? p + k : p) * size + i));
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (p + k < splits) v += x[k];
    }
    f32x4* const d = reinterpret_cast<f32x4*>(g.dW + i);
    if (g.accumulate) v += gload(d);
    gstore(d, v);
}

// Everything behind dZ for few rows in one launch: the tiles of dX, of dW, and dbias.
template <class L>
__global__ __launch_bounds__(256, 2) void dense_few_rows_kernel(const DenseProduct x, const Order order, const DenseGrads g, const GradOrder o) {
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tiles = order.row_tiles * order.col_tiles, i = (int)blockIdx.x - tiles;
    if (i < 0) dense_tile<Tile<64, 64, 2, 2, 2>, false>(x, order, xcd_order(blockIdx.x, tiles), 0, lds);
    else if (i < o.tiles) grad_tile<L>(g, o, xcd_order(i, o.tiles), lds);
    else bias_block(g, i - o.tiles, reinterpret_cast<float (*)[32]>(lds));
}

template <int V> using Grad256 = GradTile<256, 256, 4, 2, V>;
template <int V> using Grad128 = GradTile<128, 128, 2, 2, V>;
template <int V> using Grad64 = GradTile<64, 64, 2, 2, V>;

template <class L, int PER_CU>
hipError_t launch_grad(const DenseGrads& p, const GradOrder& o, hipStream_t s) {
    static std::atomic<bool> attr_set{false};
    const hipError_t e = lds_allowed(reinterpret_cast<const void*>(&dense_grad_kernel<L, PER_CU>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    const int64_t blocks = (int64_t)o.tiles * o.splits;
    if (blocks > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((dense_grad_kernel<L, PER_CU>), dim3((unsigned)blocks), dim3(64 * L::NW), L::lds, s, p, o);
    return hipGetLastError();
}
template <int V>
hipError_t launch_grad(const DenseGrads& p, const GradWay& w, hipStream_t s) {
    switch (w.tile) {
        case 0: return launch_grad<Grad256<V>, 1>(p, w.order, s);
        case 1: return launch_grad<Grad128<V>, 2>(p, w.order, s);
        default: return launch_grad<Grad64<V>, 2>(p, w.order, s);
    }
}
template <int V>
hipError_t launch_few_rows(const DenseProduct& x, const DenseGrads& g, hipStream_t s) {
    using L = Grad64<V>;
    constexpr int lds = L::lds > Tile<64, 64, 2, 2, 2>::lds ? L::lds : Tile<64, 64, 2, 2, 2>::lds;
    static std::atomic<bool> attr_set{false};
    const hipError_t e = lds_allowed(reinterpret_cast<const void*>(&dense_few_rows_kernel<L>), lds, attr_set);
    if (e != hipSuccess) return e;
    const int64_t rt = x.Y ? ceil_div(x.M, 64) : 0, ct = ceil_div(x.Q, 64);
    GradOrder o = grad_order(64, g.M, g.m, g.n, 1);
    if (!g.dW) o.tiles = 0;
    const int64_t blocks = rt * ct + o.tiles + (g.dbias ? ceil_div(g.m, 32) : 0);
    if (blocks > INT_MAX) return hipErrorInvalidValue;
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL((dense_few_rows_kernel<L>), dim3((unsigned)blocks), dim3(256), lds, s, x, Order{(int)rt, (int)ct}, g, o);
    return hipGetLastError();
}

}  // namespace

// Some 1500 work-groups, pieces of 8 rows or more (four waves)
int dense_piece_rows(int64_t M, int m) {
    const int64_t rows = align_up((size_t)ceil_div(M * ceil_div(m, kSlopeCols), 1536), 4);
    return rows < 8 ? 8 : (int)rows;
}
hipError_t launch_dense_slope(const DenseSlope& p, hipStream_t s) {
    const bool rows = p.value[0] || p.sums;
    const int64_t pieces = rows ? ceil_div(p.M, p.rows) : 0, slabs = ceil_div(p.m, kSlopeCols);
    const int64_t blocks = pieces * slabs + (p.Wt ? ceil_div(p.m, 64) * ceil_div(p.n, 64) : 0);
    if (blocks == 0) return hipSuccess;
    if (blocks > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(dense_slope_kernel, dim3((unsigned)blocks), dim3(256), 0, s, p, (int)pieces, (int)slabs);
    return hipGetLastError();
}

size_t dense_grad_partial_bytes(int64_t M, int m, int n) {
    int splits = 1;
    for (int values : {1, 3}) {
        const int k = grad_way(M, m, n, values).order.splits;
        if (k > splits) splits = k;
    }
    return splits == 1 ? 0 : (size_t)splits * (size_t)m * (size_t)n * 4;
}
hipError_t launch_dense_bwd(const DenseProduct& x, const DenseGrads& g, hipStream_t s) {
    const int values = g.values;
    const GradWay w = grad_way(g.M, g.m, g.n, values);
    if (dense_together(g.M, g.m, g.n, x.K, values)) return values == 3 ? launch_few_rows<3>(x, g, s) : launch_few_rows<1>(x, g, s);

    hipError_t e = x.Y ? launch_dense(x, s) : hipSuccess;
    if (e != hipSuccess) return e;
    if (g.dW) {
        e = values == 3 ? launch_grad<3>(g, w, s) : launch_grad<1>(g, w, s);
        if (e != hipSuccess) return e;
    }
    const int64_t blocks = g.dW && w.order.splits > 1 ? ceil_div((int64_t)g.m * g.n, 1024) : 0, more = g.dbias ? ceil_div(g.m, 32) : 0;
    if (blocks + more == 0) return hipSuccess;
    if (blocks + more > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(dense_sum_kernel, dim3((unsigned)(blocks + more)), dim3(256), 0, s, g, w.order.splits, (int)blocks);
    return hipGetLastError();
}

}  // namespace abt
