// Gradients of the dense layer: what its products are made of, and dW = dZ^T X, a contraction over the rows.
#include <atomic>
#include <climits>

#include "activation.h"
#include "dense.h"

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
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) { return u32x4{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])}; }

__device__ __forceinline__ void slope_piece(const DenseSlope& g, int piece, int col0, float (*sums)[kSlopeCols]) {
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
        for (int64_t r = first + wave; r < last; r += 4) {
            const int64_t at = r * g.m + col;
            float v[8];
            unpack8(gload(reinterpret_cast<const u32x4*>(g.dY + at)), v);
            if (g.Z) {
                float z[8];
                unpack8(gload(reinterpret_cast<const u32x4*>(g.Z + at)), z);
                with_activation(g.act, [&](auto act) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] *= slope<decltype(act)::value>(z[k]);
                });
            }
            if (g.drop.state) drop8(drop, key, (uint64_t)at >> 3, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) total[k] += v[k];
            if (!g.high) continue;
            const u32x4 high = pack8(v);
            gstore(reinterpret_cast<u32x4*>(g.high + at), high);
            if (!g.low) continue;
            float h[8], l[8];
            unpack8(high, h);
#pragma unroll
            for (int k = 0; k < 8; ++k) l[k] = __builtin_fabsf(h[k]) < __builtin_inff() ? v[k] - h[k] : 0.0f;      // (infinities and NaN are in h)
            gstore(reinterpret_cast<u32x4*>(g.low + at), pack8(l));
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
        gstore(reinterpret_cast<u32x4*>(g.Wt + (int64_t)(c0 + c) * g.m + r0 + r), v);
    }
}

__global__ __launch_bounds__(256) void dense_slope_kernel(const DenseSlope g, int pieces, int slabs) {
    __shared__ union { float sums[4][kSlopeCols]; uint16_t tile[64][72]; } lds;
    const int i = blockIdx.x, own = pieces * slabs;
    if (i < own) slope_piece(g, i / slabs, i % slabs * kSlopeCols, lds.sums);
    else transpose_block(g, i - own, lds.tile);
}

// ------------------------------------------------------------------------------------------ dW
// TP x TQ of dW by WP x WQ waves of RB x CB blocks of 32 x 32; a slab is 32 rows of both sides as they lie, in a ring of NS slots.  Both are read with the
// transposing load: sixteen lanes ask for four rows of sixteen columns, and lane i gets the four of column i.
template <int TP_, int TQ_, int WP_, int WQ_, int PLANES_, int NS_>
struct GradTile {
    static constexpr int TP = TP_, TQ = TQ_, WP = WP_, WQ = WQ_, PLANES = PLANES_, NS = NS_, NW = WP * WQ;
    static constexpr int RB = TP / (32 * WP), CB = TQ / (32 * WQ);
    static constexpr int ppart = 32 * TP * 2, qpart = 32 * TQ * 2, xbase = PLANES * ppart, slab = xbase + qpart, lds = NS * slab;
    static constexpr int NP = ppart / 1024 / NW, NQ = qpart / 1024 / NW, NL = PLANES * NP + NQ;        // load instructions per wave and slab
    static_assert(NP * NW * 1024 == ppart && NQ * NW * 1024 == qpart && RB * 32 * WP == TP && CB * 32 * WQ == TQ && TP >= 128 && TQ >= 128, "");
    static_assert(lds <= 160 * 1024 && (NS - 2) * NL < 64, "");
};

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }
// Two operands of 16 rows, whose halves are BACK bytes apart.  Before the transposing load in its builtin form the compiler waits for every load to LDS on its way,
// whichever slot of the ring it goes to: here they are issued with a wait of their own.
template <int OFF, int BACK>
__device__ __forceinline__ void read_two(uint32_t at0, uint32_t at1, u32x4& v0, u32x4& v1) {
    u32x2 a, b, c, d;
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\tds_read_b64_tr_b16 %2, %5 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %3, %5 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d) : "v"(at0), "v"(at1), "n"(OFF), "n"(OFF + BACK) : "memory");
    v0 = u32x4{a[0], a[1], b[0], b[1]};
    v1 = u32x4{c[0], c[1], d[0], d[1]};
}

struct GradOrder { int col_tiles, splits, slabs; };       // tiles across; pieces of the rows and their length in slabs

template <class L>
__device__ __forceinline__ void grad_tile(const DenseGrads& g, const GradOrder& o, int block, unsigned char* lds) {
    constexpr int RB = L::RB, CB = L::CB, NW = L::NW;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lj = lane & 31, lh = lane >> 5, li = lane & 15;
    const int wp = wave / L::WQ, wq = wave % L::WQ;
    const int split = block % o.splits, tile = block / o.splits;
    const int p0 = tile / o.col_tiles * L::TP, q0 = tile % o.col_tiles * L::TQ;
    const int pcols = g.m - p0 < L::TP ? g.m - p0 : L::TP, qcols = g.n - q0 < L::TQ ? g.n - q0 : L::TQ;
    const int64_t first = (int64_t)split * o.slabs * 32, last = first + (int64_t)o.slabs * 32 < g.M ? first + (int64_t)o.slabs * 32 : g.M;
    const int ns = (int)((last - first + 31) / 32);

    // chunk c of row r lies at c ^ 4 (r & 3): the eight rows of 64 bytes that a load asks for fall on all banks
    auto lane_offset = [&](int pitch, int width, int cols, int j) {
        const int pos = (j * NW + wave) * 64 + lane, r = pos / (pitch / 8), c = ((pos % (pitch / 8)) ^ ((r & 3) << 2)) * 8;
        return c < cols ? (r * width + c) * 2 : kBufNowhere;
    };
    int poff[L::NP], qoff[L::NQ];
#pragma unroll
    for (int j = 0; j < L::NP; ++j) poff[j] = lane_offset(L::TP, g.m, pcols, j);
#pragma unroll
    for (int j = 0; j < L::NQ; ++j) qoff[j] = lane_offset(L::TQ, g.n, qcols, j);
    auto issue = [&](int s, int slot) {
        unsigned char* const dst = lds + slot * L::slab + wave * 1024;
        const int64_t row = first + (int64_t)s * 32;
        const int rows = last - row < 32 ? (int)(last - row) : 32;            // rows past the last one read zeros
        const int64_t pbytes = ((int64_t)(rows - 1) * g.m + pcols) * 2, qbytes = ((int64_t)(rows - 1) * g.n + qcols) * 2;
        const rsrc_t high = make_rsrc(g.high + row * g.m + p0, pbytes), x = make_rsrc(g.X + row * g.n + q0, qbytes);
#pragma unroll
        for (int j = 0; j < L::NP; ++j) load_lds16(high, dst + j * (NW * 1024), poff[j], 0);
        if (L::PLANES == 2) {
            const rsrc_t low = make_rsrc(g.low + row * g.m + p0, pbytes);
#pragma unroll
            for (int j = 0; j < L::NP; ++j) load_lds16(low, dst + L::ppart + j * (NW * 1024), poff[j], 0);
        }
#pragma unroll
        for (int j = 0; j < L::NQ; ++j) load_lds16(x, dst + L::xbase + j * (NW * 1024), qoff[j], 0);
    };

    f32x16 acc[RB][CB];
#pragma unroll
    for (int a = 0; a < RB; ++a)
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    // Rows 4 lh + li / 4 and 8 more of a step of sixteen; quad t of a block's columns, taken in the order of out_row on X's side, so that a lane's sums are
    // sixteen consecutive columns of a row of dW.
    const int t = 4 * ((lane >> 4) & 1) + (li & 3), tx = 4 * (t & 1) + (t >> 1), trow = 4 * lh + (li >> 2), swz = ((li >> 2) & 3) << 2;
    uint32_t pat[RB], qat[CB];
#pragma unroll
    for (int a = 0; a < RB; ++a) pat[a] = trow * (L::TP * 2) + ((((wp * RB + a) * 4 + (t >> 1)) ^ swz) * 16) + (t & 1) * 8;
#pragma unroll
    for (int b = 0; b < CB; ++b) qat[b] = L::xbase + trow * (L::TQ * 2) + ((((wq * CB + b) * 4 + (tx >> 1)) ^ swz) * 16) + (tx & 1) * 8;
    auto step = [&](uint32_t base, auto half) {
        constexpr int H = decltype(half)::value, PO = H * 16 * L::TP * 2, QO = H * 16 * L::TQ * 2;
        static_assert(RB % 2 == 0 && CB % 2 == 0, "");
        u32x4 x[CB], z[L::PLANES][RB];
#pragma unroll
        for (int b = 0; b < CB; b += 2) read_two<QO, 8 * L::TQ * 2>(base + qat[b], base + qat[b + 1], x[b], x[b + 1]);
#pragma unroll
        for (int a = 0; a < RB; a += 2) read_two<PO, 8 * L::TP * 2>(base + pat[a], base + pat[a + 1], z[0][a], z[0][a + 1]);
        if constexpr (L::PLANES == 2)
#pragma unroll
            for (int a = 0; a < RB; a += 2) read_two<PO + L::ppart, 8 * L::TP * 2>(base + pat[a], base + pat[a + 1], z[1][a], z[1][a + 1]);
#pragma unroll
        for (int q = 0; q < L::PLANES; ++q)
#pragma unroll
            for (int a = 0; a < RB; ++a)
#pragma unroll
                for (int b = 0; b < CB; ++b) acc[a][b] = mfma_bf16(x[b], z[q][a], acc[a][b]);
    };
    int issued = 0;
    for (; issued < L::NS - 1 && issued < ns; ++issued) issue(issued, issued);
    for (int s = 0; s < ns; ++s) {
        if (issued - s - 1 >= L::NS - 2) wait_newest<(L::NS - 2) * L::NL>();
        else wait_newest<0>();
        lds_barrier();
        if (issued < ns) { issue(issued, issued % L::NS); ++issued; }
        const uint32_t base = lds_address(lds) + (s % L::NS) * L::slab;
        step(base, std::integral_constant<int, 0>{});
        step(base, std::integral_constant<int, 1>{});
    }
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

template <class L>
__global__ __launch_bounds__(64 * L::NW) void dense_grad_kernel(const DenseGrads g, const GradOrder o) {
    extern __shared__ __align__(1024) unsigned char lds[];
    grad_tile<L>(g, o, blockIdx.x, lds);
}

// dW (+)= the sum of the partials in order; behind those work-groups, 64 columns of dbias each
__global__ __launch_bounds__(256) void dense_sum_kernel(const DenseGrads g, int splits, int blocks) {
    if ((int)blockIdx.x < blocks) {
        const int64_t size = (int64_t)g.m * g.n, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
        if (i >= size) return;
        f32x4 v = {0, 0, 0, 0};
        for (int p = 0; p < splits; p += 8) {             // eight loads on their way at a time
            f32x4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = gload(reinterpret_cast<const f32x4*>(g.partials + (p + k < splits ? p + k : p) * size + i));
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (p + k < splits) v += x[k];
        }
        f32x4* const d = reinterpret_cast<f32x4*>(g.dW + i);
        if (g.accumulate) v += gload(d);
        gstore(d, v);
        return;
    }
    __shared__ float sums[4][64];
    const int c = ((int)blockIdx.x - blocks) * 64 + (threadIdx.x & 63), part = threadIdx.x >> 6;
    float v = 0.0f;
    if (c < g.m)
        for (int p = part; p < g.pieces; p += 4) v += gload(g.sums + (int64_t)p * g.m + c);
    sums[part][threadIdx.x & 63] = v;
    __syncthreads();
    if (part || c >= g.m) return;
    v = ((sums[0][c & 63] + sums[1][c & 63]) + (sums[2][c & 63] + sums[3][c & 63])) * g.alpha;
    gstore(g.dbias + c, g.accumulate ? gload(g.dbias + c) + v : v);
}

using Grad2 = GradTile<128, 256, 2, 4, 2, 4>;
using Grad1 = GradTile<128, 256, 2, 4, 1, 4>;

GradOrder grad_order(int64_t M, int m, int n) {
    const int64_t tiles = ceil_div(m, Grad2::TP) * ceil_div(n, Grad2::TQ), slabs = ceil_div(M, 32);
    int64_t splits = tiles >= 256 ? 1 : 256 / tiles;
    if (splits > slabs / 4) splits = slabs / 4 < 1 ? 1 : slabs / 4;
    const int64_t each = ceil_div(slabs, splits);
    return GradOrder{(int)ceil_div(n, Grad2::TQ), (int)ceil_div(slabs, each), (int)each};
}

template <class L>
hipError_t launch_grad(const DenseGrads& p, const GradOrder& o, hipStream_t s) {
    static std::atomic<bool> attr_set{false};
    if (!attr_set.load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&dense_grad_kernel<L>), hipFuncAttributeMaxDynamicSharedMemorySize, L::lds);
        if (e != hipSuccess) return e;
        attr_set.store(true, std::memory_order_release);
    }
    const int64_t blocks = ceil_div(p.m, L::TP) * o.col_tiles * o.splits;
    if (blocks > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((dense_grad_kernel<L>), dim3((unsigned)blocks), dim3(64 * L::NW), L::lds, s, p, o);
    return hipGetLastError();
}

}  // namespace

// Some 1500 work-groups, pieces of 8 rows or more (four waves)
int dense_piece_rows(int64_t M, int m) {
    const int64_t rows = align_up((size_t)ceil_div(M * ceil_div(m, kSlopeCols), 1536), 4);
    return rows < 8 ? 8 : (int)rows;
}
hipError_t launch_dense_slope(const DenseSlope& p, hipStream_t s) {
    const bool rows = p.high || p.sums;
    const int64_t pieces = rows ? ceil_div(p.M, p.rows) : 0, slabs = ceil_div(p.m, kSlopeCols);
    const int64_t blocks = pieces * slabs + (p.Wt ? ceil_div(p.m, 64) * ceil_div(p.n, 64) : 0);
    if (blocks == 0) return hipSuccess;
    if (blocks > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(dense_slope_kernel, dim3((unsigned)blocks), dim3(256), 0, s, p, (int)pieces, (int)slabs);
    return hipGetLastError();
}

size_t dense_grad_partial_bytes(int64_t M, int m, int n) {
    const GradOrder o = grad_order(M, m, n);
    return o.splits == 1 ? 0 : (size_t)o.splits * (size_t)m * (size_t)n * 4;
}
hipError_t launch_dense_grads(const DenseGrads& p, hipStream_t s) {
    const GradOrder o = grad_order(p.M, p.m, p.n);
    if (p.dW) {
        const hipError_t e = p.low ? launch_grad<Grad2>(p, o, s) : launch_grad<Grad1>(p, o, s);
        if (e != hipSuccess) return e;
    }
    const int64_t blocks = p.dW && o.splits > 1 ? ceil_div((int64_t)p.m * p.n, 1024) : 0, more = p.dbias ? ceil_div(p.m, 64) : 0;
    if (blocks + more == 0) return hipSuccess;
    if (blocks + more > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(dense_sum_kernel, dim3((unsigned)(blocks + more)), dim3(256), 0, s, p, o.splits, (int)blocks);
    return hipGetLastError();
}

}  // namespace abt
