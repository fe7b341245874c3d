// The factor gradients of the layer with adapters as device code: kernels of their own in adapters_grad.hip, and beside the tiles of dX for few rows in
// adapters.hip.
//     dA_a = sum over the rows i of adapter a of dY_i (s T_i)^T          dB_a = sum of (dT_i) x_i^T
// Contractions over the rows, which lie in any order: `order` lists them adapter by adapter.  The narrow operand is fp32 in three bf16 planes; the wide
// one passes through LDS as it lies, rows of 256 bytes, and both are read with the transposing load: four rows of sixteen columns per
// sixteen lanes.
#pragma once

#include "adapters_device.h"

namespace abt {
namespace {

constexpr int kPiece = 64;                                // rows of a slab; pieces are whole slabs

// VB blocks of 16 rank columns
template <int VB>
struct Grad {
    static constexpr int RP = 16 * VB, VROW = 3 * RP * 2;            // bytes of a row's planes
    static constexpr int upart = kPiece * 256, vpart = kPiece * VROW < 8192 ? 8192 : kPiece * VROW, slab = upart + vpart;
    static constexpr int NU = upart / 4096, NV = vpart / 4096, NL = NU + NV;       // load instructions per wave and slab
    static constexpr int NS = VB == 1 || VB == 4 ? 3 : 2;           // up to VB = 2 two work-groups share a compute unit
    static constexpr int list = 1024 * 4;                            // a piece's part of `order`
    static constexpr int lds = NS * slab + list;
    static_assert(lds <= 160 * 1024, "");
    // 16-byte chunks of a row change places so that the sixteen rows of a transposing load fall on all banks (32 bytes of each)
    static __device__ __forceinline__ int uswz(int row) { return (row & 7) << 1; }
    static __device__ __forceinline__ int vswz(int row) { return VB == 1 ? 0 : VB == 2 ? ((row >> 2) & 1) << 1 : VB == 4 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; }
};
constexpr int kMaxPiece = 1024;

struct Side { const uint16_t* U; const uint16_t* V; float* part; float* out; int cols, blocks; };

// 32 of a slab's rows
template <int VB, bool COLS_FIRST, int H>
__device__ __forceinline__ void half_slab(uint32_t slab, const int (&ua)[2], const int (&va)[VB], f32x4 (&acc)[2][VB]) {
    using L = Grad<VB>;
    u32x4 u[2], w[3];
    read_tr2<H * 32 * 256, 16 * 256>(slab + ua[0], slab + ua[1], u[0], u[1]);
#pragma unroll
    for (int v = 0; v < VB; ++v) {
        read_tr3<H * 32 * L::VROW, L::RP * 2, 16 * L::VROW>(slab + va[v], w);
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int b = 0; b < 2; ++b) acc[b][v] = COLS_FIRST ? mfma16(w[q], u[b], acc[b][v]) : mfma16(u[b], w[q], acc[b][v]);
    }
}

// Rows [p piece, (p + 1) piece) of the list, whatever their adapters: their sums go to slot p + a of the partials.  Or, piece = 0: all rows of adapter p (at
// most kMaxPiece), and the sum is the gradient.  COLS_FIRST: both are [cols, r] (dA), else [r, cols] (dB).
template <int VB, bool COLS_FIRST>
__device__ __forceinline__ void grad_piece(const AdapterGrads& g, const Side& side, int block, int piece, int p, unsigned char* lds) {
    using L = Grad<VB>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, lq = lane >> 4;
    const int total = __builtin_amdgcn_readfirstlane(gload(g.offsets + g.count));
    const bool whole = piece == 0;
    const int begin = whole ? __builtin_amdgcn_readfirstlane(gload(g.offsets + p)) : p * piece;
    const int end = whole ? __builtin_amdgcn_readfirstlane(gload(g.offsets + p + 1)) : begin + piece < total ? begin + piece : total;
    if (begin >= end && !whole) return;
    int* const list = reinterpret_cast<int*>(lds + L::NS * L::slab);
    for (int i = threadIdx.x; i < end - begin; i += 256) list[i] = gload(g.order + begin + i);
    // the first adapter of the piece: the one with offsets[a] <= begin < offsets[a + 1]
    int a = p;
    if (!whole) {
        int below = 0;
        for (int i = lane; i < g.count; i += 64) below += gload(g.offsets + i + 1) <= begin ? 1 : 0;
#pragma unroll
        for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
        a = __builtin_amdgcn_readfirstlane(below);
    }
    __syncthreads();
    const int col0 = block * 128, cols = side.cols - col0 < 128 ? side.cols - col0 : 128;
    const int uc = lane & 15;
    // What this lane addresses for a transposing load: row 4 lq + li / 4 of a step, four columns.  The swizzles of rows 16 apart are alike.
    const int trow = 4 * lq + (li >> 2), tcol = 4 * (li & 3);
    int ua[2], va[VB];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int c = wave * 32 + 16 * b + tcol;
        ua[b] = trow * 256 + (((c >> 3) ^ L::uswz(trow)) * 16) + (c & 7) * 2;
    }
#pragma unroll
    for (int v = 0; v < VB; ++v) {                        // of the first plane
        const int c = 16 * v + tcol;
        va[v] = L::upart + trow * L::VROW + (((c >> 3) ^ L::vswz(trow)) * 16) + (c & 7) * 2;
    }
    while (true) {
        const int a_end0 = __builtin_amdgcn_readfirstlane(gload(g.offsets + a + 1));
        const int a_begin0 = __builtin_amdgcn_readfirstlane(gload(g.offsets + a));
        const int s0 = (a_begin0 > begin ? a_begin0 : begin) - begin, s1 = (a_end0 < end ? a_end0 : end) - begin;    // in the list
        if (s1 > s0 || whole) {                           // (an adapter without rows: zeros)
            const int ns = (s1 - s0 + kPiece - 1) / kPiece;
            auto issue = [&](int s, int slot) {
                unsigned char* const dst = lds + slot * L::slab;
#pragma unroll
                for (int j = 0; j < L::NU; ++j) {         // four rows of 16 chunks
                    const int r = 4 * (wave + 4 * j) + lq, at = s0 + s * kPiece + r;
                    const int c = (uc ^ L::uswz(r)) * 8;
                    const void* src = zero_line;
                    if (at < s1 && c < cols) src = side.U + (int64_t)list[at] * side.cols + col0 + c;
                    load_lds16_at(src, dst + (wave + 4 * j) * 1024);
                }
                constexpr int CV = 6 * VB;                // chunks of a row's planes
#pragma unroll
                for (int j = 0; j < L::NV; ++j) {
                    const int pos = 64 * (wave + 4 * j) + lane, r = pos / CV, at = s0 + s * kPiece + r;
                    const int c = (pos - r * CV) ^ L::vswz(r);
                    const void* src = zero_line;
                    if (r < kPiece && at < s1) src = side.V + (int64_t)list[at] * (3 * L::RP) + c * 8;
                    load_lds16_at(src, dst + L::upart + (wave + 4 * j) * 1024);
                }
            };
            f32x4 acc[2][VB];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < VB; ++v) acc[u][v] = f32x4{0, 0, 0, 0};
            int issued = 0;
            for (; issued < L::NS - 1 && issued < ns; ++issued) issue(issued, issued);
            for (int s = 0; s < ns; ++s) {
                const int behind = issued - s - 1;
                if (behind >= L::NS - 2) wait_newest<(L::NS - 2) * L::NL>();
                else wait_newest<0>();
                lds_barrier();
                if (issued < ns) { issue(issued, issued % L::NS); ++issued; }
                const unsigned char* const us = lds + (s % L::NS) * L::slab;
                // 32 rows a step: row 16 t + 4 lq + j of it is element 4 t + j of lane group lq, on both sides
                half_slab<VB, COLS_FIRST, 0>(lds_address(us), ua, va, acc);
                half_slab<VB, COLS_FIRST, 1>(lds_address(us), ua, va, acc);
            }
            lds_barrier();                                // the slots may be loaded again
            float* const to = whole ? side.out + (int64_t)a * side.cols * g.r : side.part + (int64_t)(p + a) * side.cols * g.r;
            const bool add = whole && g.accumulate;
            auto store = [&](int64_t at, f32x4 v) {
                f32x4* const d = reinterpret_cast<f32x4*>(to + at);
                gstore(d, add ? gload(d) + v : v);
            };
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int v = 0; v < VB; ++v) {
                    if (COLS_FIRST) {
                        const int c = wave * 32 + 16 * b + li, j = 16 * v + 4 * lq;
                        if (c < cols && j < g.r) store((int64_t)(col0 + c) * g.r + j, acc[b][v]);
                    } else {
                        const int c = wave * 32 + 16 * b + 4 * lq, j = 16 * v + li;
                        if (c < cols && j < g.r) store((int64_t)j * side.cols + col0 + c, acc[b][v]);
                    }
                }
        }
        if (whole || a_end0 >= end || ++a >= g.count) return;
    }
}

// Which gradients a launch makes; part: where their partials lie
inline void grad_sides(const AdapterGrads& p, int64_t slots, Side& a, Side& b) {
    a = Side{p.dY, p.T_planes, p.partials, p.dA, p.m, p.dA ? (p.m + 127) / 128 : 0};
    b = Side{p.X, p.dT_planes, p.partials + slots * p.m * p.r, p.dB, p.n, p.dB ? (p.n + 127) / 128 : 0};
}
// block of both sides' columns
template <int VB>
__device__ __forceinline__ void grad_block(const AdapterGrads& g, const Side& a, const Side& b, int block, int piece, int p, unsigned char* lds) {
    if (block < a.blocks) grad_piece<VB, true>(g, a, block, piece, p, lds);
    else grad_piece<VB, false>(g, b, block - a.blocks, piece, p, lds);
}

}  // namespace
}  // namespace abt
