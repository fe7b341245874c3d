// A tile of the dense product with its epilogue, as device code.
#pragma once

#include <atomic>

#include "activation.h"
#include "dense.h"
#include "nt_tile.h"

namespace abt {
namespace {

inline hipError_t lds_allowed(const void* kernel, int bytes, std::atomic<bool>& done) {
    if (done.load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.store(true, std::memory_order_release);
    return e;
}

// What a tile's rows are on their way out: rows of TN bf16 values in LDS, whose 16-byte chunks change places within 128 bytes (chunk c of row r lies
// at c ^ (r & 7)), so that the lanes of a wave, which hold a row each, meet on no bank.
template <class L>
struct OutRows {
    static constexpr int CPR = L::TN / 8, count = L::TM * CPR / (64 * L::NW);       // chunks of a row; instructions per wave
    static_assert(L::TN >= 64 && L::TM * CPR % (64 * L::NW) == 0 && L::TM * L::TN * 2 <= L::lds, "");
    static __device__ __forceinline__ int at(int r, int c) { return r * (L::TN * 2) + ((c ^ (r & 7)) * 16); }
    // chunk i of this thread: its row, and its first column
    static __device__ __forceinline__ void place(int e, int& r, int& c) {
        r = e / CPR;
        c = ((e % CPR) ^ (r & 7)) * 8;
    }
    static __device__ __forceinline__ void load(const uint16_t* from, int64_t row0, int col0, int rows, int cols, int Q, int wave, int lane, unsigned char* lds) {
        const rsrc_t res = make_rsrc(from + row0 * Q + col0, ((int64_t)(rows - 1) * Q + cols) * 2);
#pragma unroll
        for (int i = 0; i < count; ++i) {
            int r, c;
            place((i * L::NW + wave) * 64 + lane, r, c);
            load_lds16(res, lds + (i * L::NW + wave) * 1024, r < rows && c < cols ? (r * Q + c) * 2 : kBufNowhere, 0);
        }
    }
    static __device__ __forceinline__ void store(uint16_t* to, int64_t row0, int col0, int rows, int cols, int Q, int wave, int lane, const unsigned char* lds) {
        const rsrc_t res = make_rsrc(to + row0 * Q + col0, ((int64_t)(rows - 1) * Q + cols) * 2);
#pragma unroll
        for (int i = 0; i < count; ++i) {
            const int e = (i * L::NW + wave) * 64 + lane;
            int r, c;
            place(e, r, c);
            buf_store16(*reinterpret_cast<const u32x4*>(lds + e * 16), res, r < rows && c < cols ? (r * Q + c) * 2 : kBufNowhere, 0);
        }
    }
};

// `block` in the order of tile_at.  PARTS: the sum over the slabs of piece `part` only, as fp32 to g.parts [pieces, M, Q]; what makes a result of them is another launch.
template <class L, bool PARTS>
__device__ __forceinline__ void dense_tile(const DenseProduct& g, const Order& order, int block, int part, unsigned char* lds) {
    constexpr int RB = L::RB, CB = L::CB, NW = L::NW;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lj = lane & 31, lh = lane >> 5;
    const int wr = wave / L::WN, wc = wave % L::WN;
    int rt, ct;
    tile_at(order, block, rt, ct);
    const int64_t row0 = (int64_t)rt * L::TM;
    const int col0 = ct * L::TN;
    const int rows = g.M - row0 < L::TM ? (int)(g.M - row0) : L::TM;
    const int cols = g.Q - col0 < L::TN ? g.Q - col0 : L::TN;

    // Load instruction j of a wave covers rows 8 (wave + NW j) .. + 7 of X, or of W: this lane's row among them and its chunk (NW is even, so the chunk
    // is the same for all j).  Rows past the last one read zeros, and so do chunks past the end of a row.
    const int lrow = 8 * wave + (lane >> 3);
    const int chunk = ((lane & 7) ^ ((lrow >> 1) & 7)) * 16;
    const int bytes = g.K * 2, all = (bytes + 127) / 128, slab0 = PARTS ? part * g.piece : 0, slabs = PARTS && all - slab0 > g.piece ? g.piece : all - slab0;
    const rsrc_t xres = make_rsrc((const char*)g.X + row0 * bytes, (int64_t)rows * bytes);
    const rsrc_t wres = make_rsrc((const char*)g.W + (int64_t)col0 * bytes, (int64_t)cols * bytes);
    int xslot = 0, wslot = L::wbase;                      // of the next parts to be requested
    auto issue = [&](int s) {
        unsigned char *const w = lds + wslot + wave * 1024, *const x = lds + xslot + wave * 1024;
        wslot = wslot == L::wbase + L::AHEAD * L::wpart ? L::wbase : wslot + L::wpart;
        xslot = xslot == L::AHEAD * L::xpart ? 0 : xslot + L::xpart;
        const int k = (slab0 + s) * 128 + chunk;
        const bool there = k < bytes;
        const int off = there ? lrow * bytes + k : kBufNowhere, step = there ? 8 * NW * bytes : 0;
#pragma unroll
        for (int j = 0; j < L::NF; ++j) load_lds16(wres, w + j * (NW * 1024), off + j * step, 0);
#pragma unroll
        for (int j = 0; j < L::NX; ++j) load_lds16(xres, x + j * (NW * 1024), off + j * step, 0);
    };
#pragma unroll
    for (int s = 0; s < L::AHEAD; ++s)
        if (s < slabs) issue(s);
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
    // the operands of a step are read while the products of the step before run, across the barrier too
    Ops o[2];
#pragma unroll
    for (int a = 0; a < RB; ++a) o[1].x[a] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < CB; ++b) o[1].f[b] = u32x4{0, 0, 0, 0};
    for (int s = 0; s < slabs; ++s) {
        // slab s has landed: loads come back in the order of issue
        if (s + L::AHEAD > slabs) wait_newest<0>();
        else wait_newest<L::behind>();
        lds_barrier();
        if (s + L::AHEAD < slabs) issue(s + L::AHEAD);    // into the slots whose reads ended before this barrier
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            read(o[j & 1], j);
            mma(o[(j + 1) & 1]);
#pragma unroll
            for (int i = 0; i < RB + CB; ++i) {           // a read behind every product
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        xat = xat == L::AHEAD * L::xpart ? 0 : xat + L::xpart;
        wat = wat == L::wbase + L::AHEAD * L::wpart ? L::wbase : wat + L::wpart;
    }
    mma(o[1]);

    if constexpr (PARTS) {
        float* const to = g.parts + ((int64_t)part * g.M + row0) * g.Q + col0;
#pragma unroll
        for (int a = 0; a < RB; ++a)
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) {             // eight columns, all there or none
                    const int r = (wr * RB + a) * 32 + lj, c = (wc * CB + b) * 32 + 16 * lh + 8 * h;
                    if (r >= rows || c >= cols) continue;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        f32x4 v;
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = acc[a][b][8 * h + 4 * q + i];
                        gstore(reinterpret_cast<f32x4*>(to + (int64_t)r * g.Q + c + 4 * q), v);
                    }
                }
        return;
    }
    // This lane has row lj of each block, and columns 16 lh .. + 15 of it; a block's bias is asked for one block ahead.
    const rsrc_t bres = make_rsrc(g.bias + col0, g.bias ? cols * 4 : 0);      // zeros without a bias
    struct Bias { f32x4 v[4]; };
    auto bias_of = [&](int b) {
        Bias bias;
#pragma unroll
        for (int q = 0; q < 4; ++q) bias.v[q] = __builtin_bit_cast(f32x4, buf_load16(bres, ((wc * CB + b) * 32 + 16 * lh + 4 * q) * 4, 0));
        return bias;
    };
    const Bias first = bias_of(0);
    lds_barrier();                                        // every wave has read its last slab, and nothing is on its way to LDS
    using O = OutRows<L>;
    // Where LDS has room for two tiles of results, Z and Y are made in one pass: Z lies behind Y (1379 rows, 2304 x 768, gelu, Z: 15.5 -> 15.2 us).
    constexpr int z_at = L::TM * L::TN * 2;
    constexpr bool both = 2 * z_at <= L::lds;
    if (g.residual && (both || !g.Z)) O::load(g.residual, row0, col0, rows, cols, g.Q, wave, lane, lds);       // comes while the rest is computed
    const DropKey key = g.drop.state ? drop_key(g.drop) : DropKey{0, 0, 0, 0};
    // Block after block, all the way to LDS: mixed by the scheduler, or with all sums alive across the choice of the activation, 113 registers of the largest tile
    // spilled.
    auto finish = [&](bool rounded_sum) {                 // Z alone, or Y (and Z)
        Bias bias = first, next = first;
#pragma unroll
        for (int b = 0; b < CB; ++b) {
            if (b + 1 < CB) next = bias_of(b + 1);
#pragma unroll
            for (int a = 0; a < RB; ++a) {
                const int r = (wr * RB + a) * 32 + lj, c = (wc * CB + b) * 32 + 16 * lh;
                float v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = acc[a][b][i] * g.alpha + bias.v[i >> 2][i & 3];
                if (both && g.Z)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        *reinterpret_cast<u32x4*>(lds + z_at + O::at(r, (c >> 3) + h)) =
                            u32x4{pack2_bf16(v[8 * h], v[8 * h + 1]), pack2_bf16(v[8 * h + 2], v[8 * h + 3]), pack2_bf16(v[8 * h + 4], v[8 * h + 5]), pack2_bf16(v[8 * h + 6], v[8 * h + 7])};
                if (!rounded_sum) {
                    if (g.act != ABT_ACT_NONE)
                        with_activation(g.act, [&](auto act) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = activate<decltype(act)::value>(v[i]);
                        });
                    if (g.drop.state) {
                        const uint64_t e = ((uint64_t)(row0 + r) * (uint32_t)g.Q + (uint32_t)(col0 + c)) >> 3;
                        drop8(g.drop, key, e, v);
                        drop8(g.drop, key, e + 1, v + 8);
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x4* const place = reinterpret_cast<u32x4*>(lds + O::at(r, (c >> 3) + h));
                    if (!rounded_sum && g.residual) {     // every lane writes where it has read
                        const u32x4 more = *place;
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[8 * h + i] += __builtin_bit_cast(float, i & 1 ? more[i >> 1] & 0xffff0000u : more[i >> 1] << 16);
                    }
                    u32x4 out;
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[i] = pack2_bf16(v[8 * h + 2 * i], v[8 * h + 2 * i + 1]);
                    *place = out;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            bias = next;
        }
        lds_barrier();
    };
    if (!both && g.Z) {
        finish(true);
        O::store(g.Z, row0, col0, rows, cols, g.Q, wave, lane, lds);
        lds_barrier();
        if (g.residual) O::load(g.residual, row0, col0, rows, cols, g.Q, wave, lane, lds);
    }
    if (g.residual) {
        wait_newest<0>();
        lds_barrier();
    }
    finish(false);
    if (both && g.Z) O::store(g.Z, row0, col0, rows, cols, g.Q, wave, lane, lds + z_at);
    O::store(g.Y, row0, col0, rows, cols, g.Q, wave, lane, lds);
}

}  // namespace
}  // namespace abt
