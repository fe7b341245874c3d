// Device code that the kernels of the layer with adapters share: small helpers, and what the backward prepares beside its first product.
#pragma once

#include <atomic>

#include "adapters.h"
#include "adapters_operands.h"

namespace abt {
namespace {

// Where loads to LDS that have nothing to fetch read zeros
__device__ const __align__(16) uint32_t zero_line[4] = {0, 0, 0, 0};

typedef __attribute__((ext_vector_type(4))) short s16x4;
__device__ __forceinline__ u32x2 read_tr(const unsigned char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(void*)p));
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }
// Before the transposing load in its builtin form the compiler waits for every load to LDS on its way, whichever slot it goes to: beside a ring of them
// they are issued here, each block with its own wait.  Operand k of a block is OFF + k STEP and, its second half, BACK bytes behind.
template <int OFF, int STEP, int BACK>
__device__ __forceinline__ void read_tr3(uint32_t at, u32x4 (&v)[3]) {
    u32x2 a, b, c, d, e, f;
    asm volatile("ds_read_b64_tr_b16 %0, %6 offset:%7\n\tds_read_b64_tr_b16 %1, %6 offset:%8\n\tds_read_b64_tr_b16 %2, %6 offset:%9\n\t"
                 "ds_read_b64_tr_b16 %3, %6 offset:%10\n\tds_read_b64_tr_b16 %4, %6 offset:%11\n\tds_read_b64_tr_b16 %5, %6 offset:%12\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(e), "=&v"(f)
                 : "v"(at), "n"(OFF), "n"(OFF + BACK), "n"(OFF + STEP), "n"(OFF + STEP + BACK), "n"(OFF + 2 * STEP), "n"(OFF + 2 * STEP + BACK));
    v[0] = u32x4{a[0], a[1], b[0], b[1]};
    v[1] = u32x4{c[0], c[1], d[0], d[1]};
    v[2] = u32x4{e[0], e[1], f[0], f[1]};
}
// two operands at addresses of their own
template <int OFF, int BACK>
__device__ __forceinline__ void read_tr2(uint32_t at0, uint32_t at1, u32x4& v0, u32x4& v1) {
    u32x2 a, b, c, d;
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\tds_read_b64_tr_b16 %2, %5 offset:%6\n\t"
                 "ds_read_b64_tr_b16 %3, %5 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d) : "v"(at0), "v"(at1), "n"(OFF), "n"(OFF + BACK));
    v0 = u32x4{a[0], a[1], b[0], b[1]};
    v1 = u32x4{c[0], c[1], d[0], d[1]};
}
// the same with halves at addresses of their own, and all of it once more OFF bytes further on
template <int OFF>
__device__ __forceinline__ void read_tr4(uint32_t at0, uint32_t back0, uint32_t at1, uint32_t back1, u32x4& v0, u32x4& v1, u32x4& w0, u32x4& w1) {
    u32x2 a, b, c, d, e, f, g, h;
    asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9\n\tds_read_b64_tr_b16 %2, %10\n\tds_read_b64_tr_b16 %3, %11\n\t"
                 "ds_read_b64_tr_b16 %4, %8 offset:%12\n\tds_read_b64_tr_b16 %5, %9 offset:%12\n\tds_read_b64_tr_b16 %6, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%12\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d), "=&v"(e), "=&v"(f), "=&v"(g), "=&v"(h) : "v"(at0), "v"(back0), "v"(at1), "v"(back1), "n"(OFF));
    v0 = u32x4{a[0], a[1], b[0], b[1]};
    v1 = u32x4{c[0], c[1], d[0], d[1]};
    w0 = u32x4{e[0], e[1], f[0], f[1]};
    w1 = u32x4{g[0], g[1], h[0], h[1]};
}
// lane l's 16 bytes at its own address go to LDS address dst + 16 l
__device__ __forceinline__ void load_lds16_at(const void* src, unsigned char* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src, (__attribute__((address_space(3))) uint32_t*)(void*)dst, 16, 0, 0);
}

inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<bool>& done) {
    if (done.load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.store(true, std::memory_order_release);
    return e;
}

// ------------------------------------------------------------------------------------------ preparation
// Work-group a < count lists the rows of adapter a, behind those of the adapters before it; four waves count and then write a quarter of the rows
// each, so the rows of an adapter stay in order.
__device__ __forceinline__ void list_rows(const AdapterPrep& p, int a, unsigned char* lds) {
    int* const mine = reinterpret_cast<int*>(lds);
    int* const below = mine + 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t each = (p.M + 255) / 256 * 64;       // whole waves of rows
    const int64_t r0 = wave * each, r1 = r0 + each < p.M ? r0 + each : p.M;
    // sixteen loads on their way at a time; ids past the wave's rows count as no adapter
    const auto ids_of = [&](int64_t r, int (&id)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) id[i] = gload(p.row_adapter + (r + 64 * i + lane < r1 ? r + 64 * i + lane : 0));
#pragma unroll
        for (int i = 0; i < 16; ++i) id[i] = r + 64 * i + lane < r1 ? id[i] : -1;
    };
    int m = 0, b = 0, id[16];
    for (int64_t r = r0; r < r1; r += 1024) {
        ids_of(r, id);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            m += id[i] == a;
            b += id[i] >= 0 && id[i] < a;
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        m += __shfl_xor(m, d);
        b += __shfl_xor(b, d);
    }
    if (lane == 0) { mine[wave] = m; below[wave] = b; }
    __syncthreads();
    int at = 0, before = 0, all = 0;
    for (int w = 0; w < 4; ++w) {
        before += below[w];
        at += w < wave ? mine[w] : 0;
        all += mine[w];
    }
    if (threadIdx.x == 0) {
        gstore(p.offsets + a, before);
        if (a == p.count - 1) gstore(p.offsets + a + 1, before + all);
    }
    at += before;
    for (int64_t r = r0; r < r1; r += 1024) {
        if (r1 - r0 > 1024) ids_of(r, id);                // (else they are still here)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint64_t who = __ballot(id[i] == a);
            if (id[i] == a) gstore(p.order + at + __builtin_popcountll(who & ((1ull << lane) - 1)), (int)(r + 64 * i + lane));
            at += __builtin_popcountll(who);
        }
    }
}

// Work-groups: one per adapter for its rows, the others take tiles of 64 x 64 of W and of every adapter's B in turn: in through LDS, out through the
// transposing load, the next tile on its way meanwhile.  All dimensions are multiples of 8.
struct PrepBlocks { int list, w, b, all; };               // lists; tiles of W, of one B; all work-groups
constexpr int kPrepPitch = 144, kPrepLds = 64 * kPrepPitch;

__device__ __forceinline__ void prepare(const AdapterPrep& p, const PrepBlocks& n, int i, unsigned char* lds) {
    if (i < n.list) {
        list_rows(p, i, lds);
        return;
    }
    const int tn = (p.n + 63) / 64;
    const int64_t tiles = n.w + (int64_t)n.b * p.count;
    struct Tile { const uint16_t* src; uint16_t* dst; int rows, cols, r0, c0; };
    const auto tile_of = [&](int64_t k) {
        if (k < n.w) return Tile{p.W, p.Wt, p.m, p.n, (int)(k / tn) * 64, (int)(k % tn) * 64};
        const int64_t a = (k - n.w) / n.b;
        const int t = (int)((k - n.w) - a * n.b);
        return Tile{p.B + a * p.n * p.r, p.Bt + a * p.n * p.r, p.r, p.n, t / tn * 64, t % tn * 64};
    };
    u32x4 v[2];
    const auto load = [&](const Tile& t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = threadIdx.x + 256 * h, r = t.r0 + (e >> 3), c = t.c0 + (e & 7) * 8;
            v[h] = gload(reinterpret_cast<const u32x4*>(t.src + (r < t.rows && c < t.cols ? (int64_t)r * t.cols + c : 0)));
        }
    };
    int64_t k = i - n.list;
    if (k >= tiles) return;
    Tile t = tile_of(k);
    load(t);
    while (true) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int e = threadIdx.x + 256 * h;
            *reinterpret_cast<u32x4*>(lds + (e >> 3) * kPrepPitch + (e & 7) * 16) = v[h];
        }
        lds_barrier();
        const Tile done = t;
        k += n.all - n.list;
        if (k < tiles) {
            t = tile_of(k);
            load(t);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {                     // sixteen lanes: sixteen columns, eight rows
            const int l = threadIdx.x & 15, g = (threadIdx.x >> 4) + 16 * h, r8 = (g & 7) * 8, c16 = (g >> 3) * 16;
            const unsigned char* const at = lds + (r8 + (l >> 2)) * kPrepPitch + (c16 + 4 * (l & 3)) * 2;
            const u32x2 a = read_tr(at), b = read_tr(at + 4 * kPrepPitch);
            const int c = done.c0 + c16 + l, r = done.r0 + r8;
            if (c < done.cols && r < done.rows) gstore(reinterpret_cast<u32x4*>(done.dst + (int64_t)c * done.rows + r), u32x4{a[0], a[1], b[0], b[1]});
        }
        if (k >= tiles) return;
        lds_barrier();                                    // the tile's place is free
    }
}

inline PrepBlocks prep_blocks(const AdapterPrep& p) {
    const int64_t tm = ceil_div(p.m, 64), tn = ceil_div(p.n, 64), tr = ceil_div(p.r, 64);
    PrepBlocks n{p.order ? p.count : 0, p.W ? (int)(tm * tn) : 0, p.B ? (int)(tn * tr) : 0, 0};
    const int64_t tiles = n.w + (int64_t)n.b * p.count;
    // four tiles each, but no more work-groups than leave room for those of the product beside them
    const int64_t each = ceil_div(tiles, 4);
    n.all = n.list + (int)(each < 128 ? each : 128);
    return n;
}

}  // namespace
}  // namespace abt
