// Gradients of the adapters, and what the backward prepares.
//     dA_a = sum over the rows i of adapter a of dY_i (s T_i)^T          dB_a = sum of (dT_i) x_i^T
// Contractions over the rows, which lie in any order: `order` lists them adapter by adapter.  The list is cut into pieces of equal length
// whatever the adapters; a work-group has 128 columns of dY or X and one piece, and leaves the sums of each adapter in it as a partial of
// its own (piece p and adapter a meet in slot p + a: along the list either grows by one, so no two meetings share a slot).  A second
// launch adds an adapter's partials in order.  No atomics: the same call gives the same bits.
//
// The narrow operand is fp32 in three bf16 planes (see adapters.hip); the wide one passes through LDS as it lies, rows of 256 bytes, and both are
// read with the transposing load: four rows of sixteen columns per sixteen lanes.
#include <atomic>

#include "adapters.h"

namespace abt {
namespace {

typedef __attribute__((ext_vector_type(4))) short s16x4;

constexpr int kPiece = 64;                                // rows of a slab; pieces are whole slabs

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ u32x2 read_tr(const unsigned char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(void*)p));
}
// lane l's 16 bytes at its own address go to LDS address dst + 16 l
__device__ __forceinline__ void load_lds16_at(const void* src, unsigned char* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src, (__attribute__((address_space(3))) uint32_t*)(void*)dst, 16, 0, 0);
}

// VB blocks of 16 rank columns
template <int VB>
struct Grad {
    static constexpr int RP = 16 * VB, VROW = 3 * RP * 2;            // bytes of a row's planes
    static constexpr int upart = kPiece * 256, vpart = kPiece * VROW < 8192 ? 8192 : kPiece * VROW, slab = upart + vpart;
    static constexpr int NU = upart / 4096, NV = vpart / 4096, NL = NU + NV;       // load instructions per wave and slab
    static constexpr int NS = VB == 8 ? 2 : VB == 4 ? 3 : 4;
    static constexpr int list = 4096 * 4;                            // a piece's part of `order`
    static constexpr int lds = NS * slab + list;
    static_assert(lds <= 160 * 1024, "");
    // 16-byte chunks of a row change places so that the sixteen rows of a transposing load fall on all banks (32 bytes of each)
    static __device__ __forceinline__ int uswz(int row) { return (row & 7) << 1; }
    static __device__ __forceinline__ int vswz(int row) { return VB == 1 ? 0 : VB == 2 ? ((row >> 2) & 1) << 1 : VB == 4 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; }
};
constexpr int kMaxPiece = 4096;

struct Side { const uint16_t* U; const uint16_t* V; float* part; int cols, blocks; };

// COLS_FIRST: the partial is [cols, r] (dA), else [r, cols] (dB)
template <int VB, bool COLS_FIRST>
__device__ __forceinline__ void grad_piece(const AdapterGrads& g, const Side& side, int block, int piece, int p, unsigned char* lds) {
    using L = Grad<VB>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, lq = lane >> 4;
    const int total = __builtin_amdgcn_readfirstlane(gload(g.offsets + g.count));
    const int begin = p * piece, end = begin + piece < total ? begin + piece : total;
    if (begin >= end) return;
    int* const list = reinterpret_cast<int*>(lds + L::NS * L::slab);
    for (int i = threadIdx.x; i < end - begin; i += 256) list[i] = gload(g.order + begin + i);
    // the first adapter of the piece: the one with offsets[a] <= begin < offsets[a + 1]
    int a = 0;
    {
        int below = 0;
        for (int i = lane; i < g.count; i += 64) below += gload(g.offsets + i + 1) <= begin ? 1 : 0;
#pragma unroll
        for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
        a = __builtin_amdgcn_readfirstlane(below);
    }
    __syncthreads();
    const int col0 = block * 128, cols = side.cols - col0 < 128 ? side.cols - col0 : 128;
    const int uc = lane & 15;
    while (true) {
        const int a_end0 = __builtin_amdgcn_readfirstlane(gload(g.offsets + a + 1));
        const int a_begin0 = __builtin_amdgcn_readfirstlane(gload(g.offsets + a));
        const int s0 = (a_begin0 > begin ? a_begin0 : begin) - begin, s1 = (a_end0 < end ? a_end0 : end) - begin;    // in the list
        if (s1 > s0) {
            const int ns = (s1 - s0 + kPiece - 1) / kPiece;
            auto issue = [&](int s, int slot) {
                unsigned char* const dst = lds + slot * L::slab;
#pragma unroll
                for (int j = 0; j < L::NU; ++j) {         // four rows of 16 chunks
                    const int r = 4 * (wave + 4 * j) + lq, at = s0 + s * kPiece + r;
                    const int c = (uc ^ L::uswz(r)) * 8;
                    const void* src = g.zeros;
                    if (at < s1 && c < cols) src = side.U + (int64_t)list[at] * side.cols + col0 + c;
                    load_lds16_at(src, dst + (wave + 4 * j) * 1024);
                }
                constexpr int CV = 6 * VB;                // chunks of a row's planes
#pragma unroll
                for (int j = 0; j < L::NV; ++j) {
                    const int pos = 64 * (wave + 4 * j) + lane, r = pos / CV, at = s0 + s * kPiece + r;
                    const int c = (pos - r * CV) ^ L::vswz(r);
                    const void* src = g.zeros;
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
                else if (L::NS > 3 && behind == L::NS - 3) wait_newest<(L::NS > 3 ? L::NS - 3 : 0) * L::NL>();
                else wait_newest<0>();
                lds_barrier();
                if (issued < ns) { issue(issued, issued % L::NS); ++issued; }
                const unsigned char* const us = lds + (s % L::NS) * L::slab;
                const unsigned char* const vs = us + L::upart;
#pragma unroll
                for (int h = 0; h < 2; ++h) {             // 32 rows: row 32 h + 16 t + 4 lq + j is element 4 t + j of lane group lq, on both sides
                    const int r0 = 32 * h + 4 * lq + (li >> 2);
                    auto operand = [&](const unsigned char* base, int pitch, int sw0, int sw1, int col) {
                        const int c = col + 4 * (li & 3);                  // of the four columns that this lane addresses
                        const u32x2 x = read_tr(base + r0 * pitch + (((c >> 3) ^ sw0) * 16) + (c & 7) * 2);
                        const u32x2 y = read_tr(base + (r0 + 16) * pitch + (((c >> 3) ^ sw1) * 16) + (c & 7) * 2);
                        return u32x4{x[0], x[1], y[0], y[1]};
                    };
                    u32x4 u[2];
#pragma unroll
                    for (int b = 0; b < 2; ++b) u[b] = operand(us, 256, L::uswz(r0), L::uswz(r0 + 16), wave * 32 + 16 * b);
#pragma unroll
                    for (int v = 0; v < VB; ++v)
#pragma unroll
                        for (int q = 0; q < 3; ++q) {
                            const u32x4 w = operand(vs, L::VROW, L::vswz(r0), L::vswz(r0 + 16), q * L::RP + 16 * v);
#pragma unroll
                            for (int b = 0; b < 2; ++b) acc[b][v] = COLS_FIRST ? mfma16(w, u[b], acc[b][v]) : mfma16(u[b], w, acc[b][v]);
                        }
                }
            }
            lds_barrier();                                // the slots may be loaded again
            float* const to = side.part + (int64_t)(p + a) * side.cols * g.r;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int v = 0; v < VB; ++v) {
                    if (COLS_FIRST) {
                        const int c = wave * 32 + 16 * b + li, j = 16 * v + 4 * lq;
                        if (c < cols && j < g.r) gstore(reinterpret_cast<f32x4*>(to + (int64_t)(col0 + c) * g.r + j), acc[b][v]);
                    } else {
                        const int c = wave * 32 + 16 * b + 4 * lq, j = 16 * v + li;
                        if (c < cols && j < g.r) gstore(reinterpret_cast<f32x4*>(to + (int64_t)j * side.cols + col0 + c), acc[b][v]);
                    }
                }
        }
        if (a_end0 >= end || ++a >= g.count) return;
    }
}

template <int VB>
__global__ __launch_bounds__(256) void adapters_grad_kernel(const AdapterGrads g, const Side a, const Side b, int piece) {
    extern __shared__ __align__(1024) unsigned char lds[];
    if ((int)blockIdx.x < a.blocks) grad_piece<VB, true>(g, a, blockIdx.x, piece, blockIdx.y, lds);
    else grad_piece<VB, false>(g, b, (int)blockIdx.x - a.blocks, piece, blockIdx.y, lds);
}

// out[a] (+)= the partials of its pieces, in order; zeros for an adapter without rows
__global__ __launch_bounds__(256) void adapters_sum_kernel(const AdapterGrads g, const Side sa, const Side sb, int piece) {
    const int a = blockIdx.y;
    const int64_t na = sa.blocks ? (int64_t)sa.cols * g.r : 0, nb = sb.blocks ? (int64_t)sb.cols * g.r : 0;
    int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const bool first = i < na;
    if (!first) i -= na;
    if (!first && i >= nb) return;
    const int64_t size = first ? na : nb;
    const float* const part = (first ? sa.part : sb.part) + i;
    float* const out = (first ? g.dA : g.dB) + a * size + i;
    const int begin = gload(g.offsets + a), end = gload(g.offsets + a + 1);
    f32x4 v = {0, 0, 0, 0};
    if (end > begin)
        for (int p = begin / piece; p <= (end - 1) / piece; ++p) v += gload(reinterpret_cast<const f32x4*>(part + (int64_t)(p + a) * size));
    if (g.accumulate) v += gload(reinterpret_cast<const f32x4*>(out));
    gstore(reinterpret_cast<f32x4*>(out), v);
}

// ------------------------------------------------------------------------------------------ preparation
// Work-group a < count lists the rows of adapter a, behind those of the adapters before it; sixteen waves count and then write a sixteenth of the rows
// each, so the rows of an adapter stay in order.
__device__ void list_rows(const AdapterPrep& p, int a) {
    __shared__ int mine[16], below[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t each = (p.M + 1023) / 1024 * 64;       // whole waves of rows
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
    for (int w = 0; w < 16; ++w) {
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

// dst[cols, rows] = src[rows, cols]^T, one tile of 64 x 64; both dimensions multiples of 8
__device__ void transpose_tile(const uint16_t* src, uint16_t* dst, int rows, int cols, int tr, int tc) {
    __shared__ uint16_t t[64][66];
    const int e = threadIdx.x;
    if (e < 512) {
        const int r = 64 * tr + (e >> 3), c = 64 * tc + (e & 7) * 8;
        if (r < rows && c < cols) {
            const u32x4 v = gload(reinterpret_cast<const u32x4*>(src + (int64_t)r * cols + c));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t[e >> 3][(e & 7) * 8 + 2 * i] = (uint16_t)(v[i] & 0xffffu);
                t[e >> 3][(e & 7) * 8 + 2 * i + 1] = (uint16_t)(v[i] >> 16);
            }
        }
    }
    __syncthreads();
    if (e < 512) {
        const int c = 64 * tc + (e >> 3), r = 64 * tr + (e & 7) * 8;
        if (c < cols && r < rows) {
            u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (uint32_t)t[(e & 7) * 8 + 2 * i][e >> 3] | (uint32_t)t[(e & 7) * 8 + 2 * i + 1][e >> 3] << 16;
            gstore(reinterpret_cast<u32x4*>(dst + (int64_t)c * rows + r), v);
        }
    }
}

struct PrepBlocks { int list, w, a, b; };                 // work-groups of each kind: rows, tiles of W, tiles of one A, of one B

__global__ __launch_bounds__(1024) void adapters_prep_kernel(const AdapterPrep p, const PrepBlocks n) {
    int i = blockIdx.x;
    if (i < n.list) {
        if (i == 0 && threadIdx.x < 16) gstore(reinterpret_cast<u32x4*>(p.zeros) + threadIdx.x, u32x4{0, 0, 0, 0});
        list_rows(p, i);
        return;
    }
    i -= n.list;
    const int tm = (p.m + 63) / 64, tn = (p.n + 63) / 64, tr = (p.r + 63) / 64;
    if (i < n.w) { transpose_tile(p.W, p.Wt, p.m, p.n, i / tn, i % tn); return; }
    i -= n.w;
    if (i < n.a * p.count) {
        const int a = i / n.a, t = i % n.a;
        transpose_tile(p.A + (int64_t)a * p.m * p.r, p.At + (int64_t)a * p.m * p.r, p.m, p.r, t / tr, t % tr);
        return;
    }
    i -= n.a * p.count;
    const int a = i / n.b, t = i % n.b;
    transpose_tile(p.B + (int64_t)a * p.n * p.r, p.Bt + (int64_t)a * p.n * p.r, p.r, p.n, t / tn, t % tn);
    (void)tm;
}

Side side_of(const uint16_t* U, const uint16_t* V, float* part, int cols, const float* out) { return Side{U, V, part, cols, out ? (cols + 127) / 128 : 0}; }

template <int VB>
hipError_t launch_grads(const AdapterGrads& p, const Side& a, const Side& b, int piece, hipStream_t s) {
    using L = Grad<VB>;
    static std::atomic<bool> attr_set{false};
    if (!attr_set.load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&adapters_grad_kernel<VB>), hipFuncAttributeMaxDynamicSharedMemorySize, L::lds);
        if (e != hipSuccess) return e;
        attr_set.store(true, std::memory_order_release);
    }
    hipLaunchKernelGGL((adapters_grad_kernel<VB>), dim3((unsigned)(a.blocks + b.blocks), (unsigned)ceil_div(p.M, piece)), dim3(256), L::lds, s, p, a, b, piece);
    return hipGetLastError();
}

}  // namespace

// Work-groups for two per compute unit and more, pieces of whole slabs, at most what the list in LDS holds
int adapters_grad_piece(int64_t M, int m, int n) {
    const int64_t blocks = ceil_div(m, 128) + ceil_div(n, 128), pieces = ceil_div(768, blocks);
    const int64_t rows = align_up((size_t)ceil_div(M, pieces), kPiece);
    return rows > kMaxPiece ? kMaxPiece : (int)rows;
}
size_t adapters_grad_partial_bytes(int64_t M, int m, int n, int r, int count) {
    return (size_t)(ceil_div(M, adapters_grad_piece(M, m, n)) + count) * (size_t)(m + n) * (size_t)r * 4;
}

hipError_t launch_adapters_grads(const AdapterGrads& p, hipStream_t s) {
    const int piece = adapters_grad_piece(p.M, p.m, p.n);
    const int64_t pieces = ceil_div(p.M, piece);
    if (pieces > 65535 || p.count > 65535) return hipErrorInvalidValue;
    float* const second = p.partials + (pieces + p.count) * p.m * p.r;
    const Side a = side_of(p.dY, p.T_planes, p.partials, p.m, p.dA), b = side_of(p.X, p.dT_planes, second, p.n, p.dB);
    if (a.blocks + b.blocks == 0) return hipSuccess;
    hipError_t e;
    switch (plane_columns(p.r)) {
        case 16: e = launch_grads<1>(p, a, b, piece, s); break;
        case 32: e = launch_grads<2>(p, a, b, piece, s); break;
        case 64: e = launch_grads<4>(p, a, b, piece, s); break;
        default: e = launch_grads<8>(p, a, b, piece, s); break;
    }
    if (e != hipSuccess) return e;
    const int64_t quads = ((a.blocks ? (int64_t)p.m * p.r : 0) + (b.blocks ? (int64_t)p.n * p.r : 0)) / 4;
    hipLaunchKernelGGL(adapters_sum_kernel, dim3((unsigned)ceil_div(quads, 256), (unsigned)p.count), dim3(256), 0, s, p, a, b, piece);
    return hipGetLastError();
}

hipError_t launch_adapters_prep(const AdapterPrep& p, hipStream_t s) {
    const int64_t tm = ceil_div(p.m, 64), tn = ceil_div(p.n, 64), tr = ceil_div(p.r, 64);
    const PrepBlocks n{p.order ? p.count : 0, p.W ? (int)(tm * tn) : 0, p.A ? (int)(tm * tr) : 0, p.B ? (int)(tn * tr) : 0};
    const int64_t blocks = n.list + (int64_t)n.w + (int64_t)(n.a + n.b) * p.count;
    if (blocks == 0) return hipSuccess;
    if (blocks > (1ll << 31) - 1) return hipErrorInvalidValue;
    hipLaunchKernelGGL(adapters_prep_kernel, dim3((unsigned)blocks), dim3(1024), 0, s, p, n);
    return hipGetLastError();
}

}  // namespace abt
