// The layer with adapters for a few rows, as single tokens of many requests are: T_i = B_a x_i, then Y_i = W x_i + A_a T_i.
// Little is reused, so the operands go from memory to registers.  Two launches:
//   first    T beside the dense product.  T: a work-group per row and eight of its rank's rows of B, one a wave.  The dense product: 64 columns, up to
//            64 rows and a part of the contraction, which eight waves share out, 128 bytes of every row at a time; with 16 columns and the whole
//            contraction per work-group the rows of X, read by every work-group, were several times the bytes of W.
//   second   adds the parts in order, and the adapters: 16 columns a work-group, eight waves that share out the adapters of the rows.
// A row or two of narrow adapters go in one launch.
// Bound by the bytes of W and of the adapters in use, and by the latency of two launches where these are few: 48 rows of 4096 x 4096 in 8 bits with 24 adapters of r = 16
// 10.0 and 5.8 us (23 MB, 1.5 TB/s; a copy's rate would be 4.9 us); one row of 768 x 768, r = 8, 5.9 us (1.2 MB).
#include <type_traits>

#include "adapters.h"
#include "adapters_operands.h"

namespace abt {
namespace {

__device__ __forceinline__ float lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }

// T of one row: row j of its adapter's B by each wave
__device__ __forceinline__ void t_of_row(const AdapterProduct& g, const uint16_t* X, const uint16_t* B, int n, int64_t row, int j) {
    const int lane = threadIdx.x & 63;
    if (j >= g.r) return;
    const int a = __builtin_amdgcn_readfirstlane(gload(g.row_adapter + row));
    const bool have = a >= 0 && a < g.count;
    float sum = 0.0f, s = 1.0f;
    int rank = 0;
    if (have) {
        // (rows past the rank are there: they are read beside the rank and not used)
        const int k = g.ranks ? gload(g.ranks + a) : g.r;
        if (g.scales) s = gload(g.scales + a);
        const uint16_t* const x = X + row * n;
        const uint16_t* const b = B + ((int64_t)a * g.r + j) * n;
        float other = 0.0f;
        const auto add = [&](u32x4 xv, u32x4 bv) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum += lo(xv[i]) * lo(bv[i]);
                other += hi(xv[i]) * hi(bv[i]);
            }
        };
        const auto at = [&](const uint16_t* p, int c) { return gload(reinterpret_cast<const u32x4*>(p + c)); };
        int c = lane * 8;
        for (; c + 3584 < n; c += 4096) {                 // eight pieces on their way at a time
            u32x4 v[8][2];
#pragma unroll
            for (int i = 0; i < 8; ++i) { v[i][0] = at(x, c + 512 * i); v[i][1] = at(b, c + 512 * i); }
#pragma unroll
            for (int i = 0; i < 8; ++i) add(v[i][0], v[i][1]);
        }
        for (; c + 512 < n; c += 1024) {
            const u32x4 x0 = at(x, c), b0 = at(b, c), x1 = at(x, c + 512), b1 = at(b, c + 512);
            add(x0, b0);
            add(x1, b1);
        }
        if (c < n) add(at(x, c), at(b, c));
        sum += other;
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        rank = k > g.r ? g.r : k;
        if (j >= rank) sum = 0.0f;
    }
    if (lane) return;
    if (g.T) gstore(g.T + row * g.r + j, sum);
    // what is past the rank is zero whatever the scale
    if (g.Tb) gstore(g.Tb + row * g.r + j, (uint16_t)(pack2_bf16(j < rank ? s * sum : 0.0f, 0.0f) & 0xffffu));
}

// T alone, for tiles of Y after it
__global__ __launch_bounds__(512) void adapters_t_rows_kernel(const AdapterProduct g) {
    const int per = g.r / 8, w = blockIdx.x;
    t_of_row(g, g.E, g.F, g.ke, w / per, (w % per) * 8 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
}

struct FewParts { int col_blocks, blocks16, row_groups, splits, units; float* sums; const uint16_t* X; const uint16_t* B; };   // X as the adapters see it

// RB blocks of 16 rows
template <int RB, bool F8>
__global__ __launch_bounds__(512) void few_first_kernel(const AdapterProduct g, const FewParts f) {
    constexpr int CB = 4;
    __shared__ __align__(16) f32x4 sums[4 * RB * CB * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nbase = f.col_blocks * f.row_groups * f.splits;
    int w = blockIdx.x;
    if (w >= nbase) {
        w -= nbase;
        const int per = g.r / 8;
        t_of_row(g, f.X, f.B, g.kmain, w / per, (w % per) * 8 + wave);
        return;
    }
    const int cb = w % f.col_blocks;
    w /= f.col_blocks;
    const int split = w % f.splits, row0 = w / f.splits * 64;
    const int li = lane & 15, lq = lane >> 4;
    const int rows = (int)g.M - row0 < 64 ? (int)g.M - row0 : 64, col0 = cb * 64;
    const int cols = g.Q - col0 < 64 ? g.Q - col0 : 64;
    const int bytes = g.kmain * (F8 ? 1 : 2);
    // a unit is 128 bytes of every row; lanes past the last row, column or byte read zeros
    const rsrc_t xres = make_rsrc((const char*)g.X + (int64_t)row0 * bytes, (int64_t)rows * bytes);
    const rsrc_t wres = make_rsrc((const char*)g.W + (int64_t)col0 * bytes, (int64_t)cols * bytes);
    f32x4 acc[RB][CB];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[b][c] = f32x4{0, 0, 0, 0};
    const int end = (split + 1) * f.units;
    for (int u = split * f.units + wave; u < end; u += 8) {
        const int at0 = u * 128 + lq * 16, at1 = at0 + 64;
        u32x4 w0[CB], w1[CB], x0[RB], x1[RB];
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            w0[c] = buf_load16(wres, at0 < bytes ? (16 * c + li) * bytes + at0 : kBufNowhere, 0);
            w1[c] = buf_load16(wres, at1 < bytes ? (16 * c + li) * bytes + at1 : kBufNowhere, 0);
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            x0[b] = buf_load16(xres, at0 < bytes ? (16 * b + li) * bytes + at0 : kBufNowhere, 0);
            x1[b] = buf_load16(xres, at1 < bytes ? (16 * b + li) * bytes + at1 : kBufNowhere, 0);
        }
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                if constexpr (F8) {
                    acc[b][c] = mfma16_f8(w0[c], w1[c], x0[b], x1[b], acc[b][c]);
                } else {
                    acc[b][c] = mfma16(w0[c], x0[b], acc[b][c]);
                    acc[b][c] = mfma16(w1[c], x1[b], acc[b][c]);
                }
            }
    }
    // the waves' sums: those of waves w and w + 4 first, then the four in order
    auto at = [&](int who, int t) -> f32x4& { return sums[(who * RB * CB + t) * 64 + lane]; };
    if (wave >= 4)
#pragma unroll
        for (int t = 0; t < RB * CB; ++t) at(wave - 4, t) = acc[t / CB][t % CB];
    __syncthreads();
    if (wave < 4)
#pragma unroll
        for (int t = 0; t < RB * CB; ++t) at(wave, t) = acc[t / CB][t % CB] + at(wave, t);
    __syncthreads();
    // parts lie as [split][16 columns][row]: whole lines for whoever stores or adds them
    float* const out = f.sums + (int64_t)split * f.blocks16 * g.M * 16;
    for (int t = wave; t < RB * CB; t += 8) {
        const f32x4 v = (at(0, t) + at(1, t)) + (at(2, t) + at(3, t));
        const int row = 16 * (t / CB) + li, c = 16 * (t % CB) + 4 * lq;      // lane: row li of the block, four columns
        if (row < rows && c < cols) gstore(reinterpret_cast<f32x4*>(out + ((int64_t)(cb * CB + t % CB) * g.M + row0 + row) * 16 + 4 * lq), v);
    }
}

template <int RB, bool F8>
__global__ __launch_bounds__(512) void few_second_kernel(const AdapterProduct g, const FewParts f) {
    __shared__ __align__(16) f32x4 sums[8 * RB * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, lq = lane >> 4;
    const int row0 = blockIdx.y * 64, rows = (int)g.M - row0 < 64 ? (int)g.M - row0 : 64;
    const int col0 = blockIdx.x * 16, cols = g.Q - col0 < 16 ? g.Q - col0 : 16;
    const int id0 = gload(g.row_adapter + row0 + (lane < rows ? lane : 0));
    // the dense product of this lane's row and four columns, by the waves that finish a block of rows
    const int row = 16 * wave + li, c0 = 4 * lq;
    const bool out = wave < RB && row < rows && c0 < cols;
    f32x4 v = {0, 0, 0, 0};
    float xs = 1.0f, ws[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    if (out) {
        const float* const from = f.sums + ((int64_t)blockIdx.x * g.M + row0 + row) * 16 + c0;
        const int64_t step = (int64_t)f.blocks16 * g.M * 16;
        for (int s = 0; s < f.splits; s += 4) {           // four on their way at a time
            f32x4 part[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) part[i] = gload(reinterpret_cast<const f32x4*>(from + (s + i < f.splits ? s + i : s) * step));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (s + i < f.splits) v += part[i];
        }
        if constexpr (F8) {
            xs = gload(g.x_scale + row0 + row);
#pragma unroll
            for (int i = 0; i < 4; ++i) ws[i] = gload(g.w_scale + col0 + c0 + i);
        }
    }
    f32x4 acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = f32x4{0, 0, 0, 0};
    // The adapters of the rows in the order in which they occur, every eighth of them by this wave, four at a time with their loads together.
    const int id = lane < rows && id0 >= 0 && id0 < g.count ? id0 : -1;
    const int rank0 = g.ranks && id >= 0 ? gload(g.ranks + id) : g.r;
    const rsrc_t eres = make_rsrc(g.E + (int64_t)row0 * g.r, (int64_t)rows * g.r * 2);
    uint64_t left = __ballot(id >= 0);
    float bad = 0.0f;
    for (int k = 0; left;) {
        uint64_t of[4] = {0, 0, 0, 0};             // its rows
        rsrc_t fres[4];
        int who[4] = {0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            int a = 0;
            while (left && !of[q]) {
                const int first = __builtin_ctzll(left);
                a = __builtin_amdgcn_readlane(id, first);
                const uint64_t same = __ballot(id == a);
                left &= ~same;
                if ((k++ & 7) == wave) { of[q] = same; who[q] = first; }
            }
            fres[q] = make_rsrc(g.F + ((int64_t)a * g.Q + col0) * g.r, of[q] ? (int64_t)cols * g.r * 2 : 0);
        }
        if (!of[0]) break;
        for (int j = 0; j < g.r; j += 32) {
            const int c = j + lq * 8;
            u32x4 f[4], t[4][RB];
#pragma unroll
            for (int q = 0; q < 4; ++q) {                 // (columns past the rank are there: they are read beside it and masked)
                f[q] = buf_load16(fres[q], c < g.r ? (li * g.r + c) * 2 : kBufNowhere, 0);
#pragma unroll
                for (int b = 0; b < RB; ++b)
                    t[q][b] = buf_load16(eres, c < g.r && ((of[q] >> (16 * b + li)) & 1) ? ((16 * b + li) * g.r + c) * 2 : kBufNowhere, 0);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (!of[q]) break;
                const int rank = __builtin_amdgcn_readlane(rank0, who[q]);
                if (rank - j < 32) f[q] = first_of(f[q], rank - c);            // (T is zero there)
                bad += zero_times(f[q]);
#pragma unroll
                for (int b = 0; b < RB; ++b) acc[b] = mfma16(f[q], t[q][b], acc[b]);
            }
        }
    }
    // lane: row 16 b + li, columns 4 lq .. + 3
#pragma unroll
    for (int b = 0; b < RB; ++b) sums[(wave * RB + b) * 64 + lane] = acc[b];
    // Where an adapter is not finite: all of it again, each into its own rows alone.
    if (any_not_finite(bad)) {
#pragma unroll
        for (int b = 0; b < RB; ++b) sums[(wave * RB + b) * 64 + lane] = f32x4{0, 0, 0, 0};
        left = __ballot(id >= 0);
        for (int k = 0; left; ++k) {
            const int first = __builtin_ctzll(left), a = __builtin_amdgcn_readlane(id, first), rank = __builtin_amdgcn_readlane(rank0, first);
            const uint64_t same = __ballot(id == a);
            left &= ~same;
            if ((k & 7) != wave) continue;
            const rsrc_t fres = make_rsrc(g.F + ((int64_t)a * g.Q + col0) * g.r, (int64_t)cols * g.r * 2);
            for (int j = 0; j < g.r; j += 32) {
                const int c = j + lq * 8;
                const u32x4 f = first_of(buf_load16(fres, c < g.r ? (li * g.r + c) * 2 : kBufNowhere, 0), rank - c);
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    const bool own = (same >> (16 * b + li)) & 1;
                    const u32x4 t = buf_load16(eres, c < g.r && own ? ((16 * b + li) * g.r + c) * 2 : kBufNowhere, 0);
                    f32x4& to = sums[(wave * RB + b) * 64 + lane];
                    const f32x4 sum = mfma16(f, t, to);
                    if (own) to = sum;
                }
            }
        }
    }
    __syncthreads();
    if (!out) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= xs * ws[i];
    f32x4 low = sums[wave * 64 + lane];
#pragma unroll
    for (int w = 1; w < 8; ++w) low += sums[(w * RB + wave) * 64 + lane];
    v += low;
    gstore(reinterpret_cast<u32x2*>(g.Y + (int64_t)(row0 + row) * g.Q + col0 + c0), u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])});
}

// One launch where there is next to nothing to share: up to 32 values of T in all (at r = 8 four rows), which every work-group computes for itself.  16
// columns a work-group, whose eight waves share out the contraction, the values of T and the adapters.
constexpr int kOneT = 32, kOneRows = kOneT / 8, kOnePitch = kOneT + 8;      // values of T; rows; LDS values per row of T, rank columns and zeros behind them
template <bool F8>
__global__ __launch_bounds__(512) void few_one_kernel(const AdapterProduct g, const uint16_t* X, const uint16_t* B) {
    __shared__ __align__(16) f32x4 sums[8 * 64];
    __shared__ __align__(16) uint16_t ts[kOneRows * kOnePitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, lq = lane >> 4;
    const int M = (int)g.M, n = g.kmain, r = g.r;
    const int col0 = blockIdx.x * 16, cols = g.Q - col0 < 16 ? g.Q - col0 : 16;
    const int id0 = gload(g.row_adapter + (lane < M ? lane : 0));
    if (threadIdx.x < kOneRows * kOnePitch / 8) *reinterpret_cast<u32x4*>(ts + 8 * threadIdx.x) = u32x4{0, 0, 0, 0};
    const int id = lane < M && id0 >= 0 && id0 < g.count ? id0 : -1;
    const int rank0 = g.ranks && id >= 0 ? gload(g.ranks + id) : r;
    const float scale0 = g.scales && id >= 0 ? gload(g.scales + id) : 1.0f;
    // T: values wave, wave + 8, .., value v is column v % r of row v / r
    float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const uint16_t *xp[4], *bp[4];
    bool have[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int v = wave + 8 * i, row = v / r;
        const int a = row < M ? __builtin_amdgcn_readlane(id, row) : -1;
        have[i] = a >= 0;
        xp[i] = X + (int64_t)(have[i] ? row : 0) * n;
        bp[i] = B + ((int64_t)(have[i] ? a : 0) * r + (v - row * r)) * n;
    }
#pragma unroll 2
    for (int c = lane * 8; c < n; c += 512) {
        u32x4 x[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (have[i]) {
                x[i] = gload(reinterpret_cast<const u32x4*>(xp[i] + c));
                b[i] = gload(reinterpret_cast<const u32x4*>(bp[i] + c));
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (have[i])
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    t[i] += lo(x[i][k]) * lo(b[i][k]);
                    t[i] += hi(x[i][k]) * hi(b[i][k]);
                }
    }
    // the dense product, 128 bytes of every row at a time
    const int bytes = n * (F8 ? 1 : 2), units = (bytes + 127) / 128;
    const rsrc_t xres = make_rsrc(g.X, (int64_t)M * bytes), wres = make_rsrc((const char*)g.W + (int64_t)col0 * bytes, (int64_t)cols * bytes);
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll 4
    for (int u = wave; u < units; u += 8) {
        const int at0 = u * 128 + lq * 16, at1 = at0 + 64;
        const u32x4 w0 = buf_load16(wres, at0 < bytes ? li * bytes + at0 : kBufNowhere, 0), w1 = buf_load16(wres, at1 < bytes ? li * bytes + at1 : kBufNowhere, 0);
        const u32x4 x0 = buf_load16(xres, at0 < bytes ? li * bytes + at0 : kBufNowhere, 0), x1 = buf_load16(xres, at1 < bytes ? li * bytes + at1 : kBufNowhere, 0);
        if constexpr (F8) {
            acc = mfma16_f8(w0, w1, x0, x1, acc);
        } else {
            acc = mfma16(w0, x0, acc);
            acc = mfma16(w1, x1, acc);
        }
    }
    if constexpr (F8) {
        const float xs = gload(g.x_scale + (li < M ? li : 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= xs * (4 * lq < cols ? gload(g.w_scale + col0 + 4 * lq + i) : 0.0f);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 32; d; d >>= 1) t[i] += __shfl_xor(t[i], d);
    __syncthreads();                                      // (the zeros are there)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int v = wave + 8 * i, row = v / r, j = v - row * r;
        if (row >= M) break;
        const bool in = j < __builtin_amdgcn_readlane(rank0, row) && have[i];
        const float value = in ? t[i] : 0.0f;
        if (lane == 0) {
            if (g.T && blockIdx.x == 0) gstore(g.T + (int64_t)row * r + j, value);
            if (in) ts[row * kOnePitch + j] = (uint16_t)(pack2_bf16(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scale0), row)) * value, 0.0f) & 0xffffu);
        }
    }
    __syncthreads();
    // the adapters of the rows, every eighth by this wave
    uint64_t left = __ballot(id >= 0);
    for (int k = 0; left; ++k) {
        const int first = __builtin_ctzll(left), a = __builtin_amdgcn_readlane(id, first), rank = __builtin_amdgcn_readlane(rank0, first);
        const uint64_t same = __ballot(id == a);
        left &= ~same;
        if ((k & 7) != wave) continue;
        const rsrc_t fres = make_rsrc(g.F + ((int64_t)a * g.Q + col0) * r, (int64_t)cols * r * 2);
        const int c = lq * 8;
        const u32x4 f = first_of(buf_load16(fres, c < r ? (li * r + c) * 2 : kBufNowhere, 0), rank - c);
        const u32x4 e = (same >> li) & 1 ? *reinterpret_cast<const u32x4*>(ts + li * kOnePitch + c) : u32x4{0, 0, 0, 0};
        const f32x4 sum = mfma16(f, e, acc);
        acc = (same >> li) & 1 ? sum : acc;               // (zero times an infinity is NaN in the other rows)
    }
    sums[wave * 64 + lane] = acc;
    __syncthreads();
    if (wave || li >= M || 4 * lq >= cols) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) acc += sums[w * 64 + lane];
    gstore(reinterpret_cast<u32x2*>(g.Y + (int64_t)li * g.Q + col0 + 4 * lq), u32x2{pack2_bf16(acc[0], acc[1]), pack2_bf16(acc[2], acc[3])});
}
// Where the contraction is so short that its parts are not missed.  us, one launch / two, rows of W 768 x 768 5.9 / 7.2 (one row, r = 16) and 6.5 / 7.2 (two), 2304 x
// 768 6.8 / 7.4 (two); 4096 x 2048 in 8 bits 8.3 / 8.4 (two), 4096 x 4096 15.3 / 13.3 and in 8 bits 11.7 / 9.6 (one).
bool few_in_one(const AdapterProduct& p, bool fp8) {
    return p.M * p.r <= kOneT && (int64_t)p.kmain * (fp8 ? 1 : 2) <= 3072;
}

FewParts few_parts(int64_t M, int Q, int n, bool fp8) {
    FewParts f{};
    f.col_blocks = (Q + 63) / 64;
    f.blocks16 = (Q + 15) / 16;
    f.row_groups = (int)((M + 63) / 64);
    const int units = (n * (fp8 ? 1 : 2) + 127) / 128;
    // one work-group per compute unit, but for each of its eight waves at least one unit
    int splits = 256 / (f.col_blocks * f.row_groups);
    const int most = (units + 7) / 8;
    splits = splits > most ? most : splits;
    splits = splits < 1 ? 1 : splits;
    f.units = (units + splits - 1) / splits;
    f.splits = (units + f.units - 1) / f.units;
    return f;
}

template <bool F8>
hipError_t few(const AdapterProduct& p, const FewParts& f, hipStream_t s) {
    const dim3 first((unsigned)(f.col_blocks * f.row_groups * f.splits + p.M * (p.r / 8))), second((unsigned)ceil_div(p.Q, 16), (unsigned)f.row_groups);
    const auto launch = [&](auto rb) {
        constexpr int RB = decltype(rb)::value;
        hipLaunchKernelGGL((few_first_kernel<RB, F8>), first, dim3(512), 0, s, p, f);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((few_second_kernel<RB, F8>), second, dim3(512), 0, s, p, f);
        return hipGetLastError();
    };
    if (p.M <= 16) return launch(std::integral_constant<int, 1>{});
    if (p.M <= 32) return launch(std::integral_constant<int, 2>{});
    if (p.M <= 48) return launch(std::integral_constant<int, 3>{});
    return launch(std::integral_constant<int, 4>{});
}

}  // namespace

size_t adapters_few_sums_bytes(int64_t M, int m, int n) {
    const int s8 = few_parts(M, m, n, true).splits, s16 = few_parts(M, m, n, false).splits;
    return (size_t)(s8 > s16 ? s8 : s16) * (size_t)M * align_up((size_t)m, 16) * 4;
}

hipError_t launch_adapters_t_rows(const AdapterProduct& p, hipStream_t s) {
    hipLaunchKernelGGL(adapters_t_rows_kernel, dim3((unsigned)(p.M * (p.r / 8))), dim3(512), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_adapters_few(const AdapterProduct& p, const uint16_t* X, const uint16_t* B, float* sums, bool fp8, hipStream_t s) {
    if (p.M > kAdapterFewRows || p.e_pitch != p.r || p.ke != p.r) return hipErrorInvalidValue;
    if (few_in_one(p, fp8)) {
        const dim3 grid((unsigned)ceil_div(p.Q, 16));
        if (fp8) hipLaunchKernelGGL(few_one_kernel<true>, grid, dim3(512), 0, s, p, X, B);
        else hipLaunchKernelGGL(few_one_kernel<false>, grid, dim3(512), 0, s, p, X, B);
        return hipGetLastError();
    }
    FewParts f = few_parts(p.M, p.Q, p.kmain, fp8);
    f.sums = sums; f.X = X; f.B = B;
    return fp8 ? few<true>(p, f, s) : few<false>(p, f, s);
}

}  // namespace abt
