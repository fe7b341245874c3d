// Group norm with an activation over channels-last images:
//     Y = act(gain (X - mean) rstd + shift),   mean and 1 / rstd^2 - eps over the pixels and the channels of a group of one image
//     dpre = dY act'(..), u = dpre gain, x^ = (X - mean) rstd:   dX = rstd (u - mean(u) - x^ mean(u x^)),   dgain = sum dpre x^,   dshift = sum dpre
// Where all pixels of an image fit a work-group's registers over a slab of channels that holds whole groups, a work-group reads them once and does everything (`whole` kernels);
// otherwise pieces of the pixels leave sums per channel in a first launch and are normalised in a second, which reads again.
// Threads: eight channels each, TC of them (a power of two) across the slab, the others down the pixels.
// Bound by memory and, little less, by vector work: a value is looked at three times, 16 instructions forward (silu) and 17 backward (relu) where there is one pass over memory; loads,
// sums and stores of a work-group follow each other, and two work-groups or more per compute unit overlap them in part.  us (GB/s): 256 x 196 x 256 bf16 forward 13.3 (3900), 64 x 3136 x 64
// 17.3 (3000), 128 x 784 x 128 backward, relu, 20 (3900) and 4 for the gradients of the channels; in pieces 64 x 3136 x 64 backward 30, 1 x 4096 x 2048 17 and 21; 1 x 49 x 512 fp32 4.6.
#include <climits>

#include "activation.h"
#include "group_norm.h"
#include "group_norm_plan.h"
#include "nt_tile.h"
#include "vec8.h"

namespace abt {
namespace {

__device__ __forceinline__ float lanes_sum(float v, int from, int to) {      // over lanes whose numbers differ in the bits from .. to / 2
    for (int d = from; d < to; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// The sums of each unit of the slab over all threads, in chan[q pitch ..]: a thread has U units, of its eight channels or of eight / U of them added up; lanes with the same ones
// first, then the waves.  `waves` holds K pitch values for each wave.
template <int THREADS, int K, int U>
__device__ __forceinline__ void channel_sums(float (&v)[K][U], int shift, int units, int pitch, float* waves, float* chan) {
    constexpr int NW = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tc = lane & ((1 << shift) - 1);
    for (int d = 1 << shift; d < 64; d <<= 1)
#pragma unroll
        for (int q = 0; q < K; ++q)
#pragma unroll
            for (int k = 0; k < U; ++k) v[q][k] += __shfl_xor(v[q][k], d);
    if (lane == tc && U * tc < units)
#pragma unroll
        for (int q = 0; q < K; ++q)
#pragma unroll
            for (int k = 0; k < U; ++k) waves[(q * NW + wave) * pitch + U * tc + k] = v[q][k];
    __syncthreads();
    for (int c = threadIdx.x; c < units; c += THREADS)
#pragma unroll
        for (int q = 0; q < K; ++q) {
            float s = waves[q * NW * pitch + c];
#pragma unroll
            for (int w = 1; w < NW; ++w) s += waves[(q * NW + w) * pitch + c];
            chan[q * pitch + c] = s;
        }
    __syncthreads();
}

// f(group, lane of `lanes`, lanes): the work-group's threads in teams of a power of two of up to 64, a team for a group
template <int THREADS, class F>
__device__ __forceinline__ void by_group(int groups, int entries, F&& f) {
    const int ls = entries <= 1 ? 0 : entries > 32 ? 6 : 32 - __builtin_clz(entries - 1);
    for (int g = threadIdx.x >> ls; g < groups; g += THREADS >> ls) f(g, (int)threadIdx.x & ((1 << ls) - 1), 1 << ls);
}

// ------------------------------------------------------------------------------------------ everything at once
// Pixel r of NV: row + r step, where row = thread / TC.  U: units of a thread's eight channels; a group is a whole number of units.
template <bool BF16, int THREADS, int NV, int U>
__global__ __launch_bounds__(THREADS) void gn_whole_fwd_kernel(const GroupNorm g, const GroupSplit sp) {
    extern __shared__ float lds[];
    const int pitch = sp.width;
    float *const waves = lds, *const chan = waves + THREADS / 64 * pitch, *const stat = chan + pitch;
    const unsigned block = xcd_order(blockIdx.x, gridDim.x);                 // the slabs of an image, which share lines of memory, on one XCD
    const int slab = block % (unsigned)sp.slabs, c0 = slab * sp.width, width = g.C - c0 < sp.width ? g.C - c0 : sp.width;
    const int64_t image = g.image0 + block / (unsigned)sp.slabs;
    const int tc = threadIdx.x & ((1 << sp.shift) - 1), row = threadIdx.x >> sp.shift, step = THREADS >> sp.shift;
    const bool there = 8 * tc < width;
    const int64_t base = image * g.pixels * g.C + c0 + 8 * tc;
    Raw8<BF16> x[NV];
#pragma unroll
    for (int r = 0; r < NV; ++r)
        if (there && row + r * step < g.pixels) x[r] = raw8<BF16>(g.X, base + (int64_t)(row + r * step) * g.C);
    float gain[8], shift[8];
    if (there) load8<false>(g.gain, c0 + 8 * tc, gain), load8<false>(g.shift, c0 + 8 * tc, shift);
    const int cpg = g.C / g.groups, groups = width / cpg, upg = cpg * U / 8;         // units of a group
    const float inv = 1.0f / ((float)g.pixels * (float)cpg);
    int mine[U];                                          // the groups of this thread's units
#pragma unroll
    for (int k = 0; k < U; ++k) mine[k] = (U * tc + k) / upg;
    float sum[1][U], mean[U], rstd[U];
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {                // the mean, then the squares around it
#pragma unroll
        for (int k = 0; k < U; ++k) sum[0][k] = 0.0f;
#pragma unroll
        for (int r = 0; r < NV; ++r)
            if (there && row + r * step < g.pixels) {
                float v[8];
                values<BF16>(x[r], v);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float d = pass ? v[k] - mean[k * U / 8] : v[k];
                    sum[0][k * U / 8] += pass ? d * d : d;
                }
            }
        channel_sums<THREADS, 1, U>(sum, sp.shift, width / 8 * U, pitch, waves, chan);
        by_group<THREADS>(groups, upg, [&](int q, int l, int lanes) {
            float s = 0.0f;
            for (int c = l; c < upg; c += lanes) s += chan[q * upg + c];
            s = lanes_sum(s, 1, lanes);
            if (l) return;
            s *= inv;
            if (pass) s = 1.0f / __builtin_sqrtf(s + g.eps);
            stat[pass * pitch + q] = s;
            gstore((pass ? g.rstd : g.mean) + image * g.groups + c0 / cpg + q, s);
        });
        __syncthreads();
        if (there)
#pragma unroll
            for (int k = 0; k < U; ++k) (pass ? rstd : mean)[k] = stat[pass * pitch + mine[k]];
    }
    if (!there) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) gain[k] *= rstd[k * U / 8], shift[k] -= mean[k * U / 8] * gain[k];
    with_activation(g.act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < NV; ++r)
            if (row + r * step < g.pixels) {
                float v[8];
                values<BF16>(x[r], v);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = activate<decltype(act)::value>(v[k] * gain[k] + shift[k]);
                store8<BF16>(g.Y, base + (int64_t)(row + r * step) * g.C, v);
            }
    });
}

// A channel in front of the activation, x G + S; and its dX = rstd (dpre gain - first - x^ second) as dpre G + (x P + Q)
struct Front {
    float G, S, mean;
    __device__ __forceinline__ float pre(float x) const { return x * G + S; }
};
// of eight channels; and 1 / sqrt(var + eps) of their groups
__device__ __forceinline__ void fronts_of(const GroupNorm& g, int64_t image, int channel, int cpg, Front (&f)[8], float (&rstd)[8]) {
    float gain[8], shift[8];
    load8<false>(g.gain, channel, gain), load8<false>(g.shift, channel, shift);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t q = image * g.groups + (channel + k) / cpg;
        rstd[k] = gload(g.rstd + q);
        f[k].mean = gload(g.mean + q);
        f[k].G = gain[k] * rstd[k];
        f[k].S = shift[k] - f[k].mean * f[k].G;
    }
}
struct Slopes {
    float G, S, P, Q;
    __device__ __forceinline__ float pre(float x) const { return x * G + S; }
    __device__ __forceinline__ float of(float x, float dpre) const { return dpre * G + (x * P + Q); }
};
__device__ __forceinline__ Slopes slopes_of(const Front& f, float rstd, float first, float second) {
    const float P = -rstd * rstd * second;
    return Slopes{f.G, f.S, P, -rstd * first - f.mean * P};
}

// sums [2, N, C] of dpre and of dpre x^
template <bool BF16, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void gn_whole_bwd_kernel(const GroupNorm g, const GroupSplit sp) {
    extern __shared__ float lds[];
    const int pitch = sp.width;
    float *const waves = lds, *const chan = waves + 2 * (THREADS / 64) * pitch, *const stat = chan + 2 * pitch;
    const unsigned block = xcd_order(blockIdx.x, gridDim.x);                 // the slabs of an image, which share lines of memory, on one XCD
    const int slab = block % (unsigned)sp.slabs, c0 = slab * sp.width, width = g.C - c0 < sp.width ? g.C - c0 : sp.width;
    const int64_t image = g.image0 + block / (unsigned)sp.slabs;
    const int tc = threadIdx.x & ((1 << sp.shift) - 1), row = threadIdx.x >> sp.shift, step = THREADS >> sp.shift;
    const bool there = 8 * tc < width;
    const int64_t base = image * g.pixels * g.C + c0 + 8 * tc;
    const int cpg = g.C / g.groups, groups = width / cpg;
    const float inv = 1.0f / ((float)g.pixels * (float)cpg);
    Raw8<BF16> x[NV], dy[NV];
#pragma unroll
    for (int r = 0; r < NV; ++r)
        if (there && row + r * step < g.pixels) {
            x[r] = raw8<BF16>(g.X, base + (int64_t)(row + r * step) * g.C);
            dy[r] = raw8<BF16>(g.dY, base + (int64_t)(row + r * step) * g.C);
        }
    Front f[8];
    float rstd[8];
    if (there) fronts_of(g, image, c0 + 8 * tc, cpg, f, rstd);
    float sum[2][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[0][k] = sum[1][k] = 0.0f;
    with_activation(g.act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < NV; ++r)
            if (there && row + r * step < g.pixels) {
                float v[8], d[8];
                values<BF16>(x[r], v), values<BF16>(dy[r], d);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float dpre = through<decltype(act)::value>(f[k].pre(v[k]), d[k]);
                    sum[0][k] += dpre;
                    sum[1][k] += dpre * (v[k] - f[k].mean);
                }
            }
    });
    if (there)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[1][k] *= rstd[k];
    channel_sums<THREADS, 2, 8>(sum, sp.shift, width, pitch, waves, chan);
    for (int c = threadIdx.x; c < width; c += THREADS)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const float s = chan[q * pitch + c];
            float* const out = q ? g.dgain : g.dshift;
            if (g.N > 1) gstore(g.sums + (q * g.N + image) * g.C + c0 + c, s);
            else if (out) gstore(out + c0 + c, g.accumulate ? gload(out + c0 + c) + s : s);      // one image: these are the gradients
        }
    if (!g.Y) return;
    by_group<THREADS>(groups, cpg, [&](int q, int l, int lanes) {
        float s = 0.0f, t = 0.0f;
        for (int c = l; c < cpg; c += lanes) {
                const float w = gload(g.gain + c0 + q * cpg + c);
                s += chan[q * cpg + c] * w;
                t += chan[pitch + q * cpg + c] * w;
            }
        s = lanes_sum(s, 1, lanes), t = lanes_sum(t, 1, lanes);
        if (l == 0) stat[q] = s * inv, stat[pitch + q] = t * inv;
    });
    __syncthreads();
    if (!there) return;
    // (computed again from what lies in registers: kept, the values in between spilled)
#pragma unroll
    for (int r = 0; r < NV; ++r)
#pragma unroll
        for (int k = 0; k < (BF16 ? 4 : 8); ++k) asm volatile("" : "+v"(x[r].w[k]), "+v"(dy[r].w[k]));
    Slopes c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = slopes_of(f[k], rstd[k], stat[(8 * tc + k) / cpg], stat[pitch + (8 * tc + k) / cpg]);
    with_activation(g.act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < NV; ++r)
            if (row + r * step < g.pixels) {
                float v[8], d[8];
                values<BF16>(x[r], v), values<BF16>(dy[r], d);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = c[k].of(v[k], through<decltype(act)::value>(c[k].pre(v[k]), d[k]));
                store8<BF16>(g.Y, base + (int64_t)(row + r * step) * g.C, v);
            }
    });
}

// ------------------------------------------------------------------------------------------ in pieces
struct Piece { int c0, width, piece, tc, first, last, step; int64_t image, base; bool there; };
__device__ __forceinline__ Piece piece_of(const GroupNorm& g, const GroupSplit& sp, unsigned blocks) {
    Piece p;
    unsigned block = xcd_order(blockIdx.x, blocks);
    const int slab = (int)(block % (unsigned)sp.slabs);
    block /= (unsigned)sp.slabs;
    p.piece = (int)(block % (unsigned)sp.pieces);
    p.image = g.image0 + block / (unsigned)sp.pieces;
    p.c0 = slab * sp.width;
    p.width = g.C - p.c0 < sp.width ? g.C - p.c0 : sp.width;
    p.tc = threadIdx.x & ((1 << sp.shift) - 1);
    p.there = 8 * p.tc < p.width;
    p.first = p.piece * sp.rows + (threadIdx.x >> sp.shift);
    p.last = g.pixels - p.piece * sp.rows < sp.rows ? g.pixels : (p.piece + 1) * sp.rows;
    p.step = 256 >> sp.shift;
    p.base = p.image * g.pixels * g.C + p.c0 + 8 * p.tc;
    return p;
}

// f(row, X, dY) for this thread's rows of the piece, four rows on their way at a time
template <bool BF16, bool BOTH, class F>
__device__ __forceinline__ void by_rows(const GroupNorm& g, const Piece& p, F&& f) {
    constexpr int B = BF16 ? 4 : 2;
    for (int r = p.first; r < p.last; r += B * p.step) {
        Raw8<BF16> x[B], dy[B];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int64_t at = p.base + (int64_t)(r + i * p.step < p.last ? r + i * p.step : r) * g.C;
            x[i] = raw8<BF16>(g.X, at);
            if (BOTH) dy[i] = raw8<BF16>(g.dY, at);
        }
#pragma unroll
        for (int i = 0; i < B; ++i) {
            if (r + i * p.step >= p.last) break;
            float v[8], d[8];
            values<BF16>(x[i], v);
            if (BOTH) values<BF16>(dy[i], d);
            f(r + i * p.step, v, d);
        }
    }
}

// The groups of a slab, of which the first and the last may reach into others.  A group q has a partial of its own in each slab s that it touches, at slot q + s of groups + slabs:
// from one partial to the next either number grows by one, so no two share a slot.
struct SlabGroups { int cpg, first, count; };
__device__ __forceinline__ SlabGroups groups_of(const GroupNorm& g, const Piece& p) {
    const int cpg = g.C / g.groups, first = p.c0 / cpg;
    return SlabGroups{cpg, first, (p.c0 + p.width - 1) / cpg - first + 1};
}
__device__ __forceinline__ int slots(const GroupNorm& g, const GroupSplit& sp) { return g.groups + sp.slabs; }
// where the slots of an image's piece begin
__device__ __forceinline__ const float* slots_of(const float* sums, const GroupNorm& g, const GroupSplit& sp, int64_t image, int piece) {
    return sums + (image * sp.pieces + piece) * slots(g, sp) * 2;
}

// per slot: the mean of a piece's pixels in the group's channels in this slab, and the squares around it
template <bool BF16>
__global__ __launch_bounds__(256) void gn_pieces_kernel(const GroupNorm g, const GroupSplit sp) {
    __shared__ float waves[4 * kMaxSlab], chan[kMaxSlab], means[kMaxSlab];
    const Piece p = piece_of(g, sp, gridDim.x);
    const SlabGroups sg = groups_of(g, p);
    const float inv = 1.0f / (float)(p.last - p.piece * sp.rows);
    float mean[8], square[8], sum[1][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) mean[k] = square[k] = 0.0f;
    float count = 0.0f;
    if (p.there)
        by_rows<BF16, false>(g, p, [&](int, const float (&v)[8], const float (&)[8]) {           // each thread's own mean and squares (Welford)
            count += 1.0f;
            const float part = 1.0f / count;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = v[k] - mean[k];
                mean[k] += d * part;
                square[k] += d * (v[k] - mean[k]);
            }
        });
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[0][k] = mean[k] * count;
    channel_sums<256, 1, 8>(sum, sp.shift, p.width, kMaxSlab, waves, chan);
    // what the group has of this slab
    auto begin = [&](int q) { return q * sg.cpg > p.c0 ? q * sg.cpg - p.c0 : 0; };
    auto end = [&](int q) { return (q + 1) * sg.cpg < p.c0 + p.width ? (q + 1) * sg.cpg - p.c0 : p.width; };
    float* const out = const_cast<float*>(slots_of(g.sums, g, sp, p.image, p.piece)) + 2 * (sg.first + p.c0 / sp.width);
    by_group<256>(sg.count, sg.cpg < p.width ? sg.cpg : p.width, [&](int q, int l, int lanes) {
        const int b = begin(sg.first + q), e = end(sg.first + q);
        float s = 0.0f;
        for (int c = b + l; c < e; c += lanes) s += chan[c];
        s = lanes_sum(s, 1, lanes) * inv / (float)(e - b);
        if (l) return;
        means[q] = s;
        gstore(out + 2 * q, s);
    });
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float d = p.there ? mean[k] - means[(p.c0 + 8 * p.tc + k) / sg.cpg - sg.first] : 0.0f;
        sum[0][k] = square[k] + count * d * d;
    }
    channel_sums<256, 1, 8>(sum, sp.shift, p.width, kMaxSlab, waves, chan);
    by_group<256>(sg.count, sg.cpg < p.width ? sg.cpg : p.width, [&](int q, int l, int lanes) {
        const int b = begin(sg.first + q), e = end(sg.first + q);
        float s = 0.0f;
        for (int c = b + l; c < e; c += lanes) s += chan[c];
        s = lanes_sum(s, 1, lanes);
        if (l == 0) gstore(out + 2 * q + 1, s);
    });
}

// f(slab, piece) for this lane's share of the partials of group q
template <class F>
__device__ __forceinline__ void by_partial(const SlabGroups& sg, const GroupSplit& sp, int q, int l, int lanes, F&& f) {
    const int s0 = q * sg.cpg / sp.width, s1 = ((q + 1) * sg.cpg - 1) / sp.width, touched = s1 - s0 + 1;
    for (int e = l; e < sp.pieces * touched; e += lanes) f(s0 + e % touched, e / touched);
}
__device__ __forceinline__ int partials(const SlabGroups& sg, const GroupSplit& sp) { return sp.pieces * ((sg.cpg + sp.width - 2) / sp.width + 1); }      // at most

template <bool BF16>
__global__ __launch_bounds__(256) void gn_apply_kernel(const GroupNorm g, const GroupSplit sp) {
    __shared__ float stat[2][kMaxSlab];
    const Piece p = piece_of(g, sp, gridDim.x);
    const SlabGroups sg = groups_of(g, p);
    const float inv = 1.0f / ((float)g.pixels * (float)sg.cpg);
    by_group<256>(sg.count, partials(sg, sp), [&](int i, int l, int lanes) {
        const int q = sg.first + i;
        auto weight = [&](int slab, int piece) {          // values behind a partial
            const int c0 = slab * sp.width, b = q * sg.cpg > c0 ? q * sg.cpg : c0, e = (q + 1) * sg.cpg < c0 + sp.width ? (q + 1) * sg.cpg : c0 + sp.width;
            const int left = g.pixels - piece * sp.rows;
            return (float)(e - b) * (float)(left < sp.rows ? left : sp.rows);
        };
        float s = 0.0f, t = 0.0f;
        by_partial(sg, sp, q, l, lanes, [&](int slab, int piece) { s += gload(slots_of(g.sums, g, sp, p.image, piece) + 2 * (q + slab)) * weight(slab, piece); });
        const float mean = lanes_sum(s, 1, lanes) * inv;
        by_partial(sg, sp, q, l, lanes, [&](int slab, int piece) {
            const float* const at = slots_of(g.sums, g, sp, p.image, piece) + 2 * (q + slab);
            const float d = gload(at) - mean;
            t += gload(at + 1) + weight(slab, piece) * d * d;
        });
        t = lanes_sum(t, 1, lanes) * inv;
        if (l) return;
        const float rstd = 1.0f / __builtin_sqrtf(t + g.eps);
        stat[0][i] = mean, stat[1][i] = rstd;
        if (p.piece == 0 && q * sg.cpg >= p.c0) gstore(g.mean + p.image * g.groups + q, mean), gstore(g.rstd + p.image * g.groups + q, rstd);
    });
    __syncthreads();
    if (!p.there) return;
    float gain[8], shift[8];
    load8<false>(g.gain, p.c0 + 8 * p.tc, gain), load8<false>(g.shift, p.c0 + 8 * p.tc, shift);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int q = (p.c0 + 8 * p.tc + k) / sg.cpg - sg.first;
        gain[k] *= stat[1][q];
        shift[k] -= stat[0][q] * gain[k];
    }
    with_activation(g.act, [&](auto act) {
        by_rows<BF16, false>(g, p, [&](int r, const float (&v)[8], const float (&)[8]) {
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = activate<decltype(act)::value>(v[k] * gain[k] + shift[k]);
            store8<BF16>(g.Y, p.base + (int64_t)r * g.C, y);
        });
    });
}

// sums [2, N pieces, C] of dpre and of dpre x^, and behind them per slot the same times the gain, over the group's channels in this slab
__device__ __forceinline__ float* slot_base(const GroupNorm& g, const GroupSplit& sp) { return g.sums + 2 * g.N * sp.pieces * g.C; }
template <bool BF16>
__global__ __launch_bounds__(256) void gn_bwd_pieces_kernel(const GroupNorm g, const GroupSplit sp) {
    __shared__ float waves[8 * kMaxSlab], chan[2 * kMaxSlab];
    const Piece p = piece_of(g, sp, gridDim.x);
    const int cpg = g.C / g.groups;
    float sum[2][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[0][k] = sum[1][k] = 0.0f;
    if (p.there) {
        Front f[8];
        float rstd[8];
        fronts_of(g, p.image, p.c0 + 8 * p.tc, cpg, f, rstd);
        with_activation(g.act, [&](auto act) {
            by_rows<BF16, true>(g, p, [&](int, const float (&x)[8], const float (&dy)[8]) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float dpre = through<decltype(act)::value>(f[k].pre(x[k]), dy[k]);
                    sum[0][k] += dpre;
                    sum[1][k] += dpre * (x[k] - f[k].mean);
                }
            });
        });
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[1][k] *= rstd[k];
    }
    channel_sums<256, 2, 8>(sum, sp.shift, p.width, kMaxSlab, waves, chan);
    for (int c = threadIdx.x; c < p.width; c += 256)
#pragma unroll
        for (int q = 0; q < 2; ++q) gstore(g.sums + ((q * g.N + p.image) * sp.pieces + p.piece) * g.C + p.c0 + c, chan[q * kMaxSlab + c]);
    const SlabGroups sg = groups_of(g, p);
    float* const out = const_cast<float*>(slots_of(slot_base(g, sp), g, sp, p.image, p.piece)) + 2 * (sg.first + p.c0 / sp.width);
    by_group<256>(sg.count, cpg < p.width ? cpg : p.width, [&](int i, int l, int lanes) {
        const int q = sg.first + i, b = q * cpg > p.c0 ? q * cpg - p.c0 : 0, e = (q + 1) * cpg < p.c0 + p.width ? (q + 1) * cpg - p.c0 : p.width;
        float s = 0.0f, t = 0.0f;
        for (int c = b + l; c < e; c += lanes) {
            const float w = gload(g.gain + p.c0 + c);
            s += chan[c] * w;
            t += chan[kMaxSlab + c] * w;
        }
        s = lanes_sum(s, 1, lanes), t = lanes_sum(t, 1, lanes);
        if (l == 0) gstore(out + 2 * i, s), gstore(out + 2 * i + 1, t);
    });
}

// dshift (block even) or dgain of eight channels from `rows` rows of sums
__device__ __forceinline__ void channel_gradients(const GroupNorm& g, int64_t rows, int block, float (*lds)[8]) {
    float* const out = block & 1 ? g.dgain : g.dshift;
    if (!out) return;
    const int c = block / 2 * 8 + (threadIdx.x & 7), part = threadIdx.x >> 3;
    const float* const from = g.sums + (block & 1) * rows * g.C + c;          // (C is a multiple of eight)
    float s = 0.0f;
    for (int64_t r = part; r < rows; r += 256) {          // eight loads on their way at a time
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = gload(from + (r + 32 * k < rows ? r + 32 * k : r) * g.C);
#pragma unroll
        for (int k = 0; k < 8; ++k) s += r + 32 * k < rows ? v[k] : 0.0f;
    }
    lds[part][threadIdx.x & 7] = s;
    __syncthreads();
    if (part) return;
    for (int k = 1; k < 32; ++k) s += lds[k][threadIdx.x];
    gstore(out + c, g.accumulate ? gload(out + c) + s : s);
}

template <bool BF16>
__global__ __launch_bounds__(256) void gn_bwd_apply_kernel(const GroupNorm g, const GroupSplit sp, unsigned blocks) {
    __shared__ float stat[2][kMaxSlab];
    if (blockIdx.x >= blocks) {
        channel_gradients(g, g.N * sp.pieces, (int)(blockIdx.x - blocks), reinterpret_cast<float (*)[8]>(&stat[0][0]));
        return;
    }
    const Piece p = piece_of(g, sp, blocks);
    const SlabGroups sg = groups_of(g, p);
    const int cpg = sg.cpg;
    const float inv = 1.0f / ((float)g.pixels * (float)cpg);
    by_group<256>(sg.count, partials(sg, sp), [&](int i, int l, int lanes) {
        const int q = sg.first + i;
        float s = 0.0f, t = 0.0f;
        by_partial(sg, sp, q, l, lanes, [&](int slab, int piece) {
            const float* const at = slots_of(slot_base(g, sp), g, sp, p.image, piece) + 2 * (q + slab);
            s += gload(at);
            t += gload(at + 1);
        });
        s = lanes_sum(s, 1, lanes), t = lanes_sum(t, 1, lanes);
        if (l == 0) stat[0][i] = s * inv, stat[1][i] = t * inv;
    });
    __syncthreads();
    if (!p.there) return;
    Front f[8];
    Slopes c[8];
    float rstd[8];
    fronts_of(g, p.image, p.c0 + 8 * p.tc, cpg, f, rstd);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int q = (p.c0 + 8 * p.tc + k) / cpg - sg.first;
        c[k] = slopes_of(f[k], rstd[k], stat[0][q], stat[1][q]);
    }
    with_activation(g.act, [&](auto act) {
        by_rows<BF16, true>(g, p, [&](int r, const float (&x)[8], const float (&dy)[8]) {
            float y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = c[k].of(x[k], through<decltype(act)::value>(c[k].pre(x[k]), dy[k]));
            store8<BF16>(g.Y, p.base + (int64_t)r * g.C, y);
        });
    });
}

__global__ __launch_bounds__(256) void gn_channels_kernel(const GroupNorm g, int64_t rows) {
    __shared__ float lds[32][8];
    channel_gradients(g, rows, blockIdx.x, lds);
}
// Many rows: sums of 1024 of them each first, [2, rows / 1024, C] behind what the other launches leave
constexpr int kManyRows = 4096, kRowsOfSum = 1024;
__global__ __launch_bounds__(256) void gn_rows_kernel(const GroupNorm g, int64_t rows, float* out) {
    __shared__ float lds[32][8];
    const unsigned chunks = (unsigned)((rows + kRowsOfSum - 1) / kRowsOfSum), chunk = blockIdx.x % chunks, block = blockIdx.x / chunks;
    const int c = (int)(block / 2) * 8 + (threadIdx.x & 7), part = threadIdx.x >> 3, q = block & 1;
    const int64_t first = (int64_t)chunk * kRowsOfSum, last = first + kRowsOfSum < rows ? first + kRowsOfSum : rows;
    const float* const from = g.sums + q * rows * g.C + c;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < kRowsOfSum / 32; ++i) {
        const int64_t r = first + part + 32 * i;
        if (r < last) s += gload(from + r * g.C);
    }
    lds[part][threadIdx.x & 7] = s;
    __syncthreads();
    if (part) return;
    for (int k = 1; k < 32; ++k) s += lds[k][threadIdx.x];
    gstore(out + ((int64_t)q * chunks + chunk) * g.C + c, s);
}

// ------------------------------------------------------------------------------------------ which
// f(g, blocks, last) for launches of fewer than 2^32 threads, some images each
template <class F>
hipError_t by_images(GroupNorm g, int64_t blocks_per_image, F&& f) {
    const int64_t most = (1 << 21) / blocks_per_image;
    for (g.image0 = 0; g.image0 < g.N; g.image0 += most) {
        const int64_t left = g.N - g.image0;
        f(g, (unsigned)((left < most ? left : most) * blocks_per_image), left <= most);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool BF16, bool BWD, int THREADS, int NV>
hipError_t launch_whole(const GroupNorm& all, const GroupSplit& sp, hipStream_t s) {
    const unsigned lds = (unsigned)(((BWD ? 2 : 1) * (THREADS / 64 + 1) + 2) * sp.width * 4);      // 40 KB at most: 512 threads backward, or 1024 forward, and 512 channels
    const int cpg = all.C / all.groups;
    return by_images(all, sp.slabs, [&](const GroupNorm& g, unsigned blocks, bool) {
        if constexpr (BWD) hipLaunchKernelGGL((gn_whole_bwd_kernel<BF16, THREADS, NV>), dim3(blocks), dim3(THREADS), lds, s, g, sp);
        else if (cpg % 8 == 0) hipLaunchKernelGGL((gn_whole_fwd_kernel<BF16, THREADS, NV, 1>), dim3(blocks), dim3(THREADS), lds, s, g, sp);
        else if (cpg % 4 == 0) hipLaunchKernelGGL((gn_whole_fwd_kernel<BF16, THREADS, NV, 2>), dim3(blocks), dim3(THREADS), lds, s, g, sp);
        else hipLaunchKernelGGL((gn_whole_fwd_kernel<BF16, THREADS, NV, 8>), dim3(blocks), dim3(THREADS), lds, s, g, sp);
    });
}
// what group_plan can answer with
template <bool BF16, bool BWD>
hipError_t launch_whole(const GroupNorm& g, const GroupPlan& p, hipStream_t s) {
    const int kernel = p.threads + (p.vectors <= 2 ? 2 : p.vectors <= 4 ? 4 : p.vectors <= 8 ? 8 : 16);
    switch (kernel) {
        case 256 + 2: return launch_whole<BF16, BWD, 256, 2>(g, p.sp, s);
        case 256 + 4: return launch_whole<BF16, BWD, 256, 4>(g, p.sp, s);
        case 512 + 8: return launch_whole<BF16, BWD, 512, 8>(g, p.sp, s);
    }
    if constexpr (BWD)
        if (kernel == 256 + 8) return launch_whole<BF16, true, 256, 8>(g, p.sp, s);
    if constexpr (BWD && BF16) {
        if (kernel == 256 + 16) return launch_whole<true, true, 256, 16>(g, p.sp, s);
        if (kernel == 512 + 16) return launch_whole<true, true, 512, 16>(g, p.sp, s);
    }
    if constexpr (!BWD) {
        if (kernel == 512 + 4) return launch_whole<BF16, false, 512, 4>(g, p.sp, s);
        if (kernel == 1024 + 8) return launch_whole<BF16, false, 1024, 8>(g, p.sp, s);
    }
    if constexpr (!BWD && BF16)
        if (kernel == 1024 + 16) return launch_whole<true, false, 1024, 16>(g, p.sp, s);
    return hipErrorInvalidValue;
}

template <bool BF16>
hipError_t pieces_fwd(const GroupNorm& all, const GroupSplit& sp, hipStream_t s) {
    const int64_t per_image = (int64_t)sp.slabs * sp.pieces;
    const hipError_t e = by_images(all, per_image, [&](const GroupNorm& g, unsigned blocks, bool) { hipLaunchKernelGGL((gn_pieces_kernel<BF16>), dim3(blocks), dim3(256), 0, s, g, sp); });
    if (e != hipSuccess) return e;
    return by_images(all, per_image, [&](const GroupNorm& g, unsigned blocks, bool) { hipLaunchKernelGGL((gn_apply_kernel<BF16>), dim3(blocks), dim3(256), 0, s, g, sp); });
}
// dgain and dshift from `rows` rows of sums
hipError_t channel_sums_of(GroupNorm g, int64_t rows, float* more, hipStream_t s) {
    if (rows > kManyRows) {
        const int64_t chunks = ceil_div(rows, kRowsOfSum), blocks = chunks * (g.C / 4);
        if (blocks >= 1 << 24) return hipErrorInvalidValue;
        hipLaunchKernelGGL(gn_rows_kernel, dim3((unsigned)blocks), dim3(256), 0, s, g, rows, more);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        g.sums = more;
        rows = chunks;
    }
    hipLaunchKernelGGL(gn_channels_kernel, dim3((unsigned)(g.C / 4)), dim3(256), 0, s, g, rows);
    return hipGetLastError();
}
// Where those sums lie: behind the sums of the channels and the partials
int64_t floats_before(int64_t N, int C, int groups, const GroupPlan& p) { return N * p.sp.pieces * (2 * (int64_t)C + (p.threads ? 0 : 2 * (int64_t)(groups + p.sp.slabs))); }

template <bool BF16>
hipError_t pieces_bwd(const GroupNorm& all, const GroupSplit& sp, float* more, hipStream_t s) {
    const int64_t per_image = (int64_t)sp.slabs * sp.pieces, rows = all.N * sp.pieces;
    const bool channels = all.dgain || all.dshift;
    hipError_t e = by_images(all, per_image, [&](const GroupNorm& g, unsigned blocks, bool) { hipLaunchKernelGGL((gn_bwd_pieces_kernel<BF16>), dim3(blocks), dim3(256), 0, s, g, sp); });
    if (e != hipSuccess) return e;
    if (!all.Y) return channel_sums_of(all, rows, more, s);
    e = by_images(all, per_image, [&](const GroupNorm& g, unsigned blocks, bool last) {      // the gradients of the channels beside the last images
        hipLaunchKernelGGL((gn_bwd_apply_kernel<BF16>), dim3(blocks + (last && channels && rows <= kManyRows ? (unsigned)g.C / 4 : 0)), dim3(256), 0, s, g, sp, blocks);
    });
    return e != hipSuccess || !channels || rows <= kManyRows ? e : channel_sums_of(all, rows, more, s);
}

template <bool BF16>
hipError_t fwd(const GroupNorm& g, hipStream_t s) {
    const GroupPlan p = group_plan(g.N, g.pixels, g.C, g.groups, BF16, false);
    return p.threads ? launch_whole<BF16, false>(g, p, s) : pieces_fwd<BF16>(g, p.sp, s);
}
template <bool BF16>
hipError_t bwd(const GroupNorm& g, hipStream_t s) {
    const GroupPlan p = group_plan(g.N, g.pixels, g.C, g.groups, BF16, true);
    float* const more = g.sums + floats_before(g.N, g.C, g.groups, p);
    if (!p.threads) return pieces_bwd<BF16>(g, p.sp, more, s);
    const hipError_t e = launch_whole<BF16, true>(g, p, s);
    return e != hipSuccess || g.N == 1 || (!g.dgain && !g.dshift) ? e : channel_sums_of(g, g.N, more, s);
}

}  // namespace

size_t group_norm_sum_bytes(int64_t N, int pixels, int C, int groups, bool bf16, bool backward) {
    const GroupPlan p = group_plan(N, pixels, C, groups, bf16, backward);
    if (!backward) return p.threads ? 0 : (size_t)(N * p.sp.pieces * (groups + p.sp.slabs)) * 8;
    if (p.threads && N == 1) return 0;
    const int64_t rows = N * p.sp.pieces;
    return (size_t)(floats_before(N, C, groups, p) + (rows > kManyRows ? ceil_div(rows, kRowsOfSum) * 2 * C : 0)) * 4;
}
hipError_t launch_group_norm_fwd(const GroupNorm& p, bool bf16, hipStream_t s) { return bf16 ? fwd<true>(p, s) : fwd<false>(p, s); }
hipError_t launch_group_norm_bwd(const GroupNorm& p, bool bf16, hipStream_t s) { return bf16 ? bwd<true>(p, s) : bwd<false>(p, s); }

}  // namespace abt
