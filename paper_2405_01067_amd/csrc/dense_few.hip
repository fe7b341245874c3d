// The dense layer of a few rows: a work-group has 16 CB columns of up to 16 RB rows, its eight waves share out the contraction, and the sums meet in LDS,
// where the epilogue takes them.  W goes from memory to registers once; X is read by every work-group, from L2.
// Bound by latency (one row of 768 x 768: 4.2 us) and by what reaches a compute unit, some 35 KB a us of W and X together: 4096 x 4096 takes 8 us for a row, 10 for 16, 18 for 48.
// Deeper rings (four steps), sixteen waves and 32 columns were no faster.
#include "activation.h"
#include "adapters_operands.h"
#include "dense.h"
#include "nt_tile.h"

namespace abt {
namespace {

// D steps of a wave are on their way at a time.
template <int RB, int CB, int NW, int D>
__global__ __launch_bounds__(64 * NW) void dense_few_kernel(const DenseProduct g, int row_blocks) {
    __shared__ f32x4 parts[NW][RB * CB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, lq = lane >> 4;
    // the row blocks of the same columns follow each other on one XCD, whose L2 then has W once
    const int block = xcd_order(blockIdx.x, gridDim.x);
    const int64_t row0 = (int64_t)(block % row_blocks) * (16 * RB);
    const int col0 = block / row_blocks * (16 * CB);
    const int rows = g.M - row0 < 16 * RB ? (int)(g.M - row0) : 16 * RB, cols = g.Q - col0 < 16 * CB ? g.Q - col0 : 16 * CB;
    const int bytes = g.K * 2, steps = (bytes + 127) / 128;
    const rsrc_t xres = make_rsrc((const char*)g.X + row0 * bytes, (int64_t)rows * bytes);
    const rsrc_t wres = make_rsrc((const char*)g.W + (int64_t)col0 * bytes, (int64_t)cols * bytes);
    f32x4 acc[RB][CB];
#pragma unroll
    for (int a = 0; a < RB; ++a)
#pragma unroll
        for (int b = 0; b < CB; ++b) acc[a][b] = f32x4{0, 0, 0, 0};
    // a step: 64 columns, of which lane group lq has 16; the same on both sides
    struct Ops { u32x4 w[CB][2], x[RB][2]; };
    auto read = [&](Ops& o, int s) {
        const int k = s * 128 + lq * 32;                  // (steps past the last one are zeros)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = k + 16 * h < bytes ? li * bytes + k + 16 * h : kBufNowhere, step = at == kBufNowhere ? 0 : 16 * bytes;
#pragma unroll
            for (int b = 0; b < CB; ++b) o.w[b][h] = buf_load16(wres, at + b * step, 0);
#pragma unroll
            for (int a = 0; a < RB; ++a) o.x[a][h] = buf_load16(xres, at + a * step, 0);
        }
    };
    Ops ring[D];
#pragma unroll
    for (int d = 0; d < D; ++d) read(ring[d], wave + d * NW);
    for (int s = wave; s < steps; s += NW * D)
#pragma unroll
        for (int d = 0; d < D; ++d) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int a = 0; a < RB; ++a)
#pragma unroll
                    for (int b = 0; b < CB; ++b) acc[a][b] = mfma16(ring[d].w[b][h], ring[d].x[a][h], acc[a][b]);
            read(ring[d], s + (D + d) * NW);
        }
    // lane: row li of a block of rows, columns 4 lq .. + 3 of a block of columns
#pragma unroll
    for (int a = 0; a < RB; ++a)
#pragma unroll
        for (int b = 0; b < CB; ++b) parts[wave][a * CB + b][lane] = acc[a][b];
    __syncthreads();
    const DropKey key = g.drop.state ? drop_key(g.drop) : DropKey{0, 0, 0, 0};
    // a thread's four columns of a row
    for (int i = threadIdx.x; i < RB * CB * 64; i += 64 * NW) {
        const int blk = i >> 6, l = i & 63, r = 16 * (blk / CB) + (l & 15), c = 16 * (blk % CB) + 4 * (l >> 4);
        if (r >= rows || c >= cols) continue;
        const int64_t at = (row0 + r) * g.Q + col0 + c;
        u32x2 res = {0, 0};
        if (g.residual) res = gload(reinterpret_cast<const u32x2*>(g.residual + at));
        f32x4 bias = {0, 0, 0, 0};
        if (g.bias) bias = gload(reinterpret_cast<const f32x4*>(g.bias + col0 + c));
        f32x4 sum = parts[0][blk][l];
#pragma unroll
        for (int w = 1; w < NW; ++w) sum += parts[w][blk][l];
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = sum[k] * g.alpha + bias[k];
        if (g.Z) gstore(reinterpret_cast<u32x2*>(g.Z + at), u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])});
        with_activation(g.act, [&](auto act) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = activate<decltype(act)::value>(v[k]);
        });
        if (g.drop.state) {
            const u32x4 bits = drop_bits(key, (uint64_t)at >> 3);
            const bool upper = (at & 4) != 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (upper ? drop_keeps(g.drop, bits, 4 + k) : drop_keeps(g.drop, bits, k)) ? v[k] * g.drop.scale : 0.0f;
        }
        if (g.residual)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += __builtin_bit_cast(float, k & 1 ? res[k >> 1] & 0xffff0000u : res[k >> 1] << 16);
        gstore(reinterpret_cast<u32x2*>(g.Y + at), u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])});
    }
}

template <int RB, int CB, int NW, int D>
hipError_t launch_few(const DenseProduct& p, hipStream_t s) {
    const int64_t row_blocks = ceil_div(p.M, 16 * RB), blocks = row_blocks * ceil_div(p.Q, 16 * CB);
    if (blocks > (1 << 30)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((dense_few_kernel<RB, CB, NW, D>), dim3((unsigned)blocks), dim3(64 * NW), 0, s, p, (int)row_blocks);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dense_few(const DenseProduct& p, hipStream_t s) {
    return p.M <= 16 ? launch_few<1, 1, 8, 2>(p, s) : p.M <= 32 ? launch_few<2, 1, 8, 1>(p, s) : launch_few<4, 1, 8, 1>(p, s);
}

}  // namespace abt
