// The layer with adapters for a few rows, as single tokens of many requests are: T_i = B_a x_i, then Y_i = W x_i + A_a T_i.
// Nothing is reused but the rows themselves, so the operands go from memory to registers: bound by the bytes of W and of the adapters in use, and
// by the latency of two launches where these are few.
//   T: a work-group per row and eight of its rank's rows of B, two rows a wave; lanes share out the columns.
//   Y: a work-group per 16 columns; eight waves share out the contraction (128 bytes of every row at a time) and the adapters, and their
//      sums are added through LDS in order.
#include <climits>

#include "adapters.h"

namespace abt {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16_f8(u32x4 a0, u32x4 a1, u32x4 b0, u32x4 b1, f32x4 c) {
    const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
    const i32x8 b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);      // scales of 2^0
}
__device__ __forceinline__ float lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xffff0000u); }

__device__ __forceinline__ u32x4 first_of(u32x4 v, int valid) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] &= valid >= 2 * i + 2 ? 0xffffffffu : valid == 2 * i + 1 ? 0xffffu : 0u;
    return v;
}

__global__ __launch_bounds__(256) void few_t_kernel(const AdapterProduct g) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x;
    const int n = g.ke;
    int a = __builtin_amdgcn_readfirstlane(gload(g.row_adapter + row));
    const bool have = a >= 0 && a < g.count;
    const int rank0 = have ? (g.ranks ? __builtin_amdgcn_readfirstlane(gload(g.ranks + a)) : g.r) : 0;
    const int rank = rank0 > g.r ? g.r : rank0;
    const int j0 = (int)blockIdx.y * 8 + 2 * wave;        // two rows of B; r is a multiple of 8
    float sum[2] = {0.0f, 0.0f};
    if (j0 < rank) {
        const uint16_t* const x = g.E + row * g.e_pitch;
        const uint16_t* const b = g.F + ((int64_t)a * g.r + j0) * n;
#pragma unroll 4
        for (int c = lane * 8; c < n; c += 512) {
            const u32x4 xv = gload(reinterpret_cast<const u32x4*>(x + c)), b0 = gload(reinterpret_cast<const u32x4*>(b + c)),
                        b1 = gload(reinterpret_cast<const u32x4*>(b + n + c));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[0] += lo(xv[i]) * lo(b0[i]);
                sum[0] += hi(xv[i]) * hi(b0[i]);
                sum[1] += lo(xv[i]) * lo(b1[i]);
                sum[1] += hi(xv[i]) * hi(b1[i]);
            }
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            sum[0] += __shfl_xor(sum[0], d);
            sum[1] += __shfl_xor(sum[1], d);
        }
        if (j0 + 1 >= rank) sum[1] = 0.0f;
    }
    if (lane) return;
    const float s = have && g.scales ? gload(g.scales + a) : 1.0f;
    if (g.T) {
        gstore(g.T + row * g.r + j0, sum[0]);
        gstore(g.T + row * g.r + j0 + 1, sum[1]);
    }
    // what is past the rank is zero whatever the scale
    if (g.Tb) gstore(reinterpret_cast<uint32_t*>(g.Tb + row * g.r + j0), pack2_bf16(j0 < rank ? s * sum[0] : 0.0f, j0 + 1 < rank ? s * sum[1] : 0.0f));
}

// RB blocks of 16 rows
template <int RB, bool F8>
__global__ __launch_bounds__(512) void few_y_kernel(const AdapterProduct g) {
    __shared__ __align__(16) f32x4 sums[8 * RB * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, lq = lane >> 4;
    const int M = (int)g.M, col0 = blockIdx.x * 16;
    const int bytes = g.kmain * (F8 ? 1 : 2), units = (bytes + 127) / 128;
    // a unit is 128 bytes of every row; lanes past the last row, column or byte read zeros
    const rsrc_t xres = make_rsrc(g.X, (int64_t)M * bytes);
    const int wrows = g.Q - col0 < 16 ? g.Q - col0 : 16;
    const rsrc_t wres = make_rsrc((const char*)g.W + (int64_t)col0 * bytes, (int64_t)wrows * bytes);
    f32x4 acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = f32x4{0, 0, 0, 0};
    auto unit = [&](int u) {
        const int at0 = u * 128 + lq * 16, at1 = at0 + 64;
        const u32x4 w0 = buf_load16(wres, at0 < bytes ? li * bytes + at0 : kBufNowhere, 0);
        const u32x4 w1 = buf_load16(wres, at1 < bytes ? li * bytes + at1 : kBufNowhere, 0);
        u32x4 x0[RB], x1[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            x0[b] = buf_load16(xres, at0 < bytes ? (16 * b + li) * bytes + at0 : kBufNowhere, 0);
            x1[b] = buf_load16(xres, at1 < bytes ? (16 * b + li) * bytes + at1 : kBufNowhere, 0);
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            if constexpr (F8) {
                acc[b] = mfma16_f8(w0, w1, x0[b], x1[b], acc[b]);
            } else {
                acc[b] = mfma16(w0, x0[b], acc[b]);
                acc[b] = mfma16(w1, x1[b], acc[b]);
            }
        }
    };
    int u = wave;
    for (; u + 24 < units; u += 32) {                     // four at a time, their loads together
        unit(u);
        unit(u + 8);
        unit(u + 16);
        unit(u + 24);
    }
    for (; u < units; u += 8) unit(u);
    if constexpr (F8) {
        float ws[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ws[i] = 4 * lq + i < wrows ? gload(g.w_scale + col0 + 4 * lq + i) : 0.0f;
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const float xs = 16 * b + li < M ? gload(g.x_scale + 16 * b + li) : 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[b][i] *= xs * ws[i];
        }
    }
    // the adapters of the rows, every eighth of those that occur
    int ids = lane < M ? gload(g.row_adapter + lane) : -1;
    if (ids >= g.count) ids = -1;
    int mine[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) mine[b] = 16 * b + li < M ? gload(g.row_adapter + 16 * b + li) : -1;
    const rsrc_t eres = make_rsrc(g.E, (int64_t)M * g.r * 2);
    int a = -1;
    for (int k = 0;; ++k) {
        int best = ids > a ? ids : INT_MAX;
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const int o = __shfl_xor(best, d);
            best = o < best ? o : best;
        }
        a = __builtin_amdgcn_readfirstlane(best);
        if (a == INT_MAX) break;
        if ((k & 7) != wave) continue;
        int rank = g.ranks ? __builtin_amdgcn_readfirstlane(gload(g.ranks + a)) : g.r;
        rank = rank > g.r ? g.r : rank;
        const rsrc_t fres = make_rsrc(g.F + ((int64_t)a * g.Q + col0) * g.r, (int64_t)wrows * g.r * 2);
        for (int j = 0; j < rank; j += 32) {
            const int c = j + lq * 8;
            u32x4 f = buf_load16(fres, c < rank ? (li * g.r + c) * 2 : kBufNowhere, 0);
            u32x4 t[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) t[b] = buf_load16(eres, c < rank && mine[b] == a ? ((16 * b + li) * g.r + c) * 2 : kBufNowhere, 0);
            if (rank - j < 32 && (rank & 7)) f = first_of(f, rank - c);            // (T is zero there)
#pragma unroll
            for (int b = 0; b < RB; ++b) acc[b] = mfma16(f, t[b], acc[b]);
        }
    }
    // lane: row 16 b + li, columns 4 lq .. + 3
#pragma unroll
    for (int b = 0; b < RB; ++b) sums[(wave * RB + b) * 64 + lane] = acc[b];
    __syncthreads();
    if (wave >= RB) return;
    f32x4 v = sums[wave * 64 + lane];
#pragma unroll
    for (int w = 1; w < 8; ++w) v += sums[(w * RB + wave) * 64 + lane];
    const int row = 16 * wave + li, c = 4 * lq;
    if (row < M && c < wrows) gstore(reinterpret_cast<u32x2*>(g.Y + (int64_t)row * g.Q + col0 + c), u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])});
}

template <bool F8>
hipError_t few_y(const AdapterProduct& p, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div(p.Q, 16));
    if (p.M <= 16) hipLaunchKernelGGL((few_y_kernel<1, F8>), grid, dim3(512), 0, s, p);
    else if (p.M <= 32) hipLaunchKernelGGL((few_y_kernel<2, F8>), grid, dim3(512), 0, s, p);
    else hipLaunchKernelGGL((few_y_kernel<4, F8>), grid, dim3(512), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adapters_few_t(const AdapterProduct& p, hipStream_t s) {
    if (p.M > kAdapterFewT) return hipErrorInvalidValue;
    hipLaunchKernelGGL(few_t_kernel, dim3((unsigned)p.M, (unsigned)ceil_div(p.r, 8)), dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_adapters_few_y(const AdapterProduct& p, bool fp8, hipStream_t s) {
    if (p.M > kAdapterFewRows || p.e_pitch != p.r) return hipErrorInvalidValue;
    return fp8 ? few_y<true>(p, s) : few_y<false>(p, s);
}

}  // namespace abt
