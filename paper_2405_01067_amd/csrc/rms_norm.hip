// Root-mean-square norm of rows with the addition of the residual, forward and backward:
//     h = x + res,  s = (mean h^2 + eps)^(-1/2),  y = h s g           also q ~ y / scale in 8-bit floats, scale = max |y| / 448
//     dX = dH + s (dY g - h s^2 mean(dY g h)),  dg = sum over rows of dY h s
// A row stays in registers from its one read to its last write: one wave per row up to 2048 columns, a work-group of four
// waves per row beyond (two waves in a range of the backward).  The backward forms s again from h, which it has in registers anyway, so the forward keeps nothing for it.
// Statistics and gradients of the gain are fp32; y is formed from h before h is rounded.  Bound by memory: 50432 x 768
// in bf16 with the residual 61 us (310 MB, 5.1 TB/s; part of it from the last-level cache); backward of 12608 x 768 17.9 us and 4.0 for the gain's sums (77 MB, 4.3 TB/s); 48 x 4096 with 8
// bits 4.2 us, latency of the load, two sums over the work-group and the stores.
#include <type_traits>

#include "common.h"

namespace abt {
namespace {

typedef __attribute__((ext_vector_type(8))) float f32x8;

__device__ __forceinline__ f32x8 load8(const float* p) {
    const f32x4 a = gload(reinterpret_cast<const f32x4*>(p)), b = gload(reinterpret_cast<const f32x4*>(p + 4));
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ f32x8 unpack8(u32x4 v) {
    f32x8 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        o[2 * j] = __builtin_bit_cast(float, v[j] << 16);
        o[2 * j + 1] = __builtin_bit_cast(float, v[j] & 0xffff0000u);
    }
    return o;
}
__device__ __forceinline__ f32x8 load8(const uint16_t* p) { return unpack8(gload(reinterpret_cast<const u32x4*>(p))); }
__device__ __forceinline__ void store8(float* p, f32x8 v) {
    gstore(reinterpret_cast<f32x4*>(p), f32x4{v[0], v[1], v[2], v[3]});
    gstore(reinterpret_cast<f32x4*>(p + 4), f32x4{v[4], v[5], v[6], v[7]});
}
__device__ __forceinline__ void store8(uint16_t* p, f32x8 v) {
    gstore(reinterpret_cast<u32x4*>(p), u32x4{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])});
}

constexpr int kNormThreads = 256;
constexpr int kNormBlocks = 1 << 23;                       // of a launch, which has fewer than 2^32 threads

// Sum or largest value over the lanes of a row: WPR waves of the work-group, in a fixed order.
template <int WPR, bool MAX>
__device__ __forceinline__ float over_row(float v, float* part) {
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const float o = __shfl_xor(v, d);
        v = MAX ? fmaxf(v, o) : v + o;
    }
    if constexpr (WPR > 1) {
        __syncthreads();                                  // (the values of the call before have been read)
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        const float* const p = part + (WPR == 2 ? threadIdx.x >> 7 << 1 : 0);
        v = MAX ? fmaxf(p[0], p[1]) : p[0] + p[1];
        if constexpr (WPR == 4) v = MAX ? fmaxf(v, fmaxf(p[2], p[3])) : v + (p[2] + p[3]);
    }
    return v;
}

// V: pieces of eight columns per lane; lane l of a row has the pieces l, l + 64 WPR, ..
template <class T, int WPR, int V, bool Q8>
__global__ __launch_bounds__(kNormThreads) void rms_norm_fwd_kernel(const T* X, const T* R, const float* gain, float eps, T* H, T* Y, uint8_t* Yq, float* scale,
                                                                    int64_t M, int n) {
    __shared__ float part[4];
    const int64_t row = (int64_t)blockIdx.x * (4 / WPR) + threadIdx.x / (64 * WPR);
    if (row >= M) return;                                 // whole waves; whole work-groups where they share a row
    const int l = threadIdx.x % (64 * WPR);
    f32x8 h[V], g[V];
    const int64_t base = row * n;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (l + 64 * WPR * i) * 8;
        if (c < n) {
            h[i] = load8(X + base + c);
            if (R) h[i] += load8(R + base + c);
            g[i] = load8(gain + c);
        } else {
            h[i] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
            g[i] = h[i];
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += h[i][j] * h[i][j];
    const float s = 1.0f / sqrtf(over_row<WPR, false>(sum, part) / (float)n + eps);
    float largest = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (l + 64 * WPR * i) * 8;
        if (c < n && H) store8(H + base + c, h[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * s * g[i][j];
        if (c < n && Y) store8(Y + base + c, h[i]);
        if constexpr (Q8)
#pragma unroll
            for (int j = 0; j < 8; ++j) largest = fmaxf(largest, fabsf(h[i][j]));
    }
    if constexpr (Q8) {
        // A row of zeros, or of values below 1e-30 (whose factor would not be finite), has scale 0 and values 0; one with an infinity has scale
        // infinity, one with NaN keeps them among its values.
        largest = over_row<WPR, true>(largest, part);
        if (largest < 1e-30f) largest = 0.0f;
        const float inv = largest > 0.0f ? 448.0f / largest : 0.0f;
        if (l == 0) gstore(scale + row, largest * (1.0f / 448.0f));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (l + 64 * WPR * i) * 8;
            if (c < n) {
                u32x2 w;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    int v = __builtin_amdgcn_cvt_pk_fp8_f32(h[i][4 * j] * inv, h[i][4 * j + 1] * inv, 0, false);
                    v = __builtin_amdgcn_cvt_pk_fp8_f32(h[i][4 * j + 2] * inv, h[i][4 * j + 3] * inv, v, true);
                    w[j] = (uint32_t)v;
                }
                gstore(reinterpret_cast<u32x2*>(Yq + base + c), w);
            }
        }
    }
}

// Work-group b takes rows b (4 / WPR), .. in steps of the grid and leaves its sum of the gain's gradient in sums[b, n].
template <class T, int WPR, int V>
__global__ __launch_bounds__(kNormThreads) void rms_norm_bwd_kernel(const T* dY, const T* Hin, const float* gain, float eps, const T* dH, T* dX, float* sums,
                                                                    int64_t M, int n) {
    __shared__ float part[4];
    constexpr int RPB = 4 / WPR;
    __shared__ __align__(16) float rows_of[RPB > 1 ? (RPB - 1) * 512 * WPR * V : 4];
    const int sub = threadIdx.x / (64 * WPR), l = threadIdx.x % (64 * WPR);
    f32x8 dg[V], g[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (l + 64 * WPR * i) * 8;
        dg[i] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
        g[i] = c < n ? load8(gain + c) : dg[i];
    }
    for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < M; row0 += (int64_t)gridDim.x * RPB) {
        const int64_t base = (row0 + sub) * n;
        const int cols = row0 + sub < M ? n : 0;          // all rows of the work-group meet at the barriers, also one that is not there
        f32x8 h[V], u[V], r[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (l + 64 * WPR * i) * 8;
            if (c < cols) {
                h[i] = load8(Hin + base + c);
                u[i] = load8(dY + base + c);
                if (dH) r[i] = load8(dH + base + c);
            } else {
                h[i] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
                u[i] = h[i];
            }
            if (!(c < cols && dH)) r[i] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
        }
        float hh = 0.0f, uh = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                hh += h[i][j] * h[i][j];
                uh += u[i][j] * g[i][j] * h[i][j];
            }
        hh = over_row<WPR, false>(hh, part);
        uh = over_row<WPR, false>(uh, part);
        // (a row that is not there has h = 0: without eps its factor would be infinite, and its part in dg NaN)
        const float s = cols ? 1.0f / sqrtf(hh / (float)n + eps) : 0.0f;
        const float k = s * s * (uh / (float)n);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (l + 64 * WPR * i) * 8;
            f32x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = r[i][j] + s * (u[i][j] * g[i][j] - k * h[i][j]);
                dg[i][j] += u[i][j] * (h[i][j] * s);
            }
            if (c < cols && dX) store8(dX + base + c, o);
        }
    }
    if (!sums) return;
    if constexpr (RPB > 1) {                              // the sums of the work-group's rows, in order
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (sub)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<f32x4*>(rows_of + (((sub - 1) * V + i) * 2 + j) * 256 * WPR + l * 4) =
                        f32x4{dg[i][4 * j], dg[i][4 * j + 1], dg[i][4 * j + 2], dg[i][4 * j + 3]};
        __syncthreads();
        if (sub) return;
#pragma unroll
        for (int w = 0; w < RPB - 1; ++w)
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(rows_of + ((w * V + i) * 2 + j) * 256 * WPR + l * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dg[i][4 * j + e] += v[e];
                }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (l + 64 * WPR * i) * 8;
        if (c < n) store8(sums + (int64_t)blockIdx.x * n + c, dg[i]);
    }
}

// dgain[c] = sum over b of sums[b, c]: 64 columns a work-group, sixteen waves that share the rows
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* sums, int rows, int n, float* out, int accumulate) {
    __shared__ float part[16][64];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + l;
    float v = 0.0f;
    if (c < n) {
        int b = w;
        for (; b + 112 < rows; b += 128) {                // eight loads on their way at a time
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = gload(sums + (int64_t)(b + 16 * i) * n + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v += x[i];
        }
        for (; b < rows; b += 16) v += gload(sums + (int64_t)b * n + c);
    }
    part[w][l] = v;
    __syncthreads();
    if (w || c >= n) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) v += part[i][l];
    gstore(out + c, accumulate ? gload(out + c) + v : v);
}

// f(waves per row, pieces per lane) as constants; pairs: two waves per row where n is more than 2048 and at most 4096
template <class F>
hipError_t by_width(int n, bool pairs, F&& f) {
    const auto c = [](auto v) { return v; };
    if (pairs) return n <= 3072 ? f(std::integral_constant<int, 2>{}, c(std::integral_constant<int, 3>{})) : f(std::integral_constant<int, 2>{}, c(std::integral_constant<int, 4>{}));
    if (n <= 2048) {
        switch ((n + 511) / 512) {
            case 1: return f(std::integral_constant<int, 1>{}, c(std::integral_constant<int, 1>{}));
            case 2: return f(std::integral_constant<int, 1>{}, c(std::integral_constant<int, 2>{}));
            case 3: return f(std::integral_constant<int, 1>{}, c(std::integral_constant<int, 3>{}));
            default: return f(std::integral_constant<int, 1>{}, c(std::integral_constant<int, 4>{}));
        }
    }
    switch ((n + 2047) / 2048) {
        case 2: return f(std::integral_constant<int, 4>{}, c(std::integral_constant<int, 2>{}));
        case 3: return f(std::integral_constant<int, 4>{}, c(std::integral_constant<int, 3>{}));
        case 4: return f(std::integral_constant<int, 4>{}, c(std::integral_constant<int, 4>{}));
        case 5: case 6: return f(std::integral_constant<int, 4>{}, c(std::integral_constant<int, 6>{}));
        default: return f(std::integral_constant<int, 4>{}, c(std::integral_constant<int, 8>{}));
    }
}

template <class T>
hipError_t fwd(const void* X, const void* R, const float* gain, float eps, void* H, void* Y, void* Yq, float* scale, int64_t M, int n, hipStream_t s) {
    return by_width(n, false, [&](auto wpr, auto v) {
        constexpr int W = decltype(wpr)::value, V = decltype(v)::value;
        const auto from = [&](auto* p, int64_t at) { return p ? p + at : p; };
        for (int64_t row = 0; row < M; row += (int64_t)kNormBlocks * (4 / W)) {
            const int64_t rows = M - row < (int64_t)kNormBlocks * (4 / W) ? M - row : (int64_t)kNormBlocks * (4 / W), at = row * n;
            const dim3 grid((unsigned)ceil_div(rows, 4 / W));
            if (Yq) hipLaunchKernelGGL((rms_norm_fwd_kernel<T, W, V, true>), grid, dim3(kNormThreads), 0, s, from((const T*)X, at), from((const T*)R, at), gain, eps,
                                       from((T*)H, at), from((T*)Y, at), (uint8_t*)Yq + at, scale + row, rows, n);
            else hipLaunchKernelGGL((rms_norm_fwd_kernel<T, W, V, false>), grid, dim3(kNormThreads), 0, s, from((const T*)X, at), from((const T*)R, at), gain, eps,
                                    from((T*)H, at), from((T*)Y, at), nullptr, nullptr, rows, n);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

}  // namespace

// Two waves per row in the backward of many rows of bf16: fewer rounds of the 512 work-groups.  us, two / four waves: 600 x 2304 9.1 / 10.5, 4096 x 2304 19.2 / 22.2,
// 12608 x 2304 43.3 / 51.9, 8190 x 4096 39.0 / 43.0; but 48 x 4096 7.4 / 6.5, fp32 2100 x 3000 21.9 / 20.9 and 8190 x 4096 82.7 / 76.2, and the
// forward, whose grid is not bounded, 8190 x 4096 44.2 / 40.5.
static bool row_pairs(int64_t M, int n, bool bf16) { return bf16 && M > 512 && n > 2048 && n <= 4096; }
// One row per wave, pair or work-group up to two work-groups per compute unit, beyond several
int rms_norm_bwd_blocks(int64_t M, int n, bool bf16) {
    const int64_t b = ceil_div(M, n <= 2048 ? 4 : row_pairs(M, n, bf16) ? 2 : 1);
    return (int)(b < 512 ? b : 512);
}

hipError_t launch_rms_norm_fwd(const void* X, const void* R, const float* gain, float eps, void* H, void* Y, void* Yq, float* scale, int64_t M, int n, bool bf16,
                               hipStream_t s) {
    return bf16 ? fwd<uint16_t>(X, R, gain, eps, H, Y, Yq, scale, M, n, s) : fwd<float>(X, R, gain, eps, H, Y, Yq, scale, M, n, s);
}

hipError_t launch_rms_norm_bwd(const void* dY, const void* H, const float* gain, float eps, const void* dH, void* dX, float* dgain, float* sums, int64_t M, int n,
                               bool bf16, int accumulate, hipStream_t s) {
    const int blocks = rms_norm_bwd_blocks(M, n, bf16);
    float* const to = dgain ? sums : nullptr;
    const hipError_t e = by_width(n, row_pairs(M, n, bf16), [&](auto wpr, auto v) {
        constexpr int W = decltype(wpr)::value, V = decltype(v)::value;
        if (bf16 || W == 2) hipLaunchKernelGGL((rms_norm_bwd_kernel<uint16_t, W, V>), dim3((unsigned)blocks), dim3(kNormThreads), 0, s, (const uint16_t*)dY,
                                     (const uint16_t*)H, gain, eps, (const uint16_t*)dH, (uint16_t*)dX, to, M, n);
        else if constexpr (W != 2) hipLaunchKernelGGL((rms_norm_bwd_kernel<float, W, V>), dim3((unsigned)blocks), dim3(kNormThreads), 0, s, (const float*)dY, (const float*)H, gain,
                                eps, (const float*)dH, (float*)dX, to, M, n);
        return hipGetLastError();
    });
    if (e != hipSuccess || !dgain) return e;
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)ceil_div(n, 64)), dim3(1024), 0, s, sums, blocks, n, dgain, accumulate);
    return hipGetLastError();
}

}  // namespace abt
