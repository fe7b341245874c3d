// Gradients of the adapters for many rows.  The list of the rows is cut into pieces of equal length whatever the adapters; a work-group has 128 columns of
// dY or X and one piece, and leaves the sums of each adapter in it as a partial of its own (piece p and adapter a meet in slot p + a:
// along the list either grows by one, so no two meetings share a slot).  A second launch adds an adapter's partials in order.
// No atomics: the same call gives the same bits.
// Bound by memory and by waits for the slabs: 12608 rows of 2304 and 768 columns, r = 16, 24.5 us alone (77 MB, 3.2 TB/s; 3.7 GFLOP three times over for the planes), the sums of
// 8 adapters' partials 4.9 us.
#include <climits>

#include "adapters_grad.h"

namespace abt {
namespace {

template <int VB>
__global__ __launch_bounds__(256) void adapters_grad_kernel(const AdapterGrads g, const Side a, const Side b, int piece) {
    extern __shared__ __align__(1024) unsigned char lds[];
    const int blocks = a.blocks + b.blocks;
    grad_block<VB>(g, a, b, (int)blockIdx.x % blocks, piece, (int)blockIdx.x / blocks, lds);
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
    if (end > begin) {
        const int last = (end - 1) / piece;
        for (int p = begin / piece; p <= last; p += 8) {  // eight loads on their way at a time
            f32x4 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = gload(reinterpret_cast<const f32x4*>(part + (int64_t)((p + i < last ? p + i : last) + a) * size));
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (p + i <= last) v += x[i];
        }
    }
    if (g.accumulate) v += gload(reinterpret_cast<const f32x4*>(out));
    gstore(reinterpret_cast<f32x4*>(out), v);
}

template <int VB>
hipError_t launch_grads(const AdapterGrads& p, const Side& a, const Side& b, int piece, hipStream_t s) {
    using L = Grad<VB>;
    static std::atomic<bool> attr_set{false};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&adapters_grad_kernel<VB>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((adapters_grad_kernel<VB>), dim3((unsigned)((a.blocks + b.blocks) * ceil_div(p.M, piece))), dim3(256), L::lds, s, p, a, b, piece);
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

hipError_t launch_adapters_grads(const AdapterGrads& p, const AdapterProduct* x, hipStream_t s) {
    const int piece = adapters_grad_piece(p.M, p.m, p.n);
    const int64_t pieces = ceil_div(p.M, piece);
    if (p.count > 65535) return hipErrorInvalidValue;
    Side a, b;
    grad_sides(p, pieces + p.count, a, b);
    if (a.blocks + b.blocks == 0) return hipSuccess;
    if ((a.blocks + b.blocks) * pieces > INT_MAX) return hipErrorInvalidValue;
    hipError_t e;
    if (x) e = launch_adapters_dx_grad_pieces(*x, p, piece, s);
    else switch (plane_columns(p.r)) {
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

}  // namespace abt
