// Y = residual + drop(act(X W^T + bias)) for many rows: tiles of the product whose epilogue runs in the accumulators.  The residual comes straight to LDS
// while activation and mask are computed, and results and the sum before the activation leave through LDS as whole rows.
#include <climits>

#include "dense_tile.h"

namespace abt {
namespace {

template <class L>
__global__ __launch_bounds__(64 * L::NW) void dense_kernel(const DenseProduct g, const Order order) {
    extern __shared__ __align__(1024) unsigned char lds[];
    dense_tile<L>(g, order, blockIdx.x, lds);
}

template <class L>
hipError_t launch_tile(const DenseProduct& p, hipStream_t s) {
    static std::atomic<bool> attr_set{false};
    const hipError_t e = lds_allowed(reinterpret_cast<const void*>(&dense_kernel<L>), L::lds, attr_set);
    if (e != hipSuccess) return e;
    const int64_t rt = ceil_div(p.M, L::TM), ct = ceil_div(p.Q, L::TN);
    if (rt * ct > INT_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((dense_kernel<L>), dim3((unsigned)(rt * ct)), dim3(64 * L::NW), L::lds, s, p, Order{(int)rt, (int)ct});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dense_tiles(const DenseProduct& p, hipStream_t s) { return launch_tile<Tile<128, 128, 2, 2, 1>>(p, s); }

}  // namespace abt
