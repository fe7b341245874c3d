// C ABI of the group norm: validation; documented in include/abtrain.h.
#include <climits>
#include <cmath>

#include "api_util.h"
#include "group_norm.h"

using namespace abt;

namespace {

bool sizes_fit(int64_t N, int64_t pixels, int64_t C, int64_t groups) {
    return N >= 1 && N <= (1 << 28) && pixels >= 1 && pixels <= (1 << 28) && C >= 8 && C <= ABT_GROUP_NORM_MAX_CHANNELS && C % 8 == 0 && groups >= 1 && groups <= C &&
           C % groups == 0 && N * pixels <= (1ll << 36);
}

}  // namespace

extern "C" {

size_t lr_group_norm_workspace_bytes(int64_t N, int64_t pixels, int64_t C, int64_t groups, int dt, int backward) {
    if ((dt != ABT_F32 && dt != ABT_BF16) || !sizes_fit(N, pixels, C, groups)) return 0;
    return align_up(group_norm_sum_bytes(N, (int)pixels, (int)C, (int)groups, dt == ABT_BF16, backward != 0), 256);
}

int lr_group_norm_fwd(const void* X, const float* gain, const float* shift, double eps, void* Y, float* mean, float* rstd,
                      int64_t N, int64_t pixels, int64_t C, int64_t groups, int act, int dt, void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != ABT_F32 && dt != ABT_BF16) return ABT_EDTYPE;
    if (!X || !gain || !shift || !Y || !mean || !rstd || !(eps >= 0.0) || !std::isfinite(eps) || act < ABT_ACT_NONE || act > ABT_ACT_SILU) return ABT_EINVAL;
    if (!sizes_fit(N, pixels, C, groups)) return ABT_ESHAPE;
    if (!aligned(X, 16) || !aligned(gain, 16) || !aligned(shift, 16) || !aligned(Y, 16) || !aligned(mean, 4) || !aligned(rstd, 4)) return ABT_EALIGN;
    const size_t need = lr_group_norm_workspace_bytes(N, pixels, C, groups, dt, 0);
    if (need && (!workspace || workspace_bytes < need)) return ABT_EWORKSPACE;
    if (need && !aligned(workspace, 256)) return ABT_EALIGN;
    GroupNorm p{};
    p.X = X; p.gain = gain; p.shift = shift; p.Y = Y; p.mean = mean; p.rstd = rstd; p.sums = (float*)workspace;
    p.N = N; p.pixels = (int)pixels; p.C = (int)C; p.groups = (int)groups; p.act = act; p.eps = (float)eps;
    return launch_group_norm_fwd(p, dt == ABT_BF16, (hipStream_t)stream) == hipSuccess ? ABT_OK : ABT_EHIP;
}

int lr_group_norm_bwd(const void* dY, const void* X, const float* gain, const float* shift, const float* mean, const float* rstd,
                      void* dX, float* dgain, float* dshift, int64_t N, int64_t pixels, int64_t C, int64_t groups, int act, int dt, int accumulate,
                      void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != ABT_F32 && dt != ABT_BF16) return ABT_EDTYPE;
    if (!dY || !X || !gain || !shift || !mean || !rstd || act < ABT_ACT_NONE || act > ABT_ACT_SILU) return ABT_EINVAL;
    if (!sizes_fit(N, pixels, C, groups)) return ABT_ESHAPE;
    if (!aligned(dY, 16) || !aligned(X, 16) || !aligned(gain, 16) || !aligned(shift, 16) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dX, 16) || !aligned(dgain, 16) ||
        !aligned(dshift, 16))
        return ABT_EALIGN;
    const size_t need = lr_group_norm_workspace_bytes(N, pixels, C, groups, dt, 1);
    if (need && (!workspace || workspace_bytes < need)) return ABT_EWORKSPACE;
    if (need && !aligned(workspace, 256)) return ABT_EALIGN;
    if (!dX && !dgain && !dshift) return ABT_OK;
    GroupNorm p{};
    p.X = X; p.dY = dY; p.gain = gain; p.shift = shift; p.Y = dX; p.mean = const_cast<float*>(mean); p.rstd = const_cast<float*>(rstd); p.sums = (float*)workspace;
    p.dgain = dgain; p.dshift = dshift;
    p.N = N; p.pixels = (int)pixels; p.C = (int)C; p.groups = (int)groups; p.act = act; p.accumulate = accumulate;
    return launch_group_norm_bwd(p, dt == ABT_BF16, (hipStream_t)stream) == hipSuccess ? ABT_OK : ABT_EHIP;
}

}  // extern "C"
