// The group norm of channels-last images (group_norm.hip): what group_norm_api.hip calls.
#pragma once

#include "common.h"

namespace abt {

// X, dY, Y, dX [N, pixels, C]; C a multiple of 8 and of `groups`
struct GroupNorm {
    const void* X; const void* dY;         // dY: backward
    const float* gain; const float* shift;
    void* Y;                               // or dX (backward; may be NULL)
    float* mean; float* rstd;              // [N, groups], written by the forward
    float* sums;                           // workspace
    float* dgain; float* dshift;           // may be NULL
    int64_t N;
    int64_t image0;                        // set by the launchers: the first image of a launch
    int pixels, C, groups, act, accumulate;
    float eps;
};
size_t group_norm_sum_bytes(int64_t N, int pixels, int C, int groups, bool bf16, bool backward);
hipError_t launch_group_norm_fwd(const GroupNorm& p, bool bf16, hipStream_t s);
hipError_t launch_group_norm_bwd(const GroupNorm& p, bool bf16, hipStream_t s);

}  // namespace abt
