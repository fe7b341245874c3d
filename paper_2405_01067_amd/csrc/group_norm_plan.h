// How a call of the group norm is split: rules on sizes alone (plain C++, no device code).
#pragma once

#include <initializer_list>

#include "int_util.h"

namespace abt {

constexpr int kMaxSlab = 512;                             // channels: 64 threads across

// Slabs of the channels, of `width` each (the last may have fewer) and TC = 2^shift threads across; pieces of the pixels
struct GroupSplit { int width, slabs, shift, pieces, rows; };

inline int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

// How a call is split; threads, vectors: of the `whole` kernels, threads = 0 for the others
struct GroupPlan { GroupSplit sp; int threads, vectors; };
// Threads of the `whole` kernels and vectors of eight values that each holds at most, in the order in which they are tried.  A thread's registers hold 16 vectors of bf16, 8 of
// fp32, or with 1024 threads 16 and 8 of one tensor (the backward has two, and what 1024 threads could hold, 512 do).
struct GroupThreads { int threads, vectors; };
constexpr GroupThreads kGroupForward[] = {{256, 4}, {512, 4}, {512, 8}, {1024, 8}, {1024, 16}}, kGroupBackward[] = {{256, 8}, {512, 8}, {512, 16}};
inline int threads_across(int width) {                           // as a power of two's exponent
    int shift = 0;
    while ((8 << shift) < width) ++shift;
    return shift;
}
inline GroupPlan group_plan(int64_t N, int pixels, int C, int groups, bool bf16, bool backward) {
    GroupPlan p{};
    const int cpg = C / groups, unit = cpg / gcd(cpg, 8) * 8, wide = 64;      // whole groups and vectors; 128 bytes in bf16, 256 in fp32
    const int most_vectors = bf16 ? 16 : 8;
    const bool much = N * pixels * C * (bf16 ? 2 : 4) > (8 << 20);            // more than a few MB
    if (unit <= kMaxSlab) {
        auto whole = [&](int width) {                     // a multiple of unit
            const int shift = threads_across(width);
            // Forward: four vectors a thread with up to 512 threads; eight with as few threads as that takes; or as many as fit.  us, threads: 64 x 196 x 1024 fp32 25.4 with 512, 26.3 with 256;
            // 128 x 784 x 128, 32 wide, 13.8 with 512, 14.6 with 1024, 14.9 with 256.
            auto fits = [&](const GroupThreads& t) {
                const int vectors = (int)ceil_div(pixels, t.threads >> shift);
                if (vectors > t.vectors || vectors > most_vectors) return false;
                p = GroupPlan{GroupSplit{width, (int)ceil_div(C, width), shift, 1, pixels}, t.threads, vectors};
                return true;
            };
            if (backward) {
                for (const GroupThreads& t : kGroupBackward)
                    if (fits(t)) return true;
            } else {
                for (const GroupThreads& t : kGroupForward)
                    if (fits(t)) return true;
            }
            return false;
        };
        auto units = [&](int width) { return width < unit ? unit : width / unit * unit; };
        // Two pixels a thread at least, with wider slabs; or enough work-groups for all compute units, with narrower ones, which read no more from memory as the slabs of an image are on one
        // XCD: two each in the forward of more than a few MB.  There 16 channels at least (backward: 64 bytes), and not fewer work-groups than compute units; with less than
        // that, fewer work-groups only where a work-group does not take longer than two launches.  us, width (threads):
        // 256 x 196 x 256 13.2 at 64 (256), 13.5 at 32 (256), 15.8 at 16 (256); 1000 x 16 x 256 11.0 at 64 (256), 6.4 at 256 (256); 128 x 784 x 128 15.3 at 64 (512), 13.8 at 32 (512), 14.2 at 16
        // (256); 64 x 3136 x 64 21.2 at 32 (1024), 17.5 at 16 (512), 22.0 at 8 (512), in pieces 22; 32 x 49 x 512 4.5 at 64 (256), 6.3 at 16 (256); 4 x 784 x 128 10.4 at 64 (512), 5.6 at 8 (512);
        // 2 x 1024 x 640 12.5 at 40 (512), in pieces 10.7; backward, sums of the channels included, 24.7 and 11.3; 4 x 784 x 128 18.0 at 64 (512), 12.0 at 32, in pieces 10.9, 9.1 at 8 (512);
        // 16 x 3136 x 256 30.3 at 16 (512), in pieces 28.9.
        // Backward of more than a few MB, where that makes two work-groups for each compute unit: the widest slab that 256 threads hold.  us, width (threads), without the sums of the channels:
        // 128 x 784 x 128 24.6 at 32 (256), 25.5 at 64 (512); 256 x 196 x 256 24.7 at 128 (256), 26.6 at 64 (256); 256 x 49 x 512 15.7 at 128 (256), 18.7 at 64 (256).
        if (backward && much)
            for (int wider : {256, 128, 64, 32}) {
                const int w = units(wider), vectors = (int)ceil_div(pixels, 256 >> threads_across(w));
                if (w > C || N * ceil_div(C, w) < 512 || vectors > most_vectors) continue;
                return GroupPlan{GroupSplit{w, (int)ceil_div(C, w), threads_across(w), 1, pixels}, 256, vectors};
            }
        const int64_t most = backward ? 20480 : 32768;    // values of a work-group
        const int least = !much ? 8 : backward && bf16 ? 32 : 16;
        int width = wide;
        while (2 * (256 >> threads_across(width)) > pixels && width < 256 && N * ceil_div(C, 2 * width) >= 256) width *= 2;
        while (width > least && N * ceil_div(C, width) < (much && !backward ? 512 : 256)) width /= 2;
        if (width > C) width = C / 8 * 8;
        for (; width >= 8; width /= 2) {
            const int w = units(width);
            if (much && w < least) break;
            if (N * ceil_div(C, w) < 256 && (much || (int64_t)pixels * w > most)) {
                if (much || w > width) break;
                continue;
            }
            if (whole(w)) return p;
            if (w > width) break;
        }
        p = GroupPlan{};
    }
    const int width = C < wide ? C : wide, shift = threads_across(width), slabs = (int)ceil_div(C, width), step = 256 >> shift;
    // Some 512 work-groups, four pixels or more a thread; not more partials than a work-group reads in a few steps.  us, 512 / 1024 of them, forward and backward: 64 x 3136 x 64
    // 22.7 / 26.9 (with 32 channels; now whole, 17.2), 29.8 / 40.1; 8 x 1024 x 640 15.5 / 18.1; but 16 x 3136 x 256 backward 29.1 / 28.9.
    int64_t pieces = ceil_div(512, N * slabs);
    const int64_t rows4 = ceil_div(pixels, 4 * step), read = 8192 / (width / cpg + 2);
    if (pieces > rows4) pieces = rows4;
    if (pieces > read) pieces = read;
    const int rows = (int)ceil_div(pixels, pieces);
    p.sp = GroupSplit{width, slabs, shift, (int)ceil_div(pixels, rows), rows};
    return p;
}

}  // namespace abt
