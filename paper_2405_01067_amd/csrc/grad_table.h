// The tensors of a launch of the clipping kernels as they travel in its arguments (plain C++, no device code).
#pragma once

#include <stdint.h>

namespace abt {

constexpr int kGradMaxTensors = 128;           // per launch
constexpr int kGradMaxBlocks = 1 << 23;        // of a launch, which has fewer than 2^32 threads
struct GradTensor { const void* grad; void* out; int64_t count; bool bf16; };   // count up to 2^40

struct GradTable {
    const void* grad[kGradMaxTensors];
    void* out[kGradMaxTensors];
    int64_t count[kGradMaxTensors];
    int first[kGradMaxTensors + 1];            // chunks [first[i], first[i + 1]) are those of tensor i
    uint64_t bf16[kGradMaxTensors / 64];       // types
    int n;
};
static_assert(sizeof(GradTable) <= 3840 && kGradMaxTensors % 64 == 0, "kernel arguments");

// One table after the other: the next tensors with elements in chunks of `chunk` elements, up to `limit` chunks.  A tensor of which no more fits goes on,
// at a chunk, in the table after it.
struct GradTables {
    const GradTensor* t;
    int n, at = 0;
    int64_t done = 0;                          // elements of tensor `at` that earlier tables have
    GradTables(const GradTensor* tensors, int count) : t(tensors), n(count) {}
    bool next(GradTable& a, int chunk, int limit, int& chunks) {
        a = GradTable{};
        chunks = 0;
        while (at < n && a.n < kGradMaxTensors) {
            const GradTensor& x = t[at];
            const int64_t left = x.count - done, room = (int64_t)(limit - chunks) * chunk, here = left < room ? left : room;
            if (left > 0 && here == 0) break;
            if (left > 0) {
                a.grad[a.n] = static_cast<const char*>(x.grad) + done * (x.bf16 ? 2 : 4);
                a.out[a.n] = x.out ? static_cast<char*>(x.out) + done * (x.bf16 ? 2 : 4) : nullptr;
                a.count[a.n] = here;
                a.first[a.n] = chunks;
                if (x.bf16) a.bf16[a.n >> 6] |= 1ull << (a.n & 63);
                chunks += (int)((here + chunk - 1) / chunk);
                ++a.n;
                done += here;
            }
            if (done == x.count) { ++at; done = 0; }
        }
        a.first[a.n] = chunks;
        return a.n > 0;
    }
};

}  // namespace abt
