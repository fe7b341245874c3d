// What the files that validate calls share (api.hip, adapters_api.hip).
#pragma once

#include <new>

#include "common.h"

namespace abt {

// The entry points promise not to throw: what the host-side tables of a call may throw (allocation
// failure of a std::vector) becomes a status.
template <class F>
int guarded(F&& f) {
    try { return f(); }
    catch (const std::bad_alloc&) { return ABT_ENOMEM; }
    catch (...) { return ABT_EHIP; }
}
template <class F>
size_t guarded_size(F&& f) {
    try { return f(); }
    catch (...) { return 0; }
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

}  // namespace abt
