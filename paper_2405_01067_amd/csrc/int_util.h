// Division and alignment that round up (plain C++, no device code).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace abt {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace abt
