// Sizes rounded and divided upwards.
#pragma once
#include <cstddef>

namespace acc {

inline size_t al256(size_t b) { return (b + 255) & ~(size_t)255; }
inline long up(long v, long m) { return (v + m - 1) / m * m; }
inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

}  // namespace acc
