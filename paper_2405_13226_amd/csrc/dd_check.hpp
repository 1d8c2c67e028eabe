// dd_check.hpp -- address ranges and alignment, as the C ABI's entry points
// check them before a launch (host code only).
#pragma once

#include <cstddef>
#include <cstdint>

namespace dd {
namespace check {

struct Range {
    uintptr_t lo, hi;  // [lo, hi)
};

inline Range range_of(const void *p, size_t bytes)
{
    uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return Range{a, a + bytes};
}

inline bool overlaps(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi; }

inline bool aligned(const void *p, uintptr_t n)
{
    return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0;
}

// Bytes of `rows` rows of `cols` elements at a row stride of `ld` elements.
inline size_t matrix_bytes(long long rows, long long cols, long long ld, int element)
{
    return static_cast<size_t>((rows - 1) * ld + cols) * element;
}

}  // namespace check
}  // namespace dd
