// Host-side helpers of the C ABI's translation units.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace esc {
namespace {

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// do the byte ranges [a, a + na) and [b, b + nb) share a byte?
inline bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t ua = (uintptr_t)a, ub = (uintptr_t)b;
    return na > 0 && nb > 0 && ua < ub + nb && ub < ua + na;
}

}  // namespace
}  // namespace esc
