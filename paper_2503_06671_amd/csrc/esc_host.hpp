// Host-side helpers of the C ABI's translation units.
#pragma once
#include <hip/hip_runtime.h>
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

// Planes of N images, `stride` bytes from image to image.
struct Images {
    const void *at;
    size_t stride, bytes;  // bytes: one image's
    int N;
    size_t extent() const { return (size_t)(N - 1) * stride + bytes; }
};

inline bool meet(const Images &a, const Images &b)
{
    if (!overlaps(a.at, a.extent(), b.at, b.extent())) return false;
    if (a.stride != b.stride || a.N == 1 || b.N == 1) return true;
    // the same step from image to image: parts of one tensor may lie between each other
    const uintptr_t ua = (uintptr_t)a.at, ub = (uintptr_t)b.at;
    const size_t s = a.stride, from = ub >= ua ? (ub - ua) % s : (s - (ua - ub) % s) % s;
    return from < a.bytes || from + b.bytes > s;
}
// The images of a caller's tensor of `elements` an image; false where they do not lie as they have to.
inline bool images_of(const void *at, long stride, int N, size_t elements, size_t es, Images *out)
{
    if ((uintptr_t)at % es != 0) return false;
    if (N > 1 && (stride < 0 || (size_t)stride < elements || (size_t)stride > ((size_t)1 << 46))) return false;
    *out = Images{at, (N > 1 ? (size_t)stride : elements) * es, elements * es, N};
    return true;
}
inline bool meets(const Images &a, const void *b, size_t bytes) { return b != nullptr && overlaps(a.at, a.extent(), b, bytes); }

// `blocks` blocks of `threads` by launch(first block, number): in one launch, or in several where it would have 2^32 threads or more, which HIP
// refuses.
template <typename F>
hipError_t in_launches(long blocks, int threads, F launch)
{
    const long most = 0xffffffffL / threads;
    for (long first = 0; first < blocks; first += most) {
        const hipError_t e = launch(first, (unsigned)(blocks - first < most ? blocks - first : most));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace esc
