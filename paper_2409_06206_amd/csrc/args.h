// What the entry points check about their buffers before anything is enqueued.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace gswa {

// A device buffer as a byte range, for the overlap rules of the entry points.
struct Range {
    uintptr_t lo, hi;
    Range(const void *p, size_t bytes) : lo(reinterpret_cast<uintptr_t>(p)), hi(lo + (p ? bytes : 0)) {}
};
inline bool overlap(const Range &a, const Range &b) { return a.lo < b.hi && b.lo < a.hi; }
// true when `out` shares a byte with any of the others
template <typename... R> bool overlaps_any(const Range &out, const R &...others) { return (overlap(out, others) || ...); }

// true when every pointer (null ones too) is a multiple of `bytes`, a power of two
template <typename... P> bool aligned_to(uintptr_t bytes, const P *...p)
{
    return (((reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0) && ...);
}

inline size_t to_256(size_t n) { return (n + 255) & ~size_t(255); }

} // namespace gswa
