// What the C entries share: alignment, overlap, status codes.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include "dispatch.hpp"

namespace triinv {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return a && b && na && nb && a0 < b0 + nb && b0 < a0 + na;
}
inline int finish(int rc) { return rc == LAUNCHED ? TRIINV_OK : rc == NOT_BUILT ? TRIINV_ERR_UNSUPPORTED : TRIINV_ERR_LAUNCH; }
inline bool any_dtype(int d) { return d == TRIINV_F32 || d == TRIINV_F16 || d == TRIINV_BF16; }

struct Span {
    const void* p;
    uint64_t bytes;
};
// Whether a result overlaps one of the inputs or another result.
template <size_t NI, size_t NO> bool aliased(const Span (&in)[NI], const Span (&out)[NO])
{
    for (size_t i = 0; i < NO; ++i) {
        for (const Span& x : in)
            if (overlap(x.p, x.bytes, out[i].p, out[i].bytes)) return true;
        for (size_t j = 0; j < i; ++j)
            if (overlap(out[j].p, out[j].bytes, out[i].p, out[i].bytes)) return true;
    }
    return false;
}

// Rows of `width` bytes, `stride` bytes from one to the next, as a projection's columns are.
struct Rows {
    const void* p;
    int64_t n;
    uint64_t width, stride;
    uint64_t bytes() const { return p && n > 0 && width ? (uint64_t)(n - 1) * stride + width : 0; }
};
// Whether two of them share a byte.  Those of one stride may lie beside each other in the same rows; of two strides it is the ranges that count.
inline bool overlap(const Rows& a, const Rows& b)
{
    if (!overlap(a.p, a.bytes(), b.p, b.bytes())) return false;
    if (a.n <= 1 && b.n <= 1) return true;
    const uint64_t s = a.n > 1 ? a.stride : b.stride;
    if ((a.n > 1 && b.n > 1 && a.stride != b.stride) || a.width > s || b.width > s) return true;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    const uint64_t at = b0 >= a0 ? (b0 - a0) % s : (s - (a0 - b0) % s) % s;  // where b begins in a's row
    return at < a.width || at + b.width > s;
}

}  // namespace triinv
