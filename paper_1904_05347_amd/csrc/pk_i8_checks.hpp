// pk_i8_checks.hpp -- argument checks shared by the entry points of the 8-bit
// operators.
#pragma once

#include <stdint.h>

#include <initializer_list>

#include "pk_api_state.hpp"

namespace pk::checks {

struct Span {
    uintptr_t lo, hi;
};

// Bytes of a row-major M x N matrix of `size`-byte elements (M, N >= 1).
inline Span span(const void *p, int64_t M, int64_t N, int64_t ld, int size)
{
    return {(uintptr_t)p, (uintptr_t)p + (size_t)(((M - 1) * ld + N) * size)};
}

inline bool overlap(const Span &a, const Span &b) { return a.lo < b.hi && b.lo < a.hi; }

inline bool misaligned(const void *p, int size) { return (uintptr_t)p % (uintptr_t)size != 0; }

inline bool short_ld(int64_t ld, int64_t N) { return ld < (N > 1 ? N : 1); }

// Indexes along a row are 32-bit in the kernels, and no product of two of these
// and an element's size passes 63 bits.
inline bool too_large(std::initializer_list<int64_t> dims)
{
    for (const int64_t d : dims)
        if (d > (int64_t)1 << 30) return true;
    return false;
}

}  // namespace pk::checks
