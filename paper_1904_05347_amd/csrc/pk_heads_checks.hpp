// pk_heads_checks.hpp -- argument checks of the attention operators: where strided
// tensors lie and whether two of them share memory.  Plain integer arithmetic,
// which the CPU tests evaluate too.
#pragma once

#include <stdint.h>

#include "../../include/pk.h"

namespace pk::heads {

constexpr int64_t kMostSize = (int64_t)1 << 30;
constexpr int64_t kMostHeads = 1 << 16;
constexpr int64_t kMostCacheStride = (int64_t)1 << 40;

// Bytes that a tensor takes: runs of `run` bytes from `at`, repeated along up to
// three dimensions, their strides (bytes) descending.
struct Region {
    uintptr_t at = 0;
    int dims = 0;
    int64_t n[3] = {}, stride[3] = {};
    int64_t run = 0;
    bool empty = false;

    void add(int64_t count, int64_t step)
    {
        if (count <= 0) empty = true;
        if (count <= 1) return;
        int i = dims++;
        for (; i > 0 && stride[i - 1] < step; --i) {
            n[i] = n[i - 1];
            stride[i] = stride[i - 1];
        }
        n[i] = count;
        stride[i] = step;
    }
    // bytes from the first to the last of what dimensions `from` and inner ones span
    __int128 extent(int from) const
    {
        __int128 e = run;
        for (int i = from; i < dims; ++i) e += (__int128)(n[i] - 1) * stride[i];
        return e;
    }
    // no two of its runs share a byte (sufficient: each dimension steps over the inner ones)
    bool distinct() const
    {
        for (int i = 0; i < dims; ++i)
            if ((__int128)stride[i] < extent(i + 1)) return false;
        return true;
    }
};

// Whether b, `shift` bytes after a, may share bytes with it, from dimension `from` on.
// Where both step equally far, the inner parts are compared at the two shifts that
// bring neighbouring steps nearest; else all that lies between counts.
inline bool shared_from(const Region &a, const Region &b, int from, __int128 shift)
{
    if (shift >= a.extent(from) || -shift >= b.extent(from)) return false;
    if (from >= a.dims && from >= b.dims) return true;
    if (from >= a.dims || from >= b.dims || a.stride[from] != b.stride[from] || a.stride[from] <= 0) return true;
    const int64_t step = a.stride[from];
    if (a.extent(from + 1) > step || b.extent(from + 1) > step) return true;
    __int128 r = shift % step;
    if (r < 0) r += step;
    return shared_from(a, b, from + 1, r) || shared_from(a, b, from + 1, r - step);
}

inline bool shared(const Region &a, const Region &b)
{
    if (a.empty || b.empty || !a.run || !b.run) return false;
    return shared_from(a, b, 0, (__int128)b.at - (__int128)a.at);
}

inline Region flat(const void *p, int64_t bytes)
{
    Region r;
    r.at = (uintptr_t)p;
    r.run = bytes;
    r.empty = bytes <= 0;
    return r;
}

inline Region matrix(const void *p, int64_t rows, int64_t step_bytes, int64_t run_bytes)
{
    Region r = flat(p, run_bytes);
    r.add(rows, step_bytes);
    return r;
}

inline Region of_heads(const pk_heads &t, int64_t M, int64_t d, int size)
{
    Region r = flat(t.data, d * size);
    r.add(M, t.token_stride * size);
    r.add(t.heads, t.head_stride * size);
    return r;
}

inline Region of_cache(const void *p, const int64_t stride[3], const pk_cache &c, int64_t d, int size)
{
    Region r = flat(p, d * size);
    r.add(c.pages, stride[0] * size);
    r.add(c.page_size, stride[1] * size);
    r.add(c.heads, stride[2] * size);
    return r;
}

inline bool same_place(const pk_heads &a, const pk_heads &b, int64_t M)
{
    return a.data == b.data && (M <= 1 || a.token_stride == b.token_stride) &&
           (a.heads <= 1 || a.head_stride == b.head_stride);
}

// PK_OK, PK_ERR_INVALID_VALUE or PK_ERR_NOT_SUPPORTED for one tensor of heads;
// its memory is looked at only where it has elements.
inline int check_heads(const pk_heads &t, int64_t M, int size, bool output, int64_t d)
{
    if (t.heads < 0 || t.token_stride < 0 || t.head_stride < 0) return PK_ERR_INVALID_VALUE;
    if (t.heads > kMostHeads || t.token_stride > kMostSize || t.head_stride > kMostSize) return PK_ERR_NOT_SUPPORTED;
    if (M == 0 || t.heads == 0) return PK_OK;
    if (!t.data || (uintptr_t)t.data % (uintptr_t)size) return PK_ERR_INVALID_VALUE;
    if (output && !of_heads(t, M, d, size).distinct()) return PK_ERR_INVALID_VALUE;
    return PK_OK;
}

inline int check_cache(const pk_cache &c, int size, bool output, int64_t d)
{
    if (c.pages < 0 || c.page_size < 1 || c.heads < 0) return PK_ERR_INVALID_VALUE;
    for (int i = 0; i < 3; ++i)
        if (c.key_stride[i] < 0 || c.value_stride[i] < 0) return PK_ERR_INVALID_VALUE;
    if (c.pages > kMostSize || c.page_size > kMostSize || c.heads > kMostHeads) return PK_ERR_NOT_SUPPORTED;
    for (int i = 0; i < 3; ++i)
        if (c.key_stride[i] > kMostCacheStride || c.value_stride[i] > kMostCacheStride) return PK_ERR_NOT_SUPPORTED;
    if (c.pages == 0 || c.heads == 0) return PK_OK;
    if (!c.key || !c.value || (uintptr_t)c.key % (uintptr_t)size || (uintptr_t)c.value % (uintptr_t)size)
        return PK_ERR_INVALID_VALUE;
    const Region k = of_cache(c.key, c.key_stride, c, d, size), v = of_cache(c.value, c.value_stride, c, d, size);
    // positions in memory are 64-bit
    if (k.extent(0) > ((__int128)1 << 62) || v.extent(0) > ((__int128)1 << 62)) return PK_ERR_NOT_SUPPORTED;
    if (output && (!k.distinct() || !v.distinct() || shared(k, v))) return PK_ERR_INVALID_VALUE;
    return PK_OK;
}

}  // namespace pk::heads
