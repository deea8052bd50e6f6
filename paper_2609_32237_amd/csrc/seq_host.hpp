// seq_host.hpp -- argument checks shared by the sequence entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <numeric>
#include <utility>

#include "mi355seq.h"

namespace mi355seq {

constexpr int64_t kMaxSize = 0x7fffffff;
constexpr int64_t kMaxElements = int64_t(1) << 40;
constexpr int64_t kMaxThreads = 0xffffffff;  // of one launch

inline size_t element_bytes(int type) { return type == SEQ_FP32 ? 4 : 2; }
inline bool known_type(int type) { return type == SEQ_FP32 || type == SEQ_FP16 || type == SEQ_BF16; }
inline bool misaligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// (outer, inner) rows of `width` consecutive elements; strides in elements.
struct Rows {
    const void *p;
    int64_t so, si;
};

struct Grid {
    int64_t outer, inner, width;
    size_t bytes;  // of one element
};

inline bool strides_in_range(const Rows &a) {
    return a.so >= 0 && a.si >= 0 && a.so <= kMaxElements && a.si <= kMaxElements;
}

// Whether the rows of one output are apart from each other.
inline bool rows_apart(const Rows &a, const Grid &g) {
    int64_t n1 = g.inner, s1 = a.si, n2 = g.outer, s2 = a.so;  // axis 1: the smaller stride
    if (n1 <= 1 || (n2 > 1 && s2 < s1)) {
        std::swap(n1, n2);
        std::swap(s1, s2);
    }
    if (n1 > 1 && s1 < g.width) return false;
    const __int128 block = n1 > 1 ? (__int128)(n1 - 1) * s1 + g.width : g.width;
    return n2 <= 1 || s2 >= block;
}

inline bool same_rows(const Rows &a, const Rows &b, const Grid &g) {
    return a.p == b.p && (g.outer <= 1 || a.so == b.so) && (g.inner <= 1 || a.si == b.si);
}

// Whether two sets of rows can have an element in common: extents that meet,
// unless every row of both starts on the same grid of s elements and the rows
// sit side by side on it (slices of one wider buffer).
inline bool may_share(const Rows &a, const Rows &b, const Grid &g) {
    if (!a.p || !b.p || g.outer < 1 || g.inner < 1) return false;
    auto extent = [&](const Rows &r) {
        return (__int128)((g.outer - 1)) * r.so + (__int128)((g.inner - 1)) * r.si + g.width;
    };
    const __int128 pa = (__int128)(uintptr_t)a.p, pb = (__int128)(uintptr_t)b.p;
    if (pa + extent(a) * (__int128)g.bytes <= pb || pb + extent(b) * (__int128)g.bytes <= pa) return false;
    int64_t s = 0;
    for (const Rows *r : {&a, &b}) {
        if (g.outer > 1) s = std::gcd(s, r->so);
        if (g.inner > 1) s = std::gcd(s, r->si);
    }
    if (s == 0) return true;
    const __int128 diff = pb - pa;
    if (diff % (__int128)g.bytes != 0) return true;
    int64_t off = (int64_t)((diff / (__int128)g.bytes) % s);
    if (off < 0) off += s;
    return !(off >= g.width && s - off >= g.width);
}

// Plain byte ranges.
inline bool ranges_share(const void *a, size_t na, const void *b, size_t nb) {
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    return pa < pb ? pb - pa < na : pa - pb < nb;
}

// The status of the launch just made, read from the launch call itself.
inline int launch(const void *kernel, dim3 grid, dim3 block, void **args, size_t lds, hipStream_t stream) {
    return hipLaunchKernel(kernel, grid, block, args, lds, stream) == hipSuccess ? SEQ_OK : SEQ_EHIP;
}

}  // namespace mi355seq
