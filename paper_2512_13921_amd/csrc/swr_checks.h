// swr_checks.h -- what the C ABI's validation shares: extents and overlaps of
// strided tensors, alignment, element sizes.  Host code; nothing is dereferenced.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/swr_hybrid.h"

namespace {

constexpr int64_t kMaxExtent = (int64_t)1 << 60;
constexpr int64_t kMaxRows = 0x7fffffffLL;
constexpr int64_t kMaxWidth = (int64_t)1 << 30;
constexpr int64_t kMaxPage = 65536;

struct Dim {
    int64_t size, stride;
};

// Largest offset of a strided tensor of these dimensions (all sizes at least
// 1), or -1 for a negative stride or one whose offsets are out of range.
int64_t max_offset(std::initializer_list<Dim> dims) {
    int64_t off = 0;
    for (const Dim& d : dims) {
        if (d.stride < 0) return -1;
        if (d.size <= 1 || d.stride == 0) continue;
        if (d.size - 1 > kMaxExtent / d.stride) return -1;
        off += (d.size - 1) * d.stride;
        if (off > kMaxExtent) return -1;
    }
    return off;
}

// Dimensions (up to four) of more than one element, of the least stride first.
struct Sorted {
    Dim d[4];
    int n = 0;
    explicit Sorted(std::initializer_list<Dim> dims) {
        for (const Dim& x : dims)
            if (x.size > 1) d[n++] = x;
        for (int i = 1; i < n; ++i)
            for (int j = i; j > 0 && d[j].stride < d[j - 1].stride; --j) {
                const Dim t = d[j];
                d[j] = d[j - 1];
                d[j - 1] = t;
            }
    }
};

// Whether different indices never name the same element.
bool apart(std::initializer_list<Dim> dims) {
    const Sorted s(dims);
    int64_t need = 1;
    for (int i = 0; i < s.n; ++i) {
        if (s.d[i].stride < need) return false;
        if (s.d[i].size > kMaxExtent / s.d[i].stride) return false;
        need = s.d[i].stride * s.d[i].size;
    }
    return true;
}

// Whether two tensors of these dimensions, apart, share an element when they begin
// `distance` elements from each other.  The lesser dimensions reach less far than a
// dimension's stride, so only its two differences of indices next to the distance count.
bool meet_at(const Sorted& s, int dims, int64_t distance) {
    if (dims == 0) return distance == 0;
    const Dim& d = s.d[dims - 1];
    const int64_t below = distance / d.stride - (distance % d.stride < 0);
    for (int64_t i = below; i <= below + 1; ++i)
        if (i > -d.size && i < d.size && meet_at(s, dims - 1, distance - i * d.stride)) return true;
    return false;
}

struct Span {
    uintptr_t lo, hi;
};
Span span(const void* p, int64_t bytes) { return {(uintptr_t)p, (uintptr_t)p + (uintptr_t)(p ? bytes : 0)}; }
bool overlap(const Span& a, const Span& b) { return a.lo < b.hi && b.lo < a.hi; }
bool overlaps(const Span& out, std::initializer_list<Span> others) {
    for (const Span& s : others)
        if (overlap(out, s)) return true;
    return false;
}

bool aligned(const void* p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }
int size_of(int dtype) { return dtype == SWR_DTYPE_F32 ? 4 : dtype == SWR_DTYPE_BF16 ? 2 : 1; }
// Whether these strides are whole numbers of 16 bytes.
bool vectors(std::initializer_list<Dim> dims, int es) {
    for (const Dim& d : dims)
        if (d.size > 1 && d.stride % (16 / es) != 0) return false;
    return true;
}
bool plain(int dtype) { return dtype == SWR_DTYPE_F32 || dtype == SWR_DTYPE_BF16; }
int status(hipError_t e) { return e == hipSuccess ? SWR_OK : SWR_ERR_HIP; }

}  // namespace
