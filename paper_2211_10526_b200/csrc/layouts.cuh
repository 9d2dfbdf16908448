// Whether strided tensors that a call writes share elements.  Host arithmetic only.
#pragma once

#include <cstdint>

namespace castling {

struct Axis { long long size, stride; };   // a size of one: the stride does not count
struct Placed { uintptr_t at; Axis axis[3]; long long width; };   // rows of `width` elements

// The axes from the longest stride to the shortest.
inline void by_stride(Axis (&a)[3]) {
    for (Axis& x : a) if (x.size == 1) x.stride = 0;
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (a[j].stride < a[j + 1].stride) { const Axis t = a[j]; a[j] = a[j + 1]; a[j + 1] = t; }
}

// Each stride passes over all that the shorter ones reach: no element has two indexes.
inline bool nested(Placed t) {
    by_stride(t.axis);
    long long reach = t.width;
    for (int i = 2; i >= 0; --i) {
        if (t.axis[i].size == 1) continue;
        if (t.axis[i].stride < reach) return false;
        reach += (t.axis[i].size - 1) * t.axis[i].stride;
    }
    return true;
}

// Elements from the first to the last, both counted.
inline long long reach(const Placed& t) {
    long long n = t.width;
    for (const Axis& x : t.axis) if (x.size > 1) n += (x.size - 1) * x.stride;
    return n;
}

// Of two nested tensors: does an element of b lie in a?  Exact where an axis has one stride in both and the longer of each nest too (slices of one fused
// tensor); of others it says yes where what they reach overlaps.
// b's elements are `delta` behind a's: delta = sum of (index in a - index in b) * stride, whose shorter terms together stay below each stride, so that
// a difference of indexes is one of two.
inline bool share_elements(const Placed& a, const Placed& b, long long element_bytes) {
    const uintptr_t a_end = a.at + (uintptr_t)(reach(a) * element_bytes), b_end = b.at + (uintptr_t)(reach(b) * element_bytes);
    if (a_end <= b.at || b_end <= a.at) return false;
    struct Pair { long long na, nb, stride; } axis[3];
    for (int i = 0; i < 3; ++i) {
        const Axis &x = a.axis[i], &y = b.axis[i];
        if (x.size > 1 && y.size > 1 && x.stride != y.stride) return true;
        axis[i] = {x.size, y.size, x.size > 1 ? x.stride : y.size > 1 ? y.stride : 0};
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (axis[j].stride < axis[j + 1].stride) { const Pair t = axis[j]; axis[j] = axis[j + 1]; axis[j + 1] = t; }
    auto longer = [](long long x, long long y) { return x > y ? x : y; };
    if (!nested({0, {{longer(axis[0].na, axis[0].nb), axis[0].stride}, {longer(axis[1].na, axis[1].nb), axis[1].stride}, {longer(axis[2].na, axis[2].nb), axis[2].stride}}, longer(a.width, b.width)}))
        return true;
    struct Search {
        const Pair* axis;
        long long wa, wb;
        bool at(int i, long long delta) const {
            if (i == 3) return delta < wa && -delta < wb;
            const Pair& x = axis[i];
            if (!x.stride) return at(i + 1, delta);
            long long j = delta / x.stride;
            if (delta % x.stride < 0) --j;
            for (int more = 0; more < 2; ++more, ++j)
                if (j < x.na && -j < x.nb && at(i + 1, delta - j * x.stride)) return true;
            return false;
        }
    };
    const long long bytes = (long long)b.at - (long long)a.at;
    return Search{axis, a.width, b.width}.at(0, bytes / element_bytes);
}

}  // namespace castling
