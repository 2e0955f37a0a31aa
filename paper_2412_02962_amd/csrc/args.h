// Argument checks shared by the feed-forward sub-layer's entry points.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace pcpp {

// One array of a call: its address (may be null: not used) and size.
struct Range {
    const void* p;
    int64_t bytes;
};

inline bool aligned_to(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

inline bool ranges_overlap(const Range& a, const Range& b) {
    if (!a.p || !b.p) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

// Whether any of the n_out arrays written overlaps another of them or one of
// the n_in arrays read.
inline bool outputs_overlap(const Range* out, int n_out, const Range* in, int n_in) {
    for (int i = 0; i < n_out; ++i) {
        for (int j = i + 1; j < n_out; ++j)
            if (ranges_overlap(out[i], out[j])) return true;
        for (int j = 0; j < n_in; ++j)
            if (ranges_overlap(out[i], in[j])) return true;
    }
    return false;
}

}  // namespace pcpp
