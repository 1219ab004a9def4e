// Argument checks shared by the C entry points (not installed).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace flarepp {

inline bool aligned16(const void* ptr) { return ((uintptr_t)ptr & 15u) == 0; }
inline bool aligned4(const void* ptr) { return ((uintptr_t)ptr & 3u) == 0; }

inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + nb && b0 < a0 + na;
}

// A buffer of a call: what it writes must not overlap anything else of the call.
struct Span {
    const void* p;
    size_t bytes;
};
inline bool disjoint(const Span* outs, int n_outs, const Span* ins, int n_ins) {
    for (int i = 0; i < n_outs; ++i) {
        for (int j = 0; j < n_ins; ++j)
            if (overlaps(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return false;
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return false;
    }
    return true;
}

}  // namespace flarepp
