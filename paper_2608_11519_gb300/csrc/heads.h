// Checks of tensors [B, H, N, D] that are given by strides (flarepp_heads), shared by the entry points
// that take them (not installed).
#pragma once
#include "checks.h"
#include "flarepp_internal.h"

namespace flarepp {

struct HeadDims {
    int64_t B, H, N, D;
    int64_t bytes;  // of a value
};

inline bool empty(const HeadDims& d) { return d.B == 0 || d.H == 0 || d.N == 0 || d.D == 0; }

// Strides that a kernel can follow: none negative, and no offset beyond 2^47 values.
inline bool strides_ok(const flarepp_heads& t, const HeadDims& d) {
    const int64_t most = int64_t(1) << 47;
    const int64_t n[3] = {d.B, d.H, d.N}, s[3] = {t.stride_b, t.stride_h, t.stride_n};
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || (n[i] > 1 && s[i] > most / n[i])) return false;
    return true;
}

// Values from the first to one past the last.
inline int64_t extent(const flarepp_heads& t, const HeadDims& d) {
    if (empty(d)) return 0;
    return (d.B - 1) * t.stride_b + (d.H - 1) * t.stride_h + (d.N - 1) * t.stride_n + d.D;
}
inline Span span_of(const flarepp_heads& t, const HeadDims& d) {
    return {t.data, (size_t)(extent(t, d) * d.bytes)};
}

// No value of a tensor that is written may be another one of it: along the dimensions by stride, each
// step passes what lies within.
inline bool apart_within(const flarepp_heads& t, const HeadDims& d) {
    int64_t n[3] = {d.B, d.H, d.N}, s[3] = {t.stride_b, t.stride_h, t.stride_n};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (s[j] > s[j + 1]) {
                const int64_t a = s[j], b = n[j];
                s[j] = s[j + 1], n[j] = n[j + 1];
                s[j + 1] = a, n[j + 1] = b;
            }
    int64_t inner = d.D;
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) continue;
        if (s[i] < inner) return false;
        inner += (n[i] - 1) * s[i];
    }
    return true;
}

// Whether no value of a is one of b: their ranges lie apart, or the rows of one lie between the rows of
// the other (the parts of one buffer [B, N, parts, H, D], or [B, parts, H, N, D]).
inline bool apart(const flarepp_heads& a, const HeadDims& da, const flarepp_heads& b, const HeadDims& db) {
    const Span x = span_of(a, da), y = span_of(b, db);
    if (!overlaps(x.p, x.bytes, y.p, y.bytes)) return true;
    if (da.bytes != db.bytes || a.stride_b != b.stride_b) return false;
    const int64_t gap = (int64_t)((uintptr_t)b.data - (uintptr_t)a.data);
    if (gap % da.bytes != 0) return false;
    // The pattern that repeats: a row of all heads if the rows' strides agree, else a batch element.
    const bool rows = a.stride_n == b.stride_n && a.stride_n > 0 &&
                      (da.B == 1 || a.stride_b % a.stride_n == 0);
    const int64_t period = rows ? a.stride_n : a.stride_b;
    if (period <= 0) return false;
    HeadDims wa = da, wb = db;
    wa.B = wb.B = 1;
    if (rows) wa.N = wb.N = 1;
    int64_t at = gap / da.bytes % period;
    if (at < 0) at += period;
    return at >= extent(a, wa) && at + extent(b, wb) <= period;
}

}  // namespace flarepp
