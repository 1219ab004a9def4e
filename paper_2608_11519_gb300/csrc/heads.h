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

// Dimensions of a tensor that has more than one place along them, and of a place's values (an innermost stride of 1).
struct Strided {
    int64_t n[4], s[4];
    int dims = 0;
    void add(int64_t count, int64_t stride) {
        if (count > 1) n[dims] = count, s[dims++] = stride;
    }
    // values from the first to one past the last, of the strides below `limit`
    int64_t extent_below(int64_t limit) const {
        int64_t e = 1;
        for (int i = 0; i < dims; ++i)
            if (s[i] < limit) e += (n[i] - 1) * s[i];
        return e;
    }
    bool others_are_multiples(int64_t of) const {
        for (int i = 0; i < dims; ++i)
            if (s[i] >= of && s[i] % of) return false;
        return true;
    }
};
inline Strided strided(const flarepp_heads& t, const HeadDims& d, bool batch) {
    Strided r;
    if (batch) r.add(d.B, t.stride_b);
    r.add(d.H, t.stride_h);
    r.add(d.N, t.stride_n);
    r.add(d.D, 1);
    return r;
}

// Whether b, which begins `gap` values behind a, has none of its values, by a stride of either as a period: if every
// stride is a multiple of it or below it, a value's place within the period tells what the strides below it make of
// it, and those of a and b lie apart there. (A stride of heads: [B, N, H, parts, D]; of rows: [B, N, parts, H, D]; of
// batch elements: [B, parts, H, N, D]; and so on.)
inline bool apart_by_period(const Strided& a, const Strided& b, int64_t gap) {
    for (const Strided* t : {&a, &b})
        for (int i = 0; i < t->dims; ++i) {
            const int64_t period = t->s[i];
            if (period < 1 || !a.others_are_multiples(period) || !b.others_are_multiples(period)) continue;
            const int64_t at = (gap % period + period) % period;
            if (at >= a.extent_below(period) && at + b.extent_below(period) <= period) return true;
        }
    return false;
}

// Whether no value of a is one of b, as far as their strides show: their ranges lie apart, or they are apart by a
// period, or they have the same batch stride, in which an element of both lies, and an element's parts are apart
// (rows of a padded batch, whose stride no row's divides). Strides of dimensions of size 1 do not matter.
inline bool apart(const flarepp_heads& a, const HeadDims& da, const flarepp_heads& b, const HeadDims& db) {
    const Span x = span_of(a, da), y = span_of(b, db);
    if (!overlaps(x.p, x.bytes, y.p, y.bytes)) return true;
    if (da.bytes != db.bytes) return false;
    const int64_t bytes = (int64_t)((uintptr_t)b.data - (uintptr_t)a.data);
    if (bytes % da.bytes != 0) return false;
    const int64_t gap = bytes / da.bytes;
    if (apart_by_period(strided(a, da, true), strided(b, db, true), gap)) return true;
    if (da.B <= 1 || db.B <= 1 || a.stride_b != b.stride_b || a.stride_b < 1) return false;
    const Strided one = strided(a, da, false), other = strided(b, db, false);
    const int64_t size = a.stride_b, ea = one.extent_below(INT64_MAX), eb = other.extent_below(INT64_MAX);
    int64_t at = (gap % size + size) % size;
    for (int k = 0; k < 2; ++k, at -= size) {  // b's element in front of a's, or behind it
        const int64_t from = at < 0 ? at : 0, to = at + eb > ea ? at + eb : ea;
        if (to - from > size) continue;
        if (at >= ea || at + eb <= 0 || apart_by_period(one, other, at)) return true;
    }
    return false;
}

}  // namespace flarepp
