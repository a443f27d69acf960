// Whether rows that a call writes share memory with one another or with rows that it reads: plain arithmetic on the host, no CUDA headers.
//
// A row's elements are next to one another; rows stand at data + i * outer_stride + j * inner_stride.  Differences of two rows' places of one
// kind are multiples of a stride, so all pairs of them are gone through by a division for each difference of the inner ones.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace lce {

struct RowSet {
    const void *data;
    int64_t outer, inner;                 // how many
    int64_t outer_stride, inner_stride;   // elements, not negative, below 2^40
    int64_t length;                       // of a row, in elements
    int64_t size;                         // of an element
};

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b != 0 && (a < 0) != (b < 0)); }

// Whether some d in [from, to] has -below < at + d * stride < above.
inline bool some_between(int64_t at, int64_t stride, int64_t from, int64_t to, int64_t below, int64_t above)
{
    if (from > to) return false;
    if (stride == 0 || (from == 0 && to == 0)) return -below < at && at < above;
    const int64_t lowest = floor_div(-below - at, stride) + 1, highest = -floor_div(at - above, stride) - 1;
    return std::max(lowest, from) <= std::min(highest, to);
}

// Rows of one set, apart from one another.
inline bool rows_apart(const RowSet &a)
{
    const int64_t length = a.length * a.size, outer_stride = a.outer_stride * a.size, inner_stride = a.inner_stride * a.size;
    if (a.outer <= 0 || a.inner <= 0 || a.length <= 0) return true;
    if ((a.inner == 1 || inner_stride >= length) && (a.outer == 1 || outer_stride >= (a.inner - 1) * inner_stride + length)) return true;
    if (a.outer > 1 && outer_stride < length) return false;
    for (int64_t j = 1; j < a.inner; ++j)
        if (some_between(j * inner_stride, outer_stride, -(a.outer - 1), a.outer - 1, length, length)) return false;
    return true;
}

// Whether a row of one set shares an element with a row of the other.  Sets of different strides have more kinds of differences; past 2^20 of them only
// the first rows are looked at: true is certain, false then is not.
inline bool rows_meet(RowSet a, RowSet b)
{
    if (a.outer <= 0 || a.inner <= 0 || a.length <= 0 || b.outer <= 0 || b.inner <= 0 || b.length <= 0) return false;
    for (RowSet *s : {&a, &b}) {  // the same row again and again is one
        if (s->outer_stride == 0) s->outer = 1;
        if (s->inner_stride == 0) s->inner = 1;
    }
    const auto end = [](const RowSet &s) {
        return (__int128)reinterpret_cast<uintptr_t>(s.data) + ((__int128)(s.outer - 1) * s.outer_stride + (s.inner - 1) * s.inner_stride + s.length) * s.size;
    };
    if (end(a) <= (__int128)reinterpret_cast<uintptr_t>(b.data) || end(b) <= (__int128)reinterpret_cast<uintptr_t>(a.data)) return false;
    if (a.outer > b.outer) std::swap(a, b);
    // the outer rows of a are gone through one by one unless they are as far apart as those of b
    const bool outer_alike = a.outer == 1 || a.outer_stride * a.size == b.outer_stride * b.size, inner_alike = a.inner == 1 || b.inner == 1 || a.inner_stride * a.size == b.inner_stride * b.size;
    const int64_t most = 1 << 20, inner_pairs = inner_alike ? a.inner + b.inner : a.inner > most / b.inner ? most : a.inner * b.inner;
    if (!outer_alike && a.outer > most / inner_pairs) a.outer = b.outer = 1;
    if (!inner_alike && inner_pairs == most) a.inner = b.inner = 1;
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(b.data) - reinterpret_cast<uintptr_t>(a.data)), a_length = a.length * a.size, b_length = b.length * b.size;
    const int64_t a_outer = a.outer_stride * a.size, b_outer = b.outer_stride * b.size, a_inner = a.inner_stride * a.size, b_inner = b.inner_stride * b.size;
    // all inner rows of one outer row as one long one: views side by side in the rows of one buffer are told apart by this
    if (outer_alike && !some_between(apart, b_outer, -(a.outer - 1), b.outer - 1, (b.inner - 1) * b_inner + b_length, (a.inner - 1) * a_inner + a_length)) return false;
    const auto meet = [&](int64_t at) {
        if (outer_alike) return some_between(at, b_outer, -(a.outer - 1), b.outer - 1, b_length, a_length);
        for (int64_t i = 0; i < a.outer; ++i)
            if (some_between(at - i * a_outer, b_outer, 0, b.outer - 1, b_length, a_length)) return true;
        return false;
    };
    if (inner_alike) {
        const int64_t stride = a.inner > 1 ? a_inner : b_inner;
        for (int64_t j = -(a.inner - 1); j < b.inner; ++j)
            if (meet(apart + j * stride)) return true;
        return false;
    }
    for (int64_t i = 0; i < a.inner; ++i)
        for (int64_t j = 0; j < b.inner; ++j)
            if (meet(apart + j * b_inner - i * a_inner)) return true;
    return false;
}

}  // namespace lce
