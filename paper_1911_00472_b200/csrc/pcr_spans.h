// Memory of strided operands: whether two of them have a byte in common.  Host only.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <initializer_list>
#include <utility>

namespace pcr {

// Rows of `bytes` bytes from `at` on, `n[i]` of them `step[i]` bytes apart on each of three axes; all of them lie in from .. to
// (to = from: there are none).
struct Span {
    uintptr_t at;
    int64_t bytes, n[3];
    __int128 step[3], from, to;
    bool behind(const Span& s) const { return from >= s.to; }
};
inline Span span_of(const void* p, size_t bytes) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return {at, (int64_t)bytes, {1, 1, 1}, {0, 0, 0}, (__int128)at, (__int128)at + bytes};
}
inline Span span_of(const void* p, const int64_t (&stride)[3], int64_t n0, int64_t n1, int64_t n2, int64_t row, size_t es) {
    Span s = span_of(p, row * es);
    const int64_t n[3] = {n0, n1, n2};
    for (int i = 0; i < 3; ++i) {
        if (n[i] < 1) { s.to = s.from = 0; return s; }
        s.n[i] = n[i]; s.step[i] = (__int128)stride[i] * (int64_t)es;
        (s.step[i] < 0 ? s.from : s.to) += s.step[i] * (n[i] - 1);
    }
    return s;
}

// Whether sum of c[i] z[i] lies in lo .. hi for some 0 <= z[i] < n[i], i >= k.  `reach`: the largest sum of the terms from each
// on.  Steps that contain one another, as those of one buffer's slices do, leave one or two z[i] each; `left` bounds the rest.
inline bool sum_within(const __int128* c, const __int128* n, const __int128* reach, int k, int terms, __int128 lo, __int128 hi, int& left) {
    if (hi < 0 || lo > reach[k] || left <= 0) return left <= 0;
    if (lo <= 0 || hi >= reach[k]) return true;                   // (none of the terms, or all of them whole)
    if (k == terms) return false;
    const __int128 least = lo - reach[k + 1], first = least <= 0 ? 0 : (least + c[k] - 1) / c[k], last = hi / c[k];
    for (__int128 z = first; z <= last && z < n[k]; ++z) {
        --left;
        if (sum_within(c, n, reach, k + 1, terms, lo - c[k] * z, hi - c[k] * z, left)) return true;
    }
    return false;
}

// Whether two spans have a byte in common.  (Spans so entangled that some ten thousand steps do not tell count as if they had.)
inline bool share_memory(const Span& a, const Span& b) {
    if (a.behind(b) || b.behind(a) || a.from == a.to || b.from == b.to) return false;         // (as a rule)
    __int128 c[6], n[6], reach[7];
    int terms = 0;
    for (const Span* s : {&a, &b})
        for (int i = 0; i < 3; ++i)
            if (s->n[i] > 1 && s->step[i] != 0) { c[terms] = s->step[i] < 0 ? -s->step[i] : s->step[i]; n[terms++] = s->n[i]; }
    // A row of a begins at a.from + u, one of b at b.to - b.bytes - v, u and v sums of steps: they meet where u + v lies between
    const __int128 lo = b.to - b.bytes - a.from - a.bytes + 1, hi = b.to - a.from - 1;
    for (int i = 0; i < terms; ++i)                                   // equal steps are one, the largest come first
        for (int j = i + 1; j < terms;) {
            if (c[j] == c[i]) { n[i] += n[j] - 1; --terms; c[j] = c[terms]; n[j] = n[terms]; continue; }
            if (c[j] > c[i]) { std::swap(c[i], c[j]); std::swap(n[i], n[j]); }
            ++j;
        }
    reach[terms] = 0;
    for (int i = terms - 1; i >= 0; --i) reach[i] = reach[i + 1] + c[i] * (n[i] - 1);
    int left = 20000;
    return sum_within(c, n, reach, 0, terms, lo, hi, left);
}

}  // namespace pcr
