// Memory of strided operands: whether two of them have a byte in common.  Host only.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <utility>

namespace pcr {

// Rows of `bytes` bytes from `at` on, `n[i]` of them `step[i]` bytes apart on each of three axes.
struct Span {
    uintptr_t at;
    int64_t bytes;
    __int128 step[3];
    int64_t n[3];
};
inline Span span_of(const void* p, size_t bytes) { return {reinterpret_cast<uintptr_t>(p), (int64_t)bytes, {0, 0, 0}, {1, 1, 1}}; }
inline Span span_of(const void* p, const int64_t (&stride)[3], int64_t n0, int64_t n1, int64_t n2, int64_t row, size_t es) {
    return {reinterpret_cast<uintptr_t>(p), row * (int64_t)es, {(__int128)stride[0] * (int64_t)es, (__int128)stride[1] * (int64_t)es, (__int128)stride[2] * (int64_t)es}, {n0, n1, n2}};
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
    if (a.bytes <= 0 || b.bytes <= 0) return false;
    __int128 c[6], n[6], reach[7], from[2], to[2];
    int terms = 0;
    const Span* of[2] = {&a, &b};
    for (int s = 0; s < 2; ++s) {
        from[s] = of[s]->at; to[s] = from[s] + of[s]->bytes;
        for (int i = 0; i < 3; ++i) {
            if (of[s]->n[i] < 1) return false;
            const __int128 step = of[s]->step[i], far = step * (of[s]->n[i] - 1);
            if (far < 0) from[s] += far; else to[s] += far;
            if (far == 0) continue;
            c[terms] = step < 0 ? -step : step; n[terms++] = of[s]->n[i];
        }
    }
    if (to[0] <= from[1] || to[1] <= from[0]) return false;
    // A row of a begins at from[0] + u, one of b at to[1] - b.bytes - v, u and v sums of steps: they meet where u + v lies between
    const __int128 lo = to[1] - b.bytes - from[0] - a.bytes + 1,
                   hi = to[1] - from[0] - 1;
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
