// Rows of heads as the operators around K,V take them: element (i, j, ..., d) of a view lies at data + i * s0 + j * s1 + ... + d.
// What the host checks of them before a launch.
#pragma once
#include "bb_internal.h"
#include <algorithm>
#include <cstdlib>

#define HEADS_MAX_STRIDE (1L << 40)         // elements; what the checks below compute with it stays within 64 bits

// Up to three dimensions (tokens and heads; pages, heads and tokens) around `dim` consecutive elements.
struct HeadView {
    const void* data; long n[3], s[3]; int dim, size;
    long last() const {                     // elements from the first to behind the last one
        long e = dim;
        for (int i = 0; i < 3; ++i) e += (n[i] - 1) * s[i];
        return e;
    }
};
static inline HeadView heads_view(const void* p, long tokens, long ts, int heads, long hs, int dim, int size) {
    return HeadView{p, {tokens, heads, 1}, {tokens > 1 ? ts : 0, heads > 1 ? hs : 0, 0}, dim, size};    // (a stride over one is none)
}
static inline HeadView pages_view(const void* p, long pages, long ps, int heads, long hs, long ts, int dim, int size) {
    HeadView v{p, {pages, heads, BB_PAGE_TOKENS}, {pages > 1 ? ps : 0, heads > 1 ? hs : 0, ts}, dim, size};
    return v;
}
static inline bool refuse_view(const HeadView& v) {
    if (!v.data || (uintptr_t)v.data % v.size) return true;
    long all = 1;
    for (int i = 0; i < 3; ++i) {
        if (v.s[i] < 0 || v.s[i] > HEADS_MAX_STRIDE || v.n[i] > (1L << 31)) return true;
        if (v.s[i] && (all = std::max(all, v.n[i] * (v.s[i] >> 20 ? v.s[i] >> 20 : 1))) > 1L << 36) return true;
    }
    return false;
}
// 16-byte pieces: what the matrix kernels load.
static inline bool refuse_pieces(const HeadView& v) {
    const long unit = 16 / v.size;
    return (uintptr_t)v.data % 16 || v.s[0] % unit || v.s[1] % unit || v.s[2] % unit;
}
// An output: no element twice (each stride, from the smallest on, at least what the ones within it span).
static inline bool refuse_out_view(const HeadView& v) {
    if (refuse_view(v)) return true;
    int by[3] = {0, 1, 2};
    std::sort(by, by + 3, [&](int a, int b) { return v.s[a] < v.s[b]; });
    long span = v.dim;
    for (int i : by) {
        if (v.n[i] <= 1) continue;
        if (v.s[i] < span) return true;
        span += (v.n[i] - 1) * v.s[i];
    }
    return false;
}
// Whether an output may share an element with a tensor that the same call reads or writes.  Apart, or column ranges of rows at one distance (the parts of one
// projection's output): no.  Anything else counts as sharing.
static inline bool overlap(const HeadView& a, const HeadView& b) {
    const long a0 = (long)(uintptr_t)a.data, b0 = (long)(uintptr_t)b.data, a1 = a0 + a.last() * a.size, b1 = b0 + b.last() * b.size;
    if (a1 <= b0 || b1 <= a0) return false;
    const long ld = a.s[0] * a.size;
    if (ld == 0 || ld != b.s[0] * b.size || a.n[2] != 1 || b.n[2] != 1) return true;
    const long na = ((a.n[1] - 1) * a.s[1] + a.dim) * a.size, nb = ((b.n[1] - 1) * b.s[1] + b.dim) * b.size;     // a row's columns
    if (na > ld || nb > ld) return true;
    const long at = ((b0 - a0) % ld + ld) % ld;             // where b's columns begin, seen from a's
    return at < na || ld - at < nb;
}
static inline bool same_rows(const HeadView& a, const HeadView& b) { return a.data == b.data && a.s[0] == b.s[0] && a.s[1] == b.s[1]; }
