// Whether two matrices in memory share bytes.  Host only.
#pragma once
#include <stdint.h>

struct Rows {
    uintptr_t at;         // of the first row
    int64_t n, ld, width; // rows; bytes between two of them and of one (width <= ld where there are several)
    Rows(const void* p, int64_t n_, int64_t ld_, int64_t width_) : at((uintptr_t)p), n(p != nullptr ? n_ : 0), ld(ld_), width(width_) {}
    uintptr_t end() const { return at + (uintptr_t)((n - 1) * ld + width); }
};

static inline bool same_place(const Rows& a, const Rows& b) { return a.at == b.at && a.n == b.n && a.width == b.width && (a.n <= 1 || a.ld == b.ld); }

// Views into the same wider rows may lie between each other's rows without sharing a byte, so the ranges of addresses alone do not decide.
static inline bool overlap(const Rows& a, const Rows& b) {
    if (a.n <= 0 || b.n <= 0 || a.width <= 0 || b.width <= 0 || a.at >= b.end() || b.at >= a.end()) return false;
    if (a.n > 1 && b.n > 1 && a.ld == b.ld) {
        // row j of b begins `over` bytes behind row j + skip of a: it can meet that row and the next one
        const int64_t apart = (int64_t)(b.at - a.at);
        int64_t skip = apart / a.ld, over = apart % a.ld;
        if (over < 0) {
            over += a.ld;
            --skip;
        }
        auto meet = [&](int64_t d) { return (d > 0 ? d : 0) < a.n && (d < 0 ? -d : 0) < b.n; };  // is there a j with both rows
        return (over < a.width && meet(skip)) || (over + b.width > a.ld && meet(skip + 1));
    }
    // of every row of the one with fewer: the last row of the other that begins before its end
    const Rows &few = a.n < b.n ? a : b, &many = a.n < b.n ? b : a;
    for (int64_t i = 0; i < few.n; ++i) {
        const uintptr_t from = few.at + (uintptr_t)(i * few.ld), to = from + (uintptr_t)few.width;
        if (to <= many.at) continue;
        int64_t j = many.n > 1 ? (int64_t)((to - 1 - many.at) / (uintptr_t)many.ld) : 0;
        if (j > many.n - 1) j = many.n - 1;
        if (many.at + (uintptr_t)(j * many.ld) + (uintptr_t)many.width > from) return true;
    }
    return false;
}
