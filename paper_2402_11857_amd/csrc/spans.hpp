// Which operands share memory, for the argument checks of include/liec_train.h.  Host code; may throw std::bad_alloc where it says so.
//
// An operand is a set of runs: `many` groups at distances of `wide` bytes, each of `n` runs of `len` bytes at distances of `s`.  The
// answers are exact, with an exception for operands that lie between one another at distances that differ, where there is little to
// calculate with: the runs of two of them are looked up one by one, and more than kSpanSteps count as sharing; in a larger set such
// operands always do.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <map>
#include <queue>
#include <utility>
#include <vector>

namespace liec {

constexpr int64_t kSpanSteps = (int64_t)1 << 22;       // some 20 ms

struct Span {
    int64_t lo = 0, hi = 0;            // first byte, one past the last
    int64_t len = 0, s = 0, n = 1, wide = 0, many = 1;      // n > 1: s > len;  many > 1: wide > s;  len = 0: empty
    int64_t runs() const { return n * many; }
    int64_t extent() const { return (n - 1) * s + len; }    // of a group
};

// Strides in bytes, of either sign; runs that touch become one.
inline Span span_of(const void* data, int64_t len, int64_t s = 0, int64_t n = 1, int64_t wide = 0, int64_t many = 1) {
    Span r;
    r.lo = (int64_t)(uintptr_t)data;
    r.hi = r.lo;
    if (!data || len <= 0 || n <= 0 || many <= 0) return r;
    if (n > 1 && s < 0) r.lo += s * (n - 1), s = -s;
    if (many > 1 && wide < 0) r.lo += wide * (many - 1), wide = -wide;
    if (n == 1 || s == 0) s = 0, n = 1;
    if (many == 1 || wide == 0) wide = 0, many = 1;
    if (many > 1 && (n == 1 || wide < s)) std::swap(s, wide), std::swap(n, many);
    if (n > 1 && s <= len) {
        len += (n - 1) * s;
        s = wide, n = many, wide = 0, many = 1;
        if (n > 1 && s <= len) len += (n - 1) * s, s = 0, n = 1;
    }
    if (many > 1 && wide == n * s) n *= many, wide = 0, many = 1;
    r.len = len, r.s = s, r.n = n, r.wide = wide, r.many = many;
    r.hi = r.lo + (many - 1) * wide + r.extent();
    return r;
}

// Index of the first of the intervals [i * step, i * step + len), i >= 0, that ends after `a`.
inline int64_t first_ending_after(int64_t a, int64_t len, int64_t step) { return a < len ? 0 : step ? (a - len) / step + 1 : 0; }

// Does a span have a byte in [a, b)?  Takes one of `steps` for every group that comes into question.
inline bool span_meets(const Span& p, int64_t a, int64_t b, int64_t& steps) {
    if (p.len <= 0 || a >= b || a >= p.hi || b <= p.lo) return false;
    a -= p.lo;
    b -= p.lo;
    for (int64_t i = first_ending_after(a, p.extent(), p.wide); i < p.many && i * p.wide < b; ++i) {
        if (--steps < 0) return true;
        const int64_t in = a - i * p.wide, j = first_ending_after(in, p.len, p.s);
        if (j < p.n && j * p.s < b - i * p.wide) return true;
    }
    return false;
}
inline bool span_meets(const Span& p, int64_t a, int64_t b) {
    int64_t steps = kSpanSteps;
    return span_meets(p, a, b, steps);
}

// Do two spans share a byte?
inline bool spans_meet(const Span& a, const Span& b, int64_t& steps) {
    if (a.len <= 0 || b.len <= 0 || a.hi <= b.lo || b.hi <= a.lo) return false;
    const bool alike = (a.s == b.s || a.n == 1 || b.n == 1) && (a.wide == b.wide || a.many == 1 || b.many == 1);
    if (alike && a.runs() > 1 && b.runs() > 1) {
        // the same distances: b's runs lie at offsets of the same kind from a's, and meet one that is less than a length away
        Span d;
        d.s = std::max(a.s, b.s), d.n = a.n + b.n - 1;
        d.wide = std::max(a.wide, b.wide), d.many = a.many + b.many - 1;
        d.len = 1;
        d.lo = b.lo - a.lo - (a.n - 1) * d.s - (a.many - 1) * d.wide;
        d.hi = d.lo + (d.many - 1) * d.wide + d.extent();
        return span_meets(d, 1 - b.len, a.len, steps);
    }
    const Span &few = a.runs() <= b.runs() ? a : b, &other = a.runs() <= b.runs() ? b : a;
    for (int64_t i = 0; i < few.many; ++i)
        for (int64_t j = 0; j < few.n; ++j) {
            const int64_t at = few.lo + i * few.wide + j * few.s;
            if (--steps < 0 || span_meets(other, at, at + few.len, steps)) return true;
        }
    return false;
}
inline bool spans_meet(const Span& a, const Span& b) {
    int64_t steps = kSpanSteps;
    return spans_meet(a, b, steps);
}

// Do the runs of one kind of distance, in rows of `s` bytes from `base`, share a byte?  Every span is a rectangle of rows and columns,
// or several where its runs end beyond their row; a sweep over the rows keeps those of the present row in order of their columns.
inline bool rectangles_meet(const Span* p, size_t count, int64_t s) {
    struct Rect {
        int64_t row, rows, col, end;
    };
    std::vector<Rect> all;
    all.reserve(2 * count);
    const int64_t base = p[0].lo;
    for (size_t i = 0; i < count; ++i) {
        int64_t row = (p[i].lo - base) / s, col = (p[i].lo - base) % s, len = p[i].len;
        while (len > 0) {
            // whole rows of a single run at once
            const int64_t whole = col == 0 && p[i].n == 1 ? len / s : 0, here = whole ? whole * s : std::min(len, s - col);
            all.push_back({row, whole ? whole : p[i].n, col, whole ? s : col + here});
            row += whole ? whole : 1;
            col = 0;
            len -= here;
        }
    }
    std::sort(all.begin(), all.end(), [](const Rect& a, const Rect& b) { return a.row < b.row; });
    std::map<int64_t, int64_t> open;                            // columns: start -> end
    typedef std::pair<int64_t, int64_t> Close;                  // row after the last, start
    std::priority_queue<Close, std::vector<Close>, std::greater<Close>> close;
    for (const Rect& r : all) {
        for (; !close.empty() && close.top().first <= r.row; close.pop()) open.erase(close.top().second);
        const auto next = open.lower_bound(r.col);
        if (next != open.end() && next->first < r.end) return true;
        if (next != open.begin() && std::prev(next)->second > r.col) return true;
        open.emplace_hint(next, r.col, r.end);
        close.push({r.row + r.rows, r.col});
    }
    return false;
}

// Do any two of the spans (many = 1) share a byte, or lie between one another at distances that differ?  Reorders them.  May throw
// std::bad_alloc.
inline bool any_meet(std::vector<Span>& all) {
    all.erase(std::remove_if(all.begin(), all.end(), [](const Span& p) { return p.len <= 0; }), all.end());
    std::sort(all.begin(), all.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    for (size_t i = 0, k; i < all.size(); i = k) {
        // spans i .. k - 1 reach into one another
        int64_t reached = all[i].hi, s = all[i].s;
        bool row = true;                                        // columns of the first one's rows, in order
        for (k = i + 1; k < all.size() && all[k].lo < reached; ++k) {
            reached = std::max(reached, all[k].hi);
            if (all[k].s && s && all[k].s != s) return true;
            s = std::max(s, all[k].s);
            if (all[k].n != all[i].n || all[k].lo < all[k - 1].lo + all[k - 1].len) row = false;
        }
        if (k == i + 1) continue;
        if (!s) return true;                                    // single runs
        if (row && all[k - 1].lo + all[k - 1].len <= all[i].lo + s) continue;
        if (rectangles_meet(&all[i], k - i, s)) return true;
    }
    return false;
}

}  // namespace liec
