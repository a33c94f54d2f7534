// csrc/spans.hpp against looking at every byte.
#include <stdio.h>
#include <stdlib.h>

#include <chrono>
#include <random>

#include "spans.hpp"

using namespace liec;

static std::mt19937 rng(7);
static int64_t pick(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }

struct Given {
    int64_t at, len, s, n, wide, many;
};
constexpr int64_t kBytes = 4096, kOrigin = 1 << 16;

static Given draw(bool groups) {
    for (;;) {
        Given g;
        g.len = pick(0, 9);
        g.n = pick(1, 5);
        g.s = pick(-25, 25);
        g.many = groups ? pick(1, 5) : 1;
        g.wide = groups ? (pick(0, 3) ? pick(-120, 120) : g.s * pick(1, 5)) : 0;
        g.at = pick(1000, 1400);
        return g;
    }
}
static Span span(const Given& g) { return span_of((const void*)(uintptr_t)(kOrigin + g.at), g.len, g.s, g.n, g.wide, g.many); }
static std::vector<int> bytes(const Given& g) {
    std::vector<int> r(kBytes, 0);
    for (int64_t i = 0; i < g.many; ++i)
        for (int64_t j = 0; j < g.n; ++j)
            for (int64_t b = 0; b < g.len; ++b) r[g.at + i * g.wide + j * g.s + b]++;
    return r;
}
static void fail(const char* what, const Given& a, const Given& b) {
    printf("%s: (%ld %ld %ld %ld %ld %ld) (%ld %ld %ld %ld %ld %ld)\n", what, a.at, a.len, a.s, a.n, a.wide, a.many, b.at, b.len, b.s, b.n, b.wide, b.many);
    exit(1);
}

static void pairs() {
    int64_t met = 0, not_met = 0;
    for (int q = 0; q < 200000; ++q) {
        Given a = draw(true), b = draw(true);
        if (q % 3 == 0) b.s = a.s, b.wide = a.wide;             // of the same distances
        if (q % 6 == 0) b.s = -a.s;
        const std::vector<int> x = bytes(a), y = bytes(b);
        bool want = false;
        for (int64_t i = 0; i < kBytes; ++i) want = want || (x[i] && y[i]);
        (want ? met : not_met)++;
        if (spans_meet(span(a), span(b)) != want || spans_meet(span(b), span(a)) != want) fail("two spans", a, b);
        const int64_t lo = pick(900, 1500), hi = lo + pick(0, 40);
        bool in = false;
        for (int64_t i = lo; i < hi; ++i) in = in || x[i];
        if (span_meets(span(a), kOrigin + lo, kOrigin + hi) != in) fail("an interval", a, Given{lo, hi, 0, 0, 0, 0});
    }
    printf("pairs that share %ld, that do not %ld\n", met, not_met);
}

static void sets() {
    int64_t met = 0, not_met = 0;
    for (int q = 0; q < 100000; ++q) {
        const int64_t n = pick(1, 4), s = pick(20, 60);
        std::vector<Span> all;
        std::vector<Given> given;
        std::vector<int> count(kBytes, 0);
        bool own = false;
        for (int64_t k = pick(1, 6); k > 0; --k) {
            Given g{pick(1000, 1000 + 3 * s), pick(0, 12), s, n, 0, 1};
            if (q % 2 && pick(0, 3) == 0) g.s = pick(12, 80), own = true;
            if (pick(0, 5) == 0) g.n = 1, g.len = pick(0, 70);    // a single run
            if (pick(0, 3) == 0) g.at += g.s * (g.n - 1), g.s = -g.s;
            given.push_back(g);
            all.push_back(span(g));
            const std::vector<int> x = bytes(g);
            for (int64_t i = 0; i < kBytes; ++i) count[i] += x[i] ? 1 : 0;
        }
        bool want = false;
        for (int64_t i = 0; i < kBytes; ++i) want = want || count[i] > 1;
        (want ? met : not_met)++;
        if (any_meet(all) != want && !(own && !want)) {          // distances that differ may count as sharing
            for (const Given& g : given) printf("(%ld %ld %ld %ld) ", g.at, g.len, g.s, g.n);
            printf("sets, expected %d\n", want);
            exit(1);
        }
    }
    printf("sets that share %ld, that do not %ld\n", met, not_met);
}

// Host time must not grow with the square of the number of tensors, whatever their layout.
static void times() {
    const int64_t T = 65536, N = 8, row = T * 16;
    for (int kind = 0; kind < 4; ++kind) {
        std::vector<Span> all;
        for (int64_t i = 0; i < T; ++i) all.push_back(span_of((const void*)(uintptr_t)((1 << 20) + i * 16), 12, row, kind == 3 ? N - i % 2 : N));
        if (kind >= 1) all.push_back(span_of((const void*)(uintptr_t)((1 << 20) + row * N + 64), 100, 100, N));           // one of its own
        if (kind == 2) all.push_back(span_of((const void*)(uintptr_t)((1 << 20) + 12), 4, -row, 1));                      // a gap of theirs
        const auto t = std::chrono::steady_clock::now();
        const bool meet = any_meet(all);
        const double ms = std::chrono::duration<double, std::milli>(std::chrono::steady_clock::now() - t).count();
        printf("kind %d: %.2f ms\n", kind, ms);
        if (meet || ms > 2000) exit(1);
    }
}

int main() {
    pairs();
    sets();
    times();
    printf("spans ok\n");
    return 0;
}
