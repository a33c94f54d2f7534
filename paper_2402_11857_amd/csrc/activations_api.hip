// Host side of include/liec_activations.h: argument checks, launch shapes, launches.
#include "liec_activations.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "kernels/group_norm_held.hpp"
#include "kernels/weight_grad.hpp"
#include "operands.hpp"

using namespace liec;

namespace {

// Results are left in the memory-side cache of 256 MB for the operation that reads them next if what was read for them fits beside them;
// larger ones are streamed past it, so that a normalisation's second pass finds in it what the first one read and the next
// call's first pass does not wait for results to leave it (stats and apply of 128 images of 56 x 56 x 256 bf16, 206 MB: 41 + 79 against 55 + 76 us,
// of 268 MB 47 + 92 against 75 + 92).
bool keeps(int64_t bytes) { return bytes <= (int64_t)128 << 20; }

// Blocks of a launch whose blocks walk over the work: far more than are resident, and within what a launch may have.
uint32_t grid_of(int64_t works) { return (uint32_t)std::max<int64_t>(1, std::min<int64_t>(works, (int64_t)1 << 22)); }

LnRows rows_of(const liec_rows* r) { return LnRows{r->data, r->worker_stride, r->row_stride}; }
LnParam param_of(const liec_param* p, int type) { return p && p->data ? LnParam{p->data, p->stride, (uint32_t)type} : LnParam{nullptr, 0, (uint32_t)type}; }

// ---- checkpoints -----------------------------------------------------------------------------------------------------
constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1;

bool valid_sizes(int64_t N, int64_t R, int64_t C) {
    if ((double)N * (double)R * (double)C > (double)kMostValues) return false;
    return N >= 1 && N <= kMaxWorkers && R >= 0 && R <= kMostRows && C >= 1 && C <= ((int64_t)1 << 28);
}
bool valid_saved(const liec_checkpoint* s) { return s && s->values && s->exponents; }
Saved saved_of(const liec_checkpoint* s) { return s ? Saved{s->values, s->exponents} : Saved{nullptr, nullptr}; }
int64_t groups_of(int64_t C) { return ceil_div(C, kSavedCols); }
Span span_of_values(const liec_checkpoint* s, int64_t rows, int64_t C) { return s ? span_of(s->values, rows * C) : Span(); }
Span span_of_exponents(const liec_checkpoint* s, int64_t rows, int64_t C) { return s ? span_of(s->exponents, rows * groups_of(C)) : Span(); }

struct SavedLaunch {
    dim3 grid;
    uint32_t per, magic;
};
SavedLaunch saved_launch(int64_t N, int64_t R, int64_t C) {
    const int64_t per = 4 * groups_of(C);
    return {dim3(grid_of(ceil_div(R * per, kSavedBlock)), (uint32_t)N), (uint32_t)per, (uint32_t)((((uint64_t)1 << 32) + per - 1) / per)};
}
// Workers whose rows follow one another are one worker's: a short one fills no block.
void merge_workers(LnRows& r, int64_t& N, int64_t& R) {
    if (N > 1 && r.worker == R * r.row && N * R <= kMostRows) R *= N, N = 1;
}

template <typename T>
void run_save(LnRows x, const Saved& to, int64_t N, int64_t R, int64_t C, hipStream_t st) {
    merge_workers(x, N, R);
    const SavedLaunch l = saved_launch(N, R, C);
    k_checkpoint_save<T><<<l.grid, kBlock, 0, st>>>(R, (uint32_t)C, l.per, l.magic, x, to);
}
template <typename T>
void run_load(const Saved& from, LnRows y, int64_t N, int64_t R, int64_t C, hipStream_t st) {
    const bool keep = keeps(N * R * C * (int64_t)sizeof(T));
    merge_workers(y, N, R);
    const SavedLaunch l = saved_launch(N, R, C);
    k_checkpoint_load<T><<<l.grid, kBlock, 0, st>>>(R, (uint32_t)C, l.per, l.magic, keep, from, y);
}

// ---- group normalisation ---------------------------------------------------------------------------------------------
// Images as an operand: runs of channels at up to three distances, in the order of these.  What follows one another is one, two
// distances are a span, and of three the largest is between groups of runs (or, where that would be very many groups, that of the
// fewest).
struct ImageSpans {
    int64_t first, wide, many;         // bytes between groups, 0 for a single one
    int64_t len, s, n, t, m;           // a group: m times at distances t, n runs of len at distances s
    Span at(int64_t i) const { return span_of((const void*)(first + i * wide), len, s, n, t, m); }
};
constexpr int64_t kImageGroups = (int64_t)1 << 16;
ImageSpans image_spans(const liec_images* x, int64_t N, int64_t B, int64_t S, int64_t C, int64_t size) {
    struct {
        int64_t stride, n;
    } d[3] = {{x->row_stride * size, S}, {x->image_stride * size, B}, {x->worker_stride * size, N}};
    ImageSpans r{(int64_t)(uintptr_t)x->data, 0, 1, C * size, 0, 1, 0, 1};
    int dims = 0;
    for (const auto& e : d) {
        if (e.n == 1 || e.stride == 0) continue;
        if (e.stride < 0) r.first += (e.n - 1) * e.stride;
        d[dims++] = {llabs(e.stride), e.n};
    }
    std::sort(d, d + dims, [](const auto& a, const auto& b) { return a.stride < b.stride; });
    for (int i = 1; i < dims;) {
        if (d[i].stride != d[i - 1].n * d[i - 1].stride) {
            ++i;
            continue;
        }
        d[i - 1].n *= d[i].n;
        for (int k = i + 1; k < dims; ++k) d[k - 1] = d[k];
        --dims;
    }
    if (dims == 3) {
        if (d[2].n > kImageGroups) std::swap(d[2], *std::min_element(d, d + 3, [](const auto& a, const auto& b) { return a.n < b.n; }));
        r.wide = d[2].stride, r.many = d[2].n;
    }
    if (dims > 0) r.s = d[0].stride, r.n = d[0].n;
    if (dims > 1) r.t = d[1].stride, r.m = d[1].n;
    return r;
}
// Only groups that come near one another are looked at: a few for each where operands lie between one another.
bool images_meet(const ImageSpans& a, const Span& p, int64_t& steps) {
    const Span box = a.at(0);
    if (box.len <= 0 || p.len <= 0) return false;
    for (int64_t i = first_ending_after(p.lo - box.lo, box.hi - box.lo, a.wide); i < a.many && box.lo + i * a.wide < p.hi; ++i)
        if (--steps < 0 || spans_meet(a.at(i), p, steps)) return true;
    return false;
}
bool images_meet(const ImageSpans& a, const Span& p) {
    int64_t steps = kSpanSteps;
    return images_meet(a, p, steps);
}
bool images_meet(const ImageSpans& a, const ImageSpans& b) {
    int64_t steps = kSpanSteps;
    const ImageSpans &few = a.many <= b.many ? a : b, &other = a.many <= b.many ? b : a;
    for (int64_t i = 0; i < few.many; ++i)
        if (--steps < 0 || images_meet(other, few.at(i), steps)) return true;
    return false;
}
// Rows that are written must not share memory: each distance spans what the narrower ones cover.
bool apart(const liec_images* x, int64_t N, int64_t B, int64_t S, int64_t C) {
    std::pair<int64_t, int64_t> d[3] = {{llabs(x->row_stride), S}, {llabs(x->image_stride), B}, {llabs(x->worker_stride), N}};
    std::sort(d, d + 3);
    int64_t covered = C;
    for (const auto& [stride, n] : d) {
        if (n == 1) continue;
        if (stride < covered) return false;
        covered += (n - 1) * stride;
    }
    return true;
}
bool same(const liec_images* a, const liec_images* b, int64_t N, int64_t B, int64_t S) {
    return a->data == b->data && (N == 1 || a->worker_stride == b->worker_stride) && (B == 1 || a->image_stride == b->image_stride) &&
           (S == 1 || a->row_stride == b->row_stride);
}
bool valid_images(const liec_images* x, int64_t N, int64_t B, int64_t S, int64_t size) {
    if (!x || !x->data || !aligned_to(x->data, size) || !in_range(x->worker_stride) || !in_range(x->image_stride) || !in_range(x->row_stride)) return false;
    return (double)(S - 1) * (double)llabs(x->row_stride) + (double)(B - 1) * (double)llabs(x->image_stride) + (double)(N - 1) * (double)llabs(x->worker_stride) <=
           (double)kMostValues;
}

bool valid_norm(int64_t N, int64_t B, int64_t S, int64_t C, int64_t G) {
    if (N < 1 || N > kMaxWorkers || B < 0 || B > kMostRows || S < 0 || S > kMostRows || C < 1 || C > ((int64_t)1 << 20)) return false;
    if (G < 1 || G > C || C % G) return false;
    return (double)N * (double)B * (double)std::max<int64_t>(S, 1) * (double)C <= (double)kMostValues;
}

// Blocks that a launch should have at least, where there is work for them: of sums, whose number sets how many partial sums a group has
// (4 x 4 images of 128 x 128 x 512 bf16: 512 blocks 70 + 9 us, 1024 75 + 15, 2048 78 + 26), and of what is written from them (512 blocks
// 116 us, 1024 92, 2048 91, 8192 88).
constexpr int64_t kGnSumBlocks = 512, kGnBlocks = 2048;
constexpr int64_t kGnChain = 256;      // positions that a thread adds up

int log_of(int64_t n) {                // of the next power of two
    int r = 0;
    while (((int64_t)1 << r) < n) ++r;
    return r;
}

GnShape shape_of(int64_t N, int64_t B, int64_t S, int64_t C, int64_t G, int64_t blocks = kGnSumBlocks) {
    GnShape s{};
    const int64_t pieces = C < 8 ? C : ceil_div(C, 8);
    s.images = N * B, s.B = B, s.S = S, s.C = (uint32_t)C, s.G = (uint32_t)G, s.per_group = (uint32_t)(C / G), s.whole = C / G % 8 == 0;
    // four lanes at least where a row is not shorter: those that share an exponent of a checkpoint
    s.lanes_log = (uint32_t)std::min(6, C < 8 ? log_of(C) : std::max(2, log_of(pieces)));
    s.tiles = (uint32_t)ceil_div(pieces, (int64_t)1 << s.lanes_log);
    const int64_t threads = kBlock >> s.lanes_log;
    const int64_t want = ceil_div(blocks, std::max<int64_t>(1, s.images * s.tiles));
    s.per = std::max(ceil_div(S, want), std::min(S, kGnAhead * threads));
    s.per = std::max<int64_t>(1, std::min(s.per, kGnChain * threads));
    s.splits = (uint32_t)std::max<int64_t>(1, ceil_div(S, s.per));
    return s;
}
int64_t gn_works_of(const GnShape& s) { return s.images * s.splits * s.tiles; }
uint32_t gn_group_blocks(const GnShape& s) { return grid_of(s.images * s.G <= kGnFewGroups ? s.images * s.G : ceil_div(s.images * s.G, kBlock / 64)); }
int64_t gn_partials(const GnShape& s) { return s.images * s.splits * 2 * (int64_t)s.C; }
GnImages images_of(const liec_images* x) { return x && x->data ? GnImages{x->data, x->worker_stride, x->image_stride, x->row_stride} : GnImages{nullptr, 0, 0, 0}; }

// Does a block of up to `threads` threads hold a group's positions, `most` of them per thread?  Spans of 128 bytes per position if they
// fit, then narrower ones down to `narrow`, in multiples of `least` channels (those that share an exponent of a checkpoint, or a
// vector); rows whose groups do not come to that are taken whole.
bool hold(const GnShape& s, int64_t size, int64_t most, int64_t threads, int64_t least, int64_t narrow, GnHeld* h) {
    const int64_t pg = s.per_group, C = s.C;
    if (C < 8 || s.S > most * threads) return false;
    for (int64_t wide = 128; wide >= narrow; wide /= 2) {
        int64_t groups = ceil_div(wide / size, pg);
        while (groups < s.G && groups * pg % least) ++groups;
        h->span = (uint32_t)std::min(groups * pg, C);
        h->spans = (uint32_t)ceil_div(C, (int64_t)h->span);
        h->lanes_log = (uint32_t)std::max(log_of(ceil_div(h->span, 8)), log_of(least / 8));
        if (h->lanes_log > 6) continue;
        h->rows_log = (uint32_t)log_of(ceil_div(s.S, most));
        while (h->lanes_log + h->rows_log < 8 && ((int64_t)1 << h->rows_log) < s.S) ++h->rows_log;
        if (((int64_t)1 << (h->lanes_log + h->rows_log)) > threads) continue;
        // more images where one is small: of one worker, so as many as its number of them is a multiple of
        h->images_log = 0;
        while (h->lanes_log + h->rows_log + h->images_log < 8 && s.B % ((int64_t)2 << h->images_log) == 0) ++h->images_log;
        while (h->lanes_log + h->rows_log + h->images_log < 6) ++h->rows_log;          // whole waves
        h->rows = (uint32_t)ceil_div(s.S, (int64_t)1 << h->rows_log);
        return true;
    }
    return false;
}
// An operand whose values a block finds at distances of less than 2^31 bytes.
bool near(const GnImages& x, const GnShape& s, const GnHeld& h, int64_t size) {
    if (x.image < 0 || x.row < 0) return false;
    return ((double)(((int64_t)1 << h.images_log) - 1) * (double)x.image + (double)s.S * (double)x.row + (double)s.C) * (double)size < 2147483648.0;
}
int64_t held_threads(const GnHeld& h) { return (int64_t)1 << (h.lanes_log + h.rows_log + h.images_log); }
int64_t held_waves(const GnHeld& h) { return h.lanes_log + h.rows_log > 6 ? (int64_t)1 << (h.lanes_log + h.rows_log - 6) : 1; }
constexpr int64_t kGnHeldBytes = 64 << 10;                           // of LDS
int64_t held_bytes(const GnShape& s, const GnHeld& h, bool backward) {
    const int64_t entries = !backward && s.whole ? h.span / 8 : h.span, images = (int64_t)1 << h.images_log;
    return 4 * images * (2 * entries * held_waves(h) + (backward ? 2 * (int64_t)h.span : 0) + 2 * (h.span / s.per_group));
}
uint32_t held_grid(const GnShape& s, const GnHeld& h) { return grid_of((s.images >> h.images_log) * h.spans); }

// Images whose partial sums are in the scratch at a time: all of them, whole workers, or some of one worker's.  Many images of few
// positions would take more scratch than they take themselves, 8 bytes per image and channel.
constexpr int64_t kGnScratch = (int64_t)256 << 20;
struct GnChunk {
    int64_t workers, images;
};
int64_t gn_scratch(int64_t N, int64_t B, int64_t S, int64_t C, int64_t G) {
    const GnShape s = shape_of(N, B, S, C, G);
    return ceil_div(gn_partials(s) * (int64_t)sizeof(float) + s.images * G * (int64_t)sizeof(float2), 16) * 16;
}
GnChunk gn_chunk(int64_t N, int64_t B, int64_t S, int64_t C, int64_t G) {
    const int64_t most = std::max<int64_t>(1, kGnScratch / (shape_of(N, B, S, C, G).splits * 8 * C + 8 * G));
    return N * B <= most ? GnChunk{N, B} : B <= most ? GnChunk{most / B, B} : GnChunk{1, most};
}
// Of the chunks, the last ones among them, whose strips may be shorter.
int64_t gn_chunk_scratch(int64_t N, int64_t B, int64_t S, int64_t C, int64_t G) {
    const GnChunk c = gn_chunk(N, B, S, C, G);
    int64_t need = gn_scratch(c.workers, c.images, S, C, G);
    if (N % c.workers) need = std::max(need, gn_scratch(N % c.workers, c.images, S, C, G));
    if (B % c.images) need = std::max(need, gn_scratch(c.workers, B % c.images, S, C, G));
    return need;
}
int64_t gn_run_bytes(int64_t C) { return 2 * C * (int64_t)sizeof(double); }   // weight gradients that chunks add to

GnImages from(const GnImages& x, int64_t worker, int64_t image, int64_t size) {
    GnImages r = x;
    if (r.data) r.data = static_cast<char*>(r.data) + (worker * x.worker + image * x.image) * size;
    return r;
}
LnParam from(const LnParam& p, int64_t worker) {
    LnParam r = p;
    if (r.data) r.data = static_cast<char*>(r.data) + worker * p.stride * size_of((int)p.type);
    return r;
}
Saved from(const Saved& s, int64_t rows, int64_t C) { return s.q ? Saved{s.q + rows * C, s.e + rows * groups_of(C)} : s; }

struct GnForward {
    int64_t N;
    GnShape s, each;                   // of sums, and of what is written from them
    GnImages x, y;
    LnParam w, b;
    float *mean, *rstd, *partial, eps;
    Saved saved;
    bool keep;
    int act;
    hipStream_t st;
};

template <typename T, int K, int ACT>
void gn_held_of(const GnForward& a, const GnHeld& h) {
    const auto f = a.saved.q ? k_gn_held<T, K, ACT, true> : k_gn_held<T, K, ACT, false>;
    f<<<held_grid(a.s, h), (uint32_t)held_threads(h), (size_t)held_bytes(a.s, h, false), a.st>>>(a.s, h, a.keep, a.eps, a.mean, a.rstd, a.x, a.y, a.w, a.b, a.saved);
}
template <typename T, int K>
void gn_held_of(const GnForward& a, const GnHeld& h) {
    a.act == kActNone ? gn_held_of<T, K, kActNone>(a, h) : a.act == kActRelu ? gn_held_of<T, K, kActRelu>(a, h) : gn_held_of<T, K, kActSilu>(a, h);
}

template <typename T, int V>
void gn_forward_of(const GnForward& a) {
    const uint32_t grid = grid_of(gn_works_of(a.s));
    k_gn_stats<T, V><<<grid, kBlock, 0, a.st>>>(a.s, a.x, a.partial);
    k_gn_groups<0><<<gn_group_blocks(a.s), kBlock, 0, a.st>>>(a.s, a.partial, a.eps, a.mean, a.rstd);
    const auto apply = a.saved.q ? (a.act == kActNone ? k_gn_apply<T, V, kActNone, true> : a.act == kActRelu ? k_gn_apply<T, V, kActRelu, true> : k_gn_apply<T, V, kActSilu, true>)
                                 : (a.act == kActNone ? k_gn_apply<T, V, kActNone, false> : a.act == kActRelu ? k_gn_apply<T, V, kActRelu, false> : k_gn_apply<T, V, kActSilu, false>);
    apply<<<grid_of(gn_works_of(a.each)), kBlock, 0, a.st>>>(a.each, a.keep, a.mean, a.rstd, a.x, a.y, a.w, a.b, a.saved);
}
// Images that blocks hold.  Positions of a thread: 32 registers for values (four times as many leave two waves to a SIMD, whose loads and
// arithmetic do not overlap: 128 images of 56 x 56 x 256 bf16 116 to 125 us against 124 in two passes, of 28 x 28 x 512 with a checkpoint
// 75 against 51).  Blocks of 512 threads, two to a compute unit, before larger ones: 128 images of 28 x 28 x 512 bf16 51.8 us, with
// 1024 threads and wider spans 53.7, in two passes 71.1; fp32 with 1024 threads 113, in two passes 145.
template <typename T>
bool held_forward(const GnForward& a, GnHeld* h) {
    constexpr int most = sizeof(T) == 2 ? 8 : 4;
    if (!hold(a.s, sizeof(T), most, 512, kSavedCols, 32, h) && !hold(a.s, sizeof(T), most, kGnHeldMost, kSavedCols, 32, h)) return false;
    return held_bytes(a.s, *h, false) <= kGnHeldBytes && near(a.x, a.s, *h, sizeof(T)) && near(a.y, a.s, *h, sizeof(T));
}
template <typename T>
void gn_forward_of(const GnForward& a) {
    GnHeld h;
    if (held_forward<T>(a, &h)) {
        gn_held_of<T, sizeof(T) == 2 ? 8 : 4>(a, h);
        return;
    }
    const int64_t B = a.s.B, S = a.s.S, C = a.s.C, G = a.s.G;
    const GnChunk chunk = gn_chunk(a.N, B, S, C, G);
    for (int64_t w = 0; w < a.N; w += chunk.workers)
        for (int64_t b = 0; b < B; b += chunk.images) {
            const int64_t workers = std::min(chunk.workers, a.N - w), images = std::min(chunk.images, B - b), at = w * B + b;
            GnForward part = a;
            part.s = shape_of(workers, images, S, C, G);
            part.each = shape_of(workers, images, S, C, G, kGnBlocks);
            part.x = from(a.x, w, b, sizeof(T)), part.y = from(a.y, w, b, sizeof(T));
            part.w = from(a.w, w), part.b = from(a.b, w);
            part.mean += at * G, part.rstd += at * G;
            part.saved = from(a.saved, at * S, C);
            C < 8 ? gn_forward_of<T, 1>(part) : gn_forward_of<T, 8>(part);
        }
}

struct GnBackward {
    int64_t N;
    GnShape s, each;
    GnImages dy, x, dx;
    Saved saved;
    LnParam w, b, dw, db;
    const float *mean, *rstd;
    double* run;
    float* partial;
    int64_t scratch;                   // bytes behind `partial`
    bool keep;
    hipStream_t st;
};

// What comes of partial sums, `parts` of all workers: means for dx where there is one, and weight gradients, one sum for each worker or one over
// all of them.
void gn_after_sums(const GnBackward& a, int64_t parts, float2* means, bool first, bool last) {
    const bool shared = a.N == 1 || (a.dw.data ? a.dw : a.db).stride == 0, params = a.dw.data || a.db.data;
    const uint32_t blocks = means ? gn_group_blocks(a.s) : 0u, columns = (uint32_t)ceil_div(a.s.C, 32), workers = shared ? 1u : (uint32_t)a.N;
    if (!blocks && !params) return;
    const GnParamGrads p{shared ? parts : parts / a.N, workers, columns, a.run, first, last, a.dw, a.db};
    k_gn_after_sums<0><<<blocks + (params ? grid_of(2 * (int64_t)columns * workers) : 0u), kBlock, 0, a.st>>>(a.s, blocks, a.partial, a.w, means, p);
}

template <typename T, int K, int ACT, bool SAVED>
void gn_held_of(const GnBackward& a, const GnHeld& h) {
    k_gn_held_backward<T, K, ACT, SAVED><<<held_grid(a.s, h), (uint32_t)held_threads(h), (size_t)held_bytes(a.s, h, true), a.st>>>(
        a.s, h, a.keep, a.mean, a.rstd, a.dy, a.x, a.saved, a.dx, a.w, a.b, a.partial);
}
template <typename T, int K, int ACT>
void gn_held_of(const GnBackward& a, const GnHeld& h) { a.saved.q ? gn_held_of<T, K, ACT, true>(a, h) : gn_held_of<T, K, ACT, false>(a, h); }
template <typename T, int K>
void gn_held_of(const GnBackward& a, const GnHeld& h, int act) {
    act == kActNone ? gn_held_of<T, K, kActNone>(a, h) : act == kActRelu ? gn_held_of<T, K, kActRelu>(a, h) : gn_held_of<T, K, kActSilu>(a, h);
}

template <typename T, int V, int ACT, bool SAVED>
void gn_backward_of(const GnBackward& a, bool first, bool last) {
    const uint32_t grid = grid_of(gn_works_of(a.s));
    k_gn_sums<T, V, ACT, SAVED><<<grid, kBlock, 0, a.st>>>(a.s, a.mean, a.rstd, a.dy, a.x, a.saved, a.w, a.b, a.partial);
    float2* const means = a.dx.data ? reinterpret_cast<float2*>(a.partial + gn_partials(a.s)) : nullptr;
    gn_after_sums(a, a.s.images * a.s.splits, means, first, last);
    if (means) k_gn_dx<T, V, ACT, SAVED><<<grid_of(gn_works_of(a.each)), kBlock, 0, a.st>>>(a.each, a.keep, a.mean, a.rstd, means, a.dy, a.x, a.saved, a.dx, a.w, a.b);
}
template <typename T, int V, int ACT>
void gn_backward_of(const GnBackward& a, bool first, bool last) {
    a.saved.q ? gn_backward_of<T, V, ACT, true>(a, first, last) : gn_backward_of<T, V, ACT, false>(a, first, last);
}
template <typename T, int V>
void gn_backward_of(const GnBackward& a, int act, bool first, bool last) {
    const auto f = act == kActNone ? gn_backward_of<T, V, kActNone> : act == kActRelu ? gn_backward_of<T, V, kActRelu> : gn_backward_of<T, V, kActSilu>;
    f(a, first, last);
}
// Half as many positions, for two operands, and spans of 64 bytes at least: 128 images of 28 x 28 x 512 bf16 in spans of 32 bytes 129 us, in
// two passes 100; of 14 x 14 x 1024 fp32, held, 95 against 114.
template <typename T>
bool held_backward(const GnBackward& a, GnHeld* h) {
    if (!hold(a.s, sizeof(T), sizeof(T) == 2 ? 4 : 2, 512, 8, 64, h) || held_bytes(a.s, *h, true) > kGnHeldBytes) return false;
    const GnImages rows{nullptr, 0, a.s.S * (int64_t)a.s.C, a.s.C};      // of a checkpoint
    return near(a.x, a.s, *h, sizeof(T)) && near(a.dy, a.s, *h, sizeof(T)) && near(a.dx, a.s, *h, sizeof(T)) && near(rows, a.s, *h, 1);
}
template <typename T>
void gn_backward_of(const GnBackward& a, int act) {
    const int64_t B = a.s.B, S = a.s.S, C = a.s.C, G = a.s.G;
    GnHeld h;
    if (held_backward<T>(a, &h) && (a.s.images >> h.images_log) * 2 * C * (int64_t)sizeof(float) <= a.scratch) {
        gn_held_of<T, sizeof(T) == 2 ? 4 : 2>(a, h, act);
        return gn_after_sums(a, a.s.images >> h.images_log, nullptr, true, true);
    }
    const GnChunk chunk = gn_chunk(a.N, B, S, C, G);
    const bool over_all = (a.dw.data ? a.dw : a.db).stride == 0;
    for (int64_t w = 0; w < a.N; w += chunk.workers)
        for (int64_t b = 0; b < B; b += chunk.images) {
            const int64_t at = w * B + b;
            GnBackward part = a;
            const int64_t images = std::min(chunk.images, B - b);
            part.N = std::min(chunk.workers, a.N - w);
            part.s = shape_of(part.N, images, S, C, G);
            part.each = shape_of(part.N, images, S, C, G, kGnBlocks);
            part.dy = from(a.dy, w, b, sizeof(T)), part.x = from(a.x, w, b, sizeof(T)), part.dx = from(a.dx, w, b, sizeof(T));
            part.w = from(a.w, w), part.b = from(a.b, w), part.dw = from(a.dw, w), part.db = from(a.db, w);
            part.mean += at * G, part.rstd += at * G;
            part.saved = from(a.saved, at * S, C);
            const bool first = b == 0 && (w == 0 || !over_all), last = b + images == B && (w + part.N == a.N || !over_all);
            C < 8 ? gn_backward_of<T, 1>(part, act, first, last) : gn_backward_of<T, 8>(part, act, first, last);
        }
}

bool valid_act(int a) { return a == LIEC_ACT_NONE || a == LIEC_ACT_RELU || a == LIEC_ACT_SILU; }

// ---- weight gradients ------------------------------------------------------------------------------------------------
constexpr int64_t kWgStep = 64;        // rows that a split is a multiple of
constexpr int64_t kWgBlocks = 512;     // of a launch whose rows are split: at most, but for chains of kWgChain rows, and more than half as many if there are the rows

bool valid_weight(int64_t N, int64_t R, int64_t O, int64_t C) {
    if (N < 1 || N > kMaxWorkers || R < 0 || R > kMostRows || O < 1 || C < 1 || O > ((int64_t)1 << 24) || C > ((int64_t)1 << 24)) return false;
    const double n = (double)N, most = (double)kMostValues;
    return n * (double)O * (double)C <= most && n * (double)R * (double)O <= most && n * (double)R * (double)C <= most;
}

int64_t wg_tile(int64_t O, int64_t C) { return O > 128 && C > 128 ? 256 : O > 64 && C > 64 ? 128 : 64; }

WgShape weight_shape(int64_t N, int64_t R, int64_t O, int64_t C) {
    WgShape s{};
    const int64_t tile = wg_tile(O, C);
    s.N = (uint32_t)N, s.R = R, s.O = O, s.C = C;
    s.tiles_o = (uint32_t)ceil_div(O, tile), s.tiles_c = (uint32_t)ceil_div(C, tile);
    const int64_t blocks = N * s.tiles_o * (int64_t)s.tiles_c;
    int64_t splits = std::max<int64_t>(1, std::min(kWgBlocks / blocks, R / (4 * kWgStep)));
    splits = std::max(splits, ceil_div(R, (int64_t)kWgChain));
    s.per = std::max(kWgStep, ceil_div(ceil_div(R, splits), kWgStep) * kWgStep);
    s.splits = (uint32_t)std::max<int64_t>(1, ceil_div(R, s.per));
    return s;
}

template <typename T>
void weight_grad_of(const WgShape& s, const LnRows& dy, const Saved& x, const WgOut& dw, const LnParam& db, float* partial, hipStream_t st) {
    const uint32_t grid = grid_of((int64_t)s.N * s.splits * s.tiles_o * s.tiles_c);
    constexpr int BK = Parts<T>::n == 1 ? 64 : 32;
    const int64_t step = BK * std::max(dy.row * (int64_t)sizeof(T), s.C);
    const bool aligned = ((uintptr_t)dy.data | (uintptr_t)x.q) % 16 == 0 && (dy.row | dy.worker) * (int64_t)sizeof(T) % 16 == 0 && s.C % 16 == 0 && dy.row >= s.O &&
                         step < (int64_t)1 << 30 && s.R;
    const int64_t tile = wg_tile(s.O, s.C);
    if (aligned && tile == 256) k_weight_grad_aligned<T, 256, 256, BK, 4, 2><<<grid, 512, 0, st>>>(s, dy, x, dw, db, partial);
    else if (aligned && tile == 128) k_weight_grad_aligned<T, 128, 128, BK, 2, 2><<<grid, 256, 0, st>>>(s, dy, x, dw, db, partial);
    else if (tile == 256) k_weight_grad<T, 256, 256, BK, 4, 2><<<grid, 512, 0, st>>>(s, dy, x, dw, db, partial);
    else if (tile == 128) k_weight_grad<T, 128, 128, BK, 2, 2><<<grid, 256, 0, st>>>(s, dy, x, dw, db, partial);
    else k_weight_grad<T, 64, 64, 64, 2, 2><<<grid, 256, 0, st>>>(s, dy, x, dw, db, partial);
    if (partial) k_weight_grad_join<0><<<dim3(grid_of(ceil_div(s.O * (s.C + 1), kBlock)), s.N), kBlock, 0, st>>>(s, partial, dw, db);
}

}  // namespace

extern "C" {

liec_status liec_checkpoint_save(const liec_rows* x, const liec_checkpoint* saved, int32_t N, int64_t R, int64_t C, liec_dtype dtype, void* hip_stream) {
    if (!valid_sizes(N, R, C) || !valid_type(dtype)) return LIEC_EINVAL;
    if (R == 0) return LIEC_OK;
    const int64_t size = size_of(dtype), rows = N * R;
    if (!valid_rows(x, N, R, size) || !valid_saved(saved)) return LIEC_EINVAL;
    const Span xs = span_of_rows(x, N, R, C, size), qs = span_of_values(saved, rows, C), es = span_of_exponents(saved, rows, C);
    if (spans_meet(xs, qs) || spans_meet(xs, es) || spans_meet(qs, es)) return LIEC_EINVAL;
    const hipStream_t st = (hipStream_t)hip_stream;
    const LnRows from = rows_of(x);
    const Saved to = saved_of(saved);
    if (dtype == LIEC_F32) run_save<float>(from, to, N, R, C, st);
    else if (dtype == LIEC_BF16) run_save<bf16>(from, to, N, R, C, st);
    else run_save<f16>(from, to, N, R, C, st);
    return launched();
}

liec_status liec_checkpoint_load(const liec_checkpoint* saved, const liec_rows* y, int32_t N, int64_t R, int64_t C, liec_dtype dtype, void* hip_stream) {
    if (!valid_sizes(N, R, C) || !valid_type(dtype)) return LIEC_EINVAL;
    if (R == 0) return LIEC_OK;
    const int64_t size = size_of(dtype), rows = N * R;
    if (!valid_rows(y, N, R, size) || !valid_saved(saved) || !apart(y, N, R, C)) return LIEC_EINVAL;
    const Span ys = span_of_rows(y, N, R, C, size);
    if (spans_meet(ys, span_of_values(saved, rows, C)) || spans_meet(ys, span_of_exponents(saved, rows, C))) return LIEC_EINVAL;
    const hipStream_t st = (hipStream_t)hip_stream;
    const LnRows to = rows_of(y);
    const Saved from = saved_of(saved);
    if (dtype == LIEC_F32) run_load<float>(from, to, N, R, C, st);
    else if (dtype == LIEC_BF16) run_load<bf16>(from, to, N, R, C, st);
    else run_load<f16>(from, to, N, R, C, st);
    return launched();
}

int64_t liec_group_norm_workspace(int32_t N, int64_t B, int64_t S, int64_t C, int64_t G) {
    if (!valid_norm(N, B, S, C, G)) return -1;
    if (B == 0 || S == 0) return 0;
    return gn_run_bytes(C) + gn_chunk_scratch(N, B, S, C, G);
}

liec_status liec_group_norm(const liec_images* x, const liec_param* weight, const liec_param* bias, const liec_images* y, float* mean, float* rstd,
                            const liec_checkpoint* saved, int32_t N, int64_t B, int64_t S, int64_t C, int64_t G, float eps, liec_activation activation,
                            liec_dtype dtype, liec_dtype param_dtype, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!valid_norm(N, B, S, C, G) || !valid_type(dtype) || !valid_type(param_dtype) || !valid_act(activation) || !(eps >= 0.f) || !isfinite(eps)) return LIEC_EINVAL;
    if (B == 0 || S == 0) return LIEC_OK;
    const int64_t size = size_of(dtype), psize = size_of(param_dtype), need = liec_group_norm_workspace(N, B, S, C, G), stats = (int64_t)N * B * G * 4;
    if (!valid_images(x, N, B, S, size) || !valid_images(y, N, B, S, size) || !valid_param(weight, psize) || !valid_param(bias, psize)) return LIEC_EINVAL;
    if (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4) || (saved && !valid_saved(saved))) return LIEC_EINVAL;
    if (!valid_workspace(workspace, workspace_bytes, need) || !apart(y, N, B, S, C)) return LIEC_EINVAL;
    const ImageSpans xs = image_spans(x, N, B, S, C, size), ys = image_spans(y, N, B, S, C, size);
    if (!same(x, y, N, B, S) && images_meet(xs, ys)) return LIEC_EINVAL;
    // what is written, apart from y, and what is read, apart from x
    const Span written[] = {span_of(mean, stats), span_of(rstd, stats), span_of_values(saved, N * B * S, C), span_of_exponents(saved, N * B * S, C), span_of(workspace, need)};
    const Span read[] = {span_of_param(weight, N, C, psize), span_of_param(bias, N, C, psize)};
    for (const Span& r : read)
        if (images_meet(ys, r)) return LIEC_EINVAL;
    for (const Span& w : written) {
        if (images_meet(xs, w) || images_meet(ys, w)) return LIEC_EINVAL;
        for (const Span& r : read)
            if (spans_meet(w, r)) return LIEC_EINVAL;
        for (const Span& v : written)
            if (&v < &w && spans_meet(v, w)) return LIEC_EINVAL;
    }
    const GnForward a{N, shape_of(N, B, S, C, G), shape_of(N, B, S, C, G, kGnBlocks), images_of(x), images_of(y), param_of(weight, param_dtype), param_of(bias, param_dtype), mean, rstd,
                      reinterpret_cast<float*>(static_cast<char*>(workspace) + gn_run_bytes(C)), eps, saved_of(saved), keeps((int64_t)N * B * S * C * size), activation, (hipStream_t)hip_stream};
    if (dtype == LIEC_F32) gn_forward_of<float>(a);
    else if (dtype == LIEC_BF16) gn_forward_of<bf16>(a);
    else gn_forward_of<f16>(a);
    return launched();
}

liec_status liec_group_norm_backward(const liec_images* dy, const liec_images* x, const liec_checkpoint* saved, const float* mean, const float* rstd,
                                     const liec_param* weight, const liec_param* bias, const liec_images* dx, const liec_param* dweight,
                                     const liec_param* dbias, int32_t N, int64_t B, int64_t S, int64_t C, int64_t G, liec_activation activation,
                                     liec_dtype dtype, liec_dtype param_dtype, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!valid_norm(N, B, S, C, G) || !valid_type(dtype) || !valid_type(param_dtype) || !valid_act(activation)) return LIEC_EINVAL;
    const int64_t size = size_of(dtype), psize = size_of(param_dtype), need = liec_group_norm_workspace(N, B, S, C, G), stats = (int64_t)N * B * G * 4;
    if (x && !x->data) x = nullptr;
    if (saved && !saved->values) saved = nullptr;
    if (dx && !dx->data) dx = nullptr;
    if (dweight && !dweight->data) dweight = nullptr;
    if (dbias && !dbias->data) dbias = nullptr;
    for (const liec_param* p : {weight, bias, dweight, dbias})
        if (!valid_param(p, psize)) return LIEC_EINVAL;
    if (N > 1) {
        for (const liec_param* p : {dweight, dbias})
            if (p && p->stride && llabs(p->stride) < C) return LIEC_EINVAL;
        // one sum for all workers, or one for each: the same for both gradients
        if (dweight && dbias && (dweight->stride == 0) != (dbias->stride == 0)) return LIEC_EINVAL;
    }
    const Span dws = span_of_param(dweight, N, C, psize), dbs = span_of_param(dbias, N, C, psize), ws = span_of_param(weight, N, C, psize),
               bs = span_of_param(bias, N, C, psize);
    if (spans_meet(dws, dbs)) return LIEC_EINVAL;
    for (const Span& r : {ws, bs})
        if (spans_meet(dws, r) || spans_meet(dbs, r)) return LIEC_EINVAL;
    const bool empty = B == 0 || S == 0;
    if (!empty) {
        if (!valid_images(dy, N, B, S, size) || (x && !valid_images(x, N, B, S, size)) || (dx && !valid_images(dx, N, B, S, size))) return LIEC_EINVAL;
        if (!x == !saved || (saved && !valid_saved(saved))) return LIEC_EINVAL;
        if (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4) || !valid_workspace(workspace, workspace_bytes, need)) return LIEC_EINVAL;
        const Span read[] = {span_of(mean, stats), span_of(rstd, stats), span_of_values(saved, N * B * S, C), span_of_exponents(saved, N * B * S, C), ws, bs};
        const Span written[] = {dws, dbs, span_of(workspace, need)};
        for (const Span& w : written) {
            for (const liec_images* m : {dy, x, dx})
                if (m && images_meet(image_spans(m, N, B, S, C, size), w)) return LIEC_EINVAL;
            for (const Span& r : read)
                if (spans_meet(w, r)) return LIEC_EINVAL;
        }
        if (spans_meet(written[2], dws) || spans_meet(written[2], dbs)) return LIEC_EINVAL;
        if (dx) {
            const ImageSpans out = image_spans(dx, N, B, S, C, size);
            if (!apart(dx, N, B, S, C)) return LIEC_EINVAL;
            for (const liec_images* m : {dy, x})
                if (m && !same(dx, m, N, B, S) && images_meet(out, image_spans(m, N, B, S, C, size))) return LIEC_EINVAL;
            for (const Span& r : read)
                if (images_meet(out, r)) return LIEC_EINVAL;
        }
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    const GnBackward a{N, shape_of(N, B, S, C, G), shape_of(N, B, S, C, G, kGnBlocks), images_of(dy), images_of(x), images_of(dx), saved_of(saved),
                       param_of(weight, param_dtype), param_of(bias, param_dtype), param_of(dweight, param_dtype), param_of(dbias, param_dtype), mean, rstd,
                       static_cast<double*>(workspace), reinterpret_cast<float*>(static_cast<char*>(workspace) + (empty ? 0 : gn_run_bytes(C))),
                       empty ? 0 : need - gn_run_bytes(C), keeps((int64_t)N * B * S * C * size), st};
    if (empty) gn_after_sums(a, 0, nullptr, true, true);
    else if (dx || dweight || dbias)
        dtype == LIEC_F32 ? gn_backward_of<float>(a, activation) : dtype == LIEC_BF16 ? gn_backward_of<bf16>(a, activation) : gn_backward_of<f16>(a, activation);
    return launched();
}

int64_t liec_weight_grad_workspace(int32_t N, int64_t R, int64_t O, int64_t C) {
    if (!valid_weight(N, R, O, C)) return -1;
    const WgShape s = weight_shape(N, R, O, C);
    return s.splits > 1 ? s.splits * (int64_t)N * O * (C + 1) * (int64_t)sizeof(float) : 0;
}

liec_status liec_weight_grad(const liec_rows* dy, const liec_checkpoint* saved, const liec_matrices* dweight, const liec_param* dbias, int32_t N, int64_t R, int64_t O,
                             int64_t C, liec_dtype dtype, liec_dtype param_dtype, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!valid_weight(N, R, O, C) || !valid_type(dtype) || !valid_type(param_dtype)) return LIEC_EINVAL;
    const int64_t size = size_of(dtype), psize = size_of(param_dtype), need = liec_weight_grad_workspace(N, R, O, C);
    if (dbias && !dbias->data) dbias = nullptr;
    if (!dweight) return LIEC_EINVAL;
    const liec_rows out{dweight->data, dweight->worker_stride, dweight->row_stride};
    if (!valid_rows(&out, N, O, psize) || !apart(&out, N, O, C) || !valid_param(dbias, psize)) return LIEC_EINVAL;
    if (dbias && N > 1 && llabs(dbias->stride) < O) return LIEC_EINVAL;
    if (need && !valid_workspace(workspace, workspace_bytes, need)) return LIEC_EINVAL;
    const Span dws = span_of_rows(&out, N, O, C, psize), dbs = span_of_param(dbias, N, O, psize), scratch = span_of(workspace, need);
    if (spans_meet(dws, dbs) || spans_meet(dws, scratch) || spans_meet(dbs, scratch)) return LIEC_EINVAL;
    if (R) {
        if (!valid_rows(dy, N, R, size) || !valid_saved(saved)) return LIEC_EINVAL;
        for (const Span& r : {span_of_rows(dy, N, R, O, size), span_of_values(saved, N * R, C), span_of_exponents(saved, N * R, C)})
            if (spans_meet(dws, r) || spans_meet(dbs, r) || spans_meet(scratch, r)) return LIEC_EINVAL;
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    const WgShape s = weight_shape(N, R, O, C);
    const LnRows g = R ? rows_of(dy) : LnRows{nullptr, 0, 0};
    const WgOut dw{dweight->data, dweight->worker_stride, dweight->row_stride, (uint32_t)param_dtype};
    const LnParam db = param_of(dbias, param_dtype);
    const Saved from = R ? saved_of(saved) : Saved{nullptr, nullptr};
    float* const partial = s.splits > 1 ? static_cast<float*>(workspace) : nullptr;
    if (dtype == LIEC_F32) weight_grad_of<float>(s, g, from, dw, db, partial, st);
    else if (dtype == LIEC_BF16) weight_grad_of<bf16>(s, g, from, dw, db, partial, st);
    else weight_grad_of<f16>(s, g, from, dw, db, partial, st);
    return launched();
}

}  // extern "C"
