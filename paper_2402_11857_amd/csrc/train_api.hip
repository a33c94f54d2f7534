// Host side of include/liec_train.h: argument checks, launch shapes, launches.
#include "liec_train.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "kernels/grads.hpp"
#include "kernels/layer_norm.hpp"
#include "operands.hpp"

using namespace liec;

namespace {

constexpr int64_t kMaxGradValues = (int64_t)1 << 35;
// Thread blocks of a launch that adds up squares, 16 per compute unit; six of them are resident at a time (norm of 16 x 11.7M
// fp32 values: 2048 blocks 123 us, 4096 114).
constexpr int64_t kGradBlocks = 4096;
// Blocks of a launch whose partial sums the blocks of the scaling kernel add up again, each of them (138M values of one worker
// clipped: 512 blocks 283 us, 1024 263, 2048 273, 4096 295).  Several launches leave up to 4096 partial sums in all.
constexpr int64_t kGradParts = 1024;
// Workers with more gradients than this are squared and scaled one after the other, all others together: many launches against a
// second pass that finds nothing of the first in the caches.  One by one and together, 16 workers in bf16: clipped, 100 MB each 905
// against 783 to 806 us, 220 MB 1790 against 1748 to 1798, 270 MB 2180 against 2169 to 2230, 330 MB 2648 against 2664 to 2738; into
// rows 100 MB 1049 against 1122 to 1141, 270 MB 2746 against 3169 to 3241.  Rows would gain from 140 MB on (4 workers: 352 against 364).
constexpr int64_t kGradRowBytes = (int64_t)256 << 20;

// ---- gradients -------------------------------------------------------------------------------------------------------
// Launches that T tensors take, at most.
int64_t grad_batches(int32_t T) { return std::max<int64_t>(1, ceil_div(T, GradTable<true>::most)); }

// Partial sums of a worker that a launch may leave: what the workspace has room for.
int64_t grad_parts_per_batch(int32_t N, int32_t T) {
    return std::max<int64_t>(1, std::min<int64_t>(kGradBlocks, 16 * kGradBlocks / N) / grad_batches(T));
}

bool valid_grads(const liec_grad_tensor* t, int32_t T, int32_t N, int64_t* total) {
    if (N < 1 || N > kMaxWorkers || T < 0 || T > LIEC_GRAD_MAX_TENSORS || (T && !t)) return false;
    int64_t sum = 0;
    for (int32_t i = 0; i < T; ++i) {
        if (t[i].count < 0 || t[i].count > kMaxGradValues || !valid_type(t[i].dtype)) return false;
        sum += t[i].count;
        if (sum > kMaxGradValues) return false;
        if (t[i].count && (!t[i].data || !aligned_to(t[i].data, size_of(t[i].dtype)))) return false;
        if (t[i].stride > kMaxGradValues || t[i].stride < -kMaxGradValues) return false;
    }
    *total = sum;
    return true;
}

// Where worker 0's values to worker N - 1's of a tensor lie.
Span span_of_grads(const liec_grad_tensor& t, int32_t N) {
    const int64_t size = size_of(t.dtype);
    return span_of(t.data, t.count * size, t.stride * size, N);
}

// Do any two tensors, or two workers' values of one, share memory?  May throw std::bad_alloc.
bool grads_meet(const liec_grad_tensor* t, int32_t T, int32_t N) {
    std::vector<Span> all;
    all.reserve((size_t)T);
    for (int32_t i = 0; i < T; ++i) {
        if (t[i].count && N > 1 && llabs(t[i].stride) < t[i].count) return true;
        all.push_back(span_of_grads(t[i], N));
    }
    return any_meet(all);
}

// The norms of N workers and the partial sums are written while other blocks read the gradients, and the norms while others read
// the partial sums.  `after`: the norms come from a launch of their own, when the gradients have been read.
bool grads_apart_from(const liec_grad_tensor* t, int32_t T, int32_t N, const float* norms, bool after, const void* workspace) {
    const Span n = span_of(norms, (int64_t)N * 4), ws = span_of(workspace, liec_grads_workspace(N, T));
    if (span_meets(ws, n.lo, n.hi)) return false;
    for (int32_t i = 0; i < T; ++i) {
        const Span g = span_of_grads(t[i], N);
        if ((!after && span_meets(g, n.lo, n.hi)) || span_meets(g, ws.lo, ws.hi)) return false;
    }
    return true;
}

struct GradBatch {
    int32_t first, count;
    int64_t tiles, blocks, col;               // col: column of its first tensor
};

struct GradPlan {
    int64_t parts = 0, bytes = 0;             // of a worker: partial sums, gradients
    bool strided = false;                     // some tensor's workers do not follow one another
    std::vector<GradBatch> batches;           // those that have any values
};

// `rows`: workers that a launch works on.
bool plan_grads(const liec_grad_tensor* t, int32_t T, int32_t N, int64_t rows, bool scales, GradPlan* out) {
    try {
        const int64_t wanted = std::max<int64_t>(1, std::min(kGradBlocks / rows, scales ? kGradParts : kGradBlocks));
        const int64_t most = std::min(grad_parts_per_batch(N, T), wanted);
        out->strided = false;
        for (int32_t i = 0; i < T; ++i) out->strided = out->strided || (N > 1 && t[i].stride != t[i].count);
        const int64_t carries = out->strided ? GradTable<true>::most : GradTable<false>::most, share = ceil_div(T, std::max<int64_t>(1, ceil_div(T, carries)));
        int64_t col = 0;
        out->parts = out->bytes = 0;
        out->batches.clear();
        for (int64_t b = 0; b < T; b += share) {
            GradBatch g{(int32_t)b, (int32_t)std::min<int64_t>(share, T - b), 0, 0, col};
            for (int32_t i = 0; i < g.count; ++i) {
                const int64_t bytes = t[b + i].count * size_of(t[b + i].dtype);
                g.tiles += ceil_div(bytes, kGradTile);
                out->bytes += bytes;
                col += t[b + i].count;
            }
            if (!g.tiles) continue;
            g.blocks = std::min(ceil_div(g.tiles, kGradWaves), most);
            out->parts += g.blocks;
            out->batches.push_back(g);
        }
    } catch (const std::bad_alloc&) {
        return false;
    }
    return true;
}

template <bool STRIDED>
void fill_table(const liec_grad_tensor* t, const GradBatch& g, GradTable<STRIDED>* tab) {
    int64_t col = g.col;
    uint32_t tile = 0;
    for (int32_t i = 0; i < g.count; ++i) {
        const liec_grad_tensor& s = t[g.first + i];
        tab->data[i] = s.data;
        tab->set_stride(i, s.stride);
        tab->col[i] = col;
        tab->first[i] = tile;
        tab->type[i] = (uint8_t)s.dtype;
        col += s.count;
        tile += (uint32_t)ceil_div(s.count * size_of(s.dtype), kGradTile);
    }
    tab->col[g.count] = col;
    tab->first[g.count] = tile;
}

struct GradCall {
    const liec_grad_tensor* t;
    int32_t T, N;
    float* rows;                              // nullptr: in place
    int64_t row_stride;
    float bound, *norms;
    double* partial;
    hipStream_t st;
};

GradPass pass_of(const GradCall& c, const GradPlan& plan, const GradBatch& g, bool sums, int64_t row, uint32_t slot) {
    return GradPass{c.partial, sums ? (uint32_t)plan.parts : 0u, slot, (uint32_t)row, (uint32_t)g.tiles, (uint32_t)g.count, c.bound, c.norms, c.rows, c.row_stride};
}

template <bool STRIDED>
void launch_squares(const GradCall& c, const GradPlan& plan, int64_t row, int64_t rows, bool stream) {
    uint32_t slot = 0;
    GradTable<STRIDED> tab;
    for (const GradBatch& g : plan.batches) {
        fill_table(c.t, g, &tab);
        const GradPass a = pass_of(c, plan, g, true, row, slot);
        const dim3 grid((uint32_t)g.blocks, (uint32_t)rows);
        if (stream) k_grad_squares<true, STRIDED><<<grid, kBlock, 0, c.st>>>(a, tab);
        else k_grad_squares<false, STRIDED><<<grid, kBlock, 0, c.st>>>(a, tab);
        slot += (uint32_t)g.blocks;
    }
}

template <bool STRIDED>
void launch_scale(const GradCall& c, const GradPlan& plan, bool sums, int64_t row, int64_t rows) {
    GradTable<STRIDED> tab;
    for (const GradBatch& g : plan.batches) {
        fill_table(c.t, g, &tab);
        const GradPass a = pass_of(c, plan, g, sums, row, 0);
        const dim3 grid((uint32_t)ceil_div(g.tiles, kGradWaves), (uint32_t)rows);
        if (c.rows) k_grad_scale<true, STRIDED><<<grid, kBlock, 0, c.st>>>(a, tab);
        else k_grad_scale<false, STRIDED><<<grid, kBlock, 0, c.st>>>(a, tab);
    }
}

liec_status run_grads(const GradCall& c) {
    const int64_t N = c.N;
    const bool scales = c.rows || c.bound < INFINITY, sums = c.norms || c.bound < INFINITY;
    GradPlan plan;
    if (!plan_grads(c.t, c.T, c.N, N, scales, &plan)) return LIEC_ENOMEM;
    int64_t group = N;
    if (scales && sums && N > 1 && plan.bytes > kGradRowBytes) {
        group = 1;
        if (!plan_grads(c.t, c.T, c.N, group, scales, &plan)) return LIEC_ENOMEM;
    }
    for (int64_t r = 0; r < N; r += group) {
        if (sums) (plan.strided ? launch_squares<true> : launch_squares<false>)(c, plan, r, group, !scales);
        if (scales) (plan.strided ? launch_scale<true> : launch_scale<false>)(c, plan, sums, r, group);
    }
    if (c.norms && (!scales || plan.batches.empty())) k_grad_norms<<<(uint32_t)N, kBlock, 0, c.st>>>(c.partial, (uint32_t)plan.parts, c.norms);
    return launched();
}

// ---- layer normalisation ---------------------------------------------------------------------------------------------
constexpr int64_t kLnMost = 16384;                                   // columns that a team holds

constexpr int64_t kLnWideBlocks = 65536;                             // that walk rows no team holds

struct Team {
    int lanes, eights;                 // lanes to a row, columns of a lane in eights
};
// The smallest team that holds a row, for the forward pass, which has registers for four eights per lane (8 x 30000 rows of
// 1024 bf16 columns 162 us, with 64 lanes of two 175; 200 MB in rows of 2000 64 against 73 with 128 lanes and a barrier), ...
Team forward_team(int64_t C) {
    if (C <= 64) return {8, 1};
    if (C <= 128) return {16, 1};
    if (C <= 256) return {16, 2};
    if (C <= 512) return {32, 2};
    if (C <= 1024) return {32, 4};
    if (C <= 2048) return {64, 4};
    if (C <= 4096) return {128, 4};
    if (C <= 8192) return {256, 4};
    return {512, 4};
}
// ... and for the backward pass, whose lanes also hold the weight gradients of their columns.
Team backward_team(int64_t C) {
    if (C <= 64) return {8, 1};
    if (C <= 128) return {16, 1};
    if (C <= 256) return {16, 2};
    if (C <= 512) return {32, 2};
    if (C <= 1024) return {64, 2};
    if (C <= 2048) return {128, 2};
    if (C <= 4096) return {256, 2};
    if (C <= 8192) return {512, 2};
    return {1024, 2};
}
int64_t threads_of(const Team& t) { return t.lanes > 64 ? t.lanes : kBlock; }
int64_t teams_of(const Team& t) { return threads_of(t) / t.lanes; }

bool holds(int64_t C) { return C >= kLnShortest && C <= kLnMost; }

struct Strips {
    int64_t per, count;
};
// Rows of a block: `waves` on each of the chip's 1024 SIMDs, and two rows for each of a block's teams at least.
Strips strips_of(int32_t N, int64_t R, const Team& t, int64_t waves) {
    const int64_t want = std::max<int64_t>(1, 1024 * 64 * waves / threads_of(t) / N);
    const int64_t per = std::max(ceil_div(R, want), 2 * teams_of(t));
    return {per, ceil_div(R, per)};
}

// Strips of the backward pass, each with partial sums of its own: as many blocks as are resident at a time.  Weight gradients
// stay in registers; one vector per lane leaves room for four waves (six: as fast or 2 to 30 % slower); of two per lane two
// waves that request two rows ahead beat four that request one (2048 columns 156 against 166 us, 8192 286 against 299); 16
// waves to a row are four by themselves.  A team adds up at most kLnChain rows in fp32; where that takes more blocks, they are a
// multiple of those that are resident.
constexpr int64_t kLnChain = 256;
Strips backward_strips(int32_t N, int64_t R, int64_t C) {
    if (R == 0) return {1, 0};
    if (!holds(C)) {                   // the columns' sums, a thread per column
        const int64_t per = ceil_div(R, std::max<int64_t>(1, 1024 / N / ceil_div(C, kBlock)));
        return {per, ceil_div(R, per)};
    }
    const Team t = backward_team(C);
    // few rows: one block, whose sums need no second kernel
    if (R <= 8 * teams_of(t)) return {R, 1};
    const Strips s = strips_of(N, R, t, t.eights == 1 || t.lanes == 1024 ? 4 : 2);
    const int64_t rounds = ceil_div(s.per, kLnChain * teams_of(t));
    if (rounds == 1) return s;
    const int64_t per = ceil_div(R, s.count * rounds);
    return {per, ceil_div(R, per)};
}

LnRows rows_of(const liec_rows* r) { return r ? LnRows{r->data, r->worker_stride, r->row_stride} : LnRows{nullptr, 0, 0}; }
LnParam param_of(const liec_param* p, int type) { return p && p->data ? LnParam{p->data, p->stride, (uint32_t)type} : LnParam{nullptr, 0, (uint32_t)type}; }

bool valid_sizes(int32_t N, int64_t R, int64_t C) {
    if ((double)N * (double)R * (double)C > (double)kMostValues) return false;
    return N >= 1 && N <= kMaxWorkers && R >= 0 && R < ((int64_t)1 << 31) && C >= 1 && C <= ((int64_t)1 << 28);
}

struct LnForward {
    LnRows x, y;
    LnParam w, b;
    float *mean, *rstd, eps;
    int32_t N;
    int64_t R, C;
    hipStream_t st;
};

// Results of up to the memory-side cache's 256 MB are left there for the operation that reads them next, larger ones are
// streamed past it: rows of 2000 bf16 columns, 200 MB 73.4 against 76.6 us forward and 108 against 119 us backward, 400 MB
// 157 against 148 and 259 against 238.
bool keeps(int32_t N, int64_t R, int64_t C, int64_t size) { return N * R * C * size <= (int64_t)256 << 20; }

template <typename T, int TEAM, int EIGHTS>
void run_forward(const LnForward& a) {
    constexpr int K = EIGHTS * 8 / Vec16<T>::n, threads = TEAM > 64 ? TEAM : kBlock;
    const bool full = a.C == TEAM * EIGHTS * 8;
    // Many short-lived blocks: 8 x 8192 rows of 4096 bf16 columns 181 us, blocks that stay on the chip and request rows ahead
    // 194 to 220, although every block reads the weights again.
    const Strips s = strips_of(a.N, a.R, Team{TEAM, EIGHTS}, 32);
    const bool keep = keeps(a.N, a.R, a.C, sizeof(T));
    const dim3 grid((uint32_t)s.count, (uint32_t)a.N);
    if (full)
        k_ln_forward<T, TEAM, K, true><<<grid, threads, 0, a.st>>>((uint32_t)a.C, a.eps, a.R, keep, a.mean, a.rstd, a.x, a.y, a.w, a.b);
    else
        k_ln_forward<T, TEAM, K, false><<<grid, threads, 0, a.st>>>((uint32_t)a.C, a.eps, a.R, keep, a.mean, a.rstd, a.x, a.y, a.w, a.b);
}

template <typename T>
void forward_of(const LnForward& a) {
    if (!holds(a.C)) {
        k_ln_forward_wide<T><<<dim3((uint32_t)std::min(a.R, kLnWideBlocks), (uint32_t)a.N), a.C < kLnShortest ? 64 : kLnWide, 0, a.st>>>(
            a.C, a.eps, a.R, a.mean, a.rstd, a.x, a.y, a.w, a.b);
        return;
    }
    const Team t = forward_team(a.C);
    switch (t.lanes * t.eights) {
        case 8: return run_forward<T, 8, 1>(a);
        case 16: return run_forward<T, 16, 1>(a);
        case 32: return run_forward<T, 16, 2>(a);
        case 64: return run_forward<T, 32, 2>(a);
        case 128: return run_forward<T, 32, 4>(a);
        case 256: return run_forward<T, 64, 4>(a);
        case 512: return run_forward<T, 128, 4>(a);
        case 1024: return run_forward<T, 256, 4>(a);
        default: return run_forward<T, 512, 4>(a);
    }
}

struct LnBackward {
    LnRows dy, x, dx;
    LnParam w, dw, db;
    const float *mean, *rstd;
    float* partial;
    int32_t N;
    int64_t R, C;
    Strips strips;
    hipStream_t st;
};

template <typename T, int TEAM, int EIGHTS>
void run_backward(const LnBackward& a) {
    constexpr int K = EIGHTS * 8 / Vec16<T>::n, threads = TEAM > 64 ? TEAM : kBlock;
    // Rows requested ahead: what registers allow.  Of 16-bit rows of 4096 columns three (two: 279.5 against 273 us for 8 x 8192
    // rows, 287 against 275 for 4000 columns), of others two (5000 bf16 columns 266 against 334 us, 1000 fp32 columns 296
    // against 322).
    constexpr int P = EIGHTS == 1 || TEAM == 1024 ? 1 : TEAM == 256 && sizeof(T) == 2 ? 3 : 2;
    const bool full = a.C == TEAM * EIGHTS * 8;
    const bool keep = keeps(a.N, a.R, a.C, sizeof(T));
    const dim3 grid((uint32_t)a.strips.count, (uint32_t)a.N);
    if (full)
        k_ln_backward<T, TEAM, K, true, P><<<grid, threads, 0, a.st>>>((uint32_t)a.C, a.R, keep, a.partial, a.mean, a.rstd, a.dy, a.x, a.dx, a.w, a.dw, a.db);
    else
        k_ln_backward<T, TEAM, K, false, P><<<grid, threads, 0, a.st>>>((uint32_t)a.C, a.R, keep, a.partial, a.mean, a.rstd, a.dy, a.x, a.dx, a.w, a.dw, a.db);
}

template <typename T>
void backward_of(const LnBackward& a) {
    if (!holds(a.C)) {
        // the columns first: dx may take the place of dy or x
        if (a.dw.data || a.db.data)
            k_ln_columns_wide<T><<<dim3((uint32_t)ceil_div(a.C, kBlock), (uint32_t)a.N, (uint32_t)a.strips.count), kBlock, 0, a.st>>>(
                a.C, a.strips.per, a.R, a.partial, a.mean, a.rstd, a.dy, a.x);
        if (a.dx.data)
            k_ln_backward_wide<T><<<dim3((uint32_t)std::min(a.R, kLnWideBlocks), (uint32_t)a.N), a.C < kLnShortest ? 64 : kLnWide, 0, a.st>>>(
                a.C, a.R, a.mean, a.rstd, a.dy, a.x, a.dx, a.w);
        return;
    }
    const Team t = backward_team(a.C);
    switch (t.lanes * t.eights) {
        case 8: return run_backward<T, 8, 1>(a);
        case 16: return run_backward<T, 16, 1>(a);
        case 32: return run_backward<T, 16, 2>(a);
        case 64: return run_backward<T, 32, 2>(a);
        case 128: return run_backward<T, 64, 2>(a);
        case 256: return run_backward<T, 128, 2>(a);
        case 512: return run_backward<T, 256, 2>(a);
        case 1024: return run_backward<T, 512, 2>(a);
        default: return run_backward<T, 1024, 2>(a);
    }
}

}  // namespace

extern "C" {

int64_t liec_grads_workspace(int32_t N, int32_t T) {
    if (N < 1 || N > kMaxWorkers || T < 0 || T > LIEC_GRAD_MAX_TENSORS) return -1;
    return (int64_t)N * grad_batches(T) * grad_parts_per_batch(N, T) * (int64_t)sizeof(double);
}

liec_status liec_grad_norm(const liec_grad_tensor* tensors, int32_t T, int32_t N, float* norms, void* workspace, int64_t workspace_bytes,
                           void* hip_stream) {
    int64_t total = 0;
    if (!valid_grads(tensors, T, N, &total) || !norms || !aligned_to(norms, 4)) return LIEC_EINVAL;
    if (!valid_workspace(workspace, workspace_bytes, liec_grads_workspace(N, T))) return LIEC_EINVAL;
    if (!grads_apart_from(tensors, T, N, norms, true, workspace)) return LIEC_EINVAL;
    return run_grads(GradCall{tensors, T, N, nullptr, 0, INFINITY, norms, static_cast<double*>(workspace), (hipStream_t)hip_stream});
}

liec_status liec_clip_grads(const liec_grad_tensor* tensors, int32_t T, int32_t N, float max_norm, float* norms, void* workspace,
                            int64_t workspace_bytes, void* hip_stream) {
    int64_t total = 0;
    if (!valid_grads(tensors, T, N, &total) || !aligned_to(norms, 4) || !(max_norm >= 0.f)) return LIEC_EINVAL;
    if (!valid_workspace(workspace, workspace_bytes, liec_grads_workspace(N, T))) return LIEC_EINVAL;
    if (!grads_apart_from(tensors, T, N, norms, false, workspace)) return LIEC_EINVAL;
    try {
        if (grads_meet(tensors, T, N)) return LIEC_EINVAL;
    } catch (const std::bad_alloc&) {
        return LIEC_ENOMEM;
    }
    return run_grads(GradCall{tensors, T, N, nullptr, 0, max_norm, norms, static_cast<double*>(workspace), (hipStream_t)hip_stream});
}

liec_status liec_gather_grads(const liec_grad_tensor* tensors, int32_t T, int32_t N, float* rows, int64_t row_stride, float max_norm, float* norms,
                              void* workspace, int64_t workspace_bytes, void* hip_stream) {
    int64_t total = 0;
    if (!valid_grads(tensors, T, N, &total) || !aligned_to(norms, 4) || !(max_norm >= 0.f)) return LIEC_EINVAL;
    if (total && (!rows || !aligned_to(rows, 4))) return LIEC_EINVAL;
    if (N > 1 && (row_stride < total || row_stride > kMaxGradValues)) return LIEC_EINVAL;
    if (!valid_workspace(workspace, workspace_bytes, liec_grads_workspace(N, T))) return LIEC_EINVAL;
    const Span written = span_of(rows, total * 4, N > 1 ? row_stride * 4 : 0, N);
    if (norms || max_norm < INFINITY) {
        const Span n = span_of(norms, (int64_t)N * 4), ws = span_of(workspace, liec_grads_workspace(N, T));
        if (!grads_apart_from(tensors, T, N, norms, false, workspace) || span_meets(written, n.lo, n.hi) || span_meets(written, ws.lo, ws.hi))
            return LIEC_EINVAL;
    }
    int64_t steps = kSpanSteps;
    for (int32_t i = 0; i < T; ++i)
        if (spans_meet(written, span_of_grads(tensors[i], N), steps)) return LIEC_EINVAL;
    return run_grads(GradCall{tensors, T, N, rows, row_stride, max_norm, norms, static_cast<double*>(workspace), (hipStream_t)hip_stream});
}

liec_status liec_layer_norm(const liec_rows* x, const liec_param* weight, const liec_param* bias, const liec_rows* y, float* mean, float* rstd, int32_t N,
                            int64_t R, int64_t C, float eps, liec_dtype dtype, liec_dtype param_dtype, void* hip_stream) {
    if (!valid_sizes(N, R, C) || !valid_type(dtype) || !valid_type(param_dtype) || !(eps >= 0.f) || !isfinite(eps)) return LIEC_EINVAL;
    if (R == 0) return LIEC_OK;
    const int64_t size = size_of(dtype), psize = size_of(param_dtype);
    if (!valid_rows(x, N, R, size) || !valid_rows(y, N, R, size) || !valid_param(weight, psize) || !valid_param(bias, psize)) return LIEC_EINVAL;
    if (!aligned_to(mean, 4) || !aligned_to(rstd, 4) || !apart(y, N, R, C) || !may_write(y, x, N, R, C, size)) return LIEC_EINVAL;
    const Span ys = span_of_rows(y, N, R, C, size), ws = span_of_param(weight, N, C, psize), bs = span_of_param(bias, N, C, psize);
    const Span ms = span_of(mean, N * R * 4), rs = span_of(rstd, N * R * 4);
    if (spans_meet(ms, rs) || spans_meet(ys, ws) || spans_meet(ys, bs)) return LIEC_EINVAL;
    for (const Span& p : {span_of_rows(x, N, R, C, size), ys, ws, bs})
        if (spans_meet(ms, p) || spans_meet(rs, p)) return LIEC_EINVAL;
    const LnForward a{rows_of(x), rows_of(y), param_of(weight, param_dtype), param_of(bias, param_dtype), mean, rstd, eps, N, R, C, (hipStream_t)hip_stream};
    if (dtype == LIEC_F32) forward_of<float>(a);
    else if (dtype == LIEC_BF16) forward_of<bf16>(a);
    else forward_of<f16>(a);
    return launched();
}

int64_t liec_layer_norm_workspace(int32_t N, int64_t R, int64_t C) {
    if (!valid_sizes(N, R, C)) return -1;
    return (int64_t)N * backward_strips(N, R, C).count * 2 * C * (int64_t)sizeof(float);
}

liec_status liec_layer_norm_backward(const liec_rows* dy, const liec_rows* x, const float* mean, const float* rstd, const liec_param* weight,
                                     const liec_rows* dx, const liec_param* dweight, const liec_param* dbias, int32_t N, int64_t R, int64_t C,
                                     liec_dtype dtype, liec_dtype param_dtype, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (!valid_sizes(N, R, C) || !valid_type(dtype) || !valid_type(param_dtype)) return LIEC_EINVAL;
    const int64_t size = size_of(dtype), psize = size_of(param_dtype);
    if (!valid_param(weight, psize) || !valid_param(dweight, psize) || !valid_param(dbias, psize)) return LIEC_EINVAL;
    const bool params = (dweight && dweight->data) || (dbias && dbias->data);
    if (dx && !dx->data) dx = nullptr;
    if (R) {
        if (!valid_rows(dy, N, R, size) || !valid_rows(x, N, R, size) || (dx && !valid_rows(dx, N, R, size))) return LIEC_EINVAL;
        if (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return LIEC_EINVAL;
        if (dx && !(apart(dx, N, R, C) && may_write(dx, dy, N, R, C, size) && may_write(dx, x, N, R, C, size))) return LIEC_EINVAL;
        const int64_t need = params ? liec_layer_norm_workspace(N, R, C) : 0;
        if (params && !valid_workspace(workspace, workspace_bytes, need)) return LIEC_EINVAL;
        const Span ms = span_of(mean, N * R * 4), rs = span_of(rstd, N * R * 4), ws = span_of_param(weight, N, C, psize), scratch = span_of(workspace, need);
        if (dx)
            for (const Span& p : {ms, rs, ws})
                if (spans_meet(span_of_rows(dx, N, R, C, size), p)) return LIEC_EINVAL;
        for (const liec_rows* r : {dy, x, dx})
            if (r && spans_meet(span_of_rows(r, N, R, C, size), scratch)) return LIEC_EINVAL;
        for (const Span& p : {ms, rs, ws, span_of_param(dweight, N, C, psize), span_of_param(dbias, N, C, psize)})
            if (spans_meet(p, scratch)) return LIEC_EINVAL;
    }
    if (params) {
        const Span dw = span_of_param(dweight, N, C, psize), db = span_of_param(dbias, N, C, psize);
        if (spans_meet(dw, db) || !may_replace(dweight, weight, N, C, psize) || !may_replace(dbias, weight, N, C, psize)) return LIEC_EINVAL;
        if (R)
            for (const Span& p : {dw, db}) {
                for (const liec_rows* r : {dy, x, dx})
                    if (r && spans_meet(p, span_of_rows(r, N, R, C, size))) return LIEC_EINVAL;
                for (const float* f : {mean, rstd})
                    if (spans_meet(p, span_of(f, N * R * 4))) return LIEC_EINVAL;
            }
        // one sum for all workers, or one for each: the same for both gradients
        if (dweight && dweight->data && dbias && dbias->data && N > 1 && (dweight->stride == 0) != (dbias->stride == 0)) return LIEC_EINVAL;
        if (N > 1)
            for (const liec_param* p : {dweight, dbias})
                if (p && p->data && p->stride && llabs(p->stride) < C) return LIEC_EINVAL;
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    LnBackward a{rows_of(dy), rows_of(x), rows_of(dx), param_of(weight, param_dtype), param_of(dweight, param_dtype), param_of(dbias, param_dtype),
                 mean, rstd, static_cast<float*>(workspace), N, R, C, backward_strips(N, R, C), st};
    const LnParam& any = a.dw.data ? a.dw : a.db;
    const bool shared = any.stride == 0 || N == 1;
    const int64_t parts = shared ? (int64_t)N * a.strips.count : a.strips.count;
    const bool direct = parts == 1 && holds(C);
    if (direct) a.partial = nullptr;
    if (R && (params || a.dx.data)) {
        if (dtype == LIEC_F32) backward_of<float>(a);
        else if (dtype == LIEC_BF16) backward_of<bf16>(a);
        else backward_of<f16>(a);
    }
    if (params && !direct)
        k_ln_param_grads<<<dim3((uint32_t)ceil_div(C, 32), shared ? 1u : (uint32_t)N, 2), kBlock, 0, st>>>(static_cast<const float*>(workspace),
                                                                                                      (uint32_t)parts, C, a.dw, a.db);
    return launched();
}

}  // extern "C"
