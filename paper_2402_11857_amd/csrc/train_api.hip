// Host side of include/liec_train.h: argument checks, launch shapes, launches.
#include "liec_train.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "kernels/grads.hpp"
#include "kernels/layer_norm.hpp"

using namespace liec;

namespace {

constexpr int32_t kMaxWorkers = 65535;
constexpr int64_t kMaxGradValues = (int64_t)1 << 44;
// Thread blocks of a launch over gradients: 16 per compute unit, twice what is resident at a time.
constexpr int64_t kGradBlocks = 4096;

bool valid_type(int t) { return t == LIEC_F32 || t == LIEC_BF16 || t == LIEC_F16; }
int64_t size_of(int t) { return t == LIEC_F32 ? 4 : 2; }
bool aligned_to(const void* p, int64_t size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
liec_status launched() { return hipGetLastError() == hipSuccess ? LIEC_OK : LIEC_EDEVICE; }

// ---- gradients -------------------------------------------------------------------------------------------------------
int64_t grad_batches(int32_t T) { return std::max<int64_t>(1, ceil_div(T, kGradTensors)); }

// Partial sums of a worker that a launch may leave: enough blocks in all to fill the chip, one for each worker at least.
int64_t grad_parts_per_batch(int32_t N, int32_t T) { return std::max<int64_t>(1, kGradBlocks / N / grad_batches(T)); }

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

bool valid_workspace(const void* ws, int64_t bytes, int64_t need) { return ws && aligned_to(ws, 16) && bytes >= need; }

// Do two sets of N equally spaced byte ranges (first starts, lengths, distances) share a byte?
bool ranges_meet(uintptr_t a, int64_t an, int64_t as, uintptr_t b, int64_t bn, int64_t bs, int32_t N) {
    if (an <= 0 || bn <= 0) return false;
    const int64_t last = N - 1, d = (int64_t)(b - a);
    const int64_t alo = std::min<int64_t>(0, as * last), ahi = std::max<int64_t>(0, as * last) + an;
    const int64_t blo = d + std::min<int64_t>(0, bs * last), bhi = d + std::max<int64_t>(0, bs * last) + bn;
    if (bhi <= alo || ahi <= blo) return false;
    if (as != bs || N == 1 || as <= 0) return true;
    // the same distance: columns of one matrix.  Range i of b lies d + (i - j) * as from range j of a.
    int64_t off = d % as;
    if (off < 0) off += as;
    const int64_t row = (d - off) / as;                        // b's range i is off bytes into a's row i + row
    return (off < an && row <= last && row >= -last) || (off + bn > as && row + 1 <= last && row + 1 >= -last);
}

struct GradBatch {
    int32_t first, count;
    int64_t tiles, blocks, per;
};

struct GradLaunch {
    int64_t parts = 0;                        // partial sums per worker
    std::vector<GradBatch> batches;
};

bool plan_grads(const liec_grad_tensor* t, int32_t T, int32_t N, GradLaunch* out) {
    try {
        const int64_t most = grad_parts_per_batch(N, T);
        for (int32_t b = 0; b < T; b += kGradTensors) {
            GradBatch g{b, std::min<int32_t>(kGradTensors, T - b), 0, 0, 0};
            for (int32_t i = 0; i < g.count; ++i) g.tiles += ceil_div(t[b + i].count, kGradTile);
            if (!g.tiles) continue;
            g.per = ceil_div(g.tiles, most);
            g.blocks = ceil_div(g.tiles, g.per);
            out->parts += g.blocks;
            out->batches.push_back(g);
        }
    } catch (const std::bad_alloc&) {
        return false;
    }
    return true;
}

void fill_table(const liec_grad_tensor* t, const GradBatch& g, int64_t col0, GradTable* tab) {
    int64_t col = col0;
    uint32_t tile = 0;
    for (int32_t i = 0; i < g.count; ++i) {
        const liec_grad_tensor& s = t[g.first + i];
        tab->data[i] = s.data;
        tab->stride[i] = s.stride;
        tab->col[i] = col;
        tab->first[i] = tile;
        tab->type[i] = (uint8_t)s.dtype;
        col += s.count;
        tile += (uint32_t)ceil_div(s.count, kGradTile);
    }
    tab->col[g.count] = col;
    tab->first[g.count] = tile;
}

void launch_squares(const liec_grad_tensor* t, int32_t N, const GradLaunch& plan, double* partial, hipStream_t st) {
    uint32_t slot = 0;
    GradTable tab;
    for (const GradBatch& g : plan.batches) {
        fill_table(t, g, 0, &tab);
        k_grad_squares<<<dim3((uint32_t)g.blocks, (uint32_t)N), kBlock, 0, st>>>(partial, (uint32_t)plan.parts, slot, (uint32_t)g.count,
                                                                                 (uint32_t)g.tiles, (uint32_t)g.per, tab);
        slot += (uint32_t)g.blocks;
    }
}

// Norms and scaling; rows == nullptr: in place.
liec_status clip_into(const liec_grad_tensor* t, int32_t T, int32_t N, float* rows, int64_t row_stride, float bound, float* norms, double* partial,
                      hipStream_t st) {
    GradLaunch plan;
    if (!plan_grads(t, T, N, &plan)) return LIEC_ENOMEM;
    const bool sums = norms || bound < INFINITY;
    if (sums) launch_squares(t, N, plan, partial, st);
    if (!rows && bound == INFINITY) {
        // nothing to scale
    } else {
        int64_t col = 0;
        int32_t next = 0;
        GradTable tab;
        for (const GradBatch& g : plan.batches) {
            for (; next < g.first; ++next) col += t[next].count;   // batches without values are left out
            fill_table(t, g, col, &tab);
            k_grad_scale<<<dim3((uint32_t)g.blocks, (uint32_t)N), kBlock, 0, st>>>(partial, sums ? (uint32_t)plan.parts : 0u, bound, norms, rows, row_stride,
                                                                                   (uint32_t)g.count, (uint32_t)g.tiles, (uint32_t)g.per, tab);
        }
    }
    if (norms && ((!rows && bound == INFINITY) || plan.batches.empty()))
        k_grad_norms<<<(uint32_t)N, kBlock, 0, st>>>(partial, (uint32_t)plan.parts, norms);
    return launched();
}

// ---- layer normalisation ---------------------------------------------------------------------------------------------
constexpr int64_t kLnMost = 16384;                                   // columns that a team holds
constexpr int64_t kLnBlocks = 1024;                                  // thread blocks of a launch, 4 per compute unit

struct Team {
    int lanes, vecs;
};
// The smallest team that holds a row.
Team team_of(int64_t C) {
    const int64_t v = ceil_div(C, kLnVec);
    if (v <= 8) return {8, 1};
    if (v <= 16) return {16, 1};
    if (v <= 32) return {32, 1};
    if (v <= 64) return {64, 1};
    if (v <= 128) return {64, 2};
    if (v <= 256) return {128, 2};
    if (v <= 512) return {256, 2};
    if (v <= 1024) return {512, 2};
    return {1024, 2};
}

bool holds(int64_t C) { return C >= kLnVec && C <= kLnMost; }

struct Strips {
    int64_t per, count;
};
// Rows of a block: as many blocks as fill the chip, and two rows for each of its teams at least.
Strips strips_of(int32_t N, int64_t R, int64_t C) {
    if (R == 0) return {1, 0};
    const bool held = holds(C);
    const int64_t teams = held ? std::max(1, kBlock / team_of(C).lanes) : 1;
    // rows that no team holds: the columns' sums, a thread per column
    const int64_t want = std::max<int64_t>(1, kLnBlocks / N / (held ? 1 : ceil_div(C, kBlock)));
    const int64_t per = std::max(ceil_div(R, want), 2 * teams);
    return {per, ceil_div(R, per)};
}

bool valid_rows(const liec_rows* r, int64_t size) {
    const int64_t most = (int64_t)1 << 44;
    return r && r->data && aligned_to(r->data, size) && llabs(r->worker_stride) <= most && llabs(r->row_stride) <= most;
}
bool valid_param(const liec_param* p, int64_t size) {
    return !p || !p->data || (aligned_to(p->data, size) && llabs(p->stride) <= (int64_t)1 << 44);
}
bool same(const liec_rows* a, const liec_rows* b) {
    return a->data == b->data && a->worker_stride == b->worker_stride && a->row_stride == b->row_stride;
}
bool dense(const liec_rows* a, int32_t N, int64_t R, int64_t C) {
    return (R == 1 || a->row_stride == C) && (N == 1 || a->worker_stride == R * C);
}
// An output may be an input, and must not share memory with it otherwise; what is not dense can be told apart by its start only.
bool may_write(const liec_rows* out, const liec_rows* in, int32_t N, int64_t R, int64_t C, int64_t size) {
    if (same(out, in)) return true;
    if (out->data == in->data) return false;
    if (!dense(out, N, R, C) || !dense(in, N, R, C)) return true;
    const uintptr_t a = (uintptr_t)out->data, b = (uintptr_t)in->data, bytes = (uintptr_t)(N * R * C * size);
    return a + bytes <= b || b + bytes <= a;
}
LnRows rows_of(const liec_rows* r) { return r ? LnRows{r->data, r->worker_stride, r->row_stride} : LnRows{nullptr, 0, 0}; }
LnParam param_of(const liec_param* p, int type) { return p && p->data ? LnParam{p->data, p->stride, (uint32_t)type} : LnParam{nullptr, 0, (uint32_t)type}; }

bool valid_sizes(int32_t N, int64_t R, int64_t C) {
    return N >= 1 && N <= kMaxWorkers && R >= 0 && R < ((int64_t)1 << 31) && C >= 1 && C < ((int64_t)1 << 31);
}

struct LnForward {
    LnRows x, y;
    LnParam w, b;
    float *mean, *rstd, eps;
    int32_t N;
    int64_t R, C;
    hipStream_t st;
};

template <typename T, int TEAM, int K>
void run_forward(const LnForward& a) {
    const Strips s = strips_of(a.N, a.R, a.C);
    k_ln_forward<T, TEAM, K><<<dim3((uint32_t)s.count, (uint32_t)a.N), (TEAM > 64 ? TEAM : kBlock), 0, a.st>>>(
        (uint32_t)a.C, (uint32_t)s.per, a.eps, a.R, a.mean, a.rstd, a.x, a.y, a.w, a.b);
}

template <typename T>
void forward_of(const LnForward& a) {
    if (!holds(a.C)) {
        k_ln_forward_wide<T><<<dim3((uint32_t)a.R, (uint32_t)a.N), a.C < kLnVec ? 64 : kLnWide, 0, a.st>>>(a.C, a.eps, a.R, a.mean, a.rstd, a.x, a.y, a.w, a.b);
        return;
    }
    const Team t = team_of(a.C);
    switch (t.lanes * t.vecs) {
        case 8: return run_forward<T, 8, 1>(a);
        case 16: return run_forward<T, 16, 1>(a);
        case 32: return run_forward<T, 32, 1>(a);
        case 64: return run_forward<T, 64, 1>(a);
        case 128: return run_forward<T, 64, 2>(a);
        case 256: return run_forward<T, 128, 2>(a);
        case 512: return run_forward<T, 256, 2>(a);
        case 1024: return run_forward<T, 512, 2>(a);
        default: return run_forward<T, 1024, 2>(a);
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

template <typename T, int TEAM, int K>
void run_backward(const LnBackward& a) {
    k_ln_backward<T, TEAM, K><<<dim3((uint32_t)a.strips.count, (uint32_t)a.N), (TEAM > 64 ? TEAM : kBlock), 0, a.st>>>(
        (uint32_t)a.C, (uint32_t)a.strips.per, a.R, a.partial, a.mean, a.rstd, a.dy, a.x, a.dx, a.w, a.dw, a.db);
}

template <typename T>
void backward_of(const LnBackward& a) {
    if (!holds(a.C)) {
        // the columns first: dx may take the place of dy or x
        if (a.dw.data || a.db.data)
            k_ln_columns_wide<T><<<dim3((uint32_t)ceil_div(a.C, kBlock), (uint32_t)a.N, (uint32_t)a.strips.count), kBlock, 0, a.st>>>(
                a.C, a.strips.per, a.R, a.partial, a.mean, a.rstd, a.dy, a.x);
        if (a.dx.data)
            k_ln_backward_wide<T><<<dim3((uint32_t)a.R, (uint32_t)a.N), a.C < kLnVec ? 64 : kLnWide, 0, a.st>>>(a.C, a.R, a.mean, a.rstd, a.dy, a.x, a.dx, a.w);
        return;
    }
    const Team t = team_of(a.C);
    switch (t.lanes * t.vecs) {
        case 8: return run_backward<T, 8, 1>(a);
        case 16: return run_backward<T, 16, 1>(a);
        case 32: return run_backward<T, 32, 1>(a);
        case 64: return run_backward<T, 64, 1>(a);
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
    return clip_into(tensors, T, N, nullptr, 0, INFINITY, norms, static_cast<double*>(workspace), (hipStream_t)hip_stream);
}

liec_status liec_clip_grads(const liec_grad_tensor* tensors, int32_t T, int32_t N, float max_norm, float* norms, void* workspace,
                            int64_t workspace_bytes, void* hip_stream) {
    int64_t total = 0;
    if (!valid_grads(tensors, T, N, &total) || !aligned_to(norms, 4) || !(max_norm >= 0.f)) return LIEC_EINVAL;
    if (!valid_workspace(workspace, workspace_bytes, liec_grads_workspace(N, T))) return LIEC_EINVAL;
    try {
        std::vector<std::pair<uintptr_t, uintptr_t>> at;       // where worker 0's values start and end
        at.reserve((size_t)T);
        for (int32_t i = 0; i < T; ++i) {
            if (!tensors[i].count) continue;
            if (N > 1 && llabs(tensors[i].stride) < tensors[i].count) return LIEC_EINVAL;
            const uintptr_t p = (uintptr_t)tensors[i].data;
            at.emplace_back(p, p + (uintptr_t)(tensors[i].count * size_of(tensors[i].dtype)));
        }
        std::sort(at.begin(), at.end());
        for (size_t i = 1; i < at.size(); ++i)
            if (at[i].first < at[i - 1].second) return LIEC_EINVAL;
    } catch (const std::bad_alloc&) {
        return LIEC_ENOMEM;
    }
    return clip_into(tensors, T, N, nullptr, 0, max_norm, norms, static_cast<double*>(workspace), (hipStream_t)hip_stream);
}

liec_status liec_gather_grads(const liec_grad_tensor* tensors, int32_t T, int32_t N, float* rows, int64_t row_stride, float max_norm, float* norms,
                              void* workspace, int64_t workspace_bytes, void* hip_stream) {
    int64_t total = 0;
    if (!valid_grads(tensors, T, N, &total) || !aligned_to(norms, 4) || !(max_norm >= 0.f)) return LIEC_EINVAL;
    if (total && (!rows || !aligned_to(rows, 4))) return LIEC_EINVAL;
    if (N > 1 && (row_stride < total || row_stride > kMaxGradValues)) return LIEC_EINVAL;
    if (!valid_workspace(workspace, workspace_bytes, liec_grads_workspace(N, T))) return LIEC_EINVAL;
    for (int32_t i = 0; i < T; ++i) {
        const int64_t s = size_of(tensors[i].dtype);
        if (ranges_meet((uintptr_t)rows, total * 4, row_stride * 4, (uintptr_t)tensors[i].data, tensors[i].count * s, tensors[i].stride * s, N))
            return LIEC_EINVAL;
    }
    return clip_into(tensors, T, N, rows, row_stride, max_norm, norms, static_cast<double*>(workspace), (hipStream_t)hip_stream);
}

liec_status liec_layer_norm(const liec_rows* x, const liec_param* weight, const liec_param* bias, const liec_rows* y, float* mean, float* rstd, int32_t N,
                            int64_t R, int64_t C, float eps, liec_dtype dtype, liec_dtype param_dtype, void* hip_stream) {
    if (!valid_sizes(N, R, C) || !valid_type(dtype) || !valid_type(param_dtype) || !(eps >= 0.f) || !isfinite(eps)) return LIEC_EINVAL;
    if (R == 0) return LIEC_OK;
    const int64_t size = size_of(dtype), psize = size_of(param_dtype);
    if (!valid_rows(x, size) || !valid_rows(y, size) || !valid_param(weight, psize) || !valid_param(bias, psize)) return LIEC_EINVAL;
    if (!aligned_to(mean, 4) || !aligned_to(rstd, 4) || !may_write(y, x, N, R, C, size)) return LIEC_EINVAL;
    const LnForward a{rows_of(x), rows_of(y), param_of(weight, param_dtype), param_of(bias, param_dtype), mean, rstd, eps, N, R, C, (hipStream_t)hip_stream};
    if (dtype == LIEC_F32) forward_of<float>(a);
    else if (dtype == LIEC_BF16) forward_of<bf16>(a);
    else forward_of<f16>(a);
    return launched();
}

int64_t liec_layer_norm_workspace(int32_t N, int64_t R, int64_t C) {
    if (!valid_sizes(N, R, C)) return -1;
    return (int64_t)N * strips_of(N, R, C).count * 2 * C * (int64_t)sizeof(float);
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
        if (!valid_rows(dy, size) || !valid_rows(x, size) || (dx && !valid_rows(dx, size))) return LIEC_EINVAL;
        if (!mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return LIEC_EINVAL;
        if (dx && !(may_write(dx, dy, N, R, C, size) && may_write(dx, x, N, R, C, size))) return LIEC_EINVAL;
        if (params && !valid_workspace(workspace, workspace_bytes, liec_layer_norm_workspace(N, R, C))) return LIEC_EINVAL;
    }
    if (params) {
        // one sum for all workers, or one for each: the same for both gradients
        if (dweight && dweight->data && dbias && dbias->data && N > 1 && (dweight->stride == 0) != (dbias->stride == 0)) return LIEC_EINVAL;
        if (N > 1)
            for (const liec_param* p : {dweight, dbias})
                if (p && p->data && p->stride && llabs(p->stride) < C) return LIEC_EINVAL;
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    LnBackward a{rows_of(dy), rows_of(x), rows_of(dx), param_of(weight, param_dtype), param_of(dweight, param_dtype), param_of(dbias, param_dtype),
                 mean, rstd, static_cast<float*>(workspace), N, R, C, strips_of(N, R, C), st};
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
