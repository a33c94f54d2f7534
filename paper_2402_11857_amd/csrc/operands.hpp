// Operands of the operators around the backward pass as their entry points check them: types, alignment, strides, and which of
// them share memory.  Host code.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "liec_train.h"
#include "spans.hpp"

namespace liec {

constexpr int32_t kMaxWorkers = 65535;
inline bool valid_type(int t) { return t == LIEC_F32 || t == LIEC_BF16 || t == LIEC_F16; }
inline int64_t size_of(int t) { return t == LIEC_F32 ? 4 : 2; }
inline bool aligned_to(const void* p, int64_t size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline liec_status launched() { return hipGetLastError() == hipSuccess ? LIEC_OK : LIEC_EDEVICE; }
inline bool valid_workspace(const void* ws, int64_t bytes, int64_t need) { return ws && aligned_to(ws, 16) && bytes >= need; }

constexpr int64_t kMostValues = (int64_t)1 << 40;
inline bool in_range(int64_t stride) { return stride >= -kMostValues && stride <= kMostValues; }
inline bool valid_rows(const liec_rows* r, int32_t N, int64_t R, int64_t size) {
    if (!r || !r->data || !aligned_to(r->data, size) || !in_range(r->worker_stride) || !in_range(r->row_stride)) return false;
    return (double)(R - 1) * (double)llabs(r->row_stride) + (double)(N - 1) * (double)llabs(r->worker_stride) <= (double)kMostValues;
}
inline bool valid_param(const liec_param* p, int64_t size) { return !p || !p->data || (aligned_to(p->data, size) && in_range(p->stride)); }
// Rows that are written must not share memory: the wider of the two strides spans what the narrower one covers.
inline bool apart(const liec_rows* r, int32_t N, int64_t R, int64_t C) {
    int64_t s = llabs(r->row_stride), n = R, wide = llabs(r->worker_stride), many = N;
    if (many == 1 || (n > 1 && wide < s)) {
        std::swap(s, wide);
        std::swap(n, many);
    }
    return (n == 1 || s >= C) && (many == 1 || wide >= (n - 1) * s + C);
}
inline bool same(const liec_rows* a, const liec_rows* b, int32_t N, int64_t R) {
    return a->data == b->data && (N == 1 || a->worker_stride == b->worker_stride) && (R == 1 || a->row_stride == b->row_stride);
}
inline Span span_of_rows(const liec_rows* r, int32_t N, int64_t R, int64_t C, int64_t size) {
    return span_of(r->data, C * size, r->row_stride * size, R, r->worker_stride * size, N);
}
// An output may be an input, and must not share memory with it otherwise.
inline bool may_write(const liec_rows* out, const liec_rows* in, int32_t N, int64_t R, int64_t C, int64_t size) {
    return same(out, in, N, R) || !spans_meet(span_of_rows(out, N, R, C, size), span_of_rows(in, N, R, C, size));
}
inline Span span_of_param(const liec_param* p, int32_t N, int64_t C, int64_t size) {
    return p && p->data ? span_of(p->data, C * size, p->stride * size, N) : Span();
}
// A weight gradient may take the place of the weight, row by row: a block has read what it replaces.
inline bool may_replace(const liec_param* out, const liec_param* in, int32_t N, int64_t C, int64_t size) {
    if (in && out && in->data && in->data == out->data && (N == 1 || in->stride == out->stride)) return true;
    return !spans_meet(span_of_param(out, N, C, size), span_of_param(in, N, C, size));
}

}  // namespace liec
