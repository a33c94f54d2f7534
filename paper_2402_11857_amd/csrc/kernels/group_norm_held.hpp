// Group normalisation of images whose groups a block holds in registers: memory is read once and written once.
//
// A block takes a span of channels (whole groups) of an image, or of several small ones: 2^lanes_log lanes of 8 channels to a position,
// 2^rows_log positions at a time, 2^images_log images; a thread holds its 8 channels of up to K positions.  Sums go from a
// thread's positions over the lanes of its wave with the same channels to LDS, where a wave adds up a group.
//
//   forward    the mean first, then values and squares around it: the mean is put right by what the values around it sum up to
//   backward   sums of dz and dz (x - mu) per channel, which are also what the weight gradients add up over images, then dx
//
// Narrow spans (down to 32 bytes of a position) let larger images fit; blocks of neighbouring spans run on one die at a time, whose cache
// puts their lines together.
//
// Bound by what a block does one after another, reading, meeting, writing, as far as the compute unit's other block does not fill the
// gaps: 16 x 8 images of 7 x 7 x 2048 fp32, gradients, 43 us (3.6 TB/s; in two passes 72), 8 x 8 of 28 x 28 x 512 bf16 forward with a
// checkpoint 45 us (2.9 TB/s; in two passes 51).  Values are widened anew after each meeting (hide): kept widened they take four
// times the registers, and spill.
#pragma once
#include <type_traits>

#include "group_norm.hpp"

namespace liec {

constexpr int kGnHeldMost = 1024;      // threads

struct GnHeld {
    uint32_t span, spans;              // channels of a block, blocks of an image
    uint32_t lanes_log, rows_log, images_log;
    uint32_t rows;                     // positions of a thread
};

struct GnPlace {                       // of a thread
    uint32_t lane, row, im, first, channels;       // first channel of the block's span, and how many it has
    int64_t set, image;                // the block's images, all of one worker, and the first of them
    GnColumns k;
};
__device__ __forceinline__ int64_t gn_held_works(const GnShape& s, const GnHeld& h) { return (s.images >> h.images_log) * h.spans; }

// Blocks are dealt out to the 8 dies in turn: each takes a range of the work, neighbouring spans after one another.
__device__ __forceinline__ GnPlace gn_place(const GnShape& s, const GnHeld& h, int64_t work) {
    const int64_t works = gn_held_works(s, h), share = works >> 3;
    if (work < share << 3) work = (work & 7) * share + (work >> 3);
    GnPlace p;
    uint32_t span;
    if (works <= 0x7fffffff) {
        const uint32_t i = (uint32_t)work / h.spans;
        span = (uint32_t)work - i * h.spans;
        p.set = i;
    } else {
        p.set = work / h.spans;
        span = (uint32_t)(work - p.set * h.spans);
    }
    p.lane = threadIdx.x & ((1u << h.lanes_log) - 1);
    p.row = threadIdx.x >> h.lanes_log & ((1u << h.rows_log) - 1);
    p.im = threadIdx.x >> (h.lanes_log + h.rows_log);
    p.image = p.set << h.images_log;
    p.first = span * h.span;
    p.channels = min(h.span, s.C - p.first);
    const uint32_t at = p.first + p.lane * 8;
    p.k.any = p.lane * 8 < p.channels;
    p.k.c = min(p.k.any ? at : p.first, s.C - 8);
    p.k.skip = p.k.any ? at - p.k.c : 0;
    return p;
}
// The address of an operand's value: the same base for the block and a distance of less than 2^31 bytes.
template <typename T>
__device__ __forceinline__ T* gn_near(T* base, uint32_t bytes) {
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type byte;
    return reinterpret_cast<T*>(reinterpret_cast<byte*>(base) + bytes);
}

// v of this lane plus v of another.
template <int CTRL>
__device__ __forceinline__ float gn_add_dpp(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Sum over the lanes of a wave that hold the same channels of the same image: those that differ in bits from..to of their number, the
// same two for the whole launch.
__device__ __forceinline__ float gn_rows_sum(float v, uint32_t from, uint32_t to) {
    const auto takes = [&](uint32_t bit) { return from <= bit && bit < to; };
    if (takes(0)) v = gn_add_dpp<0xb1>(v);       // quad_perm 1 0 3 2
    if (takes(1)) v = gn_add_dpp<0x4e>(v);       // quad_perm 2 3 0 1
    if (takes(2)) v += __uint_as_float((uint32_t)__builtin_amdgcn_ds_swizzle((int)__float_as_uint(v), 4 << 10 | 0x1f));      // lane ^ 4
    if (takes(3)) v = gn_add_dpp<0x128>(v);      // row_ror:8
    if (takes(4)) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (takes(5)) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// Where sums lie in LDS: entries (channels, or 8 of them where groups are a multiple of that and nothing asks for a channel's own) of each
// image, each with a place for every wave of the image.
struct GnSums {
    uint32_t entries, waves, group;    // of a span, of an image, entries of a group
    __device__ __forceinline__ GnSums(const GnShape& s, const GnHeld& h, bool eights) {
        const uint32_t threads_log = h.lanes_log + h.rows_log;
        entries = eights ? h.span >> 3 : h.span;
        waves = threads_log > 6 ? 1u << (threads_log - 6) : 1u;
        group = eights ? s.per_group >> 3 : s.per_group;
    }
};
// Adds up a thread's sums over its wave and leaves them in LDS.
__device__ __forceinline__ void gn_leave(float (&v)[8], const GnSums& m, const GnHeld& h, const GnPlace& p, bool eights, float* lds) {
    const uint32_t threads_log = h.lanes_log + h.rows_log, inside = min(threads_log, 6u);
    const bool writes = (threadIdx.x & ((1u << inside) - 1)) >> h.lanes_log == 0 && p.k.any;
    float* const to = lds + p.im * m.entries * m.waves + (threadIdx.x >> 6 & (m.waves - 1));
    if (eights) {
        float t = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        t = gn_rows_sum(t, h.lanes_log, inside);
        if (writes) to[p.lane * m.waves] = t;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = gn_rows_sum(v[j], h.lanes_log, inside);
    if (writes) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= (int)p.k.skip) to[(p.lane * 8 + j - p.k.skip) * m.waves] = v[j];
    }
}
__device__ __forceinline__ float gn_wave_total(float v) {
#pragma unroll
    for (uint32_t bit = 0; bit < 6; ++bit) v = gn_rows_sum(v, bit, bit + 1);
    return v;
}
// For each group of each image: f(number of the group, sums of its entries in `a` and `b`).  A thread to a group where it has few entries,
// a wave otherwise.
template <bool TWO, typename F>
__device__ __forceinline__ void gn_groups_total(const GnShape& s, const GnHeld& h, const GnPlace& p, uint32_t entries, uint32_t waves, uint32_t group, const float* a,
                                                const float* b, F f) {
    const uint32_t groups = p.channels / s.per_group, many = groups << h.images_log, lane = threadIdx.x & 63, each = group * waves;
    const bool few = each <= 16;
    for (uint32_t q = few ? threadIdx.x : threadIdx.x >> 6; q < many; q += few ? blockDim.x : blockDim.x >> 6) {
        const uint32_t im = q / groups, g = q - im * groups, at = (im * entries + g * group) * waves;
        float va = 0.f, vb = 0.f;
        for (uint32_t i = few ? 0 : lane; i < each; i += few ? 1 : 64) {
            va += a[at + i];
            if (TWO) vb += b[at + i];
        }
        if (!few) {
            va = gn_wave_total(va);
            if (TWO) vb = gn_wave_total(vb);
        }
        if (few || lane == 0) f(q, va, vb);
    }
}

template <typename T, int K, int ACT, bool SAVE>
__global__ __launch_bounds__(kGnHeldMost) void k_gn_held(GnShape s, GnHeld h, bool keep, float eps, float* __restrict__ mean, float* __restrict__ rstd, GnImages x, GnImages y,
                                                         LnParam weight, LnParam bias, Saved out) {
    extern __shared__ float gn_lds[];
    const GnSums m(s, h, s.whole);
    float* const sums = gn_lds;
    float* const squares = sums + (m.entries * m.waves << h.images_log);
    float2* const stats = reinterpret_cast<float2*>(squares + (m.entries * m.waves << h.images_log));
    const uint32_t step = 1u << h.rows_log;
    const float n = (float)s.S * (float)s.per_group;
    for (int64_t work = blockIdx.x; work < gn_held_works(s, h); work += gridDim.x) {
        const GnPlace p = gn_place(s, h, work);
        const T* const from = gn_image<const T>(x, s, p.image);
        const uint32_t x_at = (uint32_t)((p.im * x.image + p.row * x.row + p.k.c) * sizeof(T)), x_step = (uint32_t)(step * x.row * sizeof(T));
        GnRaw<T, 8, false> raw[K];
        const int rows = (int)h.rows;
        const GnColumns here{0, p.k.skip, p.k.any};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k] = {};
            if (k < rows && p.row + k * step < s.S) raw[k].load(gn_near(from, x_at + k * x_step), here);
        }
        float v[8], q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < rows && p.row + k * step < s.S) {
                float f[8];
                raw[k].widen(p.k, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += f[j];
            }
        gn_leave(v, m, h, p, s.whole, sums);
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k].hide();
        __syncthreads();
        gn_groups_total<false>(s, h, p, m.entries, m.waves, m.group, sums, sums, [&](uint32_t i, float a, float) { stats[i].x = a / n; });
        __syncthreads();
        const uint32_t groups = p.channels / s.per_group;
        float mu[8];
        gn_each_group<8>(s, p.k.c, [&](int j, uint32_t g) { mu[j] = stats[p.im * groups + min(max(g, p.first / s.per_group) - p.first / s.per_group, groups - 1)].x; });
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = q[j] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < rows && p.row + k * step < s.S) {
                float d[8];
                raw[k].center(p.k, mu, d);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] += d[j];
                    q[j] = __fmaf_rn(d[j], d[j], q[j]);
                }
            }
        gn_leave(v, m, h, p, s.whole, sums);
        gn_leave(q, m, h, p, s.whole, squares);
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k].hide();
        __syncthreads();
        gn_groups_total<true>(s, h, p, m.entries, m.waves, m.group, sums, squares, [&](uint32_t i, float a, float b) {
            const float off = a / n, var = fmaxf(__fmaf_rn(-off, a, b), 0.f) / n + (off - off);
            const float mu = stats[i].x + off, rs = (float)(1.0 / sqrt((double)var + (double)eps));
            stats[i] = make_float2(mu, rs);
        });
        __syncthreads();
        float zw[8], b[8];
        {
            const int64_t worker = gn_worker(s, p.image);
            float w[8];
            gn_param<8>(weight, worker, p.k.c, 1.f, w);
            gn_param<8>(bias, worker, p.k.c, 0.f, b);
            gn_each_group<8>(s, p.k.c, [&](int j, uint32_t g) {
                const float2 t = stats[p.im * groups + min(max(g, p.first / s.per_group) - p.first / s.per_group, groups - 1)];
                mu[j] = t.x;
                zw[j] = t.y * w[j];
            });
        }
        if (p.row == 0)
            for (uint32_t g = p.lane; g < groups; g += 1u << h.lanes_log) {
                const float2 t = stats[p.im * groups + g];
                mean[(p.image + p.im) * s.G + p.first / s.per_group + g] = t.x;
                rstd[(p.image + p.im) * s.G + p.first / s.per_group + g] = t.y;
            }
        T* const to = gn_image<T>(y, s, p.image);
        const uint32_t y_at = (uint32_t)((p.im * y.image + p.row * y.row + p.k.c) * sizeof(T)), y_step = (uint32_t)(step * y.row * sizeof(T));
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < rows && p.row + k * step < s.S) {
                if (SAVE) {
                    float f[8];
                    raw[k].widen(p.k, f);
                    gn_save<8>(out, (p.image + p.im) * s.S + p.row + k * step, s, p.k, f);
                }
                if (!p.k.any) continue;
                float d[8];
                raw[k].center(p.k, mu, d);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = act_of<T, ACT>(__fmaf_rn(d[j], zw[j], b[j]));
                gn_store<T, 8>(keep, gn_near(to, y_at + k * y_step), here, d);
            }
        __syncthreads();
    }
}

__device__ __forceinline__ uint16_t gn_bits(bf16 v) { return v.bits; }
__device__ __forceinline__ uint16_t gn_bits(f16 v) { return v.bits; }
__device__ __forceinline__ uint16_t gn_bits(float) { return 0; }

template <typename T, int K, int ACT, bool SAVED>
__global__ __launch_bounds__(kGnHeldMost) void k_gn_held_backward(GnShape s, GnHeld h, bool keep, const float* __restrict__ mean, const float* __restrict__ rstd, GnImages dy,
                                                                  GnImages x, Saved saved, GnImages dx, LnParam weight, LnParam bias, float* __restrict__ partial) {
    extern __shared__ float gn_lds[];
    const GnSums m(s, h, false);
    const uint32_t size = m.entries * m.waves << h.images_log, channels = m.entries << h.images_log;
    float* const sums_h = gn_lds;
    float* const sums_1 = sums_h + size;
    float* const a_h = sums_1 + size;                                    // per channel, times its weight
    float* const a_1 = a_h + channels;
    float2* const stats = reinterpret_cast<float2*>(a_1 + channels);
    const uint32_t step = 1u << h.rows_log;
    const float n = (float)s.S * (float)s.per_group;
    for (int64_t work = blockIdx.x; work < gn_held_works(s, h); work += gridDim.x) {
        const GnPlace p = gn_place(s, h, work);
        const uint32_t saved_groups = (s.C + kSavedCols - 1) / kSavedCols;
        const T* const xs = SAVED ? nullptr : gn_image<const T>(x, s, p.image);
        const T* const gs = gn_image<const T>(dy, s, p.image);
        const int8_t* const qs = saved.q + p.image * s.S * s.C;
        const uint8_t* const es = saved.e + p.image * s.S * saved_groups;
        const uint32_t x_at = (uint32_t)((p.im * x.image + p.row * x.row + p.k.c) * sizeof(T)), x_step = (uint32_t)(step * x.row * sizeof(T));
        const uint32_t g_at = (uint32_t)((p.im * dy.image + p.row * dy.row + p.k.c) * sizeof(T)), g_step = (uint32_t)(step * dy.row * sizeof(T));
        const uint32_t row0 = p.im * (uint32_t)s.S + p.row, q_at = row0 * s.C + p.k.c, e_at = row0 * saved_groups + (p.k.c + 7) / kSavedCols;
        GnRaw<T, 8, SAVED> raw[K];
        GnRaw<T, 8, false> grad[K];
        const int rows = (int)h.rows;
        const GnColumns here{0, p.k.skip, p.k.any};
        auto load = [&](GnRaw<T, 8, SAVED>& to, GnRaw<T, 8, false>& g, uint32_t k) {
            if constexpr (SAVED) {
                to.w = ld8_bytes(gn_near(qs, q_at + k * step * s.C));
                to.e = *gn_near(es, e_at + k * step * saved_groups);
            } else {
                to.load(gn_near(xs, x_at + k * x_step), here);
            }
            g.load(gn_near(gs, g_at + k * g_step), here);
        };
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k] = {};
            grad[k] = {};
            if (k < rows && p.row + k * step < s.S) load(raw[k], grad[k], k);
        }
        GnParams<8> t;
        const GnColumns mine{p.k.c, p.k.skip, true};
        t.load(s, p.image + p.im, mine, mean, rstd, weight, bias);
        float zw[8], v_h[8], v_1[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) zw[j] = t.rs[j] * t.w[j];
        // A ReLU's dz takes the place of dy.  Where a sign was too near to tell, a thread looks at its values again in fp64.
        if (ACT == kActRelu) {
            bool near = false;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k < rows) {
                    float d[8], g[8];
                    raw[k].center(p.k, t.mu, d);
                    grad[k].widen(p.k, g);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float z = __fmaf_rn(d[j], zw[j], t.b[j]);
                        near |= fabsf(z) <= 0x1p-22f * fabsf(t.b[j]);
                        g[j] = z > 0.f ? g[j] : 0.f;
                    }
                    grad[k].narrow(g);
                    raw[k].hide();
                    grad[k].hide();
                }
            if (__builtin_expect(near, 0)) {
                // weights out of memory again, one row after the other: registers are full
                near = false;
                float w[8];
                gn_param<8>(weight, gn_worker(s, p.image), p.k.c, 1.f, w);
#pragma unroll
                for (int k = 0; k < K; ++k)
                    if (k < rows) {
                        float d[8];
                        raw[k].center(p.k, t.mu, d);
#pragma unroll
                        for (int j = 0; j < 8; ++j) near |= gn_undecided(__fmaf_rn(d[j], zw[j], t.b[j]), d[j], w[j], t.b[j]);
                        raw[k].hide();
                    }
            }
            if (__builtin_expect(near, 0)) {
                // value by value, everything read again: registers are full, and these are a few in a million
#pragma unroll 1
                for (uint32_t i = 0; i < h.rows * 8; ++i) {
                    const uint32_t k = i >> 3, j = i & 7, c = p.k.c + j;
                    if (p.row + k * step >= s.S) break;
                    float v;
                    if constexpr (SAVED) v = (float)*gn_near(qs, q_at + k * step * s.C + j) * saved_scale(*gn_near(es, e_at + k * step * saved_groups));
                    else v = widen(gn_near(xs, x_at + k * x_step)[j]);
                    const T dyv = gn_near(gs, g_at + k * g_step)[j];
                    const int64_t at = (p.image + p.im) * s.G + c / s.per_group, worker = gn_worker(s, p.image);
                    const float w = weight.data ? load_any(weight.data, worker * weight.stride + c, weight.type) : 1.f;
                    const float o = bias.data ? load_any(bias.data, worker * bias.stride + c, bias.type) : 0.f;
                    const bool on = ((double)v - (double)mean[at]) * (double)rstd[at] * (double)w + (double)o > 0.0;
                    const uint32_t bits = !on ? 0u : sizeof(T) == 4 ? __float_as_uint(widen(dyv)) : (uint32_t)gn_bits(dyv) << (16 * (j & 1));
                    const uint32_t mask = sizeof(T) == 4 ? 0xffffffffu : 0xffffu << (16 * (j & 1)), word = sizeof(T) == 4 ? j : j >> 1;
#pragma unroll
                    for (int q = 0; q < K; ++q)
#pragma unroll
                        for (int n = 0; n < (int)Eight<T>::words * 4; ++n)
                            if (q == (int)k && n == (int)word) grad[q].v.w[n >> 2][n & 3] = (grad[q].v.w[n >> 2][n & 3] & ~mask) | bits;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v_h[j] = v_1[j] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < rows && p.row + k * step < s.S) {
                float d[8], g[8];
                raw[k].center(p.k, t.mu, d);
                grad[k].widen(p.k, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (ACT == kActSilu) g[j] = dz_of<T, ACT>(g[j], __fmaf_rn(d[j], zw[j], t.b[j]));
                    v_1[j] += g[j];
                    v_h[j] = __fmaf_rn(g[j], d[j], v_h[j]);
                }
            }
#pragma unroll
        for (int j = 0; j < 8; ++j) v_h[j] *= t.rs[j];
        gn_leave(v_h, m, h, p, false, sums_h);
        gn_leave(v_1, m, h, p, false, sums_1);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k].hide();
            grad[k].hide();
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < channels; i += blockDim.x) {
            const uint32_t im = i / h.span, c = i - im * h.span;
            float th = 0.f, t1 = 0.f, w = 0.f;
            if (c < p.channels) {
                for (uint32_t j = 0; j < m.waves; ++j) {
                    th += sums_h[i * m.waves + j];
                    t1 += sums_1[i * m.waves + j];
                }
                w = weight.data ? load_any(weight.data, gn_worker(s, p.image) * weight.stride + p.first + c, weight.type) : 1.f;
            }
            sums_h[i * m.waves] = th;
            sums_1[i * m.waves] = t1;
            a_h[i] = th * w;
            a_1[i] = t1 * w;
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < p.channels; c += blockDim.x) {
            float th = 0.f, t1 = 0.f;
            for (uint32_t im = 0; im < 1u << h.images_log; ++im) {
                th += sums_h[(im * h.span + c) * m.waves];
                t1 += sums_1[(im * h.span + c) * m.waves];
            }
            float* const to = partial + (size_t)p.set * 2 * s.C + p.first + c;
            to[0] = th;
            to[s.C] = t1;
        }
        if (dx.data) {
            gn_groups_total<true>(s, h, p, m.entries, 1, m.group, a_h, a_1, [&](uint32_t i, float ah, float a1) { stats[i] = make_float2(a1 / n, ah / n); });
            __syncthreads();
            const uint32_t groups = p.channels / s.per_group;
            float k1[8], k2[8];
            gn_each_group<8>(s, p.k.c, [&](int j, uint32_t g) {
                const float2 o = stats[p.im * groups + min(max(g, p.first / s.per_group) - p.first / s.per_group, groups - 1)];
                k1[j] = t.rs[j] * o.x;
                k2[j] = t.rs[j] * (t.rs[j] * o.y);
            });
            T* const to = gn_image<T>(dx, s, p.image);
            const uint32_t d_at = (uint32_t)((p.im * dx.image + p.row * dx.row + p.k.c) * sizeof(T)), d_step = (uint32_t)(step * dx.row * sizeof(T));
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k < rows && p.row + k * step < s.S && p.k.any) {
                    float d[8], g[8];
                    raw[k].center(p.k, t.mu, d);
                    grad[k].widen(p.k, g);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (ACT == kActSilu) g[j] = dz_of<T, ACT>(g[j], __fmaf_rn(d[j], zw[j], t.b[j]));
                        d[j] = __fmaf_rn(g[j], zw[j], -__fmaf_rn(d[j], k2[j], k1[j]));
                    }
                    gn_store<T, 8>(keep, gn_near(to, d_at + k * d_step), here, d);
                }
        }
        __syncthreads();
    }
}

}  // namespace liec
