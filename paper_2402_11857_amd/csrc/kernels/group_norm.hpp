// Group normalisation with an activation function, channels last, of N workers' images, each worker with weights of its own, and
// its gradients.
//
//   forward    mu, var over the S positions and the C / G channels of a group,  rstd = 1 / sqrt(var + eps),
//              y = act((x - mu) rstd w + b)
//   backward   h = (x - mu) rstd,  z = h w + b,  dz = dy act'(z),  a = dz w,  dx = rstd (a - mean a - h mean(a h))
//              dw = sum over the worker's images and positions of dz h,  db of dz
//
// Everything starts from sums per image and channel: with P1_c = sum_s dz and P2_c = sum_s dz h, mean a and mean(a h) are sums of
// w_c P1_c and w_c P2_c over a group's channels, dw and db those of P2_c and P1_c over images; forward, a channel's mean and squares
// around it go together in the group's.  So a thread keeps 8 channels and walks positions, whatever the groups' width, and loads are
// 16 bytes wide.  The last 8 channels of a row whose length is no multiple of 8 start 8 before its end; what they share with
// the ones before is left out where it is stored.
//
// These are the kernels for images that no block holds: two passes over them, bound by memory and, with an activation, by arithmetic
// beside it.  16 x 8 images of 56 x 56 x 256 bf16, ReLU: forward 36 us for the sums (5.7 TB/s), 5 for the groups, 78 for y
// (5.2 TB/s of x and y); backward from a checkpoint 65 for the sums (4.8 TB/s), 5 for what comes of them, 98 for dx (5.3
// TB/s).
#pragma once
#include <type_traits>

#include "checkpoint.hpp"

namespace liec {

enum Act : int { kActNone = 0, kActRelu = 1, kActSilu = 2 };

struct GnImages {                      // an [N, B, S, C] tensor of unit channel stride
    void* data;
    int64_t worker, image, row;        // strides, in elements
};

struct GnShape {
    int64_t images, B, S;              // images = N * B
    uint32_t C, G, per_group;
    uint32_t lanes_log;                // a row-thread's lanes, each with 8 channels (one, where C < 8): tiles of the channels
    bool whole;                        // groups are a multiple of 8 channels
    uint32_t tiles, splits;            // a block's work: one tile, `per` of an image's positions
    int64_t per;
};

// ---- activation ------------------------------------------------------------------------------------------------------
// exp(-z), an infinity from 2^128 on, whose reciprocal is the limit, 0 (a reciprocal under 2^-126 may come as 0 too).  For results of 16
// bits the product's rounding error stays, |z| u of the exponential; for fp32 it is put right, to about 2 u.
template <typename T>
__device__ __forceinline__ float exp_minus(float z) {
    const float log2e = 1.44269502f, rest = 1.92596299e-8f;              // their sum is log2(e)
    const float t = -z * log2e, e = __builtin_amdgcn_exp2f(t);
    if (sizeof(T) == 2) return e;
    const float off = __fmaf_rn(-z, rest, __fmaf_rn(-z, log2e, -t));
    return fabsf(t) < 128.f ? __fmaf_rn(e, off * 0.693147181f, e) : e;
}

template <typename T, int ACT>
__device__ __forceinline__ float act_of(float z) {
    if (ACT == kActRelu) return z < 0.f ? 0.f : z;
    if (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.f + exp_minus<T>(z));
    return z;
}

// dz from dy and z.
template <typename T, int ACT>
__device__ __forceinline__ float dz_of(float dy, float z) {
    if (ACT == kActNone) return dy;
    if (ACT == kActRelu) return z > 0.f ? dy : 0.f;
    const float p = __builtin_amdgcn_rcpf(1.f + exp_minus<T>(z));
    return dy * (p * __fmaf_rn(z, 1.f - p, 1.f));                        // p (1 + z (1 - p))
}

// ---- a thread's channels ----------------------------------------------------------------------------------------------
struct GnColumns {
    uint32_t c, skip;                  // first channel it loads, how many of them belong to the thread before
    bool any;
};
template <int V>
__device__ __forceinline__ GnColumns gn_columns(const GnShape& s, uint32_t tile, uint32_t lane) {
    const uint32_t at = ((tile << s.lanes_log) + lane) * V;
    GnColumns r;
    r.any = at < s.C;
    r.c = V == 1 ? at : min(at, s.C - V);
    r.skip = at - r.c;
    return r;
}

// x as it lies in memory: a tensor's row or a checkpoint's.
template <typename T, int V, bool SAVED>
struct GnRaw {
    Eight<T> v;
    // What comes before and after does not share widened values, which take up to four times the registers.
    __device__ __forceinline__ void hide() {
#pragma unroll
        for (int i = 0; i < Eight<T>::words; ++i) asm volatile("" : "+v"(v.w[i]));
    }
    __device__ __forceinline__ void load(const T* row, const GnColumns& k) { v = ld_eight<T, false>(row + k.c); }
    __device__ __forceinline__ void widen(const GnColumns&, float (&f)[V]) const { widen_eight<T>(v, f); }
    __device__ __forceinline__ void narrow(const float (&f)[V]) {
#pragma unroll
        for (int i = 0; i < Eight<T>::words; ++i) {
            float part[Vec16<T>::n];
#pragma unroll
            for (int j = 0; j < Vec16<T>::n; ++j) part[j] = f[i * Vec16<T>::n + j];
            v.w[i] = Vec16<T>::narrow(part);
        }
    }
    __device__ __forceinline__ void center(const GnColumns& k, const float (&mu)[V], float (&f)[V]) const {
        widen(k, f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] -= mu[j];
    }
};
template <typename T>
struct GnRaw<T, 1, false> {
    T v;
    __device__ __forceinline__ void load(const T* row, const GnColumns& k) { v = row[k.c]; }
    __device__ __forceinline__ void widen(const GnColumns&, float (&f)[1]) const { f[0] = liec::widen(v); }
    __device__ __forceinline__ void center(const GnColumns&, const float (&mu)[1], float (&f)[1]) const { f[0] = liec::widen(v) - mu[0]; }
};
template <typename T>
struct GnRaw<T, 8, true> {
    v2u w;
    __device__ __forceinline__ void hide() { asm volatile("" : "+v"(w), "+v"(e)); }
    uint32_t e;                        // the last channel's exponent, and that of every channel that is not left out
    __device__ __forceinline__ void load(const Saved& s, int64_t row, uint32_t C, uint32_t groups, const GnColumns& k) {
        w = ld8_bytes(s.q + row * C + k.c);
        e = s.e[row * groups + (k.c + 7) / kSavedCols];
    }
    __device__ __forceinline__ void widen(const GnColumns&, float (&f)[8]) const {
        unpack4(w.x, saved_scale(e), f);
        unpack4(w.y, saved_scale(e), f + 4);
    }
    // x - mu with one rounding: q 2^k is exact
    __device__ __forceinline__ void center(const GnColumns&, const float (&mu)[8], float (&f)[8]) const {
        const float scale = saved_scale(e);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __fmaf_rn((float)(int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3))), scale, -mu[j]);
    }
};
template <typename T>
struct GnRaw<T, 1, true> {
    int8_t q;
    uint8_t e;
    __device__ __forceinline__ void load(const Saved& s, int64_t row, uint32_t C, uint32_t groups, const GnColumns& k) {
        q = s.q[row * C + k.c];
        e = s.e[row * groups];
    }
    __device__ __forceinline__ void widen(const GnColumns&, float (&f)[1]) const { f[0] = (float)q * saved_scale(e); }
    __device__ __forceinline__ void center(const GnColumns&, const float (&mu)[1], float (&f)[1]) const { f[0] = __fmaf_rn((float)q, saved_scale(e), -mu[0]); }
};

__device__ __forceinline__ int64_t gn_worker(const GnShape& s, int64_t image) {
    return s.images <= 0x7fffffff ? (int64_t)((uint32_t)image / (uint32_t)s.B) : image / s.B;
}
template <typename T>
__device__ __forceinline__ T* gn_image(const GnImages& m, const GnShape& s, int64_t image) {
    const int64_t worker = gn_worker(s, image);
    return static_cast<T*>(m.data) + worker * m.worker + (image - worker * s.B) * m.image;
}

__device__ __forceinline__ int64_t gn_works(const GnShape& s) { return s.images * s.splits * s.tiles; }

struct GnWork {
    uint32_t tile, split;
    int64_t image, first, end;         // positions
};
__device__ __forceinline__ GnWork gn_work(const GnShape& s, int64_t work) {
    GnWork r;
    if (gn_works(s) <= 0x7fffffff) {   // a division of 64 bits takes some 150 instructions
        const uint32_t strip = (uint32_t)work / s.tiles, image = strip / s.splits;
        r.tile = (uint32_t)work - strip * s.tiles;
        r.split = strip - image * s.splits;
        r.image = image;
    } else {
        const int64_t strip = work / s.tiles;
        r.tile = (uint32_t)(work - strip * s.tiles);
        r.image = strip / s.splits;
        r.split = (uint32_t)(strip - r.image * s.splits);
    }
    r.first = r.split * s.per;
    r.end = min(r.first + s.per, s.S);
    return r;
}

constexpr int kGnAhead = 4;            // positions of a thread requested together

// A thread's positions of a strip: f(first of them, how many: kGnAhead, as a constant, or one at a time for what is left), with the
// distance between them.
template <typename F>
__device__ __forceinline__ void gn_walk(const GnWork& w, uint32_t thread, uint32_t threads, F f) {
    int64_t r = w.first + thread;
    for (; r + (kGnAhead - 1) * (int64_t)threads < w.end; r += kGnAhead * threads) f(r, std::integral_constant<int, kGnAhead>{});
    for (; r < w.end; r += threads) f(r, std::integral_constant<int, 1>{});
}
constexpr int kGnTile = 512;           // channels of a tile, at most

// Stores a block's sums per channel, lds[wave][channel of the tile] of `waves` waves put together by `join`.
template <int V, typename F>
__device__ __forceinline__ void gn_store_channels(const GnShape& s, const GnWork& w, F value, float* out) {
    for (uint32_t t = threadIdx.x; t < (uint32_t)(V << s.lanes_log); t += kBlock) {
        const GnColumns k = gn_columns<V>(s, w.tile, t / V);
        if (k.any && t % V >= k.skip) {
            const float2 v = value(t);
            float* const to = out + (size_t)(w.image * s.splits + w.split) * 2 * s.C + k.c + t % V;
            to[0] = v.x;
            to[s.C] = v.y;
        }
    }
}

// ---- forward ----------------------------------------------------------------------------------------------------------
// Mean and squares around it of n and n2 values, put together.  Where one of the two has no values the square of their means' distance does not
// count, and may be beyond fp32.
__device__ __forceinline__ void gn_join(float n, float& mean, float& squares, float n2, float mean2, float squares2) {
    const float all = n + n2, share = all > 0.f ? n2 / all : 0.f, d = mean2 - mean, weight = n * share;
    mean = __fmaf_rn(d, share, mean);
    squares += weight > 0.f ? __fmaf_rn(d * d, weight, squares2) : squares2;
}

// Mean and squares around it of each channel over a strip of an image's positions.  A thread takes its values around the mean p of its
// first four (or, of less than four in all, its first): with n of them (at most 256) and m their mean, (p - m)^2 <= n / 4 of
// their variance, so that taking n (p - m)^2 off again costs at most 64 u of it per addition's u.
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void k_gn_stats(GnShape s, GnImages x, float* __restrict__ partial) {
    __shared__ float lds_mean[kBlock / 64][kGnTile], lds_squares[kBlock / 64][kGnTile], lds_n[kBlock / 64];
    const uint32_t lane = threadIdx.x & ((1u << s.lanes_log) - 1), thread = threadIdx.x >> s.lanes_log, threads = kBlock >> s.lanes_log;
    for (int64_t work = blockIdx.x; work < gn_works(s); work += gridDim.x) {
        const GnWork w = gn_work(s, work);
        const GnColumns k = gn_columns<V>(s, w.tile, lane);
        const T* const at = gn_image<const T>(x, s, w.image);
        float p[V], sum[V], squares[V], n = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = sum[j] = squares[j] = 0.f;
        const int64_t step = threads * x.row;
        if (k.any)
            gn_walk(w, thread, threads, [&](int64_t r, auto rows) {
                constexpr int R = decltype(rows)::value;
                GnRaw<T, V, false> raw[R];
                const T* const first = at + r * x.row;
#pragma unroll
                for (int u = 0; u < R; ++u) raw[u].load(first + u * step, k);
                float f[R][V];
#pragma unroll
                for (int u = 0; u < R; ++u) raw[u].widen(k, f[u]);
                if (n == 0.f) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        p[j] = f[0][j];
#pragma unroll
                        for (int u = 1; u < R; ++u) p[j] += f[u][j];
                        p[j] *= 1.f / R;
                    }
                }
#pragma unroll
                for (int u = 0; u < R; ++u)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float d = f[u][j] - p[j];
                        sum[j] += d;
                        squares[j] = __fmaf_rn(d, d, squares[j]);
                    }
                n += (float)R;
            });
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = n > 0.f ? sum[j] / n : 0.f;
            p[j] += d;
            squares[j] = fmaxf(__fmaf_rn(-d, sum[j], squares[j]), 0.f) + (d - d);      // a NaN stays one
        }
        for (uint32_t off = 1u << s.lanes_log; off < 64; off <<= 1) {
            const float n2 = __shfl_xor(n, off);
#pragma unroll
            for (int j = 0; j < V; ++j) gn_join(n, p[j], squares[j], n2, __shfl_xor(p[j], off), __shfl_xor(squares[j], off));
            n += n2;
        }
        const uint32_t wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == lane) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                lds_mean[wave][lane * V + j] = p[j];
                lds_squares[wave][lane * V + j] = squares[j];
            }
            if (lane == 0) lds_n[wave] = n;
        }
        __syncthreads();
        gn_store_channels<V>(s, w, [&](uint32_t t) {
            float many = lds_n[0];
            float2 v = make_float2(lds_mean[0][t], lds_squares[0][t]);
            for (int i = 1; i < kBlock / 64; ++i) {
                gn_join(many, v.x, v.y, lds_n[i], lds_mean[i][t], lds_squares[i][t]);
                many += lds_n[i];
            }
            return v;
        }, partial);
        __syncthreads();
    }
}

// What an image's strips left of a group's channels, neighbouring lanes on neighbouring channels: of every `parts`-th set of strips.
template <typename F>
__device__ __forceinline__ void gn_each_part(const GnShape& s, int64_t group, uint32_t part, uint32_t parts, F f) {
    const int64_t image = group / s.G;
    const uint32_t first = (uint32_t)(group - image * s.G) * s.per_group, lane = threadIdx.x & 63;
    const uint32_t wide_log = s.per_group >= 64 ? 6 : 32 - __clz((int)s.per_group), wide = 1u << wide_log, step = 64u >> wide_log;
#pragma unroll 4
    for (uint32_t split = part * step + (lane >> wide_log); split < s.splits; split += parts * step)
        for (uint32_t c = lane & (wide - 1); c < s.per_group; c += wide) f((size_t)(image * s.splits + split) * 2 * s.C + first + c, first + c, split);
}
// Two sums over each group in fp64, added up by a wave, or, of few groups, by a block: add(group, part, parts, two sums) for a lane's share,
// done(group, both) on one lane.  Block `block` of `blocks`.  A few groups are many strips each, one load after the other.  Whole calls in us,
// a wave per group and a block: 10 groups (5 images of 2466 x 66) 27 and 17; 640 (784 x 250) 25.1 and 24.5, backward 32.8 and 31.7; 1024
// (3136 x 66) 160 and 160; 2048 (196 x 500) 55.7 and 56.4; 20 480 107 and 120.
constexpr int64_t kGnFewGroups = 1024;
template <typename A, typename D>
__device__ __forceinline__ void gn_each_group_sums(const GnShape& s, uint32_t block, uint32_t blocks, A add, D done) {
    __shared__ double lds[kBlock / 64][2];
    constexpr uint32_t waves = kBlock / 64;
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const bool few = s.images * s.G <= kGnFewGroups;
    for (int64_t g = few ? block : (int64_t)block * waves + wave; g < s.images * s.G; g += few ? blocks : (int64_t)blocks * waves) {
        double a = 0.0, b = 0.0;
        add(g, few ? wave : 0u, few ? waves : 1u, a, b);
        a = wave_sum(a);
        b = wave_sum(b);
        if (few) {
            if (lane == 0) lds[wave][0] = a, lds[wave][1] = b;
            __syncthreads();
            a = lds[0][0], b = lds[0][1];
            for (uint32_t w = 1; w < waves; ++w) a += lds[w][0], b += lds[w][1];
            __syncthreads();
        }
        if (lane == 0 && (!few || wave == 0)) done(g, a, b);
    }
}

template <int>
__global__ __launch_bounds__(kBlock) void k_gn_groups(GnShape s, const float* __restrict__ partial, float eps, float* __restrict__ mean, float* __restrict__ rstd) {
    // values around one of the group's means
    const auto around = [&](int64_t g) {
        const int64_t image = g / s.G;
        return (double)partial[(size_t)image * s.splits * 2 * s.C + (uint32_t)(g - image * s.G) * s.per_group];
    };
    gn_each_group_sums(
        s, blockIdx.x, gridDim.x,
        [&](int64_t g, uint32_t part, uint32_t parts, double& sum, double& squares) {
            const double p = around(g);
            gn_each_part(s, g, part, parts, [&](size_t at, uint32_t, uint32_t split) {
                const double n = (double)min(s.per, s.S - split * s.per), d = (double)partial[at] - p;
                sum += n * d;
                squares += (double)partial[at + s.C] + n * d * d;
            });
        },
        [&](int64_t g, double sum, double squares) {
            const double n = (double)s.S * (double)s.per_group, d = sum / n, var = (squares - d * sum) / n;
            mean[g] = (float)(around(g) + d);
            rstd[g] = (float)(1.0 / sqrt((var > 0.0 ? var : var - var) + (double)eps));
        });
}

// Bits of the largest magnitude of a checkpoint's group of columns: the lanes that share it.
template <int V>
__device__ __forceinline__ uint32_t gn_largest(uint32_t a, uint32_t lanes_log) {
    if (V == 8) return max_of_quad(a);
    for (uint32_t off = 1; off < 1u << lanes_log; off <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, off));
    return a;
}

template <typename T, int V>
__device__ __forceinline__ void gn_store(bool keep, T* row, const GnColumns& k, const float (&f)[V]) {
    if constexpr (V == 8) {
        if (k.skip == 0) {
            st_eight<T>(keep, row + k.c, f);
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j >= (int)k.skip) row[k.c + j] = narrow<T>(f[j]);
}

// The checkpoint of a thread's channels of a row; all lanes that share an exponent call it together.
template <int V>
__device__ __forceinline__ void gn_save(const Saved& out, int64_t row, const GnShape& s, const GnColumns& k, const float (&f)[V]) {
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) a = max(a, k.any && j >= (int)k.skip ? key_of(f[j]) : 0u);
    const uint32_t e = saved_exponent(gn_largest<V>(a, s.lanes_log));
    if (!k.any) return;
    int8_t* const to = out.q + row * s.C + k.c;
    const uint32_t first = k.c + k.skip;
    if (first % kSavedCols == 0) out.e[row * ((s.C + kSavedCols - 1) / kSavedCols) + first / kSavedCols] = (uint8_t)e;
    if constexpr (V == 8) {
        const v2u w = pack8(f, e);
        if (k.skip == 0) {
            st8_bytes(to, w);
        } else {
#pragma unroll
            for (int j = 1; j < 8; ++j)
                if (j >= (int)k.skip) to[j] = (int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
        }
    } else {
        to[0] = e == kSavedNan ? 0 : (int8_t)(int)rintf((e == (uint32_t)kSavedMost ? saved_in_range(f[0]) : f[0]) * saved_inverse(e));
    }
}

// V neighbouring parameters of a worker.
template <int V>
__device__ __forceinline__ void gn_param(const LnParam& p, int64_t worker, uint32_t c, float none, float (&f)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = none;
    if (!p.data) return;
    const int64_t at = worker * p.stride + c;
    if constexpr (V == 8) {
        if (p.type == kF32) widen_eight<float>(ld_eight<float, false>(static_cast<const float*>(p.data) + at), f);
        else if (p.type == kBF16) widen_eight<bf16>(ld_eight<bf16, false>(static_cast<const bf16*>(p.data) + at), f);
        else widen_eight<f16>(ld_eight<f16, false>(static_cast<const f16*>(p.data) + at), f);
    } else {
        f[0] = load_any(p.data, at, p.type);
    }
}
// The groups of V neighbouring channels: f(j, group), in order.
template <int V, typename F>
__device__ __forceinline__ void gn_each_group(const GnShape& s, uint32_t c, F f) {
    uint32_t g = c / s.per_group, left = (g + 1) * s.per_group - c;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        f(j, g);
        if (--left == 0) {
            ++g;
            left = s.per_group;
        }
    }
}

template <int V>
struct GnParams {
    float mu[V], rs[V], w[V], b[V];
    __device__ __forceinline__ void load(const GnShape& s, int64_t image, const GnColumns& k, const float* mean, const float* rstd, const LnParam& weight,
                                         const LnParam& bias) {
        const int64_t worker = gn_worker(s, image);
        const uint32_t c = k.any ? k.c : 0u;
        gn_param<V>(weight, worker, c, 1.f, w);
        gn_param<V>(bias, worker, c, 0.f, b);
        mean += image * s.G;
        rstd += image * s.G;
        if (V == 8 && s.whole) {       // one group for all eight
            const uint32_t g = c / s.per_group;
#pragma unroll
            for (int j = 0; j < V; ++j) mu[j] = mean[g], rs[j] = rstd[g];
        } else {
            gn_each_group<V>(s, c, [&](int j, uint32_t g) { mu[j] = mean[g], rs[j] = rstd[g]; });
        }
    }
};

// y, and the checkpoint of x where SAVE.
template <typename T, int V, int ACT, bool SAVE>
__global__ __launch_bounds__(kBlock) void k_gn_apply(GnShape s, bool keep, const float* __restrict__ mean, const float* __restrict__ rstd, GnImages x, GnImages y,
                                                     LnParam weight, LnParam bias, Saved out) {
    const uint32_t lane = threadIdx.x & ((1u << s.lanes_log) - 1), thread = threadIdx.x >> s.lanes_log, threads = kBlock >> s.lanes_log;
    for (int64_t work = blockIdx.x; work < gn_works(s); work += gridDim.x) {
        const GnWork w = gn_work(s, work);
        const GnColumns k = gn_columns<V>(s, w.tile, lane);
        const T* const from = gn_image<const T>(x, s, w.image);
        T* const to = gn_image<T>(y, s, w.image);
        GnParams<V> p;
        p.load(s, w.image, k, mean, rstd, weight, bias);
#pragma unroll
        for (int j = 0; j < V; ++j) p.rs[j] *= p.w[j];
        const int64_t x_step = threads * x.row, y_step = threads * y.row;
        gn_walk(w, thread, threads, [&](int64_t r, auto rows) {
            constexpr int R = decltype(rows)::value;
            GnRaw<T, V, false> raw[R];
            const T* const first = from + r * x.row;
            T* const out_first = to + r * y.row;
            if (k.any) {
#pragma unroll
                for (int u = 0; u < R; ++u) raw[u].load(first + u * x_step, k);
            }
#pragma unroll
            for (int u = 0; u < R; ++u) {
                float f[V];
                if (k.any) raw[u].widen(k, f);
                if (SAVE) gn_save<V>(out, w.image * s.S + r + u * threads, s, k, f);
                if (!k.any) continue;
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] = act_of<T, ACT>(__fmaf_rn(f[j] - p.mu[j], p.rs[j], p.b[j]));
                gn_store<T, V>(keep, out_first + u * y_step, k, f);
            }
        });
    }
}

// ---- backward ---------------------------------------------------------------------------------------------------------
// A ReLU's dz of a row with the signs of z in fp64, one channel after the other.  What these few rows need stays in registers beside all
// others: sums over a strip take 180 to 195 of them with it (two waves to a SIMD), 114 to 122 without an activation.
template <int V, typename R, typename G>
__device__ __forceinline__ void gn_dz_exact(float (&g)[V], const GnParams<V>& p, const R& raw, const G& grad, const GnColumns& k) {
    float f[V];
    raw.widen(k, f);
    grad.widen(k, g);
#pragma unroll 1
    for (int j = 0; j < V; ++j) {
        float x = 0.f, mu = 0.f, rs = 0.f, w = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i == j) x = f[i], mu = p.mu[i], rs = p.rs[i], w = p.w[i], b = p.b[i];
        const bool on = ((double)x - (double)mu) * (double)rs * (double)w + (double)b > 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = i == j && !on ? 0.f : g[i];
    }
}
// dz of a thread's channels in the place of dy, with d = x - mu and zw = rstd w.  The sign of z = d zw + b decides a ReLU's gradient: in
// fp32 z is off by at most 2 u |d zw| + u |z|, so it is right unless |z| <= 4 u |b| (then |d zw| <= |b| (1 + 4 u)).  Rows with such a
// channel, a few in a million, are looked at again.  Without a bias z has the sign of d w, and is 0 where one of them is (channels
// without weights, images of one value: 128 images of 14 x 14 x 512 bf16 whose weights are zero 41 us, 34 with others, 96 if all are decided in
// fp64) or their product is too small for fp32: only then is there something to decide.
__device__ __forceinline__ bool gn_undecided(float z, float d, float w, float b) { return fabsf(z) <= 0x1p-22f * fabsf(b) && (b != 0.f || (d != 0.f && w != 0.f)); }
template <typename T, int V, int ACT, typename R, typename G>
__device__ __forceinline__ void gn_dz(float (&g)[V], const float (&d)[V], const float (&zw)[V], const GnParams<V>& p, const R& raw, const G& grad, const GnColumns& k) {
    if (ACT == kActNone) return;
    bool near = false;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float z = __fmaf_rn(d[j], zw[j], p.b[j]);
        if (ACT == kActRelu) near |= fabsf(z) <= 0x1p-22f * fabsf(p.b[j]);
        g[j] = dz_of<T, ACT>(g[j], z);
    }
    if (ACT == kActRelu && __builtin_expect(near, 0)) {
        bool undecided = false;
#pragma unroll
        for (int j = 0; j < V; ++j) undecided |= gn_undecided(__fmaf_rn(d[j], zw[j], p.b[j]), d[j], p.w[j], p.b[j]);
        if (__builtin_expect(undecided, 0)) gn_dz_exact<V>(g, p, raw, grad, k);
    }
}

// R positions of x, or its checkpoint, and dy.
template <typename T, int V, bool SAVED, int R>
__device__ __forceinline__ void gn_load(GnRaw<T, V, SAVED> (&raw)[R], GnRaw<T, V, false> (&grad)[R], const T* xs, const GnImages& x, const Saved& saved, const T* gs,
                                        const GnImages& dy, const GnShape& s, const GnWork& w, int64_t r, uint32_t threads, const GnColumns& k) {
    const int64_t x_step = threads * x.row, g_step = threads * dy.row;
    const T* const x_first = xs + r * x.row;
    const T* const g_first = gs + r * dy.row;
#pragma unroll
    for (int u = 0; u < R; ++u) {
        if constexpr (SAVED) raw[u].load(saved, w.image * s.S + r + u * threads, s.C, (s.C + kSavedCols - 1) / kSavedCols, k);
        else raw[u].load(x_first + u * x_step, k);
        grad[u].load(g_first + u * g_step, k);
    }
}

// Sums of dz h and of dz over a strip of an image's positions.
template <typename T, int V, int ACT, bool SAVED>
__global__ __launch_bounds__(kBlock) void k_gn_sums(GnShape s, const float* __restrict__ mean, const float* __restrict__ rstd, GnImages dy, GnImages x, Saved saved,
                                                    LnParam weight, LnParam bias, float* __restrict__ partial) {
    __shared__ float lds_h[kBlock / 64][kGnTile], lds_1[kBlock / 64][kGnTile];
    const uint32_t lane = threadIdx.x & ((1u << s.lanes_log) - 1), thread = threadIdx.x >> s.lanes_log, threads = kBlock >> s.lanes_log;
    for (int64_t work = blockIdx.x; work < gn_works(s); work += gridDim.x) {
        const GnWork w = gn_work(s, work);
        const GnColumns k = gn_columns<V>(s, w.tile, lane);
        const T* const xs = SAVED ? nullptr : gn_image<const T>(x, s, w.image);
        const T* const gs = gn_image<const T>(dy, s, w.image);
        GnParams<V> p;
        p.load(s, w.image, k, mean, rstd, weight, bias);
        float zw[V];
#pragma unroll
        for (int j = 0; j < V; ++j) zw[j] = p.rs[j] * p.w[j];
        float sum_h[V], sum_1[V];
#pragma unroll
        for (int j = 0; j < V; ++j) sum_h[j] = sum_1[j] = 0.f;
        if (k.any)
            gn_walk(w, thread, threads, [&](int64_t r, auto rows) {
                constexpr int R = decltype(rows)::value;
                GnRaw<T, V, SAVED> raw[R];
                GnRaw<T, V, false> grad[R];
                gn_load<T, V, SAVED, R>(raw, grad, xs, x, saved, gs, dy, s, w, r, threads, k);
#pragma unroll
                for (int u = 0; u < R; ++u) {
                    float d[V], g[V];
                    raw[u].center(k, p.mu, d);
                    grad[u].widen(k, g);
                    gn_dz<T, V, ACT>(g, d, zw, p, raw[u], grad[u], k);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        sum_1[j] += g[j];
                        sum_h[j] = __fmaf_rn(g[j], d[j], sum_h[j]);
                    }
                }
            });
#pragma unroll
        for (int j = 0; j < V; ++j) sum_h[j] *= p.rs[j];
        for (uint32_t off = 1u << s.lanes_log; off < 64; off <<= 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sum_h[j] += __shfl_xor(sum_h[j], off);
                sum_1[j] += __shfl_xor(sum_1[j], off);
            }
        }
        const uint32_t wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == lane) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                lds_h[wave][lane * V + j] = sum_h[j];
                lds_1[wave][lane * V + j] = sum_1[j];
            }
        }
        __syncthreads();
        gn_store_channels<V>(s, w, [&](uint32_t t) {
            float2 v = make_float2(lds_h[0][t], lds_1[0][t]);
            for (int i = 1; i < kBlock / 64; ++i) {
                v.x += lds_h[i][t];
                v.y += lds_1[i][t];
            }
            return v;
        }, partial);
        __syncthreads();
    }
}

// Means of a and of a h over a group: pairs [images, G].  Block `block` of `blocks`.
__device__ __forceinline__ void gn_means(const GnShape& s, uint32_t block, uint32_t blocks, const float* __restrict__ partial, const LnParam& weight,
                                         float2* __restrict__ means) {
    gn_each_group_sums(
        s, block, blocks,
        [&](int64_t g, uint32_t part, uint32_t parts, double& sum_h, double& sum_1) {
            const int64_t worker = gn_worker(s, g / s.G);
            gn_each_part(s, g, part, parts, [&](size_t at, uint32_t c, uint32_t) {
                const double w = weight.data ? (double)load_any(weight.data, worker * weight.stride + c, weight.type) : 1.0;
                sum_h += w * (double)partial[at];
                sum_1 += w * (double)partial[at + s.C];
            });
        },
        [&](int64_t g, double sum_h, double sum_1) {
            const double n = (double)s.S * (double)s.per_group;
            means[g] = make_float2((float)(sum_1 / n), (float)(sum_h / n));
        });
}

// dw and db, the sums in fp64 of partial sums: `parts` of each of `workers` (one: all of them).  Sums that take several launches go through
// `run`.
struct GnParamGrads {
    int64_t parts;
    uint32_t workers, columns;         // columns: blocks of 32 channels
    double* run;
    bool first, last;
    LnParam dw, db;
};
// 32 channels of one of the two gradients at a time per block, 8 threads to a channel.
__device__ __forceinline__ void gn_param_grads(uint32_t C, uint32_t block, uint32_t blocks, const float* __restrict__ partial, const GnParamGrads& a) {
    __shared__ double lds[8][32];
    const uint32_t col = threadIdx.x & 31, slice = threadIdx.x >> 5;
    for (int64_t i = block; i < (int64_t)a.workers * a.columns * 2; i += blocks) {
        const uint32_t which = (uint32_t)i & 1, half = (uint32_t)(i >> 1), worker = half / a.columns, c = (half - worker * a.columns) * 32 + col;
        const LnParam& out = which ? a.db : a.dw;
        if (!out.data) continue;
        const float* const p = partial + (size_t)worker * a.parts * 2 * C + (which ? C : 0);
        double sum = 0.0;
        if (c < C) {
#pragma unroll 4
            for (int64_t q = slice; q < a.parts; q += 8) sum += (double)p[(size_t)q * 2 * C + c];
        }
        lds[slice][col] = sum;
        __syncthreads();
        if (slice == 0 && c < C) {
            for (int q = 1; q < 8; ++q) sum += lds[q][col];
            double* const so_far = a.run + (which ? C : 0u) + c;
            if (!a.first) sum += *so_far;
            if (a.last) store_any(out.data, (int64_t)worker * out.stride + c, out.type, (float)sum);
            else *so_far = sum;
        }
        __syncthreads();
    }
}
// Both in one launch: the first `blocks` blocks make the means.  Either may be left out (blocks = 0; no gradients asked for).
template <int>
__global__ __launch_bounds__(kBlock) void k_gn_after_sums(GnShape s, uint32_t blocks, const float* __restrict__ partial, LnParam weight, float2* __restrict__ means,
                                                          GnParamGrads params) {
    if (blockIdx.x < blocks) gn_means(s, blockIdx.x, blocks, partial, weight, means);
    else gn_param_grads(s.C, blockIdx.x - blocks, gridDim.x - blocks, partial, params);
}

template <typename T, int V, int ACT, bool SAVED>
__global__ __launch_bounds__(kBlock) void k_gn_dx(GnShape s, bool keep, const float* __restrict__ mean, const float* __restrict__ rstd, const float2* __restrict__ means,
                                                  GnImages dy, GnImages x, Saved saved, GnImages dx, LnParam weight, LnParam bias) {
    const uint32_t lane = threadIdx.x & ((1u << s.lanes_log) - 1), thread = threadIdx.x >> s.lanes_log, threads = kBlock >> s.lanes_log;
    for (int64_t work = blockIdx.x; work < gn_works(s); work += gridDim.x) {
        const GnWork w = gn_work(s, work);
        const GnColumns k = gn_columns<V>(s, w.tile, lane);
        if (!k.any) continue;
        const T* const xs = SAVED ? nullptr : gn_image<const T>(x, s, w.image);
        const T* const gs = gn_image<const T>(dy, s, w.image);
        T* const to = gn_image<T>(dx, s, w.image);
        GnParams<V> p;
        p.load(s, w.image, k, mean, rstd, weight, bias);
        // dx = rs (dz w - m1 - d rs m2) = dz zw - (d k2 + k1)
        float zw[V], k1[V], k2[V];
        gn_each_group<V>(s, k.c, [&](int j, uint32_t g) {
            const float2 m = means[w.image * s.G + g];
            zw[j] = p.rs[j] * p.w[j];
            k1[j] = p.rs[j] * m.x;
            k2[j] = p.rs[j] * (p.rs[j] * m.y);
        });
        const int64_t step = threads * dx.row;
        gn_walk(w, thread, threads, [&](int64_t r, auto rows) {
            constexpr int R = decltype(rows)::value;
            GnRaw<T, V, SAVED> raw[R];
            GnRaw<T, V, false> grad[R];
            gn_load<T, V, SAVED, R>(raw, grad, xs, x, saved, gs, dy, s, w, r, threads, k);
            T* const first = to + r * dx.row;
#pragma unroll
            for (int u = 0; u < R; ++u) {
                float d[V], g[V];
                raw[u].center(k, p.mu, d);
                grad[u].widen(k, g);
                gn_dz<T, V, ACT>(g, d, zw, p, raw[u], grad[u], k);
#pragma unroll
                for (int j = 0; j < V; ++j) d[j] = __fmaf_rn(g[j], zw[j], -__fmaf_rn(d[j], k2[j], k1[j]));
                gn_store<T, V>(keep, first + u * step, k, d);
            }
        });
    }
}

}  // namespace liec
