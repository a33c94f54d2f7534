// Layer normalisation of N workers' activations, each worker with weights of its own, and its gradients.
//
//   forward    mu = mean_j x_j,  var = mean_j (x_j - mu)^2,  rstd = 1 / sqrt(var + eps),  y_j = (x_j - mu) rstd w_j + b_j
//   backward   h_j = (x_j - mu) rstd,  a_j = dy_j w_j,  dx_j = rstd (a_j - mean a - h_j mean(a h))
//              dw_j = sum over the worker's rows of dy_j h_j,  db_j = sum over them of dy_j
//
// A team of TEAM lanes holds one row in registers, K vectors of 8 columns per lane, so that a row is read once; teams of up
// to a wave add up inside the wave, larger ones through LDS.  All sums are fp32, of at most a few hundred terms in a chain.
// The last vector of a row that is not a multiple of 8 columns long starts 8 columns before the row's end: what it shares
// with the vector before it is left out of the sums and stored twice with the same value, and no access needs a branch.
#pragma once
#include "elements.hpp"

namespace liec {

constexpr int kLnVec = 8;
constexpr int kLnWide = 1024;          // threads that walk a row too long (or too short) for registers

struct LnRows {                        // a [workers, rows, columns] tensor of unit column stride
    void* data;
    int64_t worker, row;               // strides, in elements
};
struct LnParam {                       // a [workers, columns] tensor of unit column stride; stride 0: one row for all workers
    void* data;
    int64_t stride;
    uint32_t type;
};

// ---- sums over a team --------------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// v of this lane plus v of the lane that differs in bit 4 (bit 5) of its number.
__device__ __forceinline__ float add_lane16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __fadd_rn(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_lane32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __fadd_rn(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Sum over groups of W lanes (8 .. 64), the same bits in every lane of the group.
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
    v += dpp_move<0xb1>(v);                      // quad_perm 1 0 3 2
    v += dpp_move<0x4e>(v);                      // quad_perm 2 3 0 1
    v += dpp_move<0x141>(v);                     // row_half_mirror: the other quad of 8 lanes
    if (W >= 16) v += dpp_move<0x140>(v);        // row_mirror: the other half of 16
    if (W >= 32) v = add_lane16(v);
    if (W >= 64) v = add_lane32(v);
    return v;
}
// Sum over the lanes of a wave that have the same place in their groups of W lanes.
template <int W>
__device__ __forceinline__ float groups_sum(float v) {
    if (W <= 8) v += dpp_move<0x128>(v);         // row_ror:8
    if (W <= 16) v = add_lane16(v);
    if (W <= 32) v = add_lane32(v);
    return v;
}

// This lane's vector k of a row of C columns: where it starts, and how many of its first columns belong to the vector before
// it (8 or more: the vector lies beyond the row).  Needs C >= 8.
template <int TEAM>
__device__ __forceinline__ uint32_t vec_start(uint32_t l, int k, uint32_t C, uint32_t& skip) {
    const uint32_t c = (k * TEAM + l) * kLnVec, s = min(c, C - kLnVec);
    skip = c - s;
    return s;
}

__device__ __forceinline__ void load_param(const LnParam& p, uint32_t worker, uint32_t col, float absent, float (&f)[8]) {
    if (!p.data) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = absent;
        return;
    }
    const int64_t at = (int64_t)worker * p.stride + col;
    if (p.type == kF32) {
        Raw8<float> r;
        r.load(static_cast<const float*>(p.data) + at);
        r.widen(f);
    } else if (p.type == kBF16) {
        Raw8<bf16> r;
        r.load(static_cast<const bf16*>(p.data) + at);
        r.widen(f);
    } else {
        Raw8<f16> r;
        r.load(static_cast<const f16*>(p.data) + at);
        r.widen(f);
    }
}

// ---- forward -------------------------------------------------------------------------------------------------------
// Block (strip, worker): rows strip * per .. of the worker, TEAM lanes to a row.
template <typename T, int TEAM, int K>
__global__ __launch_bounds__((TEAM > 64 ? TEAM : kBlock)) void k_ln_forward(uint32_t C, uint32_t per, float eps, int64_t R, float* __restrict__ mean,
                                                                                float* __restrict__ rstd, LnRows x, LnRows y, LnParam w, LnParam b) {
    constexpr int THREADS = TEAM > 64 ? TEAM : kBlock, TEAMS = THREADS / TEAM, WAVES = TEAM > 64 ? TEAM / 64 : 1;
    __shared__ float lds[2][3][WAVES > 1 ? WAVES : 1];
    const uint32_t worker = blockIdx.y, l = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const int64_t begin = (int64_t)blockIdx.x * per, end = min(begin + (int64_t)per, R);
    const T* const xs = static_cast<const T*>(x.data) + (int64_t)worker * x.worker;
    T* const ys = static_cast<T*>(y.data) + (int64_t)worker * y.worker;
    uint32_t at[K], skip[K];
    float wv[K][8], bv[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] = vec_start<TEAM>(l, k, C, skip[k]);
    int64_t r = begin + team;
    Raw8<T> raw[K];
    if (r < end) {
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k].load_stream(xs + r * x.row + at[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_param(w, worker, at[k], 1.f, wv[k]);
        load_param(b, worker, at[k], 0.f, bv[k]);
    }
    const float inv = 1.f / (float)C;
    // columns that this lane's wave (of a team of several) counts, for the waves' means
    const uint32_t wave = l >> 6;
    uint32_t parity = 0;
    for (; r < end; r += TEAMS) {
        float f[K][8];
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k].widen(f[k]);
        if (r + TEAMS < end) {
#pragma unroll
            for (int k = 0; k < K; ++k) raw[k].load_stream(xs + (r + TEAMS) * x.row + at[k]);
        }
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) s += (uint32_t)j >= skip[k] ? f[k][j] : 0.f;
        float mu, m2 = 0.f;
        if (WAVES == 1) {
            mu = lanes_sum<(TEAM > 64 ? 64 : TEAM)>(s) * inv;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = f[k][j] - mu;
                    m2 = (uint32_t)j >= skip[k] ? __fmaf_rn(d, d, m2) : m2;
                }
            m2 = lanes_sum<(TEAM > 64 ? 64 : TEAM)>(m2);
        } else {
            // every wave's own sum and its squares around its own mean, put together as sums of squares around the row's mean
            s = lanes_sum<64>(s);
            uint32_t mine = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const uint32_t c0 = (k * TEAM + wave * 64) * kLnVec;
                mine += c0 < C ? min(C - c0, 64u * kLnVec) : 0u;
            }
            const float own = mine ? s / (float)mine : 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = f[k][j] - own;
                    m2 = (uint32_t)j >= skip[k] ? __fmaf_rn(d, d, m2) : m2;
                }
            m2 = lanes_sum<64>(m2);
            if ((l & 63) == 0) {
                lds[parity][0][wave] = s;
                lds[parity][1][wave] = m2;
                lds[parity][2][wave] = (float)mine;
            }
            __syncthreads();
            float total = 0.f;
#pragma unroll
            for (int q = 0; q < WAVES; ++q) total += lds[parity][0][q];
            mu = total * inv;
            m2 = 0.f;
#pragma unroll
            for (int q = 0; q < WAVES; ++q) {
                const float cnt = lds[parity][2][q];
                const float d = cnt > 0.f ? lds[parity][0][q] / cnt - mu : 0.f;
                m2 += __fmaf_rn(cnt * d, d, lds[parity][1][q]);
            }
            parity ^= 1;
        }
        const float rs = rsqrtf(__fmaf_rn(m2, inv, eps));
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = __fmaf_rn((f[k][j] - mu) * rs, wv[k][j], bv[k][j]);
            if (skip[k] < kLnVec) Raw8<T>::store(ys + r * y.row + at[k], o);
        }
        if (l == 0) {
            if (mean) mean[(int64_t)worker * R + r] = mu;
            if (rstd) rstd[(int64_t)worker * R + r] = rs;
        }
    }
}

// Rows of any length: one block per row, which it reads three times (from the caches after the first).
template <typename T>
__global__ __launch_bounds__(kLnWide) void k_ln_forward_wide(int64_t C, float eps, int64_t R, float* __restrict__ mean, float* __restrict__ rstd,
                                                             LnRows x, LnRows y, LnParam w, LnParam b) {
    __shared__ double lds_w[kLnWide / 64];
    const uint32_t worker = blockIdx.y;
    const int64_t r = blockIdx.x;
    const T* const xr = static_cast<const T*>(x.data) + (int64_t)worker * x.worker + r * x.row;
    T* const yr = static_cast<T*>(y.data) + (int64_t)worker * y.worker + r * y.row;
    double acc = 0.0;
    for (int64_t j = threadIdx.x; j < C; j += blockDim.x) acc += (double)widen(xr[j]);
    acc = block_sum_f64(acc, lds_w);
    if (threadIdx.x == 0) lds_w[0] = acc / (double)C;
    __syncthreads();
    const double mu = lds_w[0];
    __syncthreads();
    acc = 0.0;
    for (int64_t j = threadIdx.x; j < C; j += blockDim.x) {
        const double d = (double)widen(xr[j]) - mu;
        acc = __fma_rn(d, d, acc);
    }
    acc = block_sum_f64(acc, lds_w);
    if (threadIdx.x == 0) lds_w[0] = acc / (double)C;
    __syncthreads();
    const float rs = (float)(1.0 / __dsqrt_rn(lds_w[0] + (double)eps)), m = (float)mu;
    for (int64_t j = threadIdx.x; j < C; j += blockDim.x) {
        const float wj = w.data ? load_any(w.data, (int64_t)worker * w.stride + j, w.type) : 1.f;
        const float bj = b.data ? load_any(b.data, (int64_t)worker * b.stride + j, b.type) : 0.f;
        yr[j] = narrow<T>(__fmaf_rn((widen(xr[j]) - m) * rs, wj, bj));
    }
    if (threadIdx.x == 0) {
        if (mean) mean[(int64_t)worker * R + r] = m;
        if (rstd) rstd[(int64_t)worker * R + r] = rs;
    }
}

// ---- backward ------------------------------------------------------------------------------------------------------
// Block (strip, worker): dx of its rows, and their share of dw and db in registers, which it leaves in partial[worker][strip]
// (2 x C values), or in dw and db themselves where it is the only one (partial == nullptr).
template <typename T, int TEAM, int K>
__global__ __launch_bounds__((TEAM > 64 ? TEAM : kBlock)) void k_ln_backward(uint32_t C, uint32_t per, int64_t R, float* __restrict__ partial,
                                                                                 const float* __restrict__ mean, const float* __restrict__ rstd, LnRows dy,
                                                                                 LnRows x, LnRows dx, LnParam w, LnParam dw, LnParam db) {
    constexpr int THREADS = TEAM > 64 ? TEAM : kBlock, TEAMS = THREADS / TEAM, WAVES = TEAM > 64 ? TEAM / 64 : 1;
    constexpr int COLS = TEAM <= 64 ? TEAM * K * kLnVec : 1;
    __shared__ float lds[2][2][WAVES];
    __shared__ __align__(16) float sums[2][COLS];
    const uint32_t worker = blockIdx.y, l = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const int64_t begin = (int64_t)blockIdx.x * per, end = min(begin + (int64_t)per, R);
    const T* const xs = static_cast<const T*>(x.data) + (int64_t)worker * x.worker;
    const T* const gs = static_cast<const T*>(dy.data) + (int64_t)worker * dy.worker;
    T* const os = static_cast<T*>(dx.data) + (int64_t)worker * dx.worker;
    const float* const mus = mean + (int64_t)worker * R;
    const float* const rss = rstd + (int64_t)worker * R;
    uint32_t at[K], skip[K];
    float wv[K][8], aw[K][8], ab[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] = vec_start<TEAM>(l, k, C, skip[k]);
    int64_t r = begin + team;
    Raw8<T> rx[K], rg[K];
    float mu = 0.f, rs = 0.f;
    if (r < end) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            rx[k].load_stream(xs + r * x.row + at[k]);
            rg[k].load_stream(gs + r * dy.row + at[k]);
        }
        mu = mus[r];
        rs = rss[r];
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_param(w, worker, at[k], 1.f, wv[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) aw[k][j] = ab[k][j] = 0.f;
    }
    const float inv = 1.f / (float)C;
    uint32_t parity = 0;
    for (; r < end; r += TEAMS) {
        float h[K][8], a[K][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float g[8];
            rx[k].widen(h[k]);
            rg[k].widen(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = (uint32_t)j >= skip[k];
                h[k][j] = (h[k][j] - mu) * rs;
                a[k][j] = g[j] * wv[k][j];
                ab[k][j] += in ? g[j] : 0.f;
                aw[k][j] = in ? __fmaf_rn(g[j], h[k][j], aw[k][j]) : aw[k][j];
                s1 += in ? a[k][j] : 0.f;
                s2 = in ? __fmaf_rn(a[k][j], h[k][j], s2) : s2;
            }
        }
        const float rs_now = rs;
        if (r + TEAMS < end) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                rx[k].load_stream(xs + (r + TEAMS) * x.row + at[k]);
                rg[k].load_stream(gs + (r + TEAMS) * dy.row + at[k]);
            }
            mu = mus[r + TEAMS];
            rs = rss[r + TEAMS];
        }
        s1 = lanes_sum<(TEAM > 64 ? 64 : TEAM)>(s1);
        s2 = lanes_sum<(TEAM > 64 ? 64 : TEAM)>(s2);
        if (WAVES > 1) {
            if ((l & 63) == 0) {
                lds[parity][0][l >> 6] = s1;
                lds[parity][1][l >> 6] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int q = 0; q < WAVES; ++q) {
                s1 += lds[parity][0][q];
                s2 += lds[parity][1][q];
            }
            parity ^= 1;
        }
        const float c1 = s1 * inv, c2 = s2 * inv;
        if (dx.data) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = rs_now * __fmaf_rn(-h[k][j], c2, a[k][j] - c1);
                if (skip[k] < kLnVec) Raw8<T>::store(os + r * dx.row + at[k], o);
            }
        }
    }
    if (!dw.data && !db.data) return;
    float* const out = partial ? partial + ((size_t)worker * gridDim.x + blockIdx.x) * 2 * C : nullptr;
    if (TEAM <= 64) {
        // the block's teams, wave after wave, in LDS; then columns in order
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                aw[k][j] = groups_sum<TEAM>(aw[k][j]);
                ab[k][j] = groups_sum<TEAM>(ab[k][j]);
            }
        for (uint32_t q = 0; q < kBlock / 64; ++q) {
            if ((threadIdx.x >> 6) == q && (threadIdx.x & 63) < (TEAM > 64 ? 64 : TEAM)) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    float* const sw = &sums[0][(k * TEAM + l) * kLnVec];
                    float* const sb = &sums[1][(k * TEAM + l) * kLnVec];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        sw[j] = q ? sw[j] + aw[k][j] : aw[k][j];
                        sb[j] = q ? sb[j] + ab[k][j] : ab[k][j];
                    }
                }
            }
            __syncthreads();
        }
        for (uint32_t c = threadIdx.x; c < C; c += kBlock) {
            // column c is where its vector put it: the last vector of a row starts early
            const uint32_t v = c / kLnVec, s = min(v * kLnVec, C - kLnVec), i = v * kLnVec + (c - s);
            const float sw = sums[0][i], sb = sums[1][i];
            if (out) {
                out[c] = sw;
                out[C + c] = sb;
            } else {
                if (dw.data) store_any(dw.data, (int64_t)worker * dw.stride + c, dw.type, sw);
                if (db.data) store_any(db.data, (int64_t)worker * db.stride + c, db.type, sb);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (out && skip[k] == 0) {
                st16<float, false>(out + at[k], v4u{__float_as_uint(aw[k][0]), __float_as_uint(aw[k][1]), __float_as_uint(aw[k][2]), __float_as_uint(aw[k][3])});
                st16<float, false>(out + at[k] + 4, v4u{__float_as_uint(aw[k][4]), __float_as_uint(aw[k][5]), __float_as_uint(aw[k][6]), __float_as_uint(aw[k][7])});
                st16<float, false>(out + C + at[k], v4u{__float_as_uint(ab[k][0]), __float_as_uint(ab[k][1]), __float_as_uint(ab[k][2]), __float_as_uint(ab[k][3])});
                st16<float, false>(out + C + at[k] + 4, v4u{__float_as_uint(ab[k][4]), __float_as_uint(ab[k][5]), __float_as_uint(ab[k][6]), __float_as_uint(ab[k][7])});
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if ((uint32_t)j < skip[k]) continue;
                    if (out) {
                        out[at[k] + j] = aw[k][j];
                        out[C + at[k] + j] = ab[k][j];
                    } else {
                        if (dw.data) store_any(dw.data, (int64_t)worker * dw.stride + at[k] + j, dw.type, aw[k][j]);
                        if (db.data) store_any(db.data, (int64_t)worker * db.stride + at[k] + j, db.type, ab[k][j]);
                    }
                }
            }
        }
    }
}

// dw and db of group blockIdx.y: the sum of its `parts` partial sums, 32 columns per block, 8 threads to a column.
__global__ __launch_bounds__(kBlock) void k_ln_param_grads(const float* __restrict__ partial, uint32_t parts, int64_t C, LnParam dw, LnParam db) {
    __shared__ float lds[8][32];
    const LnParam& out = blockIdx.z ? db : dw;
    if (!out.data) return;
    const uint32_t col = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + col;
    const float* const p = partial + (size_t)blockIdx.y * parts * 2 * C + (blockIdx.z ? C : 0);
    float s = 0.f;
    if (c < C) {
#pragma unroll 4
        for (uint32_t q = slice; q < parts; q += 8) s += p[(size_t)q * 2 * C + c];
    }
    lds[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < C) {
        s = lds[0][col];
        for (int q = 1; q < 8; ++q) s += lds[q][col];
        store_any(out.data, (int64_t)blockIdx.y * out.stride + c, out.type, s);
    }
}

// Rows of any length: dx, one block per row.
template <typename T>
__global__ __launch_bounds__(kLnWide) void k_ln_backward_wide(int64_t C, int64_t R, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                              LnRows dy, LnRows x, LnRows dx, LnParam w) {
    __shared__ double lds_w[2][kLnWide / 64];
    const uint32_t worker = blockIdx.y;
    const int64_t r = blockIdx.x;
    const T* const xr = static_cast<const T*>(x.data) + (int64_t)worker * x.worker + r * x.row;
    const T* const gr = static_cast<const T*>(dy.data) + (int64_t)worker * dy.worker + r * dy.row;
    T* const out = static_cast<T*>(dx.data) + (int64_t)worker * dx.worker + r * dx.row;
    const float mu = mean[(int64_t)worker * R + r], rs = rstd[(int64_t)worker * R + r];
    auto weight = [&](int64_t j) { return w.data ? load_any(w.data, (int64_t)worker * w.stride + j, w.type) : 1.f; };
    double s1 = 0.0, s2 = 0.0;
    for (int64_t j = threadIdx.x; j < C; j += blockDim.x) {
        const float a = widen(gr[j]) * weight(j);
        s1 += (double)a;
        s2 += (double)a * (double)((widen(xr[j]) - mu) * rs);
    }
    s1 = block_sum_f64(s1, lds_w[0]);
    s2 = block_sum_f64(s2, lds_w[1]);
    if (threadIdx.x == 0) {
        lds_w[0][0] = s1 / (double)C;
        lds_w[1][0] = s2 / (double)C;
    }
    __syncthreads();
    const float c1 = (float)lds_w[0][0], c2 = (float)lds_w[1][0];
    for (int64_t j = threadIdx.x; j < C; j += blockDim.x) {
        const float h = (widen(xr[j]) - mu) * rs;
        out[j] = narrow<T>(rs * __fmaf_rn(-h, c2, widen(gr[j]) * weight(j) - c1));
    }
}

// The same rows' share of dw and db: block (columns, worker, strip), a thread to a column.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_ln_columns_wide(int64_t C, int64_t per, int64_t R, float* __restrict__ partial, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, LnRows dy, LnRows x) {
    const uint32_t worker = blockIdx.y, strip = blockIdx.z;
    const int64_t c = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (c >= C) return;
    const int64_t begin = (int64_t)strip * per, end = min(begin + per, R);
    const T* const xs = static_cast<const T*>(x.data) + (int64_t)worker * x.worker + c;
    const T* const gs = static_cast<const T*>(dy.data) + (int64_t)worker * dy.worker + c;
    float aw = 0.f, ab = 0.f;
#pragma unroll 4
    for (int64_t r = begin; r < end; ++r) {
        const float mu = mean[(int64_t)worker * R + r], rs = rstd[(int64_t)worker * R + r], g = widen(gs[r * dy.row]);
        ab += g;
        aw = __fmaf_rn(g, (widen(xs[r * x.row]) - mu) * rs, aw);
    }
    float* const out = partial + ((size_t)worker * gridDim.z + strip) * 2 * C;
    out[c] = aw;
    out[C + c] = ab;
}

}  // namespace liec
