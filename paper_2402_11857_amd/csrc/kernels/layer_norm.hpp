// Layer normalisation of N workers' activations, each worker with weights of its own, and its gradients.
//
//   forward    mu = mean_j x_j,  var = mean_j (x_j - mu)^2,  rstd = 1 / sqrt(var + eps),  y_j = (x_j - mu) rstd w_j + b_j
//   backward   h_j = (x_j - mu) rstd,  a_j = dy_j w_j,  dx_j = rstd (a_j - mean a - h_j mean(a h))
//              dw_j = sum over the worker's rows of dy_j h_j,  db_j = sum over them of dy_j
//
// A team of TEAM lanes holds one row in registers, K vectors of 16 bytes per lane, so that a row is read once; teams of up
// to a wave add up inside the wave, larger ones through LDS.  The sums of a row are fp32, in chains of at most 64 additions; a weight
// gradient is fp32 within a block, over at most 256 rows of a team, and fp64 from there on.  Rows that no team holds take fp64 in all.
// The last vector of a row that is not a multiple of a vector long starts a vector's length before the row's end: what it
// shares with the vector before it is left out of the sums and stored twice with the same value, and no access needs a branch.
//
// Both kernels are bound by memory.  Measured on 8 x 8192 rows of 4096 bf16 columns: forward 181 us (5.9 TB/s of x and y, a copy
// of that size 6.6), backward 274 us (5.9 TB/s of dy, x and dx; 5 us of it add up 512 partial sums).
#pragma once
#include <type_traits>

#include "elements.hpp"

namespace liec {

constexpr int kLnShortest = 8;         // columns of the shortest row that a team holds
constexpr int kLnWide = 1024;          // threads that walk a row too long (or too short) for registers

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
// Sum over groups of W lanes (2 .. 64), the same bits in every lane of the group.
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
    v += dpp_move<0xb1>(v);                      // quad_perm 1 0 3 2
    if (W >= 4) v += dpp_move<0x4e>(v);          // quad_perm 2 3 0 1
    if (W >= 8) v += dpp_move<0x141>(v);         // row_half_mirror: the other quad of 8 lanes
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
// it (V or more: the vector lies beyond the row).  A FULL row ends with the team's last vector.
template <int TEAM, int V, bool FULL>
__device__ __forceinline__ uint32_t vec_start(uint32_t l, int k, uint32_t C, uint32_t& skip) {
    const uint32_t c = (k * TEAM + l) * V, s = FULL ? c : min(c, C - V);
    skip = c - s;
    return s;
}
// Element `at` of a row.  For whole waves on one row the row's address is scalar and `at` the only part that a lane holds.
template <typename T>
__device__ __forceinline__ T* in_row(T* row, uint32_t at) {
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type byte;
    return reinterpret_cast<T*>(reinterpret_cast<byte*>(row) + (uint32_t)(at * sizeof(T)));
}
// The team that a thread belongs to, known to be the same for a whole wave where it is.
template <int TEAM>
__device__ __forceinline__ uint32_t team_index() {
    const uint32_t team = threadIdx.x / TEAM;
    if (TEAM < 64) return team;
    return __builtin_amdgcn_readfirstlane(team);
}
// Whether vector k may lie at or beyond the end of its row: rows that half as many vectors per lane hold take a smaller team,
// except for the smallest one.
template <int TEAM, int K, bool FULL>
constexpr bool may_end(int k) { return !FULL && (TEAM == 8 || k >= K / 2); }

template <int V>
__device__ __forceinline__ void load_param(const LnParam& p, uint32_t worker, uint32_t col, float absent, float (&f)[V]) {
    if (!p.data) {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = absent;
        return;
    }
    const int64_t at = (int64_t)worker * p.stride + col;
    auto load = [&](auto* from) {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = widen(from[at + j]);
    };
    if (p.type == kF32) load(static_cast<const float*>(p.data));
    else if (p.type == kBF16) load(static_cast<const bf16*>(p.data));
    else load(static_cast<const f16*>(p.data));
}

// ---- forward -------------------------------------------------------------------------------------------------------
// Block (b, worker): TEAM lanes to a row, rows dealt out to the blocks' teams in turn, the next row of a team requested ahead.
// keep: the results are left in the caches for whoever reads them next.
template <typename T, int TEAM, int K, bool FULL>
__global__ __launch_bounds__((TEAM > 64 ? TEAM : kBlock)) void k_ln_forward(uint32_t C, float eps, int64_t R, bool keep, float* __restrict__ mean,
                                                                            float* __restrict__ rstd, LnRows x, LnRows y, LnParam w, LnParam b) {
    constexpr int TEAMS = TEAM > 64 ? 1 : kBlock / TEAM, WAVES = TEAM > 64 ? TEAM / 64 : 1, V = Vec16<T>::n;
    constexpr int LANES = TEAM > 64 ? 64 : TEAM;
    __shared__ float lds[2][2][WAVES];
    const uint32_t worker = blockIdx.y, l = threadIdx.x % TEAM, team = team_index<TEAM>(), wave = l >> 6;
    const int64_t first = (int64_t)blockIdx.x * TEAMS + team, step = (int64_t)gridDim.x * TEAMS;
    const T* const xs = static_cast<const T*>(x.data) + (int64_t)worker * x.worker;
    T* const ys = static_cast<T*>(y.data) + (int64_t)worker * y.worker;
    const int64_t stat = (int64_t)worker * R;
    uint32_t at[K], skip[K];
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] = vec_start<TEAM, V, FULL>(l, k, C, skip[k]);
    v4u held[K];
    if (first < R) {
#pragma unroll
        for (int k = 0; k < K; ++k) held[k] = ld16<T, true>(in_row(xs + first * x.row, at[k]));
    }
    float wv[K][V], bv[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_param<V>(w, worker, at[k], 1.f, wv[k]);
        load_param<V>(b, worker, at[k], 0.f, bv[k]);
    }
    const float inv = 1.f / (float)C;
    // columns of this lane's wave, and of the wave whose sums this lane puts together
    const uint32_t other = l & (WAVES - 1);
    float mine = 0.f, others = 0.f, mine_inv = inv, others_inv = 0.f;
    if (WAVES > 1) {
        uint32_t left_out = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) left_out += min(skip[k], (uint32_t)V);
        mine = lanes_sum<64>((float)(K * V - left_out));
        if ((l & 63) == 0) lds[1][0][wave] = mine;
        __syncthreads();
        others = lds[1][0][other];
        mine_inv = 1.f / fmaxf(mine, 1.f);
        others_inv = 1.f / fmaxf(others, 1.f);
    }
    uint32_t parity = 0;
    for (int64_t r = first; r < R; r += step) {
        float f[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) Vec16<T>::widen(held[k], f[k]);
        if (r + step < R) {
#pragma unroll
            for (int k = 0; k < K; ++k) held[k] = ld16<T, true>(in_row(xs + (r + step) * x.row, at[k]));
        }
        float s = 0.f, m2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s += !may_end<TEAM, K, FULL>(k) || (uint32_t)j >= skip[k] ? f[k][j] : 0.f;
        s = lanes_sum<LANES>(s);
        // squares around the row's mean, or around the wave's own
        float mu = s * mine_inv;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = f[k][j] - mu;
                m2 = !may_end<TEAM, K, FULL>(k) || (uint32_t)j >= skip[k] ? __fmaf_rn(d, d, m2) : m2;
            }
        m2 = lanes_sum<LANES>(m2);
        if (WAVES > 1) {
            // waves' sums of squares around their own means, put together around the row's
            if ((l & 63) == 0) {
                lds[parity][0][wave] = s;
                lds[parity][1][wave] = m2;
            }
            __syncthreads();
            const float sq = lds[parity][0][other], mq = lds[parity][1][other];
            mu = lanes_sum<WAVES>(sq) * inv;
            const float d = __fmaf_rn(sq, others_inv, -mu);
            m2 = lanes_sum<WAVES>(__fmaf_rn(others * d, d, mq));
            parity ^= 1;
        }
        const float rs = rsqrtf(__fmaf_rn(m2, inv, eps));
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float o[V];
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = __fmaf_rn((f[k][j] - mu) * rs, wv[k][j], bv[k][j]);
            if (!may_end<TEAM, K, FULL>(k) || skip[k] < V) st16_as<T>(keep, in_row(ys + r * y.row, at[k]), Vec16<T>::narrow(o));
        }
        if (l == 0) {
            if (mean) mean[stat + r] = mu;
            if (rstd) rstd[stat + r] = rs;
        }
    }
}

// Rows of any length: a block to a row, which it reads three times (from the caches after the first).
template <typename T>
__global__ __launch_bounds__(kLnWide) void k_ln_forward_wide(int64_t C, float eps, int64_t R, float* __restrict__ mean, float* __restrict__ rstd,
                                                             LnRows x, LnRows y, LnParam w, LnParam b) {
    __shared__ double lds_w[kLnWide / 64];
    const uint32_t worker = blockIdx.y;
    for (int64_t r = blockIdx.x; r < R; r += gridDim.x) {
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
        __syncthreads();                                    // lds_w is the next row's
    }
}

// ---- backward ------------------------------------------------------------------------------------------------------
// Block (b, worker): dx of its rows, and their share of dw and db in registers, which it leaves in partial[worker][b]
// (2 x C values), or in dw and db themselves where it is the only one (partial == nullptr).  The next P rows of a
// team are requested ahead.
template <typename T, int TEAM, int K, bool FULL, int P>
__global__ __launch_bounds__((TEAM > 64 ? TEAM : kBlock), (K * Vec16<T>::n == 8 || TEAM == 1024 ? 4 : 2))
void k_ln_backward(uint32_t C, int64_t R, bool keep, float* __restrict__ partial, const float* __restrict__ mean, const float* __restrict__ rstd,
                   LnRows dy, LnRows x, LnRows dx, LnParam w, LnParam dw, LnParam db) {
    constexpr int TEAMS = TEAM > 64 ? 1 : kBlock / TEAM, WAVES = TEAM > 64 ? TEAM / 64 : 1, V = Vec16<T>::n;
    constexpr int LANES = TEAM > 64 ? 64 : TEAM, COLS = TEAM <= 64 ? TEAM * K * V : 1;
    __shared__ float lds[2][2][WAVES];
    __shared__ __align__(16) float sums[2][COLS];
    const uint32_t worker = blockIdx.y, l = threadIdx.x % TEAM, team = team_index<TEAM>();
    const int64_t first = (int64_t)blockIdx.x * TEAMS + team, step = (int64_t)gridDim.x * TEAMS;
    const T* const xs = static_cast<const T*>(x.data) + (int64_t)worker * x.worker;
    const T* const gs = static_cast<const T*>(dy.data) + (int64_t)worker * dy.worker;
    T* const os = static_cast<T*>(dx.data) + (int64_t)worker * dx.worker;
    const float* const mus = mean + (int64_t)worker * R;
    const float* const rss = rstd + (int64_t)worker * R;
    uint32_t at[K], skip[K];
    float wv[K][V], aw[K][V], ab[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) at[k] = vec_start<TEAM, V, FULL>(l, k, C, skip[k]);
    v4u rx[P][K], rg[P][K];
    float mu[P], rs[P];
    // 0, in a vector register: mean and rstd come with the row's vectors.  As scalar loads they were waited for at the next LDS
    // access (8 x 8192 rows of 4096 bf16 columns 296 -> 279 us).
    uint32_t none;
    asm volatile("v_mov_b32 %0, 0" : "=v"(none));
    auto request = [&](int64_t r, v4u (&vx)[K], v4u (&vg)[K], float& m, float& s) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            vx[k] = ld16<T, true>(in_row(xs + r * x.row, at[k]));
            vg[k] = ld16<T, true>(in_row(gs + r * dy.row, at[k]));
        }
        m = mus[r + none];
        s = rss[r + none];
    };
#pragma unroll
    for (int q = 0; q < P; ++q)
        if (first + q * step < R) request(first + q * step, rx[q], rg[q], mu[q], rs[q]);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        load_param<V>(w, worker, at[k], 1.f, wv[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) aw[k][j] = ab[k][j] = 0.f;
    }
    const float inv = 1.f / (float)C;
    uint32_t parity = 0;
    auto row = [&](int64_t r, v4u (&vx)[K], v4u (&vg)[K], float& m, float& s) {
        float h[K][V], a[K][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float g[V];
            Vec16<T>::widen(vx[k], h[k]);
            Vec16<T>::widen(vg[k], g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool in = !may_end<TEAM, K, FULL>(k) || (uint32_t)j >= skip[k];
                h[k][j] = (h[k][j] - m) * s;
                a[k][j] = g[j] * wv[k][j];
                ab[k][j] += in ? g[j] : 0.f;
                aw[k][j] = in ? __fmaf_rn(g[j], h[k][j], aw[k][j]) : aw[k][j];
                s1 += in ? a[k][j] : 0.f;
                s2 = in ? __fmaf_rn(a[k][j], h[k][j], s2) : s2;
            }
        }
        const float rs_now = s;
        if (r + P * step < R) request(r + P * step, vx, vg, m, s);
        s1 = lanes_sum<LANES>(s1);
        s2 = lanes_sum<LANES>(s2);
        if (WAVES > 1) {
            if ((l & 63) == 0) {
                lds[parity][0][l >> 6] = s1;
                lds[parity][1][l >> 6] = s2;
            }
            __syncthreads();
            s1 = lanes_sum<WAVES>(lds[parity][0][l & (WAVES - 1)]);
            s2 = lanes_sum<WAVES>(lds[parity][1][l & (WAVES - 1)]);
            parity ^= 1;
        }
        const float c1 = s1 * inv, c2 = s2 * inv;
        if (dx.data) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = rs_now * __fmaf_rn(-h[k][j], c2, a[k][j] - c1);
                if (!may_end<TEAM, K, FULL>(k) || skip[k] < V) st16_as<T>(keep, in_row(os + r * dx.row, at[k]), Vec16<T>::narrow(o));
            }
        }
    };
    for (int64_t r = first; r < R; r += P * step) {
#pragma unroll
        for (int q = 0; q < P; ++q)
            if (r + q * step < R) row(r + q * step, rx[q], rg[q], mu[q], rs[q]);
    }
    if (!dw.data && !db.data) return;
    float* const out = partial ? partial + ((size_t)worker * gridDim.x + blockIdx.x) * 2 * C : nullptr;
    if (TEAM <= 64) {
        // the block's teams, wave after wave, in LDS; then columns in order
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                aw[k][j] = groups_sum<TEAM>(aw[k][j]);
                ab[k][j] = groups_sum<TEAM>(ab[k][j]);
            }
        for (uint32_t q = 0; q < kBlock / 64; ++q) {
            if ((threadIdx.x >> 6) == q && (threadIdx.x & 63) < LANES) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    float* const sw = &sums[0][(k * TEAM + l) * V];
                    float* const sb = &sums[1][(k * TEAM + l) * V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        sw[j] = q ? sw[j] + aw[k][j] : aw[k][j];
                        sb[j] = q ? sb[j] + ab[k][j] : ab[k][j];
                    }
                }
            }
            __syncthreads();
        }
        for (uint32_t c = threadIdx.x; c < C; c += kBlock) {
            // column c is where its vector put it: the last vector of a row starts early
            const uint32_t v = c / V, s = min(v * V, C - V), i = v * V + (c - s);
            const float sw = sums[0][i], sb = sums[1][i];
            if (out) {
                out[c] = sw;
                out[C + c] = sb;
            } else {
                if (dw.data) store_any(dw.data, (int64_t)worker * dw.stride + c, dw.type, sw);
                if (db.data) store_any(db.data, (int64_t)worker * db.stride + c, db.type, sb);
            }
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            if (out && skip[k] == 0) {
                const uint32_t c = at[k] + j;
                st16<float, false>(out + c, v4u{__float_as_uint(aw[k][j]), __float_as_uint(aw[k][j + 1]), __float_as_uint(aw[k][j + 2]), __float_as_uint(aw[k][j + 3])});
                st16<float, false>(out + C + c, v4u{__float_as_uint(ab[k][j]), __float_as_uint(ab[k][j + 1]), __float_as_uint(ab[k][j + 2]), __float_as_uint(ab[k][j + 3])});
                continue;
            }
#pragma unroll
            for (int i = j; i < j + 4; ++i) {
                if ((uint32_t)i < skip[k]) continue;
                if (out) {
                    out[at[k] + i] = aw[k][i];
                    out[C + at[k] + i] = ab[k][i];
                } else {
                    if (dw.data) store_any(dw.data, (int64_t)worker * dw.stride + at[k] + i, dw.type, aw[k][i]);
                    if (db.data) store_any(db.data, (int64_t)worker * db.stride + at[k] + i, db.type, ab[k][i]);
                }
            }
        }
    }
}

// dw and db of group blockIdx.y: the sum of its `parts` partial sums, 32 columns per block, 8 threads to a column.  In fp64: the number
// of parts grows with rows and workers (65535 equal ones in fp32 were off by 1400 u).
__global__ __launch_bounds__(kBlock) void k_ln_param_grads(const float* __restrict__ partial, uint32_t parts, int64_t C, LnParam dw, LnParam db) {
    __shared__ double lds[8][32];
    const LnParam& out = blockIdx.z ? db : dw;
    if (!out.data) return;
    const uint32_t col = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + col;
    const float* const p = partial + (size_t)blockIdx.y * parts * 2 * C + (blockIdx.z ? C : 0);
    double s = 0.0;
    if (c < C) {
#pragma unroll 4
        for (uint32_t q = slice; q < parts; q += 8) s += (double)p[(size_t)q * 2 * C + c];
    }
    lds[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < C) {
        s = lds[0][col];
        for (int q = 1; q < 8; ++q) s += lds[q][col];
        store_any(out.data, (int64_t)blockIdx.y * out.stride + c, out.type, (float)s);
    }
}

// Rows of any length: dx, a block to a row.
template <typename T>
__global__ __launch_bounds__(kLnWide) void k_ln_backward_wide(int64_t C, int64_t R, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                              LnRows dy, LnRows x, LnRows dx, LnParam w) {
    __shared__ double lds_w[2][kLnWide / 64];
    const uint32_t worker = blockIdx.y;
    auto weight = [&](int64_t j) { return w.data ? load_any(w.data, (int64_t)worker * w.stride + j, w.type) : 1.f; };
    for (int64_t r = blockIdx.x; r < R; r += gridDim.x) {
        const T* const xr = static_cast<const T*>(x.data) + (int64_t)worker * x.worker + r * x.row;
        const T* const gr = static_cast<const T*>(dy.data) + (int64_t)worker * dy.worker + r * dy.row;
        T* const out = static_cast<T*>(dx.data) + (int64_t)worker * dx.worker + r * dx.row;
        const float mu = mean[(int64_t)worker * R + r], rs = rstd[(int64_t)worker * R + r];
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
        __syncthreads();                                    // lds_w is the next row's
    }
}

// The same rows' share of dw and db: block (columns, worker, strip), a thread to a column.  In fp64: a strip may have any number of rows.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_ln_columns_wide(int64_t C, int64_t per, int64_t R, float* __restrict__ partial, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, LnRows dy, LnRows x) {
    const uint32_t worker = blockIdx.y, strip = blockIdx.z;
    const int64_t c = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (c >= C) return;
    const int64_t begin = (int64_t)strip * per, end = min(begin + per, R);
    const T* const xs = static_cast<const T*>(x.data) + (int64_t)worker * x.worker + c;
    const T* const gs = static_cast<const T*>(dy.data) + (int64_t)worker * dy.worker + c;
    double aw = 0.0, ab = 0.0;
#pragma unroll 4
    for (int64_t r = begin; r < end; ++r) {
        const float mu = mean[(int64_t)worker * R + r], rs = rstd[(int64_t)worker * R + r], g = widen(gs[r * dy.row]);
        ab += (double)g;
        aw = __fma_rn((double)g, (double)((widen(xs[r * x.row]) - mu) * rs), aw);
    }
    float* const out = partial + ((size_t)worker * gridDim.z + strip) * 2 * C;
    out[c] = (float)aw;
    out[C + c] = (float)ab;
}

}  // namespace liec
