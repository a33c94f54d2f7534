// Gradient of a linear layer's weight from an 8-bit checkpoint of its input:
//
//   dW[o, c] = sum over rows r of dy[r, o] x[r, c],  db[o] = sum over rows of dy[r, o]       (of each worker)
//
// A product of matrices whose long axis is the rows, computed by the matrix cores from bf16 operands: x = q 2^k is one bf16 number, dy
// one (bf16), two (fp16: 11 bits) or three (fp32: 24 bits) whose sum it is exactly, so every product is exact and only their sum, in
// fp32, rounds.  Both operands lie row by row while the matrix cores take columns: they are staged in LDS as they lie, x
// widened to bf16 on the way, and read transposed, 4 rows of 16 columns by 16 lanes.
#pragma once
#include "checkpoint.hpp"

namespace liec {

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct WgShape {
    int64_t R, O, C;
    uint32_t N, splits, tiles_o, tiles_c;
    int64_t per;                       // rows of a split
};
struct WgOut {
    void* data;
    int64_t worker, row;               // strides, in elements
    uint32_t type;
};

// ---- dy as bf16 numbers ------------------------------------------------------------------------------------------------
template <typename T>
struct Parts {
    static constexpr int n = sizeof(T) == 4 ? 3 : 2;
};
template <>
struct Parts<bf16> {
    static constexpr int n = 1;
};

// Splits values into bf16 numbers by cutting bits off: what is left of a value is exact, and no part overflows.  An infinity or a NaN is
// its own first part.  Parts below the smallest bf16 number, 2^-133, are lost.
template <int P>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&w)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p == P - 1) {
            w[p] = narrow2<bf16>(a, b);
            break;
        }
        const uint32_t ha = __float_as_uint(a) & 0xffff0000u, hb = __float_as_uint(b) & 0xffff0000u;
        const bool fa = key_of(a) >= kInfKey, fb = key_of(b) >= kInfKey;
        w[p] = fa || fb ? narrow2<bf16>(fa ? a : __uint_as_float(ha), fb ? b : __uint_as_float(hb)) : hb | ha >> 16;
        a = fa ? 0.f : a - __uint_as_float(ha);
        b = fb ? 0.f : b - __uint_as_float(hb);
    }
}

// ---- tiles in LDS ------------------------------------------------------------------------------------------------------
// Rows of W columns of bf16; units of 16 columns (32 bytes) change places within a row by the row's number, so that what 16
// lanes read at a time, 4 rows at one place, and what follows it, lies on different banks.
template <int W>
__device__ __forceinline__ uint32_t wg_place(uint32_t row, uint32_t col) {
    constexpr uint32_t units = W / 16;
    const uint32_t by = units >= 8 ? row & 7 : (row >> 1) & (units - 1);
    return row * W + (((col >> 4) ^ by) << 4) + (col & 15);
}
__device__ __forceinline__ v4s wg_read(const uint16_t* at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)at);
}
__device__ __forceinline__ v8bf wg_join(v4s a, v4s b) {
    const auto r = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(v8bf, r);
}

// BM x BN values of dW per block, BK rows at a time, by WM x WN waves.
template <typename T, int BM, int BN, int BK, int WM, int WN>
struct WgTile {
    static constexpr int P = Parts<T>::n, threads = WM * WN * 64;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;           // a wave's 32 x 32 tiles
    static constexpr int a_lanes = BM / 8, a_rows = threads / a_lanes, a_loads = BK / a_rows;     // 8 columns per thread and load
    static constexpr int b_lanes = BN / 16, b_rows = threads / b_lanes, b_loads = BK < b_rows ? 1 : BK / b_rows;   // 16 columns
    static constexpr int values = BK * (P * BM + BN);                    // of a buffer
    static_assert(BK % a_rows == 0 && (BK % b_rows == 0 || b_rows % BK == 0), "whole loads");
};

template <typename T, int BM, int BN, int BK, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64) void k_weight_grad(WgShape s, LnRows dy, Saved x, WgOut dw, LnParam db, float* __restrict__ partial) {
    typedef WgTile<T, BM, BN, BK, WM, WN> W;
    constexpr int P = W::P;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][W::values];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t wave_m = wave / WN * (BM / WM), wave_n = wave % WN * (BN / WN);
    const uint32_t a_col = tid % W::a_lanes * 8, a_row = tid / W::a_lanes, b_col = tid % W::b_lanes * 16, b_row = tid / W::b_lanes;
    const bool b_mine = b_row < (uint32_t)BK;
    const uint32_t groups = (uint32_t)((s.C + kSavedCols - 1) / kSavedCols);
    const int64_t works = (int64_t)s.N * s.splits * s.tiles_o * s.tiles_c;

    for (int64_t work = blockIdx.x; work < works; work += gridDim.x) {
        const uint32_t tile_c = (uint32_t)(work % s.tiles_c), tile_o = (uint32_t)(work / s.tiles_c % s.tiles_o);
        const int64_t strip = work / s.tiles_c / s.tiles_o;
        const uint32_t split = (uint32_t)(strip % s.splits), worker = (uint32_t)(strip / s.splits);
        const int64_t o0 = (int64_t)tile_o * BM, c0 = (int64_t)tile_c * BN, r0 = split * s.per, r1 = min(r0 + s.per, s.R);
        const T* const g = static_cast<const T*>(dy.data) + (int64_t)worker * dy.worker + o0 + a_col;
        const int8_t* const q = x.q + (int64_t)worker * s.R * s.C + c0 + b_col;
        const uint8_t* const e = x.e + (int64_t)worker * s.R * groups + (uint32_t)((c0 + b_col) / kSavedCols);
        const int a_n = (int)max((int64_t)0, min((int64_t)8, s.O - o0 - a_col)), b_n = b_mine ? (int)max((int64_t)0, min((int64_t)16, s.C - c0 - b_col)) : 0;
        const bool bias = db.data && tile_c == 0;

        Eight<T> ra[W::a_loads];
        v4u rb[W::b_loads];
        uint32_t re[W::b_loads];
        float sums[8] = {};
        auto fetch = [&](int64_t r) {
#pragma unroll
            for (int i = 0; i < W::a_loads; ++i) {
                const int64_t row = r + a_row + i * W::a_rows;
                if (row < r1 && a_n == 8) {
                    ra[i] = ld_eight<T, false>(g + row * dy.row);
                } else {
                    float f[8] = {};
                    if (row < r1) {
#pragma unroll
                        for (int j = 0; j < 7; ++j)
                            if (j < a_n) f[j] = widen(g[row * dy.row + j]);
                    }
#pragma unroll
                    for (int v = 0; v < Eight<T>::words; ++v) {
                        float part[Vec16<T>::n];
#pragma unroll
                        for (int j = 0; j < Vec16<T>::n; ++j) part[j] = f[v * Vec16<T>::n + j];
                        ra[i].w[v] = Vec16<T>::narrow(part);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < W::b_loads; ++i) {
                const int64_t row = r + b_row + i * W::b_rows;
                rb[i] = v4u{0, 0, 0, 0};
                re[i] = 0;
                if (row < r1 && b_n) {
                    re[i] = e[row * groups];
                    if (b_n == 16) {
                        rb[i] = (v4u) * reinterpret_cast<const v4u_any1*>(q + row * s.C);
                    } else {
#pragma unroll
                        for (int j = 0; j < 15; ++j)
                            if (j < b_n) rb[i][j >> 2] |= (uint32_t)(uint8_t)q[row * s.C + j] << (8 * (j & 3));
                    }
                }
            }
        };
        auto stage = [&](uint16_t* to) {
#pragma unroll
            for (int i = 0; i < W::a_loads; ++i) {
                const uint32_t at = wg_place<BM>(a_row + i * W::a_rows, a_col);
                if (P == 1 && !bias) {
                    *reinterpret_cast<v4u*>(to + at) = ra[i].w[0];
                    continue;
                }
                float f[8];
                widen_eight<T>(ra[i], f);
                if (bias) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) sums[j] += f[j];
                }
                v4u w[P];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t parts[P];
                    split_pair<P>(f[2 * j], f[2 * j + 1], parts);
#pragma unroll
                    for (int p = 0; p < P; ++p) w[p][j] = parts[p];
                }
#pragma unroll
                for (int p = 0; p < P; ++p) *reinterpret_cast<v4u*>(to + p * BK * BM + at) = w[p];
            }
            if (!b_mine) return;
#pragma unroll
            for (int i = 0; i < W::b_loads; ++i) {
                float f[16];
                const float scale = saved_scale(re[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) unpack4(rb[i][j], scale, f + 4 * j);
                uint16_t* const at = to + P * BK * BM + wg_place<BN>(b_row + i * W::b_rows, b_col);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v4u w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = narrow2<bf16>(f[8 * h + 2 * j], f[8 * h + 2 * j + 1]);
                    *reinterpret_cast<v4u*>(at + 8 * h) = w;
                }
            }
        };

        v16f acc[W::TM][W::TN];
#pragma unroll
        for (int m = 0; m < W::TM; ++m)
#pragma unroll
            for (int n = 0; n < W::TN; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.f;

        // lanes 16 g .. 16 g + 15 read columns 16 (g & 1) .. of rows 8 (g >> 1) .., 4 rows at a time
        const uint32_t k_at = lane >> 5 << 3 | (lane >> 2 & 3), col_at = (lane & 16) | (lane & 3) << 2;
        fetch(r0);
        int buffer = 0;
        for (int64_t r = r0; r < r1; r += BK) {
            stage(lds[buffer]);
            __syncthreads();
            if (r + BK < r1) fetch(r + BK);
            const uint16_t* const at = lds[buffer];
#pragma unroll
            for (int kk = 0; kk < BK; kk += 16) {
                v8bf a[P][W::TM], b[W::TN];
#pragma unroll
                for (int n = 0; n < W::TN; ++n) {
                    const uint16_t* const p = at + P * BK * BM;
                    b[n] = wg_join(wg_read(p + wg_place<BN>(kk + k_at, wave_n + 32 * n + col_at)), wg_read(p + wg_place<BN>(kk + k_at + 4, wave_n + 32 * n + col_at)));
                }
#pragma unroll
                for (int p = P - 1; p >= 0; --p)
#pragma unroll
                    for (int m = 0; m < W::TM; ++m) {
                        const uint16_t* const from = at + p * BK * BM;
                        a[p][m] = wg_join(wg_read(from + wg_place<BM>(kk + k_at, wave_m + 32 * m + col_at)), wg_read(from + wg_place<BM>(kk + k_at + 4, wave_m + 32 * m + col_at)));
#pragma unroll
                        for (int n = 0; n < W::TN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[p][m], b[n], acc[m][n], 0, 0, 0);
                    }
            }
            buffer ^= 1;
        }

        // a lane has column lane & 31 of rows (i & 3) + 8 (i >> 2) + 4 (lane >> 5)
        float* const part = partial ? partial + ((int64_t)split * s.N + worker) * s.O * (s.C + 1) : nullptr;
#pragma unroll
        for (int n = 0; n < W::TN; ++n) {
            const int64_t c = c0 + wave_n + 32 * n + (lane & 31);
            if (c >= s.C) continue;
#pragma unroll
            for (int m = 0; m < W::TM; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int64_t o = o0 + wave_m + 32 * m + (i & 3) + 8 * (i >> 2) + 4 * (lane >> 5);
                    if (o >= s.O) continue;
                    if (part) part[o * s.C + c] = acc[m][n][i];
                    else store_any(dw.data, (int64_t)worker * dw.worker + o * dw.row + c, dw.type, acc[m][n][i]);
                }
        }
        __syncthreads();
        if (bias) {
            float* const rows = reinterpret_cast<float*>(lds[0]);        // [a_rows][BM]
            static_assert(sizeof(lds) >= W::a_rows * BM * sizeof(float), "room for the sums");
#pragma unroll
            for (int j = 0; j < 8; ++j) rows[a_row * BM + a_col + j] = sums[j];
            __syncthreads();
            for (uint32_t t = tid; t < (uint32_t)BM; t += W::threads) {
                if (o0 + t >= s.O) continue;
                float v = 0.f;
                for (int i = 0; i < W::a_rows; ++i) v += rows[i * BM + t];
                if (part) part[s.O * s.C + o0 + t] = v;
                else store_any(db.data, (int64_t)worker * db.stride + o0 + t, db.type, v);
            }
            __syncthreads();
        }
    }
}

// The splits' sums, added up in fp64 in order.
template <int>
__global__ __launch_bounds__(kBlock) void k_weight_grad_join(WgShape s, const float* __restrict__ partial, WgOut dw, LnParam db) {
    const int64_t row = s.C + 1, size = s.O * row;
    const uint32_t worker = blockIdx.y;
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < size; i += (int64_t)gridDim.x * kBlock) {
        const bool bias = i >= s.O * s.C;
        if (bias && !db.data) break;
        double v = 0.0;
        for (uint32_t p = 0; p < s.splits; ++p) v += (double)partial[((int64_t)p * s.N + worker) * size + i];
        if (bias) store_any(db.data, (int64_t)worker * db.stride + i - s.O * s.C, db.type, (float)v);
        else store_any(dw.data, (int64_t)worker * dw.worker + i / s.C * dw.row + i % s.C, dw.type, (float)v);
    }
}

}  // namespace liec
