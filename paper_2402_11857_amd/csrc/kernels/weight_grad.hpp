// Gradient of a linear layer's weight from an 8-bit checkpoint of its input:
//
//   dW[o, c] = sum over rows r of dy[r, o] x[r, c],  db[o] = sum over rows of dy[r, o]       (of each worker)
//
// A product of matrices whose long axis is the rows, computed by the matrix cores from bf16 operands: x = q 2^k is one bf16 number, dy
// one (bf16), two (fp16: 11 bits) or three (fp32: 24 bits) whose sum it is exactly, so every product is exact and only their sum, in
// fp32, rounds.  Both operands lie row by row while the matrix cores take columns: they are staged in LDS as they lie, x
// widened to bf16 on the way, and read transposed, 4 rows of 16 columns by 16 lanes.
//
// Large products are bound by the matrix cores and what feeds them (with 256 x 256 values per block a step's products and its traffic
// through LDS take about as long): 8 products of 4096 x 4096 x 4096 from bf16 1083 to 1122 us, 980 to 1015 TFLOP/s, where plain bf16
// products of a library reach 930 to 1280.  On the way there: 128 x 128 values per block 2175 us; 256 x 256, a die on tiles that share
// rows 1726; loads without edges, stores to LDS beside the products 1361; dy from memory to LDS by itself, rows placed so that
// reads use all banks 1178; exponents as words, reads of one place and a distance 1125; x's halves in turn 1083.  Left out: operands read a
// unit ahead (1100 to 1143), 64 x 128 and 128 x 64 values per wave in blocks of 128 x 256 (1270 to 1360), waves of 128 x 64 instead of 64
// x 128 (1094), other waves' priority raised (1112).
#pragma once
#include <type_traits>

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
// Rows of W columns of bf16; groups of 32 columns (64 bytes) change places within a row by the row's number, so that what half a
// wave reads at a time, 4 rows of 32 columns, lies on 64 different banks.
template <int W>
__device__ __forceinline__ uint32_t wg_place(uint32_t row, uint32_t col) {
    const uint32_t by = W >= 128 ? row & 3 : row >> 1 & 1;
    return row * W + (((col >> 5) ^ by) << 5) + (col & 31);
}
// x's rows: besides, the halves of every other 16 columns change places, so that 16 lanes that store 8 columns of 16 each use all banks.
template <int W>
__device__ __forceinline__ uint32_t wg_place_x(uint32_t row, uint32_t col) {
    return wg_place<W>(row, col ^ (col >> 1 & 8));
}
__device__ __forceinline__ uint32_t wg_address(const uint16_t* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint16_t*)p;
}
__device__ __forceinline__ v4s wg_read(uint32_t at, uint32_t further) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)((__attribute__((address_space(3))) char*)(uintptr_t)at + further));
}
__device__ __forceinline__ v4s wg_read(const uint16_t* p) { return wg_read(wg_address(p), 0); }
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

// The bias is added up in fp32 over at most so many rows of a thread (a step's, where rows are at distances of 16 bytes), and in fp64 beyond.
// Chains over whole splits were off by up to 440 u of rows of one sign (2048 rows, each three bf16 numbers), those of 256 additions
// are by less than 86.
constexpr int kWgBiasChain = 256;
constexpr int kWgChain = 8192;         // rows of a split, at most: products of them are added up in fp32

struct WgWork {
    uint32_t tile_o, tile_c, split, worker;
};
// Neighbouring blocks run on different dies, each with a cache of its own: a die takes a range of the work, and walks through the tiles of
// a strip in bands of kWgBand tiles of o, so that what it works on at a time shares rows of dy and x.
constexpr uint32_t kWgDies = 8, kWgBand = 4;
__device__ __forceinline__ WgWork wg_work(const WgShape& s, int64_t works, int64_t work) {
    const int64_t share = works / kWgDies;
    if (work < share * kWgDies) work = work % kWgDies * share + work / kWgDies;
    const int64_t tiles = (int64_t)s.tiles_o * s.tiles_c, strip = work / tiles, in = work - strip * tiles;
    const int64_t band = in / ((int64_t)kWgBand * s.tiles_c), at = in - band * kWgBand * s.tiles_c;
    const uint32_t rows = (uint32_t)min((int64_t)kWgBand, s.tiles_o - band * kWgBand);
    WgWork r;
    r.worker = (uint32_t)(strip / s.splits);
    r.split = (uint32_t)(strip - (int64_t)r.worker * s.splits);
    r.tile_c = (uint32_t)(at / rows);
    r.tile_o = (uint32_t)(band * kWgBand + at - (int64_t)r.tile_c * rows);
    return r;
}

template <typename T, int BM, int BN, int BK, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64) void k_weight_grad(WgShape s, LnRows dy, Saved x, WgOut dw, LnParam db, float* __restrict__ partial) {
    typedef WgTile<T, BM, BN, BK, WM, WN> W;
    constexpr int P = W::P;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][W::values];
    constexpr bool once = W::a_rows * kWgBiasChain >= kWgChain;          // a thread's rows of a split are one chain
    __shared__ double totals[once ? 1 : W::threads / 64][BM];            // of a wave's rows
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t wave_m = wave / WN * (BM / WM), wave_n = wave % WN * (BN / WN);
    const uint32_t a_col = tid % W::a_lanes * 8, a_row = tid / W::a_lanes, b_col = tid % W::b_lanes * 16, b_row = tid / W::b_lanes;
    const bool b_mine = b_row < (uint32_t)BK;
    const uint32_t groups = (uint32_t)((s.C + kSavedCols - 1) / kSavedCols);
    const int64_t works = (int64_t)s.N * s.splits * s.tiles_o * s.tiles_c;

    for (int64_t work = blockIdx.x; work < works; work += gridDim.x) {
        const WgWork w = wg_work(s, works, work);
        const uint32_t tile_c = w.tile_c, tile_o = w.tile_o, split = w.split, worker = w.worker;
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
                uint16_t* const at = to + P * BK * BM;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v4u w;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = narrow2<bf16>(f[8 * h + 2 * j], f[8 * h + 2 * j + 1]);
                    *reinterpret_cast<v4u*>(at + wg_place_x<BN>(b_row + i * W::b_rows, b_col + 8 * h)) = w;
                }
            }
        };

        bool some = false;             // totals there
        auto add_up = [&] {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float v = sums[j];
#pragma unroll
                for (int off = W::a_lanes; off < 64; off <<= 1) v += __shfl_xor(v, off);
                if (lane < (uint32_t)W::a_lanes) totals[wave][a_col + j] = some ? totals[wave][a_col + j] + (double)v : (double)v;
                sums[j] = 0.f;
            }
            some = true;
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
        [[maybe_unused]] int left = kWgBiasChain / W::a_loads;
        for (int64_t r = r0; r < r1; r += BK) {
            stage(lds[buffer]);
            if constexpr (!once) {
                if (bias && --left == 0) {
                    add_up();
                    left = kWgBiasChain / W::a_loads;
                }
            }
            __syncthreads();
            if (r + BK < r1) fetch(r + BK);
            const uint16_t* const at = lds[buffer];
#pragma unroll
            for (int kk = 0; kk < BK; kk += 16) {
                v8bf a[P][W::TM], b[W::TN];
#pragma unroll
                for (int n = 0; n < W::TN; ++n) {
                    const uint16_t* const p = at + P * BK * BM;
                    b[n] = wg_join(wg_read(p + wg_place_x<BN>(kk + k_at, wave_n + 32 * n + col_at)), wg_read(p + wg_place_x<BN>(kk + k_at + 4, wave_n + 32 * n + col_at)));
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
        auto store = [&](auto put) {
#pragma unroll
            for (int n = 0; n < W::TN; ++n) {
                const int64_t c = c0 + wave_n + 32 * n + (lane & 31);
#pragma unroll
                for (int m = 0; m < W::TM; ++m) {
                    const int64_t o = o0 + wave_m + 32 * m + 4 * (lane >> 5);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c < s.C && o + (i & 3) + 8 * (i >> 2) < s.O) put(o + (i & 3) + 8 * (i >> 2), c, acc[m][n][i]);
                }
            }
        };
        const int64_t out = (int64_t)worker * dw.worker;
        if (part) store([&](int64_t o, int64_t c, float v) { part[o * s.C + c] = v; });
        else if (dw.type == kF32) store([&](int64_t o, int64_t c, float v) { static_cast<float*>(dw.data)[out + o * dw.row + c] = v; });
        else store([&](int64_t o, int64_t c, float v) { store_any(dw.data, out + o * dw.row + c, dw.type, v); });
        __syncthreads();
        if (bias) {
            float* const rows = reinterpret_cast<float*>(lds[0]);        // [a_rows][BM]
            static_assert(sizeof(lds) >= W::a_rows * BM * sizeof(float), "room for the sums");
#pragma unroll
            for (int j = 0; j < 8; ++j) rows[a_row * BM + a_col + j] = sums[j];
            __syncthreads();
            for (uint32_t t = tid; t < (uint32_t)BM; t += W::threads) {
                if (o0 + t >= s.O) continue;
                std::conditional_t<once, float, double> v = 0;
                for (int i = 0; i < W::a_rows; ++i) v += rows[i * BM + t];
                if constexpr (!once) {
                    for (int i = 0; some && i < W::threads / 64; ++i) v += totals[i][t];
                }
                if (part) part[s.O * s.C + o0 + t] = (float)v;
                else store_any(db.data, (int64_t)worker * db.stride + o0 + t, db.type, (float)v);
            }
            __syncthreads();
        }
    }
}

// ---- operands at distances of 16 bytes ---------------------------------------------------------------------------------
// Rows of dy, and of values of the checkpoint, that start at multiples of 16 bytes.  Loads go through buffer descriptors that end with the
// split's last row, beyond which they return zeros: rows that fill up the last step are none, and columns beyond a row's
// end, other rows' values, reach columns of the tile that are not stored.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t wg_buffer(const void* from, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(from), 0, (uint32_t)max((int64_t)0, min(bytes, (int64_t)0xfffffff0)), 0x00020000);
}

__device__ __forceinline__ v4u wg_words(const void* from, int64_t bytes) {
    const uint64_t at = (uint64_t)(uintptr_t)from;
    return v4u{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)max((int64_t)0, min(bytes, (int64_t)0xfffffff0)), 0x00020000u};
}
// 16 bytes per lane from an offset in the buffer to LDS, at `to` (the same for the wave) + 16 * lane.  The compiler does not know that it is
// under way: wg_wait waits for it.  m0 is reserved, so that no list of changed registers may name it, and nothing else here uses it.
__device__ __forceinline__ void wg_load_to_lds(v4u buffer, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %0, 0 offen lds" : : "s"(buffer), "v"(offset), "s"(to) : "memory");
}
// All waves meet; what they stored to LDS is there, and so is what they load, except for each wave's newest LATE loads (-1: none that the
// compiler does not know of, and it waits by itself where it uses one).
template <int LATE>
__device__ __forceinline__ void wg_wait() {
    static_assert(LATE == 4 || LATE <= 0, "what there is a wait for");
    if constexpr (LATE == 4) asm volatile("s_waitcnt vmcnt(4)" : : : "memory");
    else if constexpr (LATE == 0) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
__device__ __forceinline__ void wg_wait_all() { wg_wait<0>(); }

template <typename T, int BM, int BN, int BK, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64, 2) void k_weight_grad_aligned(WgShape s, LnRows dy, Saved x, WgOut dw, LnParam db, float* __restrict__ partial) {
    typedef WgTile<T, BM, BN, BK, WM, WN> W;
    constexpr int P = W::P, size = sizeof(T);
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][W::values];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t wave_m = wave / WN * (BM / WM), wave_n = wave % WN * (BN / WN);
    const uint32_t a_col = tid % W::a_lanes * 8, a_row = tid / W::a_lanes, b_col = tid % W::b_lanes * 16, b_row = tid / W::b_lanes;
    const uint32_t groups = (uint32_t)((s.C + kSavedCols - 1) / kSavedCols);
    const int64_t works = (int64_t)s.N * s.splits * s.tiles_o * s.tiles_c;

    for (int64_t work = blockIdx.x; work < works; work += gridDim.x) {
        const WgWork w = wg_work(s, works, work);
        const int64_t o0 = (int64_t)w.tile_o * BM, c0 = (int64_t)w.tile_c * BN, r0 = w.split * s.per, r1 = min(r0 + s.per, s.R);
        const T* const g = static_cast<const T*>(dy.data) + (int64_t)w.worker * dy.worker + o0;
        const int8_t* const q = x.q + (int64_t)w.worker * s.R * s.C + c0;
        const uint8_t* const e = x.e + (int64_t)w.worker * s.R * groups + c0 / kSavedCols;
        // bytes up to the end of the last row, the last 16 of them whole
        const int64_t g_end = ((r1 - 1) * dy.row + s.O - o0) * size + 15 & ~(int64_t)15, q_end = (r1 - 1) * s.C + s.C - c0, e_end = (r1 - 1) * groups + groups - c0 / kSavedCols;
        const uint32_t g_at = (uint32_t)((a_row * dy.row + a_col) * size), q_at = (uint32_t)(b_row * s.C + b_col), e_at = b_row * groups + b_col / kSavedCols;
        const uint32_t g_step = (uint32_t)(W::a_rows * dy.row * size), q_step = (uint32_t)(W::b_rows * s.C), e_step = W::b_rows * groups;
        const bool bias = db.data && w.tile_c == 0;

        v4u ra[P == 1 ? 1 : W::a_loads][Eight<T>::words], rb[W::b_loads];
        uint32_t re[W::b_loads];
        // bf16 rows of dy go from memory to LDS by themselves, 1024 bytes per wave and instruction: a lane's 16 bytes land at its place, so
        // it asks for the columns that belong there
        const uint32_t direct_row = wave * (W::a_loads * 512 / BM) + lane * 8 / BM, direct_col = lane * 8 % BM;
        auto direct_a = [&](int64_t r, uint16_t* to) {
            const v4u from = wg_words(g + r * dy.row, g_end - r * dy.row * size);
            const uint32_t at = __builtin_amdgcn_readfirstlane(wg_address(to) + wave * W::a_loads * 1024);
#pragma unroll
            for (int i = 0; i < W::a_loads; ++i) {
                const uint32_t row = direct_row + i * 512 / BM;
                wg_load_to_lds(from, (uint32_t)((row * dy.row + (wg_place<BM>(row, direct_col) - row * BM)) * size), at + i * 1024);
            }
        };
        auto fetch_a = [&](int64_t r) {
            const auto from = wg_buffer(g + r * dy.row, g_end - r * dy.row * size);
#pragma unroll
            for (int i = 0; i < W::a_loads; ++i)
#pragma unroll
                for (int v = 0; v < Eight<T>::words; ++v) ra[i][v] = __builtin_amdgcn_raw_buffer_load_b128(from, g_at + i * g_step + 16 * v, 0, 0);
        };
        auto fetch_b = [&](int64_t r) {
            const auto from = wg_buffer(q + r * s.C, q_end - r * s.C), scales = wg_buffer(e + r * groups, e_end - r * groups);
#pragma unroll
            for (int i = 0; i < W::b_loads; ++i) {
                rb[i] = __builtin_amdgcn_raw_buffer_load_b128(from, q_at + i * q_step, 0, 0);
                re[i] = __builtin_amdgcn_raw_buffer_load_b8(scales, e_at + i * e_step, 0, 0);
            }
        };
        auto stage_a = [&](uint16_t* to, int i) {
            const uint32_t at = wg_place<BM>(a_row + i * W::a_rows, a_col);
            Eight<T> raw;
#pragma unroll
            for (int v = 0; v < Eight<T>::words; ++v) raw.w[v] = ra[i][v];
            float f[8];
            widen_eight<T>(raw, f);
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
        };
        auto stage_b = [&](uint16_t* to, int i) {
            float f[16];
            const float scale = saved_scale(re[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack4(rb[i][j], scale, f + 4 * j);
            uint16_t* const at = to + P * BK * BM;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v4u w;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = narrow2<bf16>(f[8 * h + 2 * j], f[8 * h + 2 * j + 1]);
                *reinterpret_cast<v4u*>(at + wg_place_x<BN>(b_row + i * W::b_rows, b_col + 8 * h)) = w;
            }
        };

        v16f acc[W::TM][W::TN];
        float sums[W::TM];
#pragma unroll
        for (int m = 0; m < W::TM; ++m) {
            sums[m] = 0.f;
#pragma unroll
            for (int n = 0; n < W::TN; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.f;
        }
        // Lanes 16 g .. 16 g + 15 read columns 16 (g & 1) .. of rows 8 (g >> 1) .., 4 rows at a time.  Where a lane's places of a column
        // tile begin; other rows' are a multiple of 4 rows further, so at distances that instructions hold.
        const uint32_t k_at = lane >> 5 << 3 | (lane >> 2 & 3), col_at = (lane & 16) | (lane & 3) << 2;
        uint32_t a_at[W::TM], b_at[W::TN];
#pragma unroll
        for (int m = 0; m < W::TM; ++m) a_at[m] = wg_address(lds[0]) + 2 * wg_place<BM>(k_at, wave_m + 32 * m + col_at);
#pragma unroll
        for (int n = 0; n < W::TN; ++n) b_at[n] = wg_address(lds[0] + P * BK * BM) + 2 * wg_place_x<BN>(k_at, wave_n + 32 * n + col_at);
        // a step's products in BK / 16 * P units
        constexpr int units = BK / 16 * P;
        v8bf a[W::TM], b[W::TN];
        auto read_unit = [&](uint32_t buffer, int u) {
            const int kk = u / P * 16, p = P - 1 - u % P;
            if (u % P == 0) {
#pragma unroll
                for (int n = 0; n < W::TN; ++n) b[n] = wg_join(wg_read(b_at[n] + buffer, 2 * kk * BN), wg_read(b_at[n] + buffer, 2 * (kk + 4) * BN));
            }
#pragma unroll
            for (int m = 0; m < W::TM; ++m)
                a[m] = wg_join(wg_read(a_at[m] + buffer, 2 * (p * BK + kk) * BM), wg_read(a_at[m] + buffer, 2 * (p * BK + kk + 4) * BM));
        };
        auto multiply = [&](int u, auto with_bias) {
#pragma unroll
            for (int m = 0; m < W::TM; ++m) {
#pragma unroll
                for (int n = 0; n < W::TN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[m], b[n], acc[m][n], 0, 0, 0);
                if (with_bias && (uint32_t)(u / P % WN) == wave % WN) {
                    const v4u words = __builtin_bit_cast(v4u, a[m]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float lo, hi;
                        widen2<bf16>(words[j], lo, hi);
                        sums[m] += lo;
                        sums[m] += hi;
                    }
                }
            }
        };
        // every step, without a branch: one per 256 rows took 5 of 64 us more, where a quarter of the blocks add up the bias
        double total[W::TM] = {};
        auto add_up = [&] {
#pragma unroll
            for (int m = 0; m < W::TM; ++m) {
                total[m] += (double)sums[m];
                sums[m] = 0.f;
            }
        };
        // A step multiplies one buffer while the next is filled: dy's rows are on their way from its start (bf16) or, like x's, from
        // the end of the step before, and x is widened and stored beside the last products.  (dy's loads on the way to LDS are newer than x's, and
        // the compiler, which does not count them, waits for all of them where it needs the last of x's: half way through the step.)
        auto steps_of = [&](auto with_bias) {
            if constexpr (P == 1) {
                direct_a(r0, lds[0]);
            } else {
                fetch_a(r0);
#pragma unroll
                for (int i = 0; i < W::a_loads; ++i) stage_a(lds[0], i);
                fetch_a(r0 + BK);
            }
            fetch_b(r0);
#pragma unroll
            for (int i = 0; i < W::b_loads; ++i) stage_b(lds[0], i);
            fetch_b(r0 + BK);
            wg_wait_all();
            // the loop's registers for these hold words, not bytes to be widened at its head, where the loads are still under way
#pragma unroll
            for (int i = 0; i < W::b_loads; ++i) asm volatile("" : "+v"(re[i]));
            int buffer = 0;
            for (int64_t r = r0; r < r1; r += BK) {
                const uint32_t at = buffer ? sizeof(lds[0]) : 0;
                uint16_t* const next = lds[buffer ^ 1];
                if constexpr (P == 1) direct_a(r + BK, next);
#pragma unroll
                for (int u = 0; u < units; ++u) {
                    read_unit(at, u);
                    multiply(u, with_bias);
                    // the last third, or the last two of four: their share of what is stored
                    constexpr int late = P == 1 ? 2 : P, first = units - late;
                    if (u < first) continue;
                    if constexpr (P > 1) {
#pragma unroll
                        for (int i = 0; i < W::a_loads; ++i)
                            if (i * late / W::a_loads == u - first) stage_a(next, i);
                    }
#pragma unroll
                    for (int i = 0; i < W::b_loads; ++i)
                        if ((i + 1) * late / W::b_loads - 1 == u - first) stage_b(next, i);
                }
                if constexpr (P > 1) fetch_a(r + 2 * BK);
                fetch_b(r + 2 * BK);
                if (with_bias) add_up();
                wg_wait<P == 1 ? 2 * W::b_loads : -1>();
                buffer ^= 1;
            }
        };
        if (bias) steps_of(std::true_type{});
        else steps_of(std::false_type{});
        wg_wait_all();                 // also for loads to LDS that no step waited for

        // a lane has column lane & 31 of rows (i & 3) + 8 (i >> 2) + 4 (lane >> 5)
        float* const part = partial ? partial + ((int64_t)w.split * s.N + w.worker) * s.O * (s.C + 1) : nullptr;
        auto store = [&](auto put) {
#pragma unroll
            for (int n = 0; n < W::TN; ++n) {
                const int64_t c = c0 + wave_n + 32 * n + (lane & 31);
#pragma unroll
                for (int m = 0; m < W::TM; ++m) {
                    const int64_t o = o0 + wave_m + 32 * m + 4 * (lane >> 5);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c < s.C && o + (i & 3) + 8 * (i >> 2) < s.O) put(o + (i & 3) + 8 * (i >> 2), c, acc[m][n][i]);
                }
            }
        };
        const int64_t out = (int64_t)w.worker * dw.worker;
        if (part) store([&](int64_t o, int64_t c, float v) { part[o * s.C + c] = v; });
        else if (dw.type == kF32) store([&](int64_t o, int64_t c, float v) { static_cast<float*>(dw.data)[out + o * dw.row + c] = v; });
        else store([&](int64_t o, int64_t c, float v) { store_any(dw.data, out + o * dw.row + c, dw.type, v); });
        if (bias) {
            double* const rows = reinterpret_cast<double*>(lds[0]);      // [2 WN][BM]
#pragma unroll
            for (int m = 0; m < W::TM; ++m) rows[(wave % WN * 2 + (lane >> 5)) * BM + wave_m + 32 * m + (lane & 31)] = total[m];
            __syncthreads();
            for (uint32_t t = tid; t < (uint32_t)BM; t += W::threads) {
                if (o0 + t >= s.O) continue;
                double v = 0.0;
                for (int i = 0; i < 2 * WN; ++i) v += rows[i * BM + t];
                if (part) part[s.O * s.C + o0 + t] = (float)v;
                else store_any(db.data, (int64_t)w.worker * db.stride + o0 + t, db.type, (float)v);
            }
        }
        __syncthreads();
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
