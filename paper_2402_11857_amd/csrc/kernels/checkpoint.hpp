// Activation checkpoints in 8 bits: every 32 columns of a row share a power of two.
//
//   a = max |x| of the 32,  k the smallest integer from -126 on with a < 127.5 * 2^k,  q = x / 2^k rounded to nearest, ties to
//   even (|q| <= 127),  x stands as q * 2^k;  the byte is k + 127, or 255 where a is an infinity or a NaN.  k ends at 121: the few
//   fp32 and bf16 numbers beyond 127 * 2^121 stand as that, since 2^128 is none of them
//
// A power of two makes both directions exact up to the one rounding of q, and leaves numbers of 7 bits that bf16 holds: matrix
// products from a checkpoint need no rounding of their own.  It costs up to one bit against a scale of full precision.
//
// Both directions are bound by memory: 8 x 8192 rows of 4096 bf16 columns 135 to 145 us to save and 131 to 134 us to load (6.0 and 6.1
// TB/s; a copy reaches 6.67).
#pragma once
#include "elements.hpp"

namespace liec {

constexpr int kSavedCols = 32;         // columns that share an exponent
constexpr int kSavedMost = 248;        // largest exponent byte of numbers: 127 * 2^121 is finite, 64 * 2^122 is not
constexpr uint32_t kSavedNan = 255;    // exponent byte of 32 columns that held an infinity or a NaN

struct Saved {                         // contiguous values [rows, C] and exponents [rows, ceil(C / 32)]
    int8_t* q;
    uint8_t* e;
};

// ---- one group of columns -------------------------------------------------------------------------------------------
// Exponent byte for a largest magnitude with the bits `a`: 2^(e - 133) <= a < 2^(e - 132), one more from 127.5 / 128 of that on.
__device__ __forceinline__ uint32_t saved_exponent(uint32_t a) {
    if (a >= 0x7f800000u) return kSavedNan;
    return (uint32_t)min(max(((int)((a + 0x10000u) >> 23)) - 6, 1), kSavedMost);
}
// 2^(127 - e), what values are multiplied by.
__device__ __forceinline__ float saved_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }
// 2^(e - 127), what integers are multiplied by (0: zero); a NaN for 255.
__device__ __forceinline__ float saved_scale(uint32_t e) { return __uint_as_float(e << 23 | (e + 1) >> 8 << 22); }

// Four integers to and from a word.
__device__ __forceinline__ uint32_t pack4(const float* f, float inverse) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w |= ((uint32_t)(int)rintf(f[j] * inverse) & 0xffu) << (8 * j);
    return w;
}
// Values from 127.5 * 2^121 on, where the exponent ends, stand as 127.
__device__ __forceinline__ float saved_in_range(float v) { return fminf(fmaxf(v, -127.f * 0x1p121f), 127.f * 0x1p121f); }
__device__ __forceinline__ v2u pack8(const float (&f)[8], uint32_t e) {
    const float inverse = saved_inverse(e);
    v2u w;
    if (__builtin_expect(e == (uint32_t)kSavedMost, 0)) {
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = saved_in_range(f[j]);
        w = v2u{pack4(g, inverse), pack4(g + 4, inverse)};
    } else {
        w = v2u{pack4(f, inverse), pack4(f + 4, inverse)};
    }
    return e == kSavedNan ? v2u{0, 0} : w;
}
__device__ __forceinline__ void unpack4(uint32_t w, float s, float* f) {
    f[0] = (float)(int8_t)w * s;
    f[1] = (float)(int8_t)(w >> 8) * s;
    f[2] = (float)(int8_t)(w >> 16) * s;
    f[3] = (float)(int8_t)(w >> 24) * s;
}

typedef uint32_t v2u_any1 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t v4u_any1 __attribute__((ext_vector_type(4), aligned(1)));
__device__ __forceinline__ v2u ld8_bytes(const int8_t* p) { return (v2u)*reinterpret_cast<const v2u_any1*>(p); }
__device__ __forceinline__ void st8_bytes(int8_t* p, v2u v) { *reinterpret_cast<v2u_any1*>(p) = (v2u_any1)v; }

// ---- 8 values of any type ----------------------------------------------------------------------------------------------
template <typename T>
struct Eight {                         // as they lie in memory
    static constexpr int words = 8 * sizeof(T) / 16;
    v4u w[words];
};
template <typename T, bool NT>
__device__ __forceinline__ Eight<T> ld_eight(const T* p) {
    Eight<T> r;
#pragma unroll
    for (int i = 0; i < Eight<T>::words; ++i) r.w[i] = ld16<T, NT>(p + i * Vec16<T>::n);
    return r;
}
template <typename T>
__device__ __forceinline__ void widen_eight(const Eight<T>& r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < Eight<T>::words; ++i) {
        float part[Vec16<T>::n];
        Vec16<T>::widen(r.w[i], part);
#pragma unroll
        for (int j = 0; j < Vec16<T>::n; ++j) f[i * Vec16<T>::n + j] = part[j];
    }
}
template <typename T>
__device__ __forceinline__ void st_eight(bool keep, T* p, const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < Eight<T>::words; ++i) {
        float part[Vec16<T>::n];
#pragma unroll
        for (int j = 0; j < Vec16<T>::n; ++j) part[j] = f[i * Vec16<T>::n + j];
        st16_as<T>(keep, p + i * Vec16<T>::n, Vec16<T>::narrow(part));
    }
}

// Largest magnitude's bits among lanes that differ in their lowest two bits only.
__device__ __forceinline__ uint32_t max_of_quad(uint32_t a) {
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xb1, 0xf, 0xf, true));      // quad_perm 1 0 3 2
    return max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4e, 0xf, 0xf, true));   // quad_perm 2 3 0 1
}

// ---- whole rows ------------------------------------------------------------------------------------------------------
// A thread takes 8 columns, four lanes a group of 32: a row is 4 * ceil(C / 32) such eights, some at its end empty.  The eights of
// all rows of a worker are dealt out in order, kSavedDeep * 256 to a block, so that rows of any length fill the lanes.
constexpr int kSavedDeep = 4;
constexpr int kSavedBlock = kBlock * kSavedDeep;

// Row and eight of the n-th of a worker's eights; `in` and `row`: those of the block's first.  A block crosses few rows, or many short
// ones: magic = ceil(2^32 / per), exact while n * per < 2^32.
struct SavedPlace {
    int64_t row;
    uint32_t eight;
};
__device__ __forceinline__ SavedPlace saved_place(int64_t row, uint32_t in, uint32_t n, uint32_t per, uint32_t magic) {
    n += in;
    const uint32_t rows = per >= (uint32_t)kSavedBlock ? (n >= per) : __umulhi(n, magic);
    return {row + rows, n - rows * per};
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_checkpoint_save(int64_t R, uint32_t C, uint32_t per, uint32_t magic, LnRows x, Saved out) {
    const uint32_t worker = blockIdx.y;
    const T* const from = static_cast<const T*>(x.data) + (int64_t)worker * x.worker;
    const uint32_t groups = per >> 2;
    for (int64_t b = blockIdx.x; b * kSavedBlock < R * per; b += gridDim.x) {
        const int64_t first = b * kSavedBlock, row0 = first / per;
        const uint32_t in0 = (uint32_t)(first - row0 * per);
        SavedPlace at[kSavedDeep];
        Eight<T> raw[kSavedDeep];
        uint32_t n[kSavedDeep];
#pragma unroll
        for (int u = 0; u < kSavedDeep; ++u) {
            at[u] = saved_place(row0, in0, u * kBlock + threadIdx.x, per, magic);
            n[u] = at[u].row < R && at[u].eight * 8 < C ? min(8u, C - at[u].eight * 8) : 0u;
            if (n[u] == 8) raw[u] = ld_eight<T, true>(from + at[u].row * x.row + at[u].eight * 8);
        }
#pragma unroll
        for (int u = 0; u < kSavedDeep; ++u) {
            float f[8];
            if (n[u] == 8) {
                widen_eight<T>(raw[u], f);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = 0.f;
                const T* const p = from + at[u].row * x.row + at[u].eight * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < (int)n[u]) f[j] = widen(p[j]);
            }
            uint32_t a = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) a = max(a, key_of(f[j]));
            const uint32_t e = saved_exponent(max_of_quad(a));
            const v2u w = pack8(f, e);
            const int64_t row = (int64_t)worker * R + at[u].row;
            int8_t* const to = out.q + row * C + at[u].eight * 8;
            if (n[u] == 8) {
                st8_bytes(to, w);
            } else {
                for (uint32_t j = 0; j < n[u]; ++j) to[j] = (int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
            }
            if (n[u] && (at[u].eight & 3) == 0) out.e[row * groups + (at[u].eight >> 2)] = (uint8_t)e;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_checkpoint_load(int64_t R, uint32_t C, uint32_t per, uint32_t magic, bool keep, Saved in, LnRows y) {
    const uint32_t worker = blockIdx.y;
    T* const to = static_cast<T*>(y.data) + (int64_t)worker * y.worker;
    const uint32_t groups = per >> 2;
    for (int64_t b = blockIdx.x; b * kSavedBlock < R * per; b += gridDim.x) {
        const int64_t first = b * kSavedBlock, row0 = first / per;
        const uint32_t in0 = (uint32_t)(first - row0 * per);
        SavedPlace at[kSavedDeep];
        v2u w[kSavedDeep];
        uint32_t e[kSavedDeep], n[kSavedDeep];
#pragma unroll
        for (int u = 0; u < kSavedDeep; ++u) {
            at[u] = saved_place(row0, in0, u * kBlock + threadIdx.x, per, magic);
            n[u] = at[u].row < R && at[u].eight * 8 < C ? min(8u, C - at[u].eight * 8) : 0u;
            const int64_t row = (int64_t)worker * R + at[u].row;
            const int8_t* const p = in.q + row * C + at[u].eight * 8;
            if (n[u]) e[u] = in.e[row * groups + (at[u].eight >> 2)];
            if (n[u] == 8) {
                w[u] = ld8_bytes(p);
            } else {
                w[u] = v2u{0, 0};
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < (int)n[u]) w[u][j >> 2] |= (uint32_t)(uint8_t)p[j] << (8 * (j & 3));
            }
        }
#pragma unroll
        for (int u = 0; u < kSavedDeep; ++u) {
            if (!n[u]) continue;
            const float s = saved_scale(e[u]);
            float f[8];
            unpack4(w[u].x, s, f);
            unpack4(w[u].y, s, f + 4);
            T* const p = to + at[u].row * y.row + at[u].eight * 8;
            if (n[u] == 8) {
                st_eight<T>(keep, p, f);
            } else {
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (j < (int)n[u]) p[j] = narrow<T>(f[j]);
            }
        }
    }
}

}  // namespace liec
