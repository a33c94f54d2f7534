// Element types of the operators around a backward pass (fp32, bf16, fp16): vectors of 16 bytes, read from
// and written to any address that is a multiple of the element's size, computed on in fp32.
#pragma once
#include "common.hpp"

namespace liec {

enum DType : uint32_t { kF32 = 0, kBF16 = 1, kF16 = 2 };

struct bf16 {
    uint16_t bits;
};
struct f16 {
    uint16_t bits;
};

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any4 __attribute__((ext_vector_type(4), aligned(4)));   // fp32 at any 4-byte address
typedef uint32_t v4u_any2 __attribute__((ext_vector_type(4), aligned(2)));   // bf16, fp16 at any 2-byte address
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// Two 16-bit values of one word as fp32; both conversions are exact.
template <typename T>
__device__ __forceinline__ void widen2(uint32_t w, float& a, float& b);
template <>
__device__ __forceinline__ void widen2<bf16>(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
}
template <>
__device__ __forceinline__ void widen2<f16>(uint32_t w, float& a, float& b) {
    const v2h h = __builtin_bit_cast(v2h, w);
    a = (float)h.x;
    b = (float)h.y;
}

// Two fp32 values rounded to 16 bits, to nearest, ties to even: what a result is stored as is rounded once, here.
template <typename T>
__device__ __forceinline__ uint32_t narrow2(float a, float b);
template <>
__device__ __forceinline__ uint32_t narrow2<bf16>(float a, float b) {
    const v2f f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2bf));
}
template <>
__device__ __forceinline__ uint32_t narrow2<f16>(float a, float b) {
    const v2f f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2h));
}

template <typename T>
__device__ __forceinline__ float widen(T v) {
    float a, b;
    widen2<T>(v.bits, a, b);
    return a;
}
template <>
__device__ __forceinline__ float widen<float>(float v) { return v; }

template <typename T>
__device__ __forceinline__ T narrow(float v) { return T{(uint16_t)narrow2<T>(v, 0.f)}; }
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }

// A value of one of the three types at index i, for operands whose type only the call knows.
__device__ __forceinline__ float load_any(const void* p, int64_t i, uint32_t type) {
    if (type == kF32) return static_cast<const float*>(p)[i];
    if (type == kBF16) return widen(static_cast<const bf16*>(p)[i]);
    return widen(static_cast<const f16*>(p)[i]);
}
__device__ __forceinline__ void store_any(void* p, int64_t i, uint32_t type, float v) {
    if (type == kF32) static_cast<float*>(p)[i] = v;
    else if (type == kBF16) static_cast<bf16*>(p)[i] = narrow<bf16>(v);
    else static_cast<f16*>(p)[i] = narrow<f16>(v);
}

// 16 bytes: 4 fp32 or 8 16-bit values.
template <typename T>
struct Vec16 {
    static constexpr int n = 8;
    typedef v4u_any2 any;
    static __device__ __forceinline__ void widen(v4u r, float (&f)[n]) {
        widen2<T>(r.x, f[0], f[1]);
        widen2<T>(r.y, f[2], f[3]);
        widen2<T>(r.z, f[4], f[5]);
        widen2<T>(r.w, f[6], f[7]);
    }
    static __device__ __forceinline__ v4u narrow(const float (&f)[n]) {
        return v4u{narrow2<T>(f[0], f[1]), narrow2<T>(f[2], f[3]), narrow2<T>(f[4], f[5]), narrow2<T>(f[6], f[7])};
    }
};
template <>
struct Vec16<float> {
    static constexpr int n = 4;
    typedef v4u_any4 any;
    static __device__ __forceinline__ void widen(v4u r, float (&f)[n]) {
        f[0] = __uint_as_float(r.x);
        f[1] = __uint_as_float(r.y);
        f[2] = __uint_as_float(r.z);
        f[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ v4u narrow(const float (&f)[n]) {
        return v4u{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};

template <typename T, bool NT>
__device__ __forceinline__ v4u ld16(const T* p) {
    typedef typename Vec16<T>::any any;
    return NT ? (v4u)__builtin_nontemporal_load(reinterpret_cast<const any*>(p)) : (v4u)*reinterpret_cast<const any*>(p);
}
template <typename T, bool NT>
__device__ __forceinline__ void st16(T* p, v4u v) {
    typedef typename Vec16<T>::any any;
    if (NT) __builtin_nontemporal_store((any)v, reinterpret_cast<any*>(p));
    else *reinterpret_cast<any*>(p) = (any)v;
}

// keep: the same for the whole launch.  The empty statements hold the two stores apart: the compiler would make them one,
// a plain one.
template <typename T>
__device__ __forceinline__ void st16_as(bool keep, T* p, v4u v) {
    if (keep) {
        asm volatile("");
        st16<T, false>(p, v);
        asm volatile("");
    } else {
        st16<T, true>(p, v);
    }
}

struct LnRows {                        // a [workers, rows, columns] tensor of unit column stride
    void* data;
    int64_t worker, row;               // strides, in elements
};
struct LnParam {                       // a [workers, columns] tensor of unit column stride; stride 0: one row for all workers
    void* data;
    int64_t stride;
    uint32_t type;
};

// 4 values of 16 bits as one streaming load.
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v2u_any2 __attribute__((ext_vector_type(2), aligned(2)));
template <typename T>
struct Half16 {
    static __device__ __forceinline__ v2u load(const T* p) { return (v2u)__builtin_nontemporal_load(reinterpret_cast<const v2u_any2*>(p)); }
};

}  // namespace liec
