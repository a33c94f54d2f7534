// Global norm of a worker's gradient tensors, and their scaling: in place or into the fp32 rows of a compressed step.
//
//   norm_i = sqrt(sum_t sum_j g_tij^2)       c_i = 1 if norm_i <= bound, else bound / norm_i       out = g * c_i
//
// The tensors of all workers are cut into tiles of kGradTile consecutive elements of one tensor and one worker; a tile is
// read with 16-byte accesses whatever its alignment.  A block takes a run of consecutive tiles of one worker.
#pragma once
#include "elements.hpp"

namespace liec {

constexpr int kGradTile = 8192;
constexpr int kGradTensors = 128;      // tensors of one launch: what 4 KiB of kernel arguments hold

// Tensors of one launch.  Tensor t has tiles first[t] .. first[t + 1] - 1 of every worker and columns col[t] .. col[t + 1] - 1
// of a worker's row; worker i's elements start at data[t] + i * stride[t].
struct GradTable {
    const void* data[kGradTensors];
    int64_t stride[kGradTensors];
    int64_t col[kGradTensors + 1];
    uint32_t first[kGradTensors + 1];
    uint8_t type[kGradTensors];
};

// The tensor that holds tile `tile`: the last one that starts at or before it.  Every lane looks at two starts.
__device__ __forceinline__ uint32_t tensor_of(const GradTable& tab, uint32_t count, uint32_t tile) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t a = __ballot(lane < count && tab.first[min(lane, count)] <= tile);
    const uint64_t b = __ballot(lane + 64 < count && tab.first[min(lane + 64, count)] <= tile);
    return (uint32_t)(__popcll(a) + __popcll(b)) - 1u;
}

// Sum of the squares of n <= kGradTile elements, added to the thread's sums.  A square of fp32 is exact in fp64 and stays in
// its range, so neither large nor tiny gradients lose anything.
template <typename T>
__device__ __forceinline__ void square_tile(const T* __restrict__ p, uint32_t n, double (&acc)[4]) {
    constexpr int V = Vec16<T>::n, U = kGradTile / (kBlock * V);
    if (n == kGradTile) {
        v4u r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = ld16<T, false>(p + (u * kBlock + threadIdx.x) * V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[V];
            Vec16<T>::widen(r[u], f);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j & 3] = __fma_rn((double)f[j], (double)f[j], acc[j & 3]);
        }
        return;
    }
    for (uint32_t e = threadIdx.x * V; e < n; e += kBlock * V) {
        if (e + V <= n) {
            float f[V];
            Vec16<T>::widen(ld16<T, false>(p + e), f);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j & 3] = __fma_rn((double)f[j], (double)f[j], acc[j & 3]);
        } else {
            for (uint32_t j = e; j < n; ++j) {
                const double v = (double)widen(p[j]);
                acc[0] = __fma_rn(v, v, acc[0]);
            }
        }
    }
}

// Block b of worker blockIdx.y: tiles b * per .. of this launch's `tiles`, their sum of squares into partial[worker][slot + b].
__global__ __launch_bounds__(kBlock) void k_grad_squares(double* __restrict__ partial, uint32_t parts, uint32_t slot, uint32_t count,
                                                         uint32_t tiles, uint32_t per, GradTable tab) {
    __shared__ double lds_w[4];
    const uint32_t row = blockIdx.y;
    const uint32_t begin = blockIdx.x * per, end = min(begin + per, tiles);
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t t = __builtin_amdgcn_readfirstlane(tensor_of(tab, count, begin));
    for (uint32_t tile = begin; tile < end; ++tile) {
        while (tile >= tab.first[t + 1]) ++t;
        const int64_t off = (int64_t)(tile - tab.first[t]) * kGradTile;
        const uint32_t n = (uint32_t)min((int64_t)kGradTile, tab.col[t + 1] - tab.col[t] - off);
        const int64_t at = (int64_t)row * tab.stride[t] + off;
        const uint32_t type = tab.type[t];
        if (type == kF32) square_tile(static_cast<const float*>(tab.data[t]) + at, n, acc);
        else if (type == kBF16) square_tile(static_cast<const bf16*>(tab.data[t]) + at, n, acc);
        else square_tile(static_cast<const f16*>(tab.data[t]) + at, n, acc);
    }
    const double s = block_sum_f64((acc[0] + acc[1]) + (acc[2] + acc[3]), lds_w);
    if (threadIdx.x == 0) partial[(size_t)row * parts + slot + blockIdx.x] = s;
}

// The norm of a worker from its partial sums, in the same order in every block that forms it; valid in every thread.
__device__ __forceinline__ double norm_of(const double* __restrict__ partial, uint32_t parts, double* lds_w) {
    double acc = 0.0;
    for (uint32_t q = threadIdx.x; q < parts; q += kBlock) acc += partial[q];
    const double s = block_sum_f64(acc, lds_w);
    if (threadIdx.x == 0) lds_w[0] = __dsqrt_rn(s);
    __syncthreads();
    return lds_w[0];
}

__global__ __launch_bounds__(kBlock) void k_grad_norms(const double* __restrict__ partial, uint32_t parts, float* __restrict__ norms) {
    __shared__ double lds_w[4];
    const double norm = norm_of(partial + (size_t)blockIdx.x * parts, parts, lds_w);
    if (threadIdx.x == 0) norms[blockIdx.x] = (float)norm;
}

// out[0 .. n) = p[0 .. n) * c; out may be p.
template <typename T, typename O>
__device__ __forceinline__ void scale_tile(const T* p, O* out, uint32_t n, float c) {
    constexpr int V = Vec16<T>::n, U = kGradTile / (kBlock * V);
    auto put = [&](uint32_t e, v4u r) {
        float f[V];
        Vec16<T>::widen(r, f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = __fmul_rn(f[j], c);
        if constexpr (sizeof(T) == sizeof(O)) {
            st16<T, true>(reinterpret_cast<T*>(out) + e, Vec16<T>::narrow(f));
        } else {
            Raw8<float>::store(out + e, f);
        }
    };
    if (n == kGradTile) {
        v4u r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = ld16<T, true>(p + (u * kBlock + threadIdx.x) * V);
#pragma unroll
        for (int u = 0; u < U; ++u) put((u * kBlock + threadIdx.x) * V, r[u]);
        return;
    }
    for (uint32_t e = threadIdx.x * V; e < n; e += kBlock * V) {
        if (e + V <= n) {
            put(e, ld16<T, true>(p + e));
        } else {
            for (uint32_t j = e; j < n; ++j) out[j] = narrow<O>(__fmul_rn(widen(p[j]), c));
        }
    }
}

// rows == nullptr: every element of a worker times its factor, in place; nothing is touched where that factor is 1.
// Otherwise the products go to columns col[t] .. of the worker's row.  A bound of +Inf asks for no factor and reads no sums.
__global__ __launch_bounds__(kBlock) void k_grad_scale(const double* __restrict__ partial, uint32_t parts, float bound, float* __restrict__ norms,
                                                       float* rows, int64_t row_stride, uint32_t count, uint32_t tiles, uint32_t per, GradTable tab) {
    __shared__ double lds_w[4];
    const uint32_t row = blockIdx.y;
    const uint32_t begin = blockIdx.x * per, end = min(begin + per, tiles);
    float c = 1.f;
    if (parts) {
        const double norm = norm_of(partial + (size_t)row * parts, parts, lds_w);
        // a norm that is NaN is not below any bound: its worker's gradients become NaN
        if (!(norm <= (double)bound) && bound < __builtin_inff()) c = (float)((double)bound / norm);
        if (norms && blockIdx.x == 0 && threadIdx.x == 0) norms[row] = (float)norm;
    }
    if (!rows && c == 1.f) return;
    uint32_t t = __builtin_amdgcn_readfirstlane(tensor_of(tab, count, begin));
    for (uint32_t tile = begin; tile < end; ++tile) {
        while (tile >= tab.first[t + 1]) ++t;
        const int64_t off = (int64_t)(tile - tab.first[t]) * kGradTile;
        const uint32_t n = (uint32_t)min((int64_t)kGradTile, tab.col[t + 1] - tab.col[t] - off);
        const int64_t at = (int64_t)row * tab.stride[t] + off;
        const uint32_t type = tab.type[t];
        if (rows) {
            float* const out = rows + (int64_t)row * row_stride + tab.col[t] + off;
            if (type == kF32) scale_tile(static_cast<const float*>(tab.data[t]) + at, out, n, c);
            else if (type == kBF16) scale_tile(static_cast<const bf16*>(tab.data[t]) + at, out, n, c);
            else scale_tile(static_cast<const f16*>(tab.data[t]) + at, out, n, c);
        } else {
            void* const data = const_cast<void*>(tab.data[t]);
            if (type == kF32) scale_tile(static_cast<float*>(data) + at, static_cast<float*>(data) + at, n, c);
            else if (type == kBF16) scale_tile(static_cast<bf16*>(data) + at, static_cast<bf16*>(data) + at, n, c);
            else scale_tile(static_cast<f16*>(data) + at, static_cast<f16*>(data) + at, n, c);
        }
    }
}

}  // namespace liec
