// Global norm of a worker's gradient tensors, and their scaling: in place or into the fp32 rows of a compressed step.
//
//   norm_i = sqrt(sum_t sum_j g_tij^2)       c_i = 1 if norm_i <= bound, else bound / norm_i       out = g * c_i
//
// The tensors of all workers are cut into tiles of kGradTile consecutive bytes of one tensor and one worker; a tile is read
// with 16-byte accesses whatever its alignment.  Both kernels are bound by memory, and both sweep it in the order of their
// blocks: squares are added up by blocks that stay on the chip, take every gridDim.x-th tile of one worker and have the next
// one's loads under way (consecutive tiles per block: 5 % slower), scaling is done by a block per tile.  Measured: 32 x 25.6M
// bf16 values squared at 6.4 TB/s, 16 x 11.7M fp32 values squared and scaled in 351 us, 6.4 TB/s over both passes.
#pragma once
#include "elements.hpp"

namespace liec {

constexpr int kGradTile = 16384;
constexpr int kGradVecs = kGradTile / (kBlock * 16);    // 16-byte vectors of a thread

// Tensors of one launch: as many as 4 KiB of kernel arguments hold, more where every tensor's workers follow one another and no
// distances are needed (161 tensors in one launch instead of two).  Tensor t has tiles first[t] .. first[t + 1] - 1 of every
// worker and columns col[t] .. col[t + 1] - 1 of a worker's row; worker i's elements start at data[t] + i * stride(t) elements.
template <bool STRIDED>
struct GradTable {
    static constexpr int most = 128;
    const void* data[most];
    int64_t strides[most];
    int64_t col[most + 1];
    uint32_t first[most + 1];
    uint8_t type[most];
    __device__ __forceinline__ int64_t stride(uint32_t t) const { return strides[t]; }
    void set_stride(int i, int64_t s) { strides[i] = s; }
};
template <>
struct GradTable<false> {
    static constexpr int most = 184;
    const void* data[most];
    int64_t col[most + 1];
    uint32_t first[most + 1];
    uint8_t type[most];
    __device__ __forceinline__ int64_t stride(uint32_t t) const { return col[t + 1] - col[t]; }
    void set_stride(int, int64_t) {}
};

struct GradPass {
    double* partial;                   // parts sums of squares per worker; this launch's blocks leave theirs at slot ..
    uint32_t parts, slot;
    uint32_t row;                      // first worker of the launch
    uint32_t tiles, count;             // of this launch's tensors
    float bound;
    float* norms;
    float* rows;                       // nullptr: in place
    int64_t row_stride;
};

struct Tile {
    char* p;
    uint32_t bytes, type;
    int64_t col;                       // column of its first element
};

// The tensor that holds tile `tile`: the last one that starts at or before it.  Every lane looks at three starts.
template <bool STRIDED>
__device__ __forceinline__ uint32_t tensor_of(const GradTable<STRIDED>& tab, uint32_t count, uint32_t tile) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t before = 0;
#pragma unroll
    for (uint32_t q = 0; q < GradTable<STRIDED>::most; q += 64) {
        const uint64_t in = __ballot(lane + q < count && tab.first[min(lane + q, count)] <= tile);
        before += (uint32_t)__popcll(in);
    }
    return __builtin_amdgcn_readfirstlane(before - 1u);
}

// Tile `tile` of worker `row`; t: the tensor of an earlier tile, moved to this one's.
template <bool STRIDED>
__device__ __forceinline__ Tile tile_at(const GradTable<STRIDED>& tab, uint32_t tile, uint32_t row, uint32_t& t) {
    while (tile >= tab.first[t + 1]) ++t;
    const uint32_t type = tab.type[t], shift = type == kF32 ? 2 : 1;
    const int64_t off = (int64_t)(tile - tab.first[t]) * kGradTile, len = (tab.col[t + 1] - tab.col[t]) << shift;
    Tile r;
    r.p = static_cast<char*>(const_cast<void*>(tab.data[t])) + (((int64_t)row * tab.stride(t)) << shift) + off;
    r.bytes = (uint32_t)min((int64_t)kGradTile, len - off);
    r.type = type;
    r.col = tab.col[t] + (off >> shift);
    return r;
}

// ---- squares -------------------------------------------------------------------------------------------------------
template <bool NT>
__device__ __forceinline__ void load_tile(const Tile& c, v4u (&r)[kGradVecs]) {
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u) r[u] = ld16<bf16, NT>(reinterpret_cast<const bf16*>(c.p + (u * kBlock + threadIdx.x) * 16));
}

// The squares of a vector, added to the thread's sums.  A square of fp32 is exact in fp64 and stays in its range, so neither
// large nor tiny gradients lose anything.
template <typename T>
__device__ __forceinline__ void add_squares(v4u r, double (&acc)[4]) {
    float f[Vec16<T>::n];
    Vec16<T>::widen(r, f);
#pragma unroll
    for (int j = 0; j < Vec16<T>::n; ++j) acc[j & 3] = __fma_rn((double)f[j], (double)f[j], acc[j & 3]);
}

// A tile that ends early, without its loads under way.
template <typename T>
__device__ __forceinline__ void square_end(const Tile& c, double (&acc)[4]) {
    constexpr uint32_t V = Vec16<T>::n;
    const T* const p = reinterpret_cast<const T*>(c.p);
    const uint32_t n = c.bytes / sizeof(T);
    for (uint32_t e = threadIdx.x * V; e < n; e += kBlock * V) {
        if (e + V <= n) {
            add_squares<T>(ld16<T, false>(p + e), acc);
        } else {
            for (uint32_t j = e; j < n; ++j) {
                const double v = (double)widen(p[j]);
                acc[0] = __fma_rn(v, v, acc[0]);
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void square_tile(const Tile& c, const v4u (&r)[kGradVecs], double (&acc)[4]) {
    if (c.bytes == kGradTile) {
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) add_squares<T>(r[u], acc);
    } else {
        square_end<T>(c, acc);
    }
}

// Block b of a worker: every gridDim.x-th tile from b on, their sum of squares into partial[row][slot + b].  NT: past the caches,
// where nothing reads the gradients again (32 x 25.6M bf16 values 252 us, through them 282).
template <bool NT, bool STRIDED>
__global__ __launch_bounds__(kBlock) void k_grad_squares(GradPass a, GradTable<STRIDED> tab) {
    __shared__ double lds_w[4];
    const uint32_t row = a.row + blockIdx.y;
    const uint32_t begin = blockIdx.x, end = a.tiles, B = gridDim.x;
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t t = tensor_of(tab, a.count, begin);
    auto work = [&](const Tile& c, const v4u (&r)[kGradVecs]) {
        if (c.type == kF32) square_tile<float>(c, r, acc);
        else if (c.type == kBF16) square_tile<bf16>(c, r, acc);
        else square_tile<f16>(c, r, acc);
    };
    Tile ca = tile_at(tab, begin, row, t), cb;
    v4u ra[kGradVecs], rb[kGradVecs];
    if (ca.bytes == kGradTile) load_tile<NT>(ca, ra);
    for (uint32_t tile = begin; tile < end; tile += 2 * B) {
        if (tile + B < end) {
            cb = tile_at(tab, tile + B, row, t);
            if (cb.bytes == kGradTile) load_tile<NT>(cb, rb);
        }
        work(ca, ra);
        if (tile + B >= end) break;
        if (tile + 2 * B < end) {
            ca = tile_at(tab, tile + 2 * B, row, t);
            if (ca.bytes == kGradTile) load_tile<NT>(ca, ra);
        }
        work(cb, rb);
    }
    const double s = block_sum_f64((acc[0] + acc[1]) + (acc[2] + acc[3]), lds_w);
    if (threadIdx.x == 0) a.partial[(size_t)row * a.parts + a.slot + blockIdx.x] = s;
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

// A norm that is NaN is not below any bound: its worker's gradients become NaN.  A bound of +Inf asks for no factor.
__device__ __forceinline__ float factor_of(double norm, float bound) {
    return norm <= (double)bound || bound == __builtin_inff() ? 1.f : (float)((double)bound / norm);
}

__global__ __launch_bounds__(kBlock) void k_grad_norms(const double* __restrict__ partial, uint32_t parts, float* __restrict__ norms) {
    __shared__ double lds_w[4];
    const double norm = norm_of(partial + (size_t)blockIdx.x * parts, parts, lds_w);
    if (threadIdx.x == 0) norms[blockIdx.x] = (float)norm;
}

// ---- scaling -------------------------------------------------------------------------------------------------------
// Into fp32 rows 16-bit values are read 8 bytes at a time, so that a wave's stores are as contiguous as its loads.
template <typename T, bool ROWS>
__device__ __forceinline__ void load_to_scale(const Tile& c, v4u (&r)[kGradVecs]) {
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u) {
        if (ROWS && sizeof(T) == 2) {
            const v2u lo = Half16<T>::load(reinterpret_cast<const T*>(c.p + (2 * u * kBlock + threadIdx.x) * 8));
            const v2u hi = Half16<T>::load(reinterpret_cast<const T*>(c.p + ((2 * u + 1) * kBlock + threadIdx.x) * 8));
            r[u] = v4u{lo.x, lo.y, hi.x, hi.y};
        } else {
            r[u] = ld16<T, true>(reinterpret_cast<const T*>(c.p + (u * kBlock + threadIdx.x) * 16));
        }
    }
}

template <typename T, bool ROWS>
__device__ __forceinline__ void scale_tile(const Tile& c, const v4u (&r)[kGradVecs], float* out, float factor) {
    constexpr int V = Vec16<T>::n;
    constexpr bool SPLIT = ROWS && sizeof(T) == 2;
    T* const p = reinterpret_cast<T*>(c.p);
    if (c.bytes == kGradTile) {
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) {
            float f[V];
            Vec16<T>::widen(r[u], f);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = __fmul_rn(f[j], factor);
            if (SPLIT) {
#pragma unroll
                for (int h = 0; h < V; h += 4) {
                    const float o[4] = {f[h], f[h + 1], f[h + 2], f[h + 3]};
                    st16<float, true>(out + ((2 * u + h / 4) * kBlock + threadIdx.x) * 4, Vec16<float>::narrow(o));
                }
            } else {
                T* const to = ROWS ? reinterpret_cast<T*>(out) : p;
                st16<T, true>(to + (u * kBlock + threadIdx.x) * V, Vec16<T>::narrow(f));
            }
        }
        return;
    }
    const uint32_t n = c.bytes / sizeof(T);
    auto put = [&](uint32_t e, float v) {
        if (ROWS) out[e] = v;
        else p[e] = narrow<T>(v);
    };
    for (uint32_t e = threadIdx.x; e < n; e += kBlock) put(e, __fmul_rn(widen(p[e]), factor));
}

// Tile b of a worker times its factor, which every block forms from the partial sums while its loads are under way.
template <bool ROWS, bool STRIDED>
__global__ __launch_bounds__(kBlock) void k_grad_scale(GradPass a, GradTable<STRIDED> tab) {
    __shared__ double lds_w[4];
    const uint32_t row = a.row + blockIdx.y;
    uint32_t t = tensor_of(tab, a.count, blockIdx.x);
    const Tile c = tile_at(tab, blockIdx.x, row, t);
    v4u r[kGradVecs];
    if (c.bytes == kGradTile) {
        if (!ROWS || c.type == kF32) load_to_scale<bf16, false>(c, r);
        else load_to_scale<bf16, true>(c, r);
    }
    float factor = 1.f;
    if (a.parts) {
        const double norm = norm_of(a.partial + (size_t)row * a.parts, a.parts, lds_w);
        factor = factor_of(norm, a.bound);
        if (a.norms && blockIdx.x == 0 && threadIdx.x == 0) a.norms[row] = (float)norm;
    }
    if (!ROWS && factor == 1.f) return;                     // nothing to change
    float* const out = ROWS ? a.rows + (int64_t)row * a.row_stride + c.col : nullptr;
    if (c.type == kF32) scale_tile<float, ROWS>(c, r, out, factor);
    else if (c.type == kBF16) scale_tile<bf16, ROWS>(c, r, out, factor);
    else scale_tile<f16, ROWS>(c, r, out, factor);
}

}  // namespace liec
