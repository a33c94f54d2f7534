// Global norm of a worker's gradient tensors, and their scaling: in place or into the fp32 rows of a compressed step.
//
//   norm_i = sqrt(sum_t sum_j g_tij^2)       c_i = 1 if norm_i <= bound, else bound / norm_i       out = g * c_i
//
// The tensors of all workers are cut into tiles of kGradTile consecutive bytes of one tensor and one worker; a tile is read
// by one wave, with 16-byte accesses whatever its alignment (a tile per block of four waves left three of them idle on small
// tensors: 161 tensors of 52 x 158 043 fp16 values 36 us, now 12).  Both kernels are bound by memory, and both sweep it in the
// order of their blocks: squares are added up by at most 4096 blocks, whose waves take every B-th tile of one worker and have
// the next one's loads under way (consecutive tiles: 5 % slower), scaling is done by a wave per tile.  Measured: 32 x 25.6M bf16
// values squared at 6.7 TB/s, 16 x 11.7M fp32 values squared and scaled in 355 us, 6.4 TB/s over both passes.
#pragma once
#include "elements.hpp"

namespace liec {

constexpr int kGradTile = 4096;        // bytes: one wave's, four 16-byte vectors per lane
constexpr int kGradVecs = kGradTile / (64 * 16);
constexpr int kGradWaves = kBlock / 64;                 // tiles that a block works on at a time

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

__device__ __forceinline__ uint32_t lane_id() { return threadIdx.x & 63; }
// This wave's number among those of its row's blocks; the same for the whole wave, in a scalar register.
__device__ __forceinline__ uint32_t wave_of_row() { return __builtin_amdgcn_readfirstlane(blockIdx.x * kGradWaves + (threadIdx.x >> 6)); }

struct Tile {
    char* p;
    uint32_t bytes, type;
    int64_t col;                       // column of its first element
};

// The tensor that holds tile `tile`: the last one that starts at or before it.  Every lane looks at two starts, or three.
template <bool STRIDED>
__device__ __forceinline__ uint32_t tensor_of(const GradTable<STRIDED>& tab, uint32_t count, uint32_t tile) {
    const uint32_t lane = lane_id();
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
// A tile's loads: whole vectors, zeros where the tile has ended, and the values after the last whole vector, one per lane.  They
// are requested together and looked at later.
struct Held {
    v4u r[kGradVecs];
    uint32_t tail;
};

// Value `e` of a tile as it is in memory.
__device__ __forceinline__ uint32_t raw_value(const Tile& c, uint32_t e) {
    return c.type == kF32 ? reinterpret_cast<const uint32_t*>(c.p)[e] : (uint32_t)reinterpret_cast<const uint16_t*>(c.p)[e];
}
__device__ __forceinline__ float widen_raw(uint32_t v, uint32_t type) {
    if (type == kF32) return __uint_as_float(v);
    return type == kBF16 ? widen(bf16{(uint16_t)v}) : widen(f16{(uint16_t)v});
}

template <bool NT>
__device__ __forceinline__ void load_tile(const Tile& c, Held& h) {
    const uint32_t lane = lane_id();
    if (c.bytes == kGradTile) {
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) h.r[u] = ld16<bf16, NT>(reinterpret_cast<const bf16*>(c.p + (u * 64 + lane) * 16));
        return;
    }
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u) {
        h.r[u] = v4u{0, 0, 0, 0};
        const uint32_t at = (u * 64 + lane) * 16;
        if (at + 16 <= c.bytes) h.r[u] = ld16<bf16, NT>(reinterpret_cast<const bf16*>(c.p + at));
    }
    const uint32_t shift = c.type == kF32 ? 2 : 1, from = (c.bytes & ~15u) >> shift;
    h.tail = 0;
    if (from + lane < c.bytes >> shift) h.tail = raw_value(c, from + lane);
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

// A whole tile's vectors are there already; one that ends early is loaded here (with its loads under way like the others', whole
// tiles took 3 % longer).
template <bool NT, typename T>
__device__ __forceinline__ void square_tile(const Tile& c, const Held& h, double (&acc)[4]) {
    if (c.bytes == kGradTile) {
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) add_squares<T>(h.r[u], acc);
        return;
    }
    Held own;
    load_tile<NT>(c, own);
#pragma unroll
    for (int u = 0; u < kGradVecs; ++u) add_squares<T>(own.r[u], acc);
    const double v = (double)widen_raw(own.tail, c.type);
    acc[0] = __fma_rn(v, v, acc[0]);
}

// A wave of a worker's blocks: its own tile and every one a whole round of waves further; the block's sum of squares into partial[row][slot + b].  NT: past the caches,
// where nothing reads the gradients again (32 x 25.6M bf16 values 252 us, through them 282).
// 80 registers are six waves per SIMD; with 82 the norm of 32 x 25.6M bf16 values takes 250 us instead of 245.
template <bool NT, bool STRIDED>
__global__ __launch_bounds__(kBlock, 6) void k_grad_squares(GradPass a, GradTable<STRIDED> tab) {
    __shared__ double lds_w[4];
    const uint32_t row = a.row + blockIdx.y;
    const uint32_t begin = wave_of_row(), end = a.tiles, B = gridDim.x * kGradWaves;
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t t = tensor_of(tab, a.count, min(begin, end - 1));
    auto work = [&](const Tile& c, const Held& h) {
        if (c.type == kF32) square_tile<NT, float>(c, h, acc);
        else if (c.type == kBF16) square_tile<NT, bf16>(c, h, acc);
        else square_tile<NT, f16>(c, h, acc);
    };
    Tile ca = tile_at(tab, min(begin, end - 1), row, t), cb;
    Held ha, hb;
    if (ca.bytes == kGradTile) load_tile<NT>(ca, ha);
    for (uint32_t tile = begin; tile < end; tile += 2 * B) {
        if (tile + B < end) {
            cb = tile_at(tab, tile + B, row, t);
            if (cb.bytes == kGradTile) load_tile<NT>(cb, hb);
        }
        work(ca, ha);
        if (tile + B >= end) break;
        if (tile + 2 * B < end) {
            ca = tile_at(tab, tile + 2 * B, row, t);
            if (ca.bytes == kGradTile) load_tile<NT>(ca, ha);
        }
        work(cb, hb);
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
// The loads of a tile to be scaled.  SPLIT: into fp32 rows 16-bit values are read 8 bytes at a time, so that a wave's stores are
// as contiguous as its loads.
template <bool SPLIT>
__device__ __forceinline__ void load_to_scale(const Tile& c, Held& h) {
    const uint32_t lane = lane_id();
    if (!SPLIT) return load_tile<true>(c, h);
    auto load = [&](auto inside) {
#pragma unroll
        for (int u = 0; u < 2 * kGradVecs; ++u) {
            const uint32_t at = (u * 64 + lane) * 8;
            v2u v = {0, 0};
            if (inside(at + 8)) v = Half16<bf16>::load(reinterpret_cast<const bf16*>(c.p + at));
            h.r[u / 2][u % 2 * 2] = v.x;
            h.r[u / 2][u % 2 * 2 + 1] = v.y;
        }
    };
    if (c.bytes == kGradTile) return load([](uint32_t) { return true; });
    load([&](uint32_t end) { return end <= c.bytes; });
    const uint32_t from = (c.bytes & ~7u) >> 1;
    h.tail = 0;
    if (from + lane < c.bytes >> 1) h.tail = raw_value(c, from + lane);
}

template <typename T, bool ROWS>
__device__ __forceinline__ void scale_tile(const Tile& c, const Held& h, float* out, float factor) {
    constexpr int V = Vec16<T>::n;
    constexpr bool SPLIT = ROWS && sizeof(T) == 2;
    constexpr uint32_t PIECE = SPLIT ? 4 : V;               // values that are loaded and stored together
    const uint32_t lane = lane_id(), n = c.bytes / sizeof(T);
    T* const p = reinterpret_cast<T*>(c.p);
    auto store = [&](auto inside) {
#pragma unroll
        for (int u = 0; u < kGradVecs; ++u) {
            float f[V];
            Vec16<T>::widen(h.r[u], f);
#pragma unroll
            for (int j = 0; j < V; ++j) f[j] = __fmul_rn(f[j], factor);
            if (SPLIT) {
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const float o[4] = {f[i], f[i + 1], f[i + 2], f[i + 3]};
                    const uint32_t e = ((2 * u + i / 4) * 64 + lane) * 4;
                    if (inside(e + 4)) st16<float, true>(out + e, Vec16<float>::narrow(o));
                }
            } else {
                const uint32_t e = (u * 64 + lane) * V;
                T* const to = ROWS ? reinterpret_cast<T*>(out) : p;
                if (inside(e + V)) st16<T, true>(to + e, Vec16<T>::narrow(f));
            }
        }
    };
    // whole tiles without conditions, which keep the stores apart (8 x 25.6M bf16 values into rows 286 against 262 us)
    if (c.bytes == kGradTile) return store([](uint32_t) { return true; });
    store([&](uint32_t end) { return end <= n; });
    const uint32_t e = n - n % PIECE + lane;
    if (e < n) {
        const float v = __fmul_rn(widen_raw(h.tail, c.type), factor);
        if (ROWS) out[e] = v;
        else p[e] = narrow<T>(v);
    }
}

// A tile of a worker per wave, times the factor that every block forms from the partial sums while its loads are under way.
template <bool ROWS, bool STRIDED>
__global__ __launch_bounds__(kBlock) void k_grad_scale(GradPass a, GradTable<STRIDED> tab) {
    __shared__ double lds_w[4];
    const uint32_t row = a.row + blockIdx.y, tile = min(wave_of_row(), a.tiles - 1);
    uint32_t t = tensor_of(tab, a.count, tile);
    const Tile c = tile_at(tab, tile, row, t);
    Held h;
    if (!ROWS || c.type == kF32) load_to_scale<false>(c, h);
    else load_to_scale<true>(c, h);
    float factor = 1.f;
    if (a.parts) {
        const double norm = norm_of(a.partial + (size_t)row * a.parts, a.parts, lds_w);
        factor = factor_of(norm, a.bound);
        if (a.norms && blockIdx.x == 0 && threadIdx.x == 0) a.norms[row] = (float)norm;
    }
    if (!ROWS && factor == 1.f) return;                     // nothing to change
    if (wave_of_row() >= a.tiles) return;
    float* const out = ROWS ? a.rows + (int64_t)row * a.row_stride + c.col : nullptr;
    if (c.type == kF32) scale_tile<float, ROWS>(c, h, out, factor);
    else if (c.type == kBF16) scale_tile<bf16, ROWS>(c, h, out, factor);
    else scale_tile<f16, ROWS>(c, h, out, factor);
}

}  // namespace liec
