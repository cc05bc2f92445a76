// What the row-wise kernels of layer norm share: how a row is laid over threads, vectors of
// elements, sums over a row's threads.
//
// A row lies in the registers of `tpr` threads (a power of two), J vectors of V elements each:
// vector j of thread t holds columns (j tpr + t) V .. + V - 1, so that a warp's loads are
// contiguous and a group of 32 columns lies in 32 / V neighbouring lanes. V follows from the
// alignment of everything that is read or written in such vectors (16 bytes where it can). A
// row is read once.
#pragma once

#include "checkpoint.cuh"
#include "launch.cuh"

namespace bigcn {

constexpr int kRowThreads = 256;        // threads of a block, or of a row where that is more
constexpr int kMostRowThreads = 512;

template <typename T, int V> struct alignas(sizeof(T) * V) Vec {
    T v[V];
};

// Vectors of a thread that are compiled, by V. J is the least that holds a row, so a thread's
// vectors before the next smaller option are all within the row, and are taken without tests.
constexpr int kOptions[4][6] = {{1, 2, 4, 8, 16, 24}, {1, 2, 4, 8, 12, 0}, {1, 2, 4, 8, 0, 0},
                                {1, 2, 4, 0, 0, 0}};
__host__ __device__ constexpr int options_of(int V) { return V == 1 ? 0 : V == 2 ? 1 : V == 4 ? 2 : 3; }
__host__ __device__ constexpr int full_vectors(int V, int J) {
    int full = 0;
    for (int q = 0; q < 6; ++q)
        if (kOptions[options_of(V)][q] > 0 && kOptions[options_of(V)][q] < J)
            full = kOptions[options_of(V)][q];
    return full;
}

// The layout of a call: tpr threads a row, J vectors a thread, V elements a vector;
// J == 0: rows that no layout holds in registers.
struct RowLayout {
    int tpr, J;
};

// The fewest threads, `fewest` or more, that hold a row of K, with at most `warp_most`
// elements a thread where they are a warp and `most` otherwise; and then more threads while
// the rows do not fill the card (each has less to do then).
inline RowLayout row_layout(int64_t N, int K, int V, int fewest, int warp_most, int most,
                            const DeviceInfo &dev) {
    const int *options = kOptions[options_of(V)];
    const int64_t vecs = (int64_t(K) + V - 1) / V;
    auto fit = [&](int threads) {
        const int64_t need = (vecs + threads - 1) / threads;
        for (int q = 0; q < 6 && options[q] > 0; ++q)
            if (options[q] >= need)
                return options[q] * V <= (threads == 32 ? warp_most : most) ? options[q] : 0;
        return 0;
    };
    int tpr = fewest;
    while (fit(tpr) == 0 && tpr < kMostRowThreads) tpr *= 2;
    while (tpr < kRowThreads && tpr < vecs && N * tpr < int64_t(dev.sm_count) * 2 * kRowThreads)
        tpr *= 2;
    return {tpr, fit(tpr)};
}

// What stands in for a gamma or a beta that is not given, read with a stride of 0.
static __device__ __align__(32) const float kOnes[8] = {1, 1, 1, 1, 1, 1, 1, 1};
static __device__ __align__(32) const float kZeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};

// Largest V <= 16 bytes of elements by which everything in `addresses` (pointers and byte
// strides of element size es) is aligned.
inline int vector_width(size_t es, const uint64_t *addresses, int n) {
    uint64_t all = 16;
    for (int q = 0; q < n; ++q) all |= addresses[q];
    const uint64_t bytes = all & (~all + 1);        // the lowest set bit, at most 16
    return bytes <= es ? 1 : int(bytes / es);
}

// Sums over a row's threads, the same value for all of them. kWarp: the row is one warp;
// else `red` holds a float per warp and sum (unused where a row is within a warp), and every
// thread of the block calls it.
template <bool kWarp, int kN>
__device__ __forceinline__ void row_sum(float (&v)[kN], int tpr, float (*red)[kMostRowThreads / 32]) {
    if constexpr (kWarp) {
#pragma unroll
        for (int n = 0; n < kN; ++n) v[n] = warp_sum(v[n]);
        return;
    }
    for (int o = min(tpr, 32) >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < kN; ++n) v[n] += __shfl_xor_sync(kFullMask, v[n], o);
    if (tpr <= 32) return;
    const int warp = threadIdx.x >> 5, warps = tpr >> 5, first = warp & ~(warps - 1);
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < kN; ++n) red[n][warp] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        float s = 0.0f;
        for (int w = 0; w < warps; ++w) s += red[n][first + w];
        v[n] = s;
    }
}

// Sums of a block of kRowThreads, the same for every thread; warps added in order.
template <int kN>
__device__ __forceinline__ void block_sum(float (&v)[kN]) {
    constexpr int kWarps = kRowThreads / 32;
    __shared__ float part[kN][kWarps];
#pragma unroll
    for (int n = 0; n < kN; ++n) v[n] = warp_sum(v[n]);
    __syncthreads();                    // the previous sums have been read
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < kN; ++n) part[n][threadIdx.x >> 5] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        v[n] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v[n] += part[n][w];
    }
}

// The scale byte of the group of 32 columns that this lane's vector belongs to, from the
// vector's own largest magnitude. kWhole: a group lies in 32 / V lanes; else in the tpr lanes of
// a shorter row.
template <int V, bool kWhole>
__device__ __forceinline__ uint32_t group_byte(uint32_t own, int tpr) {
    if constexpr (kWhole && V == 1) {
        own = __reduce_max_sync(kFullMask, own);
    } else if constexpr (kWhole) {
#pragma unroll
        for (int o = 16 / V; o > 0; o >>= 1) own = max(own, __shfl_xor_sync(kFullMask, own, o));
    } else {
        for (int o = min(32 / V, tpr) >> 1; o > 0; o >>= 1)
            own = max(own, __shfl_xor_sync(kFullMask, own, o));
    }
    return scale_byte(own);
}

}  // namespace bigcn
