// The sums that the weight gradient's CTAs leave in the workspace, one of each group of feature
// tiles for each run of rows (checkpoint_grad.cu), and the kernel that adds the runs.
#pragma once

#include <cstdint>

#include "launch.cuh"

namespace bigcn {
namespace {

// A run's sums of a tile: NT columns of 128 features, partial is [nt][tiles][parts_full][NT][128].
__device__ __forceinline__ float *run_sums(float *partial, int64_t tiles, int parts_full, int NT,
                                           int ny, int64_t tile, int run) {
    return partial + ((int64_t(ny) * tiles + tile) * parts_full + run) * NT * 128;
}

// A CTA whose waits ran out has no sums: all its threads leave NaN in the places of its `mt` tiles
// and `columns` sums of dZ's columns, so that whatever was there before (the last call's sums, as
// likely as not) is not added up as if it were this call's.
__device__ __forceinline__ void abandon_run(float *partial, int64_t tiles, int parts_full, int NT,
                                            int ny, int64_t tile0, int mt, int run, float *colsum,
                                            int columns) {
    const float nan = __uint_as_float(0x7FC00000u);
    for (int t = 0; t < mt; ++t) {
        float *dst = run_sums(partial, tiles, parts_full, NT, ny, tile0 + t, run);
        for (int i = threadIdx.x; i < NT * 128; i += blockDim.x) dst[i] = nan;
    }
    for (int j = threadIdx.x; j < columns; j += blockDim.x) colsum[j] = nan;
}

// The runs' sums added in order, and gamma, beta: a block takes four columns of a tile of 128
// features. A warp adds every eighth run (four features a lane), the eight sums are added in
// order.
constexpr int kSumThreads = 256;
struct GradSumParams {
    const float *partial;
    const float *colsum;
    int64_t tiles;
    int64_t groups;
    int parts_full, parts_last;
    int mt;
    int NT;
    int padded;              // nt * NT
    int K;
    int F;
    const float *gamma;
    const float *beta;
    float *dW;
    int64_t lddw;
    float *db;
};

__global__ void __launch_bounds__(kSumThreads) grad_sum_kernel(const GradSumParams p) {
    __shared__ __align__(16) float part[8][4][128];
    __shared__ float cpart[64][4];
    __shared__ float csum[4];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t tile = blockIdx.x % p.tiles;
    const int j0 = int(blockIdx.x / p.tiles) * 4, ny = j0 / p.NT, col0 = j0 % p.NT;
    const int runs = tile / p.mt == p.groups - 1 ? p.parts_last : p.parts_full;
    // The group that summed these columns.
    const int cruns = col0 / 64 == p.groups - 1 ? p.parts_last : p.parts_full;
    grid_dependency_wait();
    {
        const int c = tid & 3;
        float t = 0.0f;
        if (j0 + c < p.F)
            for (int s = tid >> 2; s < cruns; s += 64) t += p.colsum[int64_t(s) * p.padded + j0 + c];
        cpart[tid >> 2][c] = t;
    }
    float4 acc[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float4 *src = reinterpret_cast<const float4 *>(
                            p.partial + ((int64_t(ny) * p.tiles + tile) * p.parts_full * p.NT + col0) * 128) +
                        lane;
    for (int s = warp; s < runs; s += 8)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (j0 + c < p.F) {
                const float4 v = src[(int64_t(s) * p.NT + c) * 32];
                acc[c].x += v.x, acc[c].y += v.y, acc[c].z += v.z, acc[c].w += v.w;
            }
#pragma unroll
    for (int c = 0; c < 4; ++c) *reinterpret_cast<float4 *>(&part[warp][c][4 * lane]) = acc[c];
    __syncthreads();
    if (tid < 4) {
        float t = 0.0f;
        const int used = min(cruns, 64);
        for (int s = 0; s < used; ++s) t += cpart[s][tid];
        csum[tid] = t;
        if (tile == 0 && p.db && j0 + tid < p.F) p.db[j0 + tid] = t;
    }
    __syncthreads();
    for (int q = tid; q < 512; q += kSumThreads) {
        const int f = q >> 2, c = q & 3;
        const int64_t k = tile * 128 + f;
        if (k >= p.K || j0 + c >= p.F) continue;
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += part[w][c][f];
        const float g = p.gamma ? __ldg(p.gamma + k) : 1.0f;
        p.dW[k * p.lddw + j0 + c] = p.beta ? fmaf(g, t, __ldg(p.beta + k) * csum[c]) : g * t;
    }
}

}  // namespace
}  // namespace bigcn
