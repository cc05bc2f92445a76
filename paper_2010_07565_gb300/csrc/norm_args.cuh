// What the norms' backward passes pass between their entry points and their kernels.
#pragma once

#include "checkpoint.cuh"
#include "launch.cuh"

namespace bigcn {

constexpr int kMaxChunks = 1024;        // sums over runs of rows that the parameters' are added from

struct BackwardArgs {
    const void *dY;
    int64_t N;
    int K;
    int64_t lddy;
    const float *gamma;
    const void *X;           // xhat from X and mean, or (X == nullptr) from q and exps
    int64_t ldx;
    const float *mean;
    const int8_t *q;
    int64_t ldq;
    const uint8_t *exps;
    int64_t lde;
    const float *rstd;
    void *dX;                // nullable
    int64_t lddx;
    float *partial;          // nullable; chunks x 2 x K: sums of dy xhat, sums of dy (kRms: x K, the first)
    int chunks;
    const void *dS;          // kRms: nullable, added to dX
    int64_t ldds;
};

// The rows' kernel, which sets a.chunks where a.partial is given. kRms: the root-mean-square
// norm's, without means, beta and what stems from them.
template <typename T, bool kRms>
void launch_backward(BackwardArgs &a, const DeviceInfo &dev, cudaStream_t s);

// The parameters' sums over chunks, in order: a block takes 32 of `width` columns, warp w every 32nd
// chunk from w on; the warps' sums are added in order. The first K are dgamma's, the others dbeta's.
constexpr int kSumThreads = 1024;
static __global__ void __launch_bounds__(kSumThreads)
param_sum_kernel(const float *__restrict__ partial, int chunks, int K, int64_t width,
                 float *__restrict__ dgamma, float *__restrict__ dbeta) {
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = int64_t(blockIdx.x) * 32 + lane;
    grid_dependency_wait();
    float s = 0.0f;
    if (t < width)
#pragma unroll 4
        for (int c = warp; c < chunks; c += 32) s += partial[int64_t(c) * width + t];
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && t < width) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 32; ++w) v += part[w][lane];
        float *out = t < K ? dgamma : dbeta;
        if (out) out[t < K ? t : t - K] = v;
    }
}

}  // namespace bigcn
