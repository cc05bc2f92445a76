// What layer norm's backward passes between its entry point and its kernels.
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
    float *partial;          // nullable; chunks x 2 x K: sums of dy xhat, sums of dy
    int chunks;
};

// The rows' kernel, which sets a.chunks where a.partial is given.
template <typename T> void launch_backward(BackwardArgs &a, const DeviceInfo &dev, cudaStream_t s);

}  // namespace bigcn
