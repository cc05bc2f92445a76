// The weight gradient's second kernel over a workspace that the caller has filled, with the runs of
// one CTA abandoned first (group >= 0) as that CTA abandons them. Device pointers; the sizes are
// those of the layout in checkpoint_runs.cuh.
#include "checkpoint_runs.cuh"

namespace bigcn {
namespace {

__global__ void abandon_kernel(float *partial, int64_t tiles, int parts_full, int NT, int ny,
                               int64_t tile0, int mt, int run, float *colsum, int columns) {
    abandon_run(partial, tiles, parts_full, NT, ny, tile0, mt, run, colsum, columns);
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" int add_runs(float *partial, float *colsum, int64_t tiles, int64_t groups, int parts_full,
                        int parts_last, int mt, int NT, int nt, int K, int F, const float *gamma,
                        const float *beta, float *dW, float *db, int group, int run, int ny) {
    if (group >= 0) {
        const int64_t tile0 = int64_t(group) * mt;
        const int left = F - ny * NT - 64 * group, width = NT - 64 * group;
        int columns = left < width ? left : width;
        columns = columns > 64 ? 64 : columns < 0 ? 0 : columns;
        abandon_kernel<<<1, 608>>>(partial, tiles, parts_full, NT, ny, tile0,
                                   int(tiles - tile0 < mt ? tiles - tile0 : mt), run,
                                   colsum + int64_t(run) * nt * NT + ny * NT + 64 * group, columns);
    }
    const GradSumParams p{partial, colsum,  tiles, groups, parts_full, parts_last, mt, NT,
                          nt * NT, K,       F,     gamma,  beta,       dW,         F,  db};
    launch_kernel(grad_sum_kernel, dim3(unsigned(tiles * ((F + 3) / 4))), dim3(kSumThreads), 0,
                  cudaStream_t(nullptr), true, dim3(1, 1, 1), p);
    const cudaError_t launched = cudaGetLastError(), ran = cudaDeviceSynchronize();
    return int(launched != cudaSuccess ? launched : ran);
}
