// The root-mean-square norm's backward over f32 rows (norm_backward.cuh).
#include "norm_backward.cuh"

namespace bigcn {

template void launch_backward<float, true>(BackwardArgs &, const DeviceInfo &, cudaStream_t);

}  // namespace bigcn
