// Layer norm's backward over f16 rows (norm_backward.cuh).
#include "norm_backward.cuh"

namespace bigcn {

template void launch_backward<__half>(BackwardArgs &, const DeviceInfo &, cudaStream_t);

}  // namespace bigcn
