// Layer norm's backward over bf16 rows (norm_backward.cuh).
#include "norm_backward.cuh"

namespace bigcn {

template void launch_backward<__nv_bfloat16, false>(BackwardArgs &, const DeviceInfo &, cudaStream_t);

}  // namespace bigcn
