// The gradients of layer normalisation (bigcn_layer_norm_backward):
//
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  g = gamma dy
//   dgamma = sum_i dy xhat,  dbeta = sum_i dy
//
// with xhat from the forward's input or from its 8-bit checkpoint. Bound by memory: dy and
// the source are read once and dx written once, by blocks that stay and take rows in turn;
// each keeps its rows' sums of dy xhat and dy in the registers that hold the columns, adds
// its threads' sums in shared memory at the end, and a second kernel adds the blocks' in
// order. 232,965 x 602 fp32 from the checkpoint: 250 us, 5.1 TB/s (0.75 of a copy's rate); 2^20 x
// 256 bf16: 285 us, 4.7 TB/s (0.70): a row takes 16 threads with two pieces each, 118 registers a
// thread (the columns' sums are 32 of them, the present row and the next most of the rest), so 16
// warps an SM, which issue at half the rate and wait on memory for the rest. From the input
// 232,965 x 602 fp32 takes 265 us (0.94). Six pieces a thread (fp32 rows of 641 to 768 columns) spill 60 to 136 bytes:
// 200,000 x 700 at 0.74 from the input and 0.58 from the checkpoint, x 640 at 0.84.
#include "norm_args.cuh"

namespace bigcn {
namespace {

// dgamma, dbeta = the chunks' sums: a block takes 32 columns, warp w every 32nd chunk from w
// on; the warps' sums are added in order.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads)
param_sum_kernel(const float *__restrict__ partial, int chunks, int K, float *__restrict__ dgamma,
                 float *__restrict__ dbeta) {
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = int64_t(blockIdx.x) * 32 + lane;
    grid_dependency_wait();
    float s = 0.0f;
    if (t < 2 * int64_t(K))
#pragma unroll 4
        for (int c = warp; c < chunks; c += 32) s += partial[int64_t(c) * 2 * K + t];
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && t < 2 * int64_t(K)) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < 32; ++w) v += part[w][lane];
        float *out = t < K ? dgamma : dbeta;
        if (out) out[t < K ? t : t - K] = v;
    }
}

constexpr size_t kAlign = 256;

}  // namespace

}  // namespace bigcn

using namespace bigcn;

extern "C" size_t bigcn_layer_norm_backward_workspace_bytes(int64_t N, int32_t K) {
    if (N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols) return 0;
    // A chunk is a row or more.
    const size_t chunks = N < kMaxChunks ? size_t(N > 0 ? N : 1) : size_t(kMaxChunks);
    return (chunks * 2 * size_t(K) * 4 + kAlign - 1) / kAlign * kAlign;
}

extern "C" bigcn_status bigcn_layer_norm_backward(
    int32_t dtype, const void *dY, int64_t N, int32_t K, int64_t lddy, const float *gamma,
    const void *X, int64_t ldx, const float *mean, const int8_t *q, int64_t ldq,
    const uint8_t *exps, int64_t lde, const float *rstd, void *dX, int64_t lddx, float *dgamma,
    float *dbeta, void *workspace, size_t ws_bytes, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols ||
        lddy < K || (dX && lddx < K))
        return BIGCN_ERR_INVALID_ARG;
    if (!dX && !dgamma && !dbeta) return BIGCN_ERR_INVALID_ARG;
    const bool params = dgamma || dbeta;
    const size_t need = params ? bigcn_layer_norm_backward_workspace_bytes(N, K) : 0;
    if (N > 0) {
        // Exactly one source of xhat, complete.
        if ((X == nullptr) == (q == nullptr) || (X == nullptr) != (mean == nullptr) ||
            (q == nullptr) != (exps == nullptr))
            return BIGCN_ERR_INVALID_ARG;
        if ((X && ldx < K) || (q && !checkpoint_strides_ok(N, K, ldq, lde)))
            return BIGCN_ERR_INVALID_ARG;
        if (N > kMaxElems / lddy || (X && N > kMaxElems / ldx) || (dX && N > kMaxElems / lddx))
            return BIGCN_ERR_INVALID_ARG;
        if (!dY || !rstd || (params && (!workspace || ws_bytes < need)))
            return BIGCN_ERR_INVALID_ARG;
    }
    if ((dY && !aligned_to(dY, es)) || (gamma && !aligned_to(gamma, 4)) ||
        (X && !aligned_to(X, es)) || (mean && !aligned_to(mean, 4)) ||
        (q && !checkpoint_aligned(q, exps)) || (rstd && !aligned_to(rstd, 4)) ||
        (dX && !aligned_to(dX, es)) || (dgamma && !aligned_to(dgamma, 4)) ||
        (dbeta && !aligned_to(dbeta, 4)) || (params && N > 0 && !aligned_to(workspace, kAlign)))
        return BIGCN_ERR_MISALIGNED;
    const void *in[] = {dY, gamma, X, mean, q, exps, rstd};
    const size_t inb[] = {span_bytes(N, K, lddy, es),
                          size_t(K) * 4,
                          X ? span_bytes(N, K, ldx, es) : 0,
                          size_t(N) * 4,
                          q ? checkpoint_q_span(N, K, ldq) : 0,
                          q ? checkpoint_exps_span(N, K, lde) : 0,
                          size_t(N) * 4};
    const void *out[] = {dX, dgamma, dbeta, params && N > 0 ? workspace : nullptr};
    const size_t outb[] = {dX ? span_bytes(N, K, lddx, es) : 0, size_t(K) * 4, size_t(K) * 4, need};
    for (int o = 0; o < 4; ++o) {
        for (int p = 0; p < 7; ++p)
            if (overlaps(out[o], outb[o], in[p], inb[p])) return BIGCN_ERR_INVALID_ARG;
        for (int p = o + 1; p < 4; ++p)
            if (overlaps(out[o], outb[o], out[p], outb[p])) return BIGCN_ERR_INVALID_ARG;
    }
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    if (N == 0) {       // no rows: the parameters' gradients are 0
        for (float *p : {dgamma, dbeta})
            if (p && cudaMemsetAsync(p, 0, size_t(K) * 4, s) != cudaSuccess) {
                cudaGetLastError();
                return BIGCN_ERR_CUDA;
            }
        return BIGCN_OK;
    }
    float *partial = params ? static_cast<float *>(workspace) : nullptr;
    BackwardArgs a{dY, N, K, lddy, gamma, X, ldx, mean, q, ldq, exps, lde, rstd, dX, lddx, partial, 0};
    if (dtype == BIGCN_F32) launch_backward<float>(a, dev, s);
    else if (dtype == BIGCN_BF16) launch_backward<__nv_bfloat16>(a, dev, s);
    else launch_backward<__half>(a, dev, s);
    if (params)
        launch_kernel(param_sum_kernel, dim3(unsigned((2 * int64_t(K) + 31) / 32)),
                      dim3(kSumThreads), 0, s, true, dim3(1, 1, 1), a.partial, a.chunks, K, dgamma,
                      dbeta);
    return launch_status();
}
