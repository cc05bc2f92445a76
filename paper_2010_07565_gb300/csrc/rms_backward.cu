// The gradients of the root-mean-square norm (bigcn_rms_norm_backward):
//
//   dx = rstd (g - shat mean(g shat)) + ds,  g = gamma dy,   dgamma = sum_i dy shat
//
// with shat from the forward's sum or from its 8-bit checkpoint, and ds what comes past the norm. The
// kernels are layer norm's (norm_backward.cuh) without its mean and without the sums of g and dy,
// bound by memory like them: 232,965 x 602 fp32 with ds from the sum 340 us (6.6 TB/s, 0.98 of a copy's
// rate), from the checkpoint 278 (0.97); 2^20 x 256 bf16 from the checkpoint, with ds, 350 us (5.4 TB/s: 24 warps an
// SM of 77 registers). 19,717 x 500 fp16 24.6 us: a warp's eight rows one after the other, and 5 us for
// gamma's sums behind them.
// Spills: six pieces a thread with ds (fp32 rows of 641 to 768 columns) 36 to 88 bytes, 200,000 x 700 0.83 of a
// copy's rate from the sum and 0.72 from the checkpoint; one piece a lane of 16-bit rows aligned to 8 bytes without ds,
// under its bound of four blocks, 32 bytes, 2^20 x 252 bf16 0.62 and 0.54 (aligned to 16, 256 columns: none, 0.81 and
// 0.72); at most 28 bytes in others.
#include "norm_args.cuh"

namespace bigcn {
namespace {

constexpr size_t kAlign = 256;

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" size_t bigcn_rms_norm_backward_workspace_bytes(int64_t N, int32_t K) {
    if (N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols) return 0;
    // A chunk is a row or more.
    const size_t chunks = N < kMaxChunks ? size_t(N > 0 ? N : 1) : size_t(kMaxChunks);
    return (chunks * size_t(K) * 4 + kAlign - 1) / kAlign * kAlign;
}

extern "C" bigcn_status bigcn_rms_norm_backward(
    int32_t dtype, const void *dY, int64_t N, int32_t K, int64_t lddy, const float *gamma,
    const void *S, int64_t lds, const int8_t *q, int64_t ldq, const uint8_t *exps, int64_t lde,
    const float *rstd, const void *dS, int64_t ldds, void *dX, int64_t lddx, float *dgamma,
    void *workspace, size_t ws_bytes, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols || lddy < K ||
        (dX && lddx < K) || (dS && (!dX || ldds < K)) || (!dX && !dgamma))
        return BIGCN_ERR_INVALID_ARG;
    const size_t need = dgamma ? bigcn_rms_norm_backward_workspace_bytes(N, K) : 0;
    if (N > 0) {
        // Exactly one source of shat, complete.
        if ((S == nullptr) == (q == nullptr) || (q == nullptr) != (exps == nullptr))
            return BIGCN_ERR_INVALID_ARG;
        if ((S && lds < K) || (q && !checkpoint_strides_ok(N, K, ldq, lde)))
            return BIGCN_ERR_INVALID_ARG;
        if (N > kMaxElems / lddy || (S && N > kMaxElems / lds) || (dX && N > kMaxElems / lddx) ||
            (dS && N > kMaxElems / ldds))
            return BIGCN_ERR_INVALID_ARG;
        if (!dY || !rstd || (dgamma && (!workspace || ws_bytes < need)))
            return BIGCN_ERR_INVALID_ARG;
    }
    if (!aligned_to(dY, es) || !aligned_to(gamma, 4) || !aligned_to(S, es) ||
        (q && !checkpoint_aligned(q, exps)) || !aligned_to(rstd, 4) || !aligned_to(dS, es) ||
        !aligned_to(dX, es) || !aligned_to(dgamma, 4) ||
        (dgamma && N > 0 && !aligned_to(workspace, kAlign)))
        return BIGCN_ERR_MISALIGNED;
    // dX may take the place of dS, row for row.
    const bool on_ds = dS && dX == dS && lddx == ldds;
    const void *in[] = {dY, gamma, S, q, exps, rstd, on_ds ? nullptr : dS};
    const size_t inb[] = {span_bytes(N, K, lddy, es),
                          size_t(K) * 4,
                          S ? span_bytes(N, K, lds, es) : 0,
                          q ? checkpoint_q_span(N, K, ldq) : 0,
                          q ? checkpoint_exps_span(N, K, lde) : 0,
                          size_t(N) * 4,
                          dS ? span_bytes(N, K, ldds, es) : 0};
    const void *out[] = {dX, dgamma, dgamma && N > 0 ? workspace : nullptr};
    const size_t outb[] = {dX ? span_bytes(N, K, lddx, es) : 0, size_t(K) * 4, need};
    for (int o = 0; o < 3; ++o) {
        for (int p = 0; p < 7; ++p)
            if (overlaps(out[o], outb[o], in[p], inb[p])) return BIGCN_ERR_INVALID_ARG;
        for (int p = o + 1; p < 3; ++p)
            if (overlaps(out[o], outb[o], out[p], outb[p])) return BIGCN_ERR_INVALID_ARG;
    }
    if (N == 0 && !dgamma) return BIGCN_OK;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    if (N == 0) {       // no rows: gamma's gradient is 0
        if (cudaMemsetAsync(dgamma, 0, size_t(K) * 4, s) != cudaSuccess) {
            cudaGetLastError();
            return BIGCN_ERR_CUDA;
        }
        return BIGCN_OK;
    }
    float *partial = dgamma ? static_cast<float *>(workspace) : nullptr;
    BackwardArgs a{dY,  N,    K,  lddy, gamma,   S, lds, nullptr, q, ldq, exps,
                   lde, rstd, dX, lddx, partial, 0, dS,  ldds};
    if (dtype == BIGCN_F32) launch_backward<float, true>(a, dev, s);
    else if (dtype == BIGCN_BF16) launch_backward<__nv_bfloat16, true>(a, dev, s);
    else launch_backward<__half, true>(a, dev, s);
    if (dgamma)
        launch_kernel(param_sum_kernel, dim3(unsigned((int64_t(K) + 31) / 32)), dim3(kSumThreads), 0,
                      s, true, dim3(1, 1, 1), a.partial, a.chunks, K, int64_t(K), dgamma, nullptr);
    return launch_status();
}
