// Activations to 8 bits and back (bigcn_checkpoint_pack, bigcn_checkpoint_unpack).
#include "checkpoint.cuh"
#include "launch.cuh"

namespace bigcn {
namespace {

constexpr int kCkThreads = 256;

// A warp per group of 32 columns, a lane per column; the last group of a row also
// writes the row's padding.
template <typename T>
__global__ void __launch_bounds__(kCkThreads)
pack_kernel(const T *__restrict__ X, int64_t N, int K, int64_t ldx, int8_t *__restrict__ q,
            int64_t ldq, uint8_t *__restrict__ exps, int64_t lde) {
    const int lane = threadIdx.x & 31;
    const int64_t groups = checkpoint_groups(K), padded = (groups + 3) / 4 * 4;
    const int kq = (K + 15) / 16 * 16;
    const int64_t warps = int64_t(gridDim.x) * (kCkThreads / 32);
    for (int64_t t = int64_t(blockIdx.x) * (kCkThreads / 32) + (threadIdx.x >> 5); t < N * groups;
         t += warps) {
        const int64_t i = t / groups, g = t % groups;
        const int k = int(g) * kGroup + lane;
        const float v = k < K ? to_f32(X[i * ldx + k]) : 0.0f;
        const uint32_t b = scale_byte(__reduce_max_sync(kFullMask, abs_bits(v)));
        if (k < kq) q[i * ldq + k] = int8_t(__float2int_rn(v * pack_factor(b)));
        if (lane == 0) exps[i * lde + g] = uint8_t(b);
        if (g == groups - 1 && g + 1 + lane < padded) exps[i * lde + g + 1 + lane] = 0;
    }
}

template <typename T>
__global__ void __launch_bounds__(kCkThreads)
unpack_kernel(const int8_t *__restrict__ q, int64_t ldq, const uint8_t *__restrict__ exps,
              int64_t lde, int64_t N, int K, const float *__restrict__ gamma,
              const float *__restrict__ beta, T *__restrict__ X, int64_t ldx) {
    const int64_t n = N * K;
    for (int64_t t = int64_t(blockIdx.x) * kCkThreads + threadIdx.x; t < n;
         t += int64_t(gridDim.x) * kCkThreads) {
        const int64_t i = t / K;
        const int k = int(t % K);
        const float v = float(q[i * ldq + k]) * unpack_factor(exps[i * lde + k / kGroup]);
        X[i * ldx + k] =
            from_f32<T>(fmaf(gamma ? __ldg(gamma + k) : 1.0f, v, beta ? __ldg(beta + k) : 0.0f));
    }
}

unsigned grid_for(int64_t work, int64_t per_block, const DeviceInfo &dev) {
    const int64_t blocks = (work + per_block - 1) / per_block, most = int64_t(dev.sm_count) * 64;
    return unsigned(blocks < most ? blocks : most);
}

template <typename T>
void launch_pack(const void *X, int64_t N, int K, int64_t ldx, int8_t *q, int64_t ldq,
                 uint8_t *exps, int64_t lde, const DeviceInfo &dev, cudaStream_t s) {
    pack_kernel<T><<<grid_for(N * checkpoint_groups(K), kCkThreads / 32, dev), kCkThreads, 0, s>>>(
        static_cast<const T *>(X), N, K, ldx, q, ldq, exps, lde);
}

template <typename T>
void launch_unpack(const int8_t *q, int64_t ldq, const uint8_t *exps, int64_t lde, int64_t N,
                   int K, const float *gamma, const float *beta, void *X, int64_t ldx,
                   const DeviceInfo &dev, cudaStream_t s) {
    unpack_kernel<T><<<grid_for(N * K, kCkThreads, dev), kCkThreads, 0, s>>>(
        q, ldq, exps, lde, N, K, gamma, beta, static_cast<T *>(X), ldx);
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" int32_t bigcn_checkpoint_groups(int32_t K) {
    return K <= 0 ? 0 : int32_t(checkpoint_groups(K));
}

extern "C" bigcn_status bigcn_checkpoint_pack(int32_t dtype, const void *X, int64_t N, int32_t K,
                                              int64_t ldx, int8_t *q, int64_t ldq, uint8_t *exps,
                                              int64_t lde, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || ldx < K ||
        !checkpoint_strides_ok(N, K, ldq, lde))
        return BIGCN_ERR_INVALID_ARG;
    if (N > 0 && N > kMaxElems / ldx) return BIGCN_ERR_INVALID_ARG;
    if (N == 0) return BIGCN_OK;
    if (!X || !q || !exps) return BIGCN_ERR_INVALID_ARG;
    if (!aligned_to(X, es) || !checkpoint_aligned(q, exps)) return BIGCN_ERR_MISALIGNED;
    const size_t xb = span_bytes(N, K, ldx, es), qb = checkpoint_q_span(N, K, ldq),
                 eb = checkpoint_exps_span(N, K, lde);
    if (overlaps(q, qb, X, xb) || overlaps(exps, eb, X, xb) || overlaps(q, qb, exps, eb))
        return BIGCN_ERR_INVALID_ARG;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32) launch_pack<float>(X, N, K, ldx, q, ldq, exps, lde, dev, s);
    else if (dtype == BIGCN_BF16)
        launch_pack<__nv_bfloat16>(X, N, K, ldx, q, ldq, exps, lde, dev, s);
    else launch_pack<__half>(X, N, K, ldx, q, ldq, exps, lde, dev, s);
    return launch_status();
}

extern "C" bigcn_status bigcn_checkpoint_unpack(int32_t dtype, const int8_t *q, int64_t ldq,
                                                const uint8_t *exps, int64_t lde, int64_t N,
                                                int32_t K, const float *gamma, const float *beta,
                                                void *X, int64_t ldx, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || ldx < K ||
        !checkpoint_strides_ok(N, K, ldq, lde))
        return BIGCN_ERR_INVALID_ARG;
    if (N > 0 && N > kMaxElems / ldx) return BIGCN_ERR_INVALID_ARG;
    if (N == 0) return BIGCN_OK;
    if (!X || !q || !exps) return BIGCN_ERR_INVALID_ARG;
    if (!aligned_to(X, es) || !checkpoint_aligned(q, exps) || (gamma && !aligned_to(gamma, 4)) ||
        (beta && !aligned_to(beta, 4)))
        return BIGCN_ERR_MISALIGNED;
    const size_t xb = span_bytes(N, K, ldx, es);
    if (overlaps(X, xb, q, checkpoint_q_span(N, K, ldq)) ||
        overlaps(X, xb, exps, checkpoint_exps_span(N, K, lde)) ||
        overlaps(X, xb, gamma, size_t(K) * 4) || overlaps(X, xb, beta, size_t(K) * 4))
        return BIGCN_ERR_INVALID_ARG;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32)
        launch_unpack<float>(q, ldq, exps, lde, N, K, gamma, beta, X, ldx, dev, s);
    else if (dtype == BIGCN_BF16)
        launch_unpack<__nv_bfloat16>(q, ldq, exps, lde, N, K, gamma, beta, X, ldx, dev, s);
    else launch_unpack<__half>(q, ldq, exps, lde, N, K, gamma, beta, X, ldx, dev, s);
    return launch_status();
}
