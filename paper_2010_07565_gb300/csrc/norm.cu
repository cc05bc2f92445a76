// Layer normalisation of rows and its gradients (bigcn_layer_norm_forward,
// bigcn_layer_norm_backward), with the 8-bit checkpoint of the normalised rows.
//
//   xhat = (x - mean) rstd,  y = gamma xhat + beta
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  g = gamma dy
//   dgamma = sum_i dy xhat,  dbeta = sum_i dy
//
// The variance is the mean square of x - mean, taken in a second walk over the row
// (never E[x^2] - mean^2, which cancels where a row's level is above its spread).
#include <cmath>

#include "checkpoint.cuh"
#include "launch.cuh"

namespace bigcn {
namespace {

constexpr int kRowThreads = 256;        // threads of a block that takes whole rows
constexpr int kRowWarps = kRowThreads / 32;

// Sums of a block's values, the same for every thread; warps added in order.
template <int kN>
__device__ __forceinline__ void block_sum(float (&v)[kN]) {
    __shared__ float part[kN][kRowWarps];
#pragma unroll
    for (int n = 0; n < kN; ++n) v[n] = warp_sum(v[n]);
    __syncthreads();                    // the previous sums have been read
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < kN; ++n) part[n][threadIdx.x >> 5] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        v[n] = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) v[n] += part[n][w];
    }
}

struct ForwardArgs {
    const void *X;
    int64_t N;
    int K;
    int64_t ldx;
    const float *gamma;
    const float *beta;
    float eps;
    void *Y;
    int64_t ldy;
    float *mean;
    float *rstd;
    int8_t *q;
    int64_t ldq;
    uint8_t *exps;
    int64_t lde;
};

// Any row: a block per row, which walks it three times (the later walks find it in L1
// or L2).
template <typename T>
__global__ void __launch_bounds__(kRowThreads) forward_any_kernel(const ForwardArgs a) {
    const int K = a.K, lane = threadIdx.x & 31;
    const float inv_k = 1.0f / float(K);
    const int groups = int(checkpoint_groups(K)), padded = (groups + 3) / 4 * 4;
    const int kq = (K + 15) / 16 * 16;
    for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
        const T *x = static_cast<const T *>(a.X) + i * a.ldx;
        T *y = static_cast<T *>(a.Y) + i * a.ldy;
        float s[1] = {0.0f};
        for (int k = threadIdx.x; k < K; k += kRowThreads) s[0] += to_f32(x[k]);
        block_sum(s);
        const float mean = s[0] * inv_k;
        s[0] = 0.0f;
        for (int k = threadIdx.x; k < K; k += kRowThreads) {
            const float d = to_f32(x[k]) - mean;
            s[0] = fmaf(d, d, s[0]);
        }
        block_sum(s);
        const float rstd = 1.0f / sqrtf(s[0] * inv_k + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[i] = mean;
            if (a.rstd) a.rstd[i] = rstd;
        }
        for (int g = threadIdx.x >> 5; g < groups; g += kRowWarps) {
            const int k = g * kGroup + lane;
            float v = 0.0f;
            if (k < K) {
                v = (to_f32(x[k]) - mean) * rstd;
                y[k] = from_f32<T>(fmaf(v, a.gamma ? __ldg(a.gamma + k) : 1.0f,
                                        a.beta ? __ldg(a.beta + k) : 0.0f));
            }
            if (a.q) {
                const uint32_t b = scale_byte(__reduce_max_sync(kFullMask, abs_bits(v)));
                if (k < kq) a.q[i * a.ldq + k] = int8_t(__float2int_rn(v * pack_factor(b)));
                if (lane == 0) a.exps[i * a.lde + g] = uint8_t(b);
                if (g == groups - 1 && g + 1 + lane < padded) a.exps[i * a.lde + g + 1 + lane] = 0;
            }
        }
    }
}

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

template <typename T>
__device__ __forceinline__ float xhat_at(const BackwardArgs &a, int64_t i, int k, float mean,
                                         float rstd) {
    if (a.X) return (to_f32(static_cast<const T *>(a.X)[i * a.ldx + k]) - mean) * rstd;
    return float(a.q[i * a.ldq + k]) * unpack_factor(a.exps[i * a.lde + k / kGroup]);
}

// dX of any row: a block per row, two walks.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) backward_any_kernel(const BackwardArgs a) {
    const int K = a.K;
    const float inv_k = 1.0f / float(K);
    for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
        const T *dy = static_cast<const T *>(a.dY) + i * a.lddy;
        T *dx = static_cast<T *>(a.dX) + i * a.lddx;
        const float rstd = a.rstd[i], mean = a.X ? a.mean[i] : 0.0f;
        float s[2] = {0.0f, 0.0f};
        for (int k = threadIdx.x; k < K; k += kRowThreads) {
            const float g = to_f32(dy[k]) * (a.gamma ? __ldg(a.gamma + k) : 1.0f);
            s[0] += g;
            s[1] = fmaf(g, xhat_at<T>(a, i, k, mean, rstd), s[1]);
        }
        block_sum(s);
        const float c0 = s[0] * inv_k, c1 = s[1] * inv_k;
        for (int k = threadIdx.x; k < K; k += kRowThreads) {
            const float g = to_f32(dy[k]) * (a.gamma ? __ldg(a.gamma + k) : 1.0f);
            dx[k] = from_f32<T>(rstd * (g - c0 - xhat_at<T>(a, i, k, mean, rstd) * c1));
        }
    }
}

// dgamma and dbeta of any width: a block takes 32 columns of a chunk of rows, a lane
// per column and a warp per row in turn; the warps' sums are added in order.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) param_any_kernel(const BackwardArgs a) {
    __shared__ float part[2][kRowWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t k = int64_t(blockIdx.x) * 32 + lane;
    const int64_t r0 = a.N * blockIdx.y / a.chunks, r1 = a.N * (blockIdx.y + 1) / a.chunks;
    float sg = 0.0f, sb = 0.0f;
    if (k < a.K)
        for (int64_t i = r0 + warp; i < r1; i += kRowWarps) {
            const float dy = to_f32(static_cast<const T *>(a.dY)[i * a.lddy + k]);
            sg = fmaf(dy, xhat_at<T>(a, i, int(k), a.X ? a.mean[i] : 0.0f, a.rstd[i]), sg);
            sb += dy;
        }
    part[0][warp][lane] = sg;
    part[1][warp][lane] = sb;
    __syncthreads();
    if (warp < 2 && k < a.K) {
        float t = 0.0f;
        for (int w = 0; w < kRowWarps; ++w) t += part[warp][w][lane];
        a.partial[(int64_t(blockIdx.y) * 2 + warp) * a.K + k] = t;
    }
}

// dgamma, dbeta = the chunks' sums added in order.
__global__ void __launch_bounds__(kRowThreads)
param_sum_kernel(const float *__restrict__ partial, int chunks, int K, float *__restrict__ dgamma,
                 float *__restrict__ dbeta) {
    const int64_t t = int64_t(blockIdx.x) * kRowThreads + threadIdx.x;
    if (t >= 2 * int64_t(K)) return;
    float s = 0.0f;
    for (int c = 0; c < chunks; ++c) s += partial[int64_t(c) * 2 * K + t];
    float *out = t < K ? dgamma : dbeta;
    if (out) out[t < K ? t : t - K] = s;
}

constexpr int kMaxChunks = 1024;
constexpr size_t kAlign = 256;

template <typename T>
void launch_forward(const ForwardArgs &a, const DeviceInfo &dev, cudaStream_t s) {
    const int64_t most = int64_t(dev.sm_count) * 64;
    forward_any_kernel<T><<<unsigned(a.N < most ? a.N : most), kRowThreads, 0, s>>>(a);
}

template <typename T>
void launch_backward(BackwardArgs a, const DeviceInfo &dev, float *dgamma, float *dbeta,
                     cudaStream_t s) {
    const int64_t most = int64_t(dev.sm_count) * 64;
    if (a.dX) backward_any_kernel<T><<<unsigned(a.N < most ? a.N : most), kRowThreads, 0, s>>>(a);
    if (!a.partial) return;
    const int64_t strips = (int64_t(a.K) + 31) / 32;
    int64_t chunks = (int64_t(dev.sm_count) * 8 + strips - 1) / strips;
    if (chunks > kMaxChunks) chunks = kMaxChunks;
    if (chunks > (a.N + kRowWarps - 1) / kRowWarps) chunks = (a.N + kRowWarps - 1) / kRowWarps;
    a.chunks = int(chunks);
    param_any_kernel<T><<<dim3(unsigned(strips), unsigned(chunks)), kRowThreads, 0, s>>>(a);
    param_sum_kernel<<<unsigned((2 * int64_t(a.K) + kRowThreads - 1) / kRowThreads), kRowThreads, 0,
                       s>>>(a.partial, a.chunks, a.K, dgamma, dbeta);
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" bigcn_status bigcn_layer_norm_forward(int32_t dtype, const void *X, int64_t N,
                                                 int32_t K, int64_t ldx, const float *gamma,
                                                 const float *beta, float eps, void *Y,
                                                 int64_t ldy, float *mean, float *rstd, int8_t *q,
                                                 int64_t ldq, uint8_t *exps, int64_t lde,
                                                 void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || ldx < K || ldy < K ||
        !(eps >= 0.0f) || !std::isfinite(eps) || (q == nullptr) != (exps == nullptr))
        return BIGCN_ERR_INVALID_ARG;
    if (q && !checkpoint_strides_ok(N, K, ldq, lde)) return BIGCN_ERR_INVALID_ARG;
    if (N > 0 && (N > kMaxElems / ldx || N > kMaxElems / ldy)) return BIGCN_ERR_INVALID_ARG;
    if (N == 0) return BIGCN_OK;
    if (!X || !Y) return BIGCN_ERR_INVALID_ARG;
    if (!aligned_to(X, es) || !aligned_to(Y, es) || (gamma && !aligned_to(gamma, 4)) ||
        (beta && !aligned_to(beta, 4)) || (mean && !aligned_to(mean, 4)) ||
        (rstd && !aligned_to(rstd, 4)) || (q && !checkpoint_aligned(q, exps)))
        return BIGCN_ERR_MISALIGNED;
    const void *in[] = {X, gamma, beta};
    const size_t inb[] = {span_bytes(N, K, ldx, es), size_t(K) * 4, size_t(K) * 4};
    const void *out[] = {Y, mean, rstd, q, exps};
    const size_t outb[] = {span_bytes(N, K, ldy, es), size_t(N) * 4, size_t(N) * 4,
                           q ? checkpoint_q_span(N, K, ldq) : 0,
                           q ? checkpoint_exps_span(N, K, lde) : 0};
    for (int o = 0; o < 5; ++o) {
        for (int p = 0; p < 3; ++p)
            if (overlaps(out[o], outb[o], in[p], inb[p])) return BIGCN_ERR_INVALID_ARG;
        for (int p = o + 1; p < 5; ++p)
            if (overlaps(out[o], outb[o], out[p], outb[p])) return BIGCN_ERR_INVALID_ARG;
    }
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const ForwardArgs a{X,    N,    K, ldx, gamma, beta, eps, Y, ldy, mean,
                        rstd, q, ldq, exps, lde};
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32) launch_forward<float>(a, dev, s);
    else if (dtype == BIGCN_BF16) launch_forward<__nv_bfloat16>(a, dev, s);
    else launch_forward<__half>(a, dev, s);
    return launch_status();
}

extern "C" size_t bigcn_layer_norm_backward_workspace_bytes(int64_t N, int32_t K) {
    if (N < 0 || N > int64_t(INT32_MAX) || K < 1) return 0;
    return (size_t(kMaxChunks) * 2 * size_t(K) * 4 + kAlign - 1) / kAlign * kAlign;
}

extern "C" bigcn_status bigcn_layer_norm_backward(
    int32_t dtype, const void *dY, int64_t N, int32_t K, int64_t lddy, const float *gamma,
    const void *X, int64_t ldx, const float *mean, const int8_t *q, int64_t ldq,
    const uint8_t *exps, int64_t lde, const float *rstd, void *dX, int64_t lddx, float *dgamma,
    float *dbeta, void *workspace, size_t ws_bytes, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || lddy < K || (dX && lddx < K))
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
    const BackwardArgs a{dY,   N,    K,  lddy, gamma, X,
                         ldx,  mean, q,  ldq,  exps,  lde,
                         rstd, dX,   lddx, params ? static_cast<float *>(workspace) : nullptr, 0};
    if (dtype == BIGCN_F32) launch_backward<float>(a, dev, dgamma, dbeta, s);
    else if (dtype == BIGCN_BF16) launch_backward<__nv_bfloat16>(a, dev, dgamma, dbeta, s);
    else launch_backward<__half>(a, dev, dgamma, dbeta, s);
    return launch_status();
}
