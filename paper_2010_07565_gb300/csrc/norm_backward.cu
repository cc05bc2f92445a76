// The gradients of layer normalisation (bigcn_layer_norm_backward):
//
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  g = gamma dy
//   dgamma = sum_i dy xhat,  dbeta = sum_i dy
//
// with xhat from the forward's input or from its 8-bit checkpoint. Bound by memory: dy and
// the source are read once and dx written once, by blocks that stay and take rows in turn;
// each keeps its rows' sums of dy xhat and dy in the registers that hold the columns, adds
// its threads' sums in shared memory at the end, and a second kernel adds the blocks' in
// order.
#include "norm.cuh"

namespace bigcn {
namespace {

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
    float v[1];
    dequantise<1>(uint8_t(a.q[i * a.ldq + k]), unpack_factor(a.exps[i * a.lde + k / kGroup]), v);
    return v[0];
}

// dX of rows that do not fit registers: a block per row, two walks.
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

// dgamma and dbeta of such rows: a block takes 32 columns of a chunk of rows, a lane
// per column and a warp per row in turn; the warps' sums are added in order.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) param_any_kernel(const BackwardArgs a) {
    __shared__ float part[2][(kRowThreads / 32)][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t k = int64_t(blockIdx.x) * 32 + lane;
    const int64_t r0 = a.N * blockIdx.y / a.chunks, r1 = a.N * (blockIdx.y + 1) / a.chunks;
    float sg = 0.0f, sb = 0.0f;
    if (k < a.K)
        for (int64_t i = r0 + warp; i < r1; i += (kRowThreads / 32)) {
            const float dy = to_f32(static_cast<const T *>(a.dY)[i * a.lddy + k]);
            sg = fmaf(dy, xhat_at<T>(a, i, int(k), a.X ? a.mean[i] : 0.0f, a.rstd[i]), sg);
            sb += dy;
        }
    part[0][warp][lane] = sg;
    part[1][warp][lane] = sb;
    __syncthreads();
    if (warp < 2 && k < a.K) {
        float t = 0.0f;
        for (int w = 0; w < (kRowThreads / 32); ++w) t += part[warp][w][lane];
        a.partial[(int64_t(blockIdx.y) * 2 + warp) * a.K + k] = t;
    }
}

// Rows in registers; a.chunks blocks, block b takes the sets of rows b, b + chunks, ...
// kWarp: a row is one warp's (tpr = 32, which makes every offset a constant), else tpr
// threads'.
template <typename T, int V, int J, bool kKept, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowThreads : kMostRowThreads, kWarp ? 2 : 1)
backward_rows_kernel(const BackwardArgs a, const int row_threads) {
    __shared__ float red[2][2][kMostRowThreads / 32];
    __shared__ float part[kMostRowThreads * V];
    constexpr int kFull = full_vectors(V, J);
    // xhat is kept in fp32 between the two uses where that takes no more registers than what
    // it was read as (a byte and its scale take two), else expanded twice.
    constexpr bool kHold = V <= 2 || (!kKept && sizeof(T) == 4);
    const int tpr = kWarp ? 32 : row_threads;
    const int t = threadIdx.x & (tpr - 1), rows = blockDim.x / tpr, slot = threadIdx.x / tpr;
    const int K = a.K, k0 = t * V, step = tpr * V, left = K - k0;
    const float inv_k = 1.0f / float(K);
    using Q = typename QWord<V>::type;
    float sg[J][V], sb[J][V];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) sg[j][e] = sb[j][e] = 0.0f;
    const float *gamma = a.gamma ? a.gamma + k0 : kOnes;
    const int gstep = a.gamma ? step : 0;
    int turn = 0;
    for (int64_t i0 = int64_t(blockIdx.x) * rows; i0 < a.N; i0 += int64_t(a.chunks) * rows) {
        const int64_t i = i0 + slot;
        const bool live = i < a.N;
        if (kWarp && !live) break;
        const int64_t at = live ? i : 0;
        const T *dy = static_cast<const T *>(a.dY) + at * a.lddy + k0;
        const T *x = static_cast<const T *>(a.X) + at * a.ldx + k0;
        const int8_t *q = a.q + at * a.ldq + k0;
        const uint8_t *exps = a.exps + at * a.lde;
        Vec<T, V> w[J];                 // dy as read
        Vec<T, V> xr[kKept ? 1 : J];
        Q qr[kKept ? J : 1];
        uint8_t er[kKept ? J : 1];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (j < kFull || j * step < left) {
                w[j] = *reinterpret_cast<const Vec<T, V> *>(dy + j * step);
                if constexpr (kKept) {
                    qr[j] = *reinterpret_cast<const Q *>(q + j * step);
                    er[j] = exps[unsigned(k0 + j * step) / kGroup];
                } else {
                    xr[j] = *reinterpret_cast<const Vec<T, V> *>(x + j * step);
                }
            }
        }
        const float rstd = a.rstd[at], mean = kKept ? 0.0f : a.mean[at];
        auto expand = [&](int j, float (&h)[V]) {
            if constexpr (kKept) {
                dequantise<V>(qr[j], unpack_factor(er[j]), h);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) h[e] = (to_f32(xr[j].v[e]) - mean) * rstd;
            }
        };
        float g[J][V];                  // gamma dy
        float h[kHold ? J : 1][V];
        float s[2] = {0.0f, 0.0f};
        if (kWarp || live) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                if (j < kFull || j * step < left) {
                    float (&hj)[V] = h[kHold ? j : 0];
                    expand(j, hj);
                    const Vec<float, V> m =
                        *reinterpret_cast<const Vec<float, V> *>(gamma + j * gstep);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float d = to_f32(w[j].v[e]);
                        sg[j][e] = fmaf(d, hj[e], sg[j][e]);
                        sb[j][e] += d;
                        g[j][e] = d * m.v[e];
                        s[0] += g[j][e];
                        s[1] = fmaf(g[j][e], hj[e], s[1]);
                    }
                }
            }
        }
        if (!a.dX) continue;
        // Two sets of sums in turn: a set is written again only after the next one's barrier.
        row_sum<kWarp>(s, tpr, red[turn]);
        turn ^= 1;
        if (!kWarp && !live) continue;
        const float c0 = s[0] * inv_k, c1 = s[1] * inv_k;
        T *dx = static_cast<T *>(a.dX) + at * a.lddx + k0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (j < kFull || j * step < left) {
                float (&hj)[V] = h[kHold ? j : 0];
                if (!kHold) expand(j, hj);
                Vec<T, V> o;
#pragma unroll
                for (int e = 0; e < V; ++e)
                    o.v[e] = from_f32<T>(rstd * (g[j][e] - c0 - hj[e] * c1));
                *reinterpret_cast<Vec<T, V> *>(dx + j * step) = o;
            }
        }
    }
    allow_dependent_launch();
    if (!a.partial) return;
    // The threads that hold the same columns, in order.
    float *out = a.partial + int64_t(blockIdx.x) * 2 * K;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (j * step >= K) break;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int k = k0 + j * step;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e)
                part[e * kMostRowThreads + threadIdx.x] = w == 0 ? sg[j][e] : sb[j][e];
            __syncthreads();
            if (slot == 0 && k < K)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float v = 0.0f;
                    for (int r = 0; r < rows; ++r) v += part[e * kMostRowThreads + r * tpr + t];
                    out[w * K + k + e] = v;
                }
        }
    }
}

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

constexpr int kMaxChunks = 1024;
constexpr size_t kAlign = 256;

template <typename T, int V, int J, bool kKept, bool kWarp>
void launch_kept(BackwardArgs &a, int tpr, const DeviceInfo &dev, cudaStream_t s) {
    const auto kernel = backward_rows_kernel<T, V, J, kKept, kWarp>;
    const int threads = tpr > kRowThreads ? tpr : kRowThreads, rows = threads / tpr;
    static const auto blocks_per_sm = [](int n) {
        int per = 1;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(
                &per, backward_rows_kernel<T, V, J, kKept, kWarp>, n, 0) != cudaSuccess)
            cudaGetLastError();
        return per > 1 ? per : 1;
    };
    static const int with[2] = {blocks_per_sm(kRowThreads), blocks_per_sm(kMostRowThreads)};
    const int per_sm = with[threads > kRowThreads];
    const int64_t sets = (a.N + rows - 1) / rows;
    int64_t blocks = int64_t(dev.sm_count) * per_sm;
    if (blocks > kMaxChunks) blocks = kMaxChunks;
    a.chunks = int(blocks < sets ? blocks : sets);
    kernel<<<unsigned(a.chunks), threads, 0, s>>>(a, tpr);
}

template <typename T, int V, int J>
void launch_rows(BackwardArgs &a, int tpr, const DeviceInfo &dev, cudaStream_t s) {
    if (tpr == 32) {
        if (a.X) launch_kept<T, V, J, false, true>(a, tpr, dev, s);
        else launch_kept<T, V, J, true, true>(a, tpr, dev, s);
    } else if constexpr (V * J <= 16) {
        if (a.X) launch_kept<T, V, J, false, false>(a, tpr, dev, s);
        else launch_kept<T, V, J, true, false>(a, tpr, dev, s);
    }
}

template <typename T, int V>
bool launch_width(BackwardArgs &a, const DeviceInfo &dev, cudaStream_t s) {
    const RowLayout r = row_layout(a.N, a.K, V, 8, 24, 16, dev);
    if (r.J == 1) launch_rows<T, V, 1>(a, r.tpr, dev, s);
    else if (r.J == 2) launch_rows<T, V, 2>(a, r.tpr, dev, s);
    else if (V <= 4 && r.J == 4) launch_rows<T, V, V <= 4 ? 4 : 1>(a, r.tpr, dev, s);
    else if (V <= 2 && r.J == 8) launch_rows<T, V, V <= 2 ? 8 : 1>(a, r.tpr, dev, s);
    else if (V == 2 && r.J == 12) launch_rows<T, V, V == 2 ? 12 : 1>(a, r.tpr, dev, s);
    else if (V == 1 && r.J == 16) launch_rows<T, V, V == 1 ? 16 : 1>(a, r.tpr, dev, s);
    else if (V == 1 && r.J == 24) launch_rows<T, V, V == 1 ? 24 : 1>(a, r.tpr, dev, s);
    else return false;
    return true;
}

template <typename T>
void launch_backward(BackwardArgs a, const DeviceInfo &dev, float *dgamma, float *dbeta,
                     cudaStream_t s) {
    const uint64_t es = sizeof(T), f = 4 / es;
    const uint64_t where[] = {uint64_t(uintptr_t(a.dY)),
                              uint64_t(a.lddy) * es,
                              uint64_t(a.K) * es,
                              uint64_t(uintptr_t(a.gamma)) / f,
                              uint64_t(uintptr_t(a.dX)),
                              a.dX ? uint64_t(a.lddx) * es : 0,
                              uint64_t(uintptr_t(a.X)),
                              a.X ? uint64_t(a.ldx) * es : 0};
    const int V = vector_width(es, where, 8);
    const bool done = V == 1   ? launch_width<T, 1>(a, dev, s)
                      : V == 2 ? launch_width<T, 2>(a, dev, s)
                      : V == 4 ? launch_width<T, 4>(a, dev, s)
                               : launch_width<T, es == 2 ? 8 : 4>(a, dev, s);
    if (!done) {
        const int64_t most = int64_t(dev.sm_count) * 64;
        if (a.dX)
            backward_any_kernel<T><<<unsigned(a.N < most ? a.N : most), kRowThreads, 0, s>>>(a);
        if (!a.partial) return;
        const int64_t strips = (int64_t(a.K) + 31) / 32;
        int64_t chunks = (int64_t(dev.sm_count) * 8 + strips - 1) / strips;
        if (chunks > kMaxChunks) chunks = kMaxChunks;
        const int64_t sets = (a.N + kRowThreads / 32 - 1) / (kRowThreads / 32);
        a.chunks = int(chunks < sets ? chunks : sets);
        param_any_kernel<T><<<dim3(unsigned(strips), unsigned(a.chunks)), kRowThreads, 0, s>>>(a);
    }
    if (!a.partial) return;
    launch_kernel(param_sum_kernel, dim3(unsigned((2 * int64_t(a.K) + 31) / 32)), dim3(kSumThreads),
                  0, s, true, dim3(1, 1, 1), a.partial, a.chunks, a.K, dgamma, dbeta);
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

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
