// Layer normalisation of rows (bigcn_layer_norm_forward), with the 8-bit checkpoint of the
// normalised rows:
//
//   xhat = (x - mean) rstd,  y = gamma xhat + beta
//
// Bound by memory: a row is read once into registers and written once, the checkpoint with
// it. The variance is the mean square of x - mean over the row in registers (never
// E[x^2] - mean^2, which cancels where a row's level is above its spread).
#include <cmath>

#include "norm.cuh"

namespace bigcn {
namespace {

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

// Rows that do not fit registers (more than 8192 columns): a block per row, which walks it
// three times; the later walks find it in L1 or L2.
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
        for (int g = threadIdx.x >> 5; g < groups; g += (kRowThreads / 32)) {
            const int k = g * kGroup + lane;
            float v = 0.0f;
            if (k < K) {
                v = (to_f32(x[k]) - mean) * rstd;
                y[k] = from_f32<T>(fmaf(v, a.gamma ? __ldg(a.gamma + k) : 1.0f,
                                        a.beta ? __ldg(a.beta + k) : 0.0f));
            }
            if (a.q) {
                const uint32_t b = scale_byte(__reduce_max_sync(kFullMask, abs_bits(v)));
                if (k < kq) a.q[i * a.ldq + k] = int8_t(q_low(v, pack_factor(b)));
                if (lane == 0) a.exps[i * a.lde + g] = uint8_t(b);
                if (g == groups - 1 && g + 1 + lane < padded) a.exps[i * a.lde + g + 1 + lane] = 0;
            }
        }
    }
}

// Rows in registers. kWarp: a row is one warp's (tpr = 32, which makes every offset a constant),
// else tpr threads'. Rows past N take part in the sums over threads and store nothing.
template <typename T, int V, int J, bool kKeep, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowThreads : kMostRowThreads, kWarp ? 4 : 2)
forward_rows_kernel(const ForwardArgs a, const int row_threads) {
    __shared__ float red[2][1][kMostRowThreads / 32];
    const int tpr = kWarp ? 32 : row_threads;
    const int t = threadIdx.x & (tpr - 1);
    const int64_t i = int64_t(blockIdx.x) * (blockDim.x / tpr) + threadIdx.x / tpr;
    const bool live = i < a.N;
    if (kWarp && !live) return;
    // Columns k0 + j step; those of this thread from `left` on are past the row. The first
    // kFull vectors are within it.
    constexpr int kFull = full_vectors(V, J);
    const int K = a.K, k0 = t * V, step = tpr * V, left = K - k0;
    const float inv_k = 1.0f / float(K);
    // The row as it was read: 16-bit elements take half the registers that way, and are
    // converted where they are used.
    Vec<T, V> x[J];
    const T *row = static_cast<const T *>(a.X) + (live ? i : 0) * a.ldx + k0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (j < kFull || j * step < left) x[j] = *reinterpret_cast<const Vec<T, V> *>(row + j * step);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) x[j].v[e] = from_f32<T>(0.0f);
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) s[0] += to_f32(x[j].v[e]);
    row_sum<kWarp>(s, tpr, red[0]);
    const float mean = s[0] * inv_k;
    s[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (j < kFull || j * step < left)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = to_f32(x[j].v[e]) - mean;
                s[0] = fmaf(d, d, s[0]);
            }
    row_sum<kWarp>(s, tpr, red[1]);
    if (!kWarp && !kKeep && !live) return;      // (with a checkpoint lanes still meet below)
    const float rstd = 1.0f / sqrtf(s[0] * inv_k + a.eps);
    if (live && t == 0) {
        if (a.mean) a.mean[i] = mean;
        if (a.rstd) a.rstd[i] = rstd;
    }
    T *out = static_cast<T *>(a.Y) + i * a.ldy + k0;
    using Q = typename QWord<V>::type;
    int8_t *qrow = a.q + i * a.ldq;
    uint8_t *erow = a.exps + i * a.lde;
    const float *gamma = a.gamma ? a.gamma + k0 : kOnes, *beta = a.beta ? a.beta + k0 : kZeros;
    const int gstep = a.gamma ? step : 0, bstep = a.beta ? step : 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (j >= kFull && j * step >= K) break;     // the same for the whole row's threads
        const bool in = (kWarp || live) && (j < kFull || j * step < left);
        uint32_t top = 0;
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            v[e] = (to_f32(x[j].v[e]) - mean) * rstd;
            if (kKeep) top = max(top, abs_bits(v[e]));
        }
        if (kKeep && j >= kFull) top = in ? top : 0u;
        if (in) {
            const Vec<float, V> g = *reinterpret_cast<const Vec<float, V> *>(gamma + j * gstep);
            const Vec<float, V> b = *reinterpret_cast<const Vec<float, V> *>(beta + j * bstep);
            Vec<T, V> w;
#pragma unroll
            for (int e = 0; e < V; ++e) w.v[e] = from_f32<T>(fmaf(v[e], g.v[e], b.v[e]));
            *reinterpret_cast<Vec<T, V> *>(out + j * step) = w;
        }
        if constexpr (kKeep) {
            const uint32_t b = group_byte<V, kWarp>(top, tpr);
            if (in) {
                *reinterpret_cast<Q *>(qrow + k0 + j * step) = quantise<V>(v, pack_factor(b));
                // A warp's step is a whole number of groups.
                if (kWarp ? (k0 & (kGroup - 1)) == 0 : ((k0 + j * step) & (kGroup - 1)) == 0)
                    erow[unsigned(k0 + j * step) / kGroup] = uint8_t(b);
            }
        }
    }
    if constexpr (kKeep)
        if (live) {
            const int groups = int(checkpoint_groups(K));
            for (int k = K + t; k < (K + 15) / 16 * 16; k += tpr) qrow[k] = 0;
            for (int g = groups + t; g < (groups + 3) / 4 * 4; g += tpr) erow[g] = 0;
        }
}

template <typename T, int V, int J, bool kWarp>
void launch_kind(const ForwardArgs &a, int tpr, cudaStream_t s) {
    const int threads = tpr > kRowThreads ? tpr : kRowThreads, rows = threads / tpr;
    const unsigned grid = unsigned((a.N + rows - 1) / rows);
    if (a.q) forward_rows_kernel<T, V, J, true, kWarp><<<grid, threads, 0, s>>>(a, tpr);
    else forward_rows_kernel<T, V, J, false, kWarp><<<grid, threads, 0, s>>>(a, tpr);
}

template <typename T, int V, int J>
void launch_rows(const ForwardArgs &a, int tpr, cudaStream_t s) {
    if (tpr == 32) launch_kind<T, V, J, true>(a, tpr, s);
    else if constexpr (V * J <= 16 || V == 8) launch_kind<T, V, J, false>(a, tpr, s);
}

template <typename T, int V>
bool launch_width(const ForwardArgs &a, const DeviceInfo &dev, cudaStream_t s) {
    const RowLayout r = row_layout(a.N, a.K, V, a.q ? 32 / V : 8, 32, V == 8 ? 32 : 16, dev);
    if (r.J == 1) launch_rows<T, V, 1>(a, r.tpr, s);
    else if (r.J == 2) launch_rows<T, V, 2>(a, r.tpr, s);
    else if (r.J == 4) launch_rows<T, V, 4>(a, r.tpr, s);
    else if (V <= 4 && r.J == 8) launch_rows<T, V, V <= 4 ? 8 : 1>(a, r.tpr, s);
    else if (V == 2 && r.J == 12) launch_rows<T, V, V == 2 ? 12 : 1>(a, r.tpr, s);
    else if (V == 1 && r.J == 16) launch_rows<T, V, V == 1 ? 16 : 1>(a, r.tpr, s);
    else if (V == 1 && r.J == 24) launch_rows<T, V, V == 1 ? 24 : 1>(a, r.tpr, s);
    else return false;
    return true;
}

template <typename T>
void launch_forward(const ForwardArgs &a, const DeviceInfo &dev, cudaStream_t s) {
    // Vectors of x and y; those of gamma and beta are fp32, q's are V bytes of 16-byte rows.
    const uint64_t es = sizeof(T), f = 4 / es;
    const uint64_t where[] = {uint64_t(uintptr_t(a.X)),
                              uint64_t(uintptr_t(a.Y)),
                              uint64_t(a.ldx) * es,
                              uint64_t(a.ldy) * es,
                              uint64_t(a.K) * es,
                              uint64_t(uintptr_t(a.gamma)) / f,
                              uint64_t(uintptr_t(a.beta)) / f};
    const int V = vector_width(es, where, 7);
    const bool done = V == 1   ? launch_width<T, 1>(a, dev, s)
                      : V == 2 ? launch_width<T, 2>(a, dev, s)
                      : V == 4 ? launch_width<T, 4>(a, dev, s)
                               : launch_width<T, es == 2 ? 8 : 4>(a, dev, s);
    if (done) return;
    const int64_t most = int64_t(dev.sm_count) * 64;
    forward_any_kernel<T><<<unsigned(a.N < most ? a.N : most), kRowThreads, 0, s>>>(a);
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
