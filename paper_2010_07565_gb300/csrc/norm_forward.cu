// Layer normalisation of rows (bigcn_layer_norm_forward), with the 8-bit checkpoint of the
// normalised rows:
//
//   xhat = (x - mean) rstd,  y = gamma xhat + beta
//
// Bound by memory: a row is read once into registers and written once, the checkpoint with
// it. 232,965 x 602 fp32 with the checkpoint: 203 us, 6.2 TB/s (0.92 of a copy's rate); 2^20 x 256
// bf16 with it: 232 us (0.86); 8191 x 8192 fp16: 61 us, 4.4 TB/s (L1 at 73 % while a block is on an
// SM, which reads gamma and beta for every row).
// The mean and the variance are those of d = x - m0 over the row in registers, m0 = sum x / K
// (never E[x^2] - mean^2, which cancels where a row's level is above its spread). m0 itself is off by
// some ulps, of the sum and of 1 / K, and an ulp of 1000 is 0.02 of xhat in a constant row (eps =
// 1e-5): with the mean of d added, the mean is off by its rounding to fp32 alone, and that of a
// constant row is its value.
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

// The row's mean and variance from m0, S1 = sum d and S2 = sum d^2: m0 + S1 / K and S2 / K - (S1 / K)^2.
// The difference cancels only where the spread is below m0's own error, some ulps of the row's
// level. In a constant row it is what the rounding of the sums leaves, at most 3 (K / 32 + 40) u of
// S2 (u = 2^-24; rows of 16384 columns: 2^-13.2; the threads of longer ones add K / 256 terms, 256 at a
// time): taken for 0. (A NaN stays one.)
__device__ __forceinline__ void finish_moments(float (&s)[2], int K, float inv_k, float &mean,
                                               float &variance) {
    const float c = s[0] * inv_k, left = fmaf(-s[0], c, s[1]);
    mean += c;
    variance = left < s[1] * fmaf(float(min(K, kRowThreads * kRun)), 0x1p-29f, 0x1p-13f) ? 0.0f : left * inv_k;
}

// Rows that do not fit registers (more than 8192 fp32 or 16384 16-bit columns): a block per
// row, which walks it three times; the later walks find it in L1 or L2.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) forward_any_kernel(const ForwardArgs a) {
    const int K = a.K, lane = threadIdx.x & 31;
    const float inv_k = 1.0f / float(K);
    const int groups = int(checkpoint_groups(K)), padded = (groups + 3) / 4 * 4;
    const int kq = (K + 15) / 16 * 16;
    for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
        const T *x = static_cast<const T *>(a.X) + i * a.ldx;
        T *y = static_cast<T *>(a.Y) + i * a.ldy;
        float s0[1], s[2], variance;
        share_sums<false, false>(K, s0, [&](int k, float (&run)[1]) { run[0] += to_f32(x[k]); });
        block_sum(s0);
        float mean = s0[0] * inv_k;
        share_sums<false, false>(K, s, [&](int k, float (&run)[2]) {
            const float d = to_f32(x[k]) - mean;
            run[0] += d;
            run[1] = fmaf(d, d, run[1]);
        });
        block_sum(s);
        finish_moments(s, K, inv_k, mean, variance);
        const float rstd = 1.0f / sqrtf(variance + a.eps);
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
                if (k < kq) a.q[i * a.ldq + k] = int8_t(b == kNanByte ? 0u : q_low(v, pack_factor(b)));
                if (lane == 0) a.exps[i * a.lde + g] = uint8_t(b);
                if (g == groups - 1 && g + 1 + lane < padded) a.exps[i * a.lde + g + 1 + lane] = 0;
            }
        }
    }
}

// Rows in registers (norm.cuh). kWarp: a row is one warp's (tpr = 32, which makes every offset a
// constant), else tpr threads'. Rows past N take part in the sums over threads and store
// nothing.
template <typename T, int A, int J, bool kKeep, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowThreads : kMostRowThreads, kWarp ? 4 : 2)
forward_rows_kernel(const ForwardArgs a, const int row_threads, const bool aligned) {
    constexpr int V = kPiece<T>, H = V / 2, kFull = full_pieces(V, J);
    __shared__ float red0[1][kMostRowThreads / 32], red[2][kMostRowThreads / 32];
    const int tpr = kWarp ? 32 : row_threads;
    const int t = threadIdx.x & (tpr - 1);
    const int64_t i = int64_t(blockIdx.x) * (blockDim.x / tpr) + threadIdx.x / tpr;
    const bool live = i < a.N;
    if (kWarp && !live) return;
    // Piece j holds columns k0 + j step ..; left - j step of them are in the row, all V where
    // j < kFull.
    const int K = a.K, k0 = t * V, step = tpr * V, left = K - k0;
    const float inv_k = 1.0f / float(K);
    const T *row = static_cast<const T *>(a.X) + (live ? i : 0) * a.ldx + k0;
    // The row as it was read: 16-bit elements take half the registers that way, so that all
    // loads are under way at once, and are expanded for each use.
    uint4 w[J];
    Raw<A> raw[J];
    const bool together = kWarp || tpr >= 32;
    const bool x_whole = whole_pieces<A>(row, together), x_odd = odd_pieces<A>(row);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        raw[j] = raw_zero<A>();
        if (j < kFull) raw[j] = load16<A>(row + j * step, x_whole, x_odd);
        else if (left > j * step)
            raw[j] = load_piece<T, A>(row + j * step, left - j * step, x_whole, x_odd);
    }
#pragma unroll
    for (int j = 0; j < J; ++j) w[j] = settled<A>(raw[j], x_odd);
    float2 s2 = both(0.0f);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        float2 x[H];
        unpack16<T>(w[j], x);
#pragma unroll
        for (int e = 0; e < H; ++e) s2 = __fadd2_rn(s2, x[e]);
    }
    float s0[1] = {s2.x + s2.y}, variance;
    row_sum<kWarp>(s0, tpr, red0);
    float mean = s0[0] * inv_k;
    // x - mean of piece j, zeros past the row.
    auto centred = [&](int j, float2 (&x)[H]) {
        unpack16<T>(w[j], x);
#pragma unroll
        for (int e = 0; e < H; ++e) x[e] = __fadd2_rn(x[e], both(-mean));
        if (j >= kFull && left < j * step + V) clear_from(x, left - j * step);
    };
    float2 s1 = both(0.0f);
    s2 = both(0.0f);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        float2 x[H];
        centred(j, x);
#pragma unroll
        for (int e = 0; e < H; ++e) {
            s1 = __fadd2_rn(s1, x[e]);
            s2 = __ffma2_rn(x[e], x[e], s2);
        }
    }
    float s[2] = {s1.x + s1.y, s2.x + s2.y};
    row_sum<kWarp>(s, tpr, red);
    finish_moments(s, K, inv_k, mean, variance);
    if (!kWarp && !kKeep && !live) return;      // (with a checkpoint lanes still meet below)
    const float rstd = 1.0f / sqrtf(variance + a.eps);
    if (live && t == 0) {
        if (a.mean) a.mean[i] = mean;
        if (a.rstd) a.rstd[i] = rstd;
    }
    T *out = static_cast<T *>(a.Y) + i * a.ldy + k0;
    const bool y_whole = whole_pieces<A>(out, together);
    int8_t *q = a.q + i * a.ldq + k0;
    uint8_t *exps = a.exps + i * a.lde;
    const int kq = (K + 15) / 16 * 16 - k0;
    const float *gamma = a.gamma ? a.gamma + k0 : kOnes, *beta = a.beta ? a.beta + k0 : kZeros;
    const int gstep = a.gamma ? step : 0, bstep = a.beta ? step : 0;
    // Two pieces at a time, whose groups' maxima share a word.
#pragma unroll
    for (int j0 = 0; j0 < J; j0 += 2) {
        constexpr int kPair = J == 1 ? 1 : 2;
        float2 x[kPair][H];
        uint32_t own[kPair], top[kPair];
#pragma unroll
        for (int u = 0; u < kPair; ++u) {
            own[u] = 0u;
            if (j0 + u >= J) continue;
            const int j = j0 + u, n = j < kFull ? V : left - j * step;
            centred(j, x[u]);
#pragma unroll
            for (int e = 0; e < H; ++e) x[u][e] = __fmul2_rn(x[u][e], both(rstd));
            if (kKeep) own[u] = top_bits(x[u]);
            if (n > 0 && (kWarp || live)) {
                float2 g[H], b[H], y[H];
                load_params(gamma + j * gstep, aligned, n, g);
                load_params(beta + j * bstep, aligned, n, b);
#pragma unroll
                for (int e = 0; e < H; ++e) y[e] = __ffma2_rn(x[u][e], g[e], b[e]);
                store_piece<T, A>(out + j * step, pack16<T>(y), n, y_whole);
            }
        }
        if constexpr (kKeep) {
            group_tops<32 / V>(own, top);
#pragma unroll
            for (int u = 0; u < kPair; ++u) {
                const int j = j0 + u;
                if (j >= J || (!kWarp && !live) || (j >= kFull && j * step >= kq)) continue;
                const uint32_t b = scale_byte(top[u]);
                *reinterpret_cast<QPiece<H> *>(q + j * step) = quantise_piece(x[u], b);
                if ((t & (32 / V - 1)) == 0 && j * step < left)
                    exps[unsigned(k0 + j * step) / kGroup] = uint8_t(b);
            }
        }
    }
    if constexpr (kKeep) {
        const int groups = int(checkpoint_groups(K));
        if (live && groups + t < (groups + 3) / 4 * 4) exps[groups + t] = 0;
    }
}

template <typename T, int A, int J>
void launch_rows(const ForwardArgs &a, int tpr, bool aligned, cudaStream_t s) {
    const int threads = tpr > kRowThreads ? tpr : kRowThreads, rows = threads / tpr;
    const unsigned grid = unsigned((a.N + rows - 1) / rows);
    if (tpr == 32) {
        if (a.q) forward_rows_kernel<T, A, J, true, true><<<grid, threads, 0, s>>>(a, tpr, aligned);
        else forward_rows_kernel<T, A, J, false, true><<<grid, threads, 0, s>>>(a, tpr, aligned);
    } else if constexpr (J <= 4) {
        if (a.q) forward_rows_kernel<T, A, J, true, false><<<grid, threads, 0, s>>>(a, tpr, aligned);
        else forward_rows_kernel<T, A, J, false, false><<<grid, threads, 0, s>>>(a, tpr, aligned);
    }
}

template <typename T, int A>
bool launch_aligned(const ForwardArgs &a, bool aligned, const DeviceInfo &dev, cudaStream_t s) {
    constexpr bool kWide = sizeof(T) == 4;      // pieces of four columns: up to eight of them
    const RowLayout r = row_layout(a.N, a.K, kPiece<T>, kWide ? 16 : 32, 32, dev);
    switch (r.J) {
    case 1: launch_rows<T, A, 1>(a, r.tpr, aligned, s); return true;
    case 2: launch_rows<T, A, 2>(a, r.tpr, aligned, s); return true;
    case 3: launch_rows<T, A, 3>(a, r.tpr, aligned, s); return true;
    case 4: launch_rows<T, A, 4>(a, r.tpr, aligned, s); return true;
    case 5: launch_rows<T, A, kWide ? 5 : 1>(a, r.tpr, aligned, s); return true;
    case 6: launch_rows<T, A, kWide ? 6 : 1>(a, r.tpr, aligned, s); return true;
    case 8: launch_rows<T, A, kWide ? 8 : 1>(a, r.tpr, aligned, s); return true;
    }
    return false;
}

template <typename T>
void launch_forward(const ForwardArgs &a, const DeviceInfo &dev, cudaStream_t s) {
    const uint64_t es = sizeof(T);
    const uint64_t rows[] = {uint64_t(uintptr_t(a.X)), uint64_t(a.ldx) * es, uint64_t(uintptr_t(a.Y)),
                             uint64_t(a.ldy) * es};
    const bool aligned = aligned_to(a.gamma, 32) && aligned_to(a.beta, 32);
    const int A = alignment_of(rows, 4);
    const bool done = A == 16  ? launch_aligned<T, 16>(a, aligned, dev, s)
                      : A == 8 ? launch_aligned<T, 8>(a, aligned, dev, s)
                      : A == 4 ? launch_aligned<T, 4>(a, aligned, dev, s)
                               : launch_aligned<T, es == 2 ? 2 : 4>(a, aligned, dev, s);
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
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols || ldx < K ||
        ldy < K || !(eps >= 0.0f) || !std::isfinite(eps) || (q == nullptr) != (exps == nullptr))
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
