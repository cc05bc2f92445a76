// The kernels of layer norm's backward and their launch, by element type: a translation unit
// instantiates launch_backward for one.
#pragma once

#include "norm_args.cuh"
#include "norm.cuh"

namespace bigcn {
namespace {

template <typename T>
__device__ __forceinline__ float xhat_at(const BackwardArgs &a, int64_t i, int k, float mean,
                                         float rstd) {
    if (a.X) return (to_f32(static_cast<const T *>(a.X)[i * a.ldx + k]) - mean) * rstd;
    return float(a.q[i * a.ldq + k]) * unpack_factor(a.exps[i * a.lde + k / kGroup]);
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

// What a row's pieces are read as: dy, and x or the checkpoint's bytes.
template <int A, int J, int H, bool kKept> struct RawRow {
    Raw<A> dy[J];
    Raw<A> x[kKept ? 1 : J];
    QPiece<H> q[kKept ? J : 1];
    uint8_t b[kKept ? J : 1];
    float rstd, mean;
    bool dy_odd, x_odd;
};

// Rows in registers (norm.cuh); a.chunks blocks, block b takes the sets of rows b, b + chunks,
// ... and keeps their sums of dy xhat and dy in the registers that hold the columns. kWarp: a
// row is one warp's. kAhead: the next row is loaded before the present one is worked on, where
// the registers allow it (16 warps an SM wait on memory otherwise).
template <typename T, int A, int J, bool kKept, bool kWarp, bool kAhead>
__global__ void __launch_bounds__(kWarp ? kRowThreads : kMostRowThreads, kWarp ? 2 : 1)
backward_rows_kernel(const BackwardArgs a, const int row_threads, const bool aligned) {
    constexpr int V = kPiece<T>, H = V / 2, kFull = full_pieces(V, J);
    __shared__ float red[2][2][kMostRowThreads / 32];
    __shared__ float part[V][kMostRowThreads];
    const int tpr = kWarp ? 32 : row_threads;
    const int t = threadIdx.x & (tpr - 1), rows = blockDim.x / tpr, slot = threadIdx.x / tpr;
    const int K = a.K, k0 = t * V, step = tpr * V, left = K - k0;
    const float inv_k = 1.0f / float(K);
    float2 sg[J][H], sb[J][H];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < H; ++e) sg[j][e] = sb[j][e] = both(0.0f);
    const float *gamma = a.gamma ? a.gamma + k0 : kOnes;
    const int gstep = a.gamma ? step : 0;

    const bool together = kWarp || tpr >= 32;
    auto load = [&](int64_t i, RawRow<A, J, H, kKept> &r) {
        if (i >= a.N) return;
        const T *dy = static_cast<const T *>(a.dY) + i * a.lddy + k0;
        const bool dy_whole = whole_pieces<A>(dy, together);
        r.dy_odd = odd_pieces<A>(dy);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (j < kFull) r.dy[j] = load16<A>(dy + j * step, dy_whole, r.dy_odd);
            else if (left > j * step)
                r.dy[j] = load_piece<T, A>(dy + j * step, left - j * step, dy_whole, r.dy_odd);
        }
        if constexpr (kKept) {
            const int8_t *q = a.q + i * a.ldq + k0;
            const uint8_t *exps = a.exps + i * a.lde;
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j < kFull || left > j * step) {
                    r.q[j] = *reinterpret_cast<const QPiece<H> *>(q + j * step);
                    r.b[j] = exps[unsigned(k0 + j * step) / kGroup];
                }
        } else {
            const T *x = static_cast<const T *>(a.X) + i * a.ldx + k0;
            const bool x_whole = whole_pieces<A>(x, together);
            r.x_odd = odd_pieces<A>(x);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                if (j < kFull) r.x[j] = load16<A>(x + j * step, x_whole, r.x_odd);
                else if (left > j * step)
                    r.x[j] = load_piece<T, A>(x + j * step, left - j * step, x_whole, r.x_odd);
            }
            r.mean = a.mean[i];
        }
        r.rstd = a.rstd[i];
    };

    const int64_t stride = int64_t(a.chunks) * rows;
    int turn = 0;
    RawRow<A, J, H, kKept> next;
    if (kAhead) load(int64_t(blockIdx.x) * rows + slot, next);
    for (int64_t i0 = int64_t(blockIdx.x) * rows; i0 < a.N; i0 += stride) {
        const int64_t i = i0 + slot;
        const bool live = i < a.N;
        if (kWarp && !live) break;
        RawRow<A, J, H, kKept> r;
        if (kAhead) {
            r = next;
            load(i + stride, next);
        } else {
            load(i, r);
        }
        // dy, xhat and gamma of piece j, n of its columns in the row, from what was read. gamma dy and
        // xhat are kept from the sums to dx where the registers allow it (up to 16 columns a thread),
        // else expanded twice. (Behind the row dy and gamma are 0 and xhat anything finite, or NaN with
        // its row.)
        constexpr bool kHold = J * V <= 16;
        float2 gk[kHold ? J : 1][H], hk[kHold ? J : 1][H];
        const float rstd = r.rstd;
        auto take = [&](int j, int n, float2 (&d)[H], float2 (&h)[H], float2 (&m)[H]) {
            unpack16<T>(settled<A>(r.dy[j], r.dy_odd), d);
            if constexpr (kKept) {
                dequantise_piece<H>(r.q[j], unpack_factor(r.b[j]), h);
            } else {
                unpack16<T>(settled<A>(r.x[j], r.x_odd), h);
#pragma unroll
                for (int e = 0; e < H; ++e)
                    h[e] = __fmul2_rn(__fadd2_rn(h[e], both(-r.mean)), both(rstd));
            }
            load_params(gamma + j * gstep, aligned, n, m);
        };
        float2 s0 = both(0.0f), s1 = both(0.0f);
        if (kWarp || live) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int n = j < kFull ? V : left - j * step;
                if (n <= 0) continue;
                float2 d[H], h[H], m[H];
                take(j, n, d, h, m);
#pragma unroll
                for (int e = 0; e < H; ++e) {
                    sg[j][e] = __ffma2_rn(d[e], h[e], sg[j][e]);
                    sb[j][e] = __fadd2_rn(sb[j][e], d[e]);
                    const float2 g = __fmul2_rn(d[e], m[e]);
                    s0 = __fadd2_rn(s0, g);
                    s1 = __ffma2_rn(g, h[e], s1);
                    if constexpr (kHold) gk[j][e] = g, hk[j][e] = h[e];
                }
            }
        }
        if (!a.dX) continue;
        // Two sets of sums in turn: a set is written again only after the next one's barrier.
        float s[2] = {s0.x + s0.y, s1.x + s1.y};
        row_sum<kWarp>(s, tpr, red[turn]);
        turn ^= 1;
        if (!kWarp && !live) continue;
        const float2 c0 = both(-s[0] * inv_k), c1 = both(-s[1] * inv_k), rs = both(rstd);
        T *dx = static_cast<T *>(a.dX) + i * a.lddx + k0;
        const bool dx_whole = whole_pieces<A>(dx, together);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int n = j < kFull ? V : left - j * step;
            if (n <= 0) continue;
            float2 d[H], h[H], m[H];
            if constexpr (!kHold) take(j, n, d, h, m);
#pragma unroll
            for (int e = 0; e < H; ++e) {
                const float2 g = kHold ? gk[kHold ? j : 0][e] : __fmul2_rn(d[e], m[e]);
                const float2 xh = kHold ? hk[kHold ? j : 0][e] : h[e];
                d[e] = __fmul2_rn(__ffma2_rn(xh, c1, __fadd2_rn(g, c0)), rs);
            }
            store_piece<T, A>(dx + j * step, pack16<T>(d), n, dx_whole);
        }
    }
    allow_dependent_launch();
    if (!a.partial) return;
    // The sums of threads that hold the same columns, tpr apart, in order.
    float *out = a.partial + int64_t(blockIdx.x) * 2 * K;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (j * step >= K) break;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < H; ++e) {
                const float2 v = w == 0 ? sg[j][e] : sb[j][e];
                part[2 * e][threadIdx.x] = v.x;
                part[2 * e + 1][threadIdx.x] = v.y;
            }
            __syncthreads();
            // A thread per column of this piece: column e of the row's thread u.
            for (int c = threadIdx.x; c < tpr * V; c += blockDim.x) {
                const int u = c / V, e = c % V, k = j * step + c;
                if (k >= K) continue;
                float v = 0.0f;
                for (int q = 0; q < rows; ++q) v += part[e][q * tpr + u];
                out[int64_t(w) * K + k] = v;
            }
        }
    }
}

template <typename T, int A, int J, bool kKept, bool kWarp>
void launch_kept(BackwardArgs &a, int tpr, bool aligned, const DeviceInfo &dev, cudaStream_t s) {
    // A row ahead where its registers and the sums' leave room for two blocks.
    constexpr bool kAhead = J * kPiece<T> <= (sizeof(T) == 4 ? 12 : 16);
    const auto kernel = backward_rows_kernel<T, A, J, kKept, kWarp, kAhead>;
    const int threads = tpr > kRowThreads ? tpr : kRowThreads, rows = threads / tpr;
    static const auto blocks_per_sm = [](int n) {
        int per = 1;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(
                &per, backward_rows_kernel<T, A, J, kKept, kWarp, kAhead>, n, 0) != cudaSuccess)
            cudaGetLastError();
        return per > 1 ? per : 1;
    };
    static const int with[2] = {blocks_per_sm(kRowThreads), blocks_per_sm(kMostRowThreads)};
    const int64_t sets = (a.N + rows - 1) / rows;
    int64_t blocks = int64_t(dev.sm_count) * with[threads > kRowThreads];
    if (blocks > kMaxChunks) blocks = kMaxChunks;
    a.chunks = int(blocks < sets ? blocks : sets);
    kernel<<<unsigned(a.chunks), threads, 0, s>>>(a, tpr, aligned);
}

template <typename T, int A, int J>
void launch_rows(BackwardArgs &a, int tpr, bool aligned, const DeviceInfo &dev, cudaStream_t s) {
    if (tpr == 32) {
        if (a.X) launch_kept<T, A, J, false, true>(a, tpr, aligned, dev, s);
        else launch_kept<T, A, J, true, true>(a, tpr, aligned, dev, s);
    } else if constexpr (J * kPiece<T> <= 16) {
        if (a.X) launch_kept<T, A, J, false, false>(a, tpr, aligned, dev, s);
        else launch_kept<T, A, J, true, false>(a, tpr, aligned, dev, s);
    }
}

template <typename T, int A>
bool launch_aligned(BackwardArgs &a, bool aligned, const DeviceInfo &dev, cudaStream_t s) {
    constexpr bool kWide = sizeof(T) == 4;      // pieces of four columns
    const RowLayout r = row_layout(a.N, a.K, kPiece<T>, 16, kWide ? 24 : 16, dev);
    switch (r.J) {
    case 1: launch_rows<T, A, 1>(a, r.tpr, aligned, dev, s); return true;
    case 2: launch_rows<T, A, 2>(a, r.tpr, aligned, dev, s); return true;
    case 3: launch_rows<T, A, kWide ? 3 : 1>(a, r.tpr, aligned, dev, s); return true;
    case 4: launch_rows<T, A, kWide ? 4 : 1>(a, r.tpr, aligned, dev, s); return true;
    case 5: launch_rows<T, A, kWide ? 5 : 1>(a, r.tpr, aligned, dev, s); return true;
    case 6: launch_rows<T, A, kWide ? 6 : 1>(a, r.tpr, aligned, dev, s); return true;
    }
    return false;
}

}  // namespace

template <typename T>
void launch_backward(BackwardArgs &a, const DeviceInfo &dev, cudaStream_t s) {
    const uint64_t es = sizeof(T);
    const uint64_t where[] = {uint64_t(uintptr_t(a.dY)), uint64_t(a.lddy) * es,
                              uint64_t(uintptr_t(a.dX)), a.dX ? uint64_t(a.lddx) * es : 0,
                              uint64_t(uintptr_t(a.X)),  a.X ? uint64_t(a.ldx) * es : 0};
    const bool aligned = aligned_to(a.gamma, 32);
    const int A = alignment_of(where, 6);
    const bool done = A == 16  ? launch_aligned<T, 16>(a, aligned, dev, s)
                      : A == 8 ? launch_aligned<T, 8>(a, aligned, dev, s)
                      : A == 4 ? launch_aligned<T, 4>(a, aligned, dev, s)
                               : launch_aligned<T, es == 2 ? 2 : 4>(a, aligned, dev, s);
    if (done) return;
    const int64_t most = int64_t(dev.sm_count) * 64;
    if (a.dX) backward_any_kernel<T><<<unsigned(a.N < most ? a.N : most), kRowThreads, 0, s>>>(a);
    if (!a.partial) return;
    const int64_t strips = (int64_t(a.K) + 31) / 32;
    int64_t chunks = (int64_t(dev.sm_count) * 8 + strips - 1) / strips;
    if (chunks > kMaxChunks) chunks = kMaxChunks;
    const int64_t sets = (a.N + kRowThreads / 32 - 1) / (kRowThreads / 32);
    a.chunks = int(chunks < sets ? chunks : sets);
    param_any_kernel<T><<<dim3(unsigned(strips), unsigned(a.chunks)), kRowThreads, 0, s>>>(a);
}

}  // namespace bigcn
