// The residual's addition and the root-mean-square norm of the sum (bigcn_rms_norm_forward), with
// the 8-bit checkpoint of the normalised rows:
//
//   s = x + r (rounded to the rows' type),  rstd = 1 / sqrt(mean(s^2) + eps),  y = gamma s rstd
//
// Bound by memory: x and r are read once into registers, s, y and the checkpoint written once.
// What is normalised is the rounded sum, which the next layers and the backward pass read. Rows,
// pieces and their accesses are norm.cuh's. 232,965 x 602 fp32 with R, S and the checkpoint 347 us, 6.9 TB/s (a
// copy's rate); 2^20 x 256 bf16 349 us, 6.9 TB/s; 400,000 x 500 fp16 without it 244 us (6.5 TB/s), x 501, rows at odd
// halves, 398: five accesses a piece. Eight pieces a thread (fp32 rows of 769 to 1024 columns, aligned to 16 bytes)
// spill 28 to 60 bytes: 200,000 x 1000 505 us, 0.94 of a copy's rate, with the checkpoint 496.
#include <cmath>

#include "norm.cuh"

namespace bigcn {
namespace {

struct RmsForwardArgs {
    const void *X;
    int64_t N;
    int K;
    int64_t ldx;
    const void *R;           // nullable: s = x
    int64_t ldr;
    const float *gamma;
    float eps;
    void *S;                 // nullable; may be R or X
    int64_t lds;
    void *Y;                 // nullable
    int64_t ldy;
    float *rstd;
    int8_t *q;
    int64_t ldq;
    uint8_t *exps;
    int64_t lde;
};

// rstd from the sum of squares. Where that has left the range in which single squares keep fp32's
// precision, it is taken again of s 2^-96 or, where eps does not cover it, of s 2^110 (whose sum stays below
// 2^124, eps's share below 2^126): `again` is a factor's sum of squares. A row with a NaN or an infinity gets NaN.
constexpr float kDown = 0x1p-96f, kUp = 0x1p110f;
__device__ __forceinline__ float squares_factor(float ss, float eps) {
    return !(ss <= 0x1p100f) ? kDown : ss < 0x1p-96f && eps < 0x1p-94f ? kUp : 1.0f;
}
// `by`: shat is s by, or (s 2^110) by where the sum was taken of that, as rstd = 2^110 by may be infinite.
struct Rstd {
    float rstd, by;
    bool up;
};
template <typename Again>
__device__ __forceinline__ Rstd rstd_of(float ss, int K, float inv_k, float eps, Again again) {
    const float f = squares_factor(ss, eps);
    if (f != 1.0f) {
        ss = again(f);
        if (!(ss < __int_as_float(0x7F800000))) {
            const float nan = __int_as_float(0x7FC00000);
            return {nan, nan, false};
        }
    }
    const float root = sqrtf(fmaf(eps * f, f, ss * inv_k)), rstd = f / root;
    return {rstd, f == kUp ? 1.0f / root : rstd, f == kUp};
}

// A word of a row times 2^110.
template <typename T> __device__ __forceinline__ uint32_t word_up(uint32_t w) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(__uint_as_float(w) * kUp);
    const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&w), __float2bfloat162_rn(kUp));
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Rows that do not fit registers: a block per row, which walks it two or three times; the later
// walks find it in L1 or L2. A thread takes the same columns in each.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) rms_forward_any_kernel(const RmsForwardArgs a) {
    const int K = a.K, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kWarps = kRowThreads / 32;
    const float inv_k = 1.0f / float(K);
    const int groups = int(checkpoint_groups(K)), padded = (groups + 3) / 4 * 4;
    const int kq = (K + 15) / 16 * 16;
    for (int64_t i = blockIdx.x; i < a.N; i += gridDim.x) {
        const T *x = static_cast<const T *>(a.X) + i * a.ldx;
        const T *r = a.R ? static_cast<const T *>(a.R) + i * a.ldr : nullptr;
        T *sum = a.S ? static_cast<T *>(a.S) + i * a.lds : nullptr;
        auto fresh = [&](int k) { return r ? from_f32<T>(to_f32(x[k]) + to_f32(r[k])) : x[k]; };
        // (Once the sum is stored it is read there: it may have taken r's or x's place.)
        auto at = [&](int k) { return to_f32(sum ? sum[k] : fresh(k)); };
        float s[1];
        share_sums<false, false>(K, s, [&](int k, float (&run)[1]) {
            const T v = fresh(k);
            if (sum) sum[k] = v;
            run[0] = fmaf(to_f32(v), to_f32(v), run[0]);
        });
        block_sum(s);
        const Rstd r_of = rstd_of(s[0], K, inv_k, a.eps, [&](float f) {
            float again[1];
            share_sums<false, false>(K, again, [&](int k, float (&run)[1]) {
                const float v = at(k) * f;
                run[0] = fmaf(v, v, run[0]);
            });
            block_sum(again);
            return again[0];
        });
        if (threadIdx.x == 0 && a.rstd) a.rstd[i] = r_of.rstd;
        const float up = r_of.up ? kUp : 1.0f;
        for (int g = warp; g < groups; g += kWarps) {
            const int k = g * kGroup + lane;
            float v = 0.0f;
            if (k < K) {
                v = at(k) * up * r_of.by;
                if (a.Y)
                    static_cast<T *>(a.Y)[i * a.ldy + k] =
                        from_f32<T>(v * (a.gamma ? __ldg(a.gamma + k) : 1.0f));
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

// Rows in registers (norm.cuh). kWarp: a row is one warp's, else row_threads threads'. Rows past N
// take part in the sums over threads and store nothing.
template <typename T, int A, int J, bool kKeep, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowThreads : kMostRowThreads, kWarp ? 3 : 2)
rms_forward_kernel(const RmsForwardArgs a, const int row_threads, const bool aligned) {
    constexpr int V = kPiece<T>, H = V / 2, kFull = full_pieces(V, J);
    __shared__ float red0[1][kMostRowThreads / 32], red1[1][kMostRowThreads / 32];
    const int tpr = kWarp ? 32 : row_threads;
    const int t = threadIdx.x & (tpr - 1);
    const int64_t i = int64_t(blockIdx.x) * (blockDim.x / tpr) + threadIdx.x / tpr;
    const bool live = i < a.N;
    if (kWarp && !live) return;
    const int K = a.K, k0 = t * V, step = tpr * V, left = K - k0;
    const float inv_k = 1.0f / float(K);
    const bool together = kWarp || tpr >= 32;
    uint4 w[J];
    {
        auto load = [&](const void *p, int64_t ld, Raw<A> (&raw)[J]) {
            const T *row = static_cast<const T *>(p) + (live ? i : 0) * ld + k0;
            const bool whole = whole_pieces<A>(row, together), odd = odd_pieces<A>(row);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                raw[j] = raw_zero<A>();
                if (j < kFull) raw[j] = load16<A>(row + j * step, whole, odd);
                else if (left > j * step)
                    raw[j] = load_piece<T, A>(row + j * step, left - j * step, whole, odd);
            }
            return odd;
        };
        Raw<A> x[J], r[J];
        const bool x_odd = load(a.X, a.ldx, x);
        if (a.R) {
            const bool r_odd = load(a.R, a.ldr, r);
            T *sum = static_cast<T *>(a.S) + i * a.lds + k0;
            const bool whole = whole_pieces<A>(sum, together);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float2 u[H], v[H];
                unpack16<T>(settled<A>(x[j], x_odd), u);
                unpack16<T>(settled<A>(r[j], r_odd), v);
#pragma unroll
                for (int e = 0; e < H; ++e) u[e] = __fadd2_rn(u[e], v[e]);
                w[j] = pack16<T>(u);
                const int n = j < kFull ? V : left - j * step;
                if (a.S && n > 0 && live) store_piece<T, A>(sum + j * step, w[j], n, whole);
            }
        } else {
#pragma unroll
            for (int j = 0; j < J; ++j) w[j] = settled<A>(x[j], x_odd);
        }
    }
    auto squares = [&](float f, float (*red)[kMostRowThreads / 32]) {
        float2 s2 = both(0.0f);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            float2 x[H];
            unpack16<T>(w[j], x);
#pragma unroll
            for (int e = 0; e < H; ++e) {
                const float2 v = __fmul2_rn(x[e], both(f));
                s2 = __ffma2_rn(v, v, s2);
            }
        }
        float s[1] = {s2.x + s2.y};
        row_sum<kWarp>(s, tpr, red);
        return s[0];
    };
    // Whether a row's sum is taken again is decided by its warps alike, but rows of a block's other
    // warps, or of other lanes, may differ: where a row is not one warp's, all take the sum again where any must.
    const float ss = squares(1.0f, red0);
    Rstd r;
    if constexpr (kWarp) {
        r = rstd_of(ss, K, inv_k, a.eps, [&](float f) { return squares(f, red1); });
    } else {
        const float f = squares_factor(ss, a.eps);
        float again = ss;
        if (__syncthreads_or(live && f != 1.0f)) again = squares(f, red1);
        r = rstd_of(ss, K, inv_k, a.eps, [&](float) { return again; });
        if (!kKeep && !live) return;            // (with a checkpoint lanes still meet below)
    }
    if (live && t == 0 && a.rstd) a.rstd[i] = r.rstd;
    // (The sum has been stored; a power of two is exact on such rows. fp16 has no magnitude as small.)
    if constexpr (!std::is_same<T, __half>::value) {
        if (r.up) {
#pragma unroll
            for (int j = 0; j < J; ++j)
                w[j] = make_uint4(word_up<T>(w[j].x), word_up<T>(w[j].y), word_up<T>(w[j].z), word_up<T>(w[j].w));
        }
    }
    T *out = static_cast<T *>(a.Y) + i * a.ldy + k0;
    const bool y_whole = whole_pieces<A>(out, together);
    int8_t *q = a.q + i * a.ldq + k0;
    uint8_t *exps = a.exps + i * a.lde;
    const int kq = (K + 15) / 16 * 16 - k0;
    const float *gamma = a.gamma ? a.gamma + k0 : kOnes;
    const int gstep = a.gamma ? step : 0;
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
            unpack16<T>(w[j], x[u]);
#pragma unroll
            for (int e = 0; e < H; ++e) x[u][e] = __fmul2_rn(x[u][e], both(r.by));
            if (kKeep) {
                // (Behind the row a zero stays one, whatever rstd is.)
                if (j >= kFull && n < V) clear_from(x[u], n);
                own[u] = top_bits(x[u]);
            }
            if (a.Y && n > 0 && (kWarp || live)) {
                float2 g[H], y[H];
                load_params(gamma + j * gstep, aligned, n, g);
#pragma unroll
                for (int e = 0; e < H; ++e) y[e] = __fmul2_rn(x[u][e], g[e]);
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
void launch_rows(const RmsForwardArgs &a, int tpr, bool aligned, cudaStream_t s) {
    const int threads = tpr > kRowThreads ? tpr : kRowThreads, rows = threads / tpr;
    const unsigned grid = unsigned((a.N + rows - 1) / rows);
    if (tpr == 32) {
        if (a.q) rms_forward_kernel<T, A, J, true, true><<<grid, threads, 0, s>>>(a, tpr, aligned);
        else rms_forward_kernel<T, A, J, false, true><<<grid, threads, 0, s>>>(a, tpr, aligned);
    } else if constexpr (J <= 4) {
        if (a.q) rms_forward_kernel<T, A, J, true, false><<<grid, threads, 0, s>>>(a, tpr, aligned);
        else rms_forward_kernel<T, A, J, false, false><<<grid, threads, 0, s>>>(a, tpr, aligned);
    }
}

template <typename T, int A>
bool launch_aligned(const RmsForwardArgs &a, bool aligned, const DeviceInfo &dev, cudaStream_t s) {
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
void launch_forward(const RmsForwardArgs &a, const DeviceInfo &dev, cudaStream_t s) {
    const uint64_t es = sizeof(T);
    const uint64_t rows[] = {uint64_t(uintptr_t(a.X)), uint64_t(a.ldx) * es,
                             uint64_t(uintptr_t(a.Y)), a.Y ? uint64_t(a.ldy) * es : 0,
                             uint64_t(uintptr_t(a.R)), a.R ? uint64_t(a.ldr) * es : 0,
                             uint64_t(uintptr_t(a.S)), a.S ? uint64_t(a.lds) * es : 0};
    const bool aligned = aligned_to(a.gamma, 32);
    const int A = alignment_of(rows, 8);
    const bool done = A == 16  ? launch_aligned<T, 16>(a, aligned, dev, s)
                      : A == 8 ? launch_aligned<T, 8>(a, aligned, dev, s)
                      : A == 4 ? launch_aligned<T, 4>(a, aligned, dev, s)
                               : launch_aligned<T, es == 2 ? 2 : 4>(a, aligned, dev, s);
    if (done) return;
    const int64_t most = int64_t(dev.sm_count) * 64;
    rms_forward_any_kernel<T><<<unsigned(a.N < most ? a.N : most), kRowThreads, 0, s>>>(a);
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" bigcn_status bigcn_rms_norm_forward(int32_t dtype, const void *X, int64_t N, int32_t K,
                                               int64_t ldx, const void *R, int64_t ldr,
                                               const float *gamma, float eps, void *S, int64_t lds,
                                               void *Y, int64_t ldy, float *rstd, int8_t *q,
                                               int64_t ldq, uint8_t *exps, int64_t lde,
                                               void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols || ldx < K ||
        (R && ldr < K) || (S && lds < K) || (Y && ldy < K) || !(eps >= 0.0f) ||
        !std::isfinite(eps) || (q == nullptr) != (exps == nullptr) || (S && !R))
        return BIGCN_ERR_INVALID_ARG;
    if (q && !checkpoint_strides_ok(N, K, ldq, lde)) return BIGCN_ERR_INVALID_ARG;
    if (N > 0 && (N > kMaxElems / ldx || (R && N > kMaxElems / ldr) || (S && N > kMaxElems / lds) ||
                  (Y && N > kMaxElems / ldy)))
        return BIGCN_ERR_INVALID_ARG;
    if (N == 0) return BIGCN_OK;
    if (!X || (!S && !Y && !rstd && !q)) return BIGCN_ERR_INVALID_ARG;
    if (!aligned_to(X, es) || !aligned_to(R, es) || !aligned_to(S, es) || !aligned_to(Y, es) ||
        !aligned_to(gamma, 4) || !aligned_to(rstd, 4) || (q && !checkpoint_aligned(q, exps)))
        return BIGCN_ERR_MISALIGNED;
    // S may take the place of R or of X, row for row.
    const bool on_r = S && S == R && lds == ldr, on_x = S && S == X && lds == ldx;
    const void *in[] = {X, R, gamma};
    const size_t inb[] = {span_bytes(N, K, ldx, es), R ? span_bytes(N, K, ldr, es) : 0,
                          size_t(K) * 4};
    const void *out[] = {S, Y, rstd, q, exps};
    const size_t outb[] = {S ? span_bytes(N, K, lds, es) : 0, Y ? span_bytes(N, K, ldy, es) : 0,
                           size_t(N) * 4, q ? checkpoint_q_span(N, K, ldq) : 0,
                           q ? checkpoint_exps_span(N, K, lde) : 0};
    for (int o = 0; o < 5; ++o) {
        for (int p = 0; p < 3; ++p) {
            if (o == 0 && ((p == 0 && on_x) || (p == 1 && on_r))) continue;
            if (overlaps(out[o], outb[o], in[p], inb[p])) return BIGCN_ERR_INVALID_ARG;
        }
        for (int p = o + 1; p < 5; ++p)
            if (overlaps(out[o], outb[o], out[p], outb[p])) return BIGCN_ERR_INVALID_ARG;
    }
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const RmsForwardArgs a{X,   N, K,   ldx,  R, ldr, gamma, eps, S,
                           lds, Y, ldy, rstd, q, ldq, exps,  lde};
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32) launch_forward<float>(a, dev, s);
    else if (dtype == BIGCN_BF16) launch_forward<__nv_bfloat16>(a, dev, s);
    else launch_forward<__half>(a, dev, s);
    return launch_status();
}
