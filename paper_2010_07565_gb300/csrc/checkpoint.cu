// Activations to 8 bits and back (bigcn_checkpoint_pack, bigcn_checkpoint_unpack).
#include "norm.cuh"

namespace bigcn {
namespace {

constexpr int kCkThreads = 256;

// Both directions lay a row over `tpr` threads (a power of two, 4 to 256) in vectors of V
// elements, as layer norm does (norm.cuh): a group of 32 columns lies in 32 / V
// neighbouring lanes (or in the row's, where it is shorter). A thread takes four vectors, J of a
// row by R rows, all loaded before the first is used; a row longer than tpr J V columns
// goes over several blocks. Bound by memory.
template <int V, int J, int R>
struct Place {
    int64_t i[R];            // rows
    int k0;                  // column of vector 0
    int step;                // columns from one vector to the next
    __device__ __forceinline__ Place(int tpr, unsigned pieces) {
        const int t = threadIdx.x & (tpr - 1), rows = kCkThreads / tpr;
        const int64_t set = blockIdx.x / pieces, piece = blockIdx.x % pieces;
#pragma unroll
        for (int r = 0; r < R; ++r) i[r] = (set * R + r) * rows + threadIdx.x / tpr;
        step = tpr * V;
        k0 = int(piece) * step * J + t * V;
    }
};

template <typename T, int V, int J, int R, bool kWhole>
__global__ void __launch_bounds__(kCkThreads)
pack_kernel(const T *__restrict__ X, int64_t N, int K, int64_t ldx, int8_t *__restrict__ q,
            int64_t ldq, uint8_t *__restrict__ exps, int64_t lde, int tpr, unsigned pieces) {
    const Place<V, J, R> at(tpr, pieces);
    Vec<T, V> x[R][J];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int k = at.k0 + j * at.step;
            if (at.i[r] < N && k < K)
                x[r][j] = *reinterpret_cast<const Vec<T, V> *>(X + at.i[r] * ldx + k);
            else
#pragma unroll
                for (int e = 0; e < V; ++e) x[r][j].v[e] = from_f32<T>(0.0f);
        }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int k = at.k0 + j * at.step;
            const bool in = at.i[r] < N && k < K;
            uint32_t top = 0;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[e] = to_f32(x[r][j].v[e]);
                top = max(top, abs_bits(v[e]));
            }
            const uint32_t b = group_byte<V, kWhole>(in ? top : 0u, tpr);
            if (in) {
                *reinterpret_cast<typename QWord<V>::type *>(q + at.i[r] * ldq + k) =
                    quantise<V>(v, pack_factor(b));
                if (k % kGroup == 0) exps[at.i[r] * lde + k / kGroup] = uint8_t(b);
            }
        }
    // The padding of the rows that end in this block's columns.
    const int t = threadIdx.x & (tpr - 1), groups = int(checkpoint_groups(K));
    if (int64_t(blockIdx.x % pieces) + 1 == pieces)
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (at.i[r] < N) {
                for (int k = K + t; k < (K + 15) / 16 * 16; k += tpr) q[at.i[r] * ldq + k] = 0;
                for (int g = groups + t; g < (groups + 3) / 4 * 4; g += tpr)
                    exps[at.i[r] * lde + g] = 0;
            }
}

template <typename T, int V, int J, int R>
__global__ void __launch_bounds__(kCkThreads)
unpack_kernel(const int8_t *__restrict__ q, int64_t ldq, const uint8_t *__restrict__ exps,
              int64_t lde, int64_t N, int K, const float *__restrict__ gamma,
              const float *__restrict__ beta, T *__restrict__ X, int64_t ldx, int tpr,
              unsigned pieces) {
    const Place<V, J, R> at(tpr, pieces);
    using Q = typename QWord<V>::type;
    Q w[R][J];
    uint8_t b[R][J];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int k = at.k0 + j * at.step;
            if (at.i[r] < N && k < K) {
                w[r][j] = *reinterpret_cast<const Q *>(q + at.i[r] * ldq + k);
                b[r][j] = exps[at.i[r] * lde + k / kGroup];
            }
        }
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int k = at.k0 + j * at.step;
        if (k >= K) continue;
        Vec<float, V> g, c;
        if (gamma) g = *reinterpret_cast<const Vec<float, V> *>(gamma + k);
        if (beta) c = *reinterpret_cast<const Vec<float, V> *>(beta + k);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (at.i[r] >= N) continue;
            Vec<T, V> x;
            float v[V];
            dequantise<V>(w[r][j], unpack_factor(b[r][j]), v);
#pragma unroll
            for (int e = 0; e < V; ++e)
                x.v[e] = from_f32<T>(gamma || beta
                                         ? fmaf(gamma ? g.v[e] : 1.0f, v[e], beta ? c.v[e] : 0.0f)
                                         : v[e]);
            *reinterpret_cast<Vec<T, V> *>(X + at.i[r] * ldx + k) = x;
        }
    }
}

// Threads of a row and the call's grid: the fewest threads (a warp, or fewer for short rows)
// that hold a row in at most four vectors, else all 256 and several blocks.
struct CkGrid {
    int tpr, J;
    unsigned pieces, blocks;
};
inline CkGrid ck_grid(int64_t N, int K, int V) {
    const int64_t vecs = (int64_t(K) + V - 1) / V;
    CkGrid g;
    g.tpr = 4;
    while (g.tpr < 32 && g.tpr < vecs) g.tpr *= 2;
    while (g.tpr < kCkThreads && int64_t(g.tpr) * 4 < vecs) g.tpr *= 2;
    g.J = vecs <= g.tpr ? 1 : vecs <= 2 * g.tpr ? 2 : 4;
    const int64_t pieces = (vecs + int64_t(g.tpr) * g.J - 1) / (int64_t(g.tpr) * g.J);
    const int64_t rows = kCkThreads / g.tpr * (4 / g.J);
    g.pieces = unsigned(pieces);
    g.blocks = unsigned((N + rows - 1) / rows * pieces);
    return g;
}

template <typename T>
struct PackArgs {
    T *X;                    // read by the packing, written by the unpacking
    int64_t N;
    int K;
    int64_t ldx;
    int8_t *q;
    int64_t ldq;
    uint8_t *exps;
    int64_t lde;
    const float *gamma;
    const float *beta;
};

template <typename T, int V, int J>
void launch_vectors(const PackArgs<T> &a, bool pack, const CkGrid &g, cudaStream_t s) {
    if (pack && g.tpr >= 32)
        pack_kernel<T, V, J, 4 / J, true><<<g.blocks, kCkThreads, 0, s>>>(
            a.X, a.N, a.K, a.ldx, a.q, a.ldq, a.exps, a.lde, g.tpr, g.pieces);
    else if (pack)
        pack_kernel<T, V, J, 4 / J, false><<<g.blocks, kCkThreads, 0, s>>>(
            a.X, a.N, a.K, a.ldx, a.q, a.ldq, a.exps, a.lde, g.tpr, g.pieces);
    else
        unpack_kernel<T, V, J, 4 / J><<<g.blocks, kCkThreads, 0, s>>>(
            a.q, a.ldq, a.exps, a.lde, a.N, a.K, a.gamma, a.beta, a.X, a.ldx, g.tpr, g.pieces);
}

template <typename T, int V>
void launch_width(const PackArgs<T> &a, bool pack, cudaStream_t s) {
    const CkGrid g = ck_grid(a.N, a.K, V);
    if (g.J == 1) launch_vectors<T, V, 1>(a, pack, g, s);
    else if (g.J == 2) launch_vectors<T, V, 2>(a, pack, g, s);
    else launch_vectors<T, V, 4>(a, pack, g, s);
}

template <typename T>
void launch_type(const PackArgs<T> &a, bool pack, cudaStream_t s) {
    const uint64_t es = sizeof(T), f = 4 / es;
    const uint64_t where[] = {uint64_t(uintptr_t(a.X)), uint64_t(a.ldx) * es, uint64_t(a.K) * es,
                              uint64_t(uintptr_t(a.gamma)) / f, uint64_t(uintptr_t(a.beta)) / f};
    const int V = vector_width(es, where, 5);
    if (V == 1) launch_width<T, 1>(a, pack, s);
    else if (V == 2) launch_width<T, 2>(a, pack, s);
    else if (V == 4) launch_width<T, 4>(a, pack, s);
    else launch_width<T, es == 2 ? 8 : 4>(a, pack, s);
}

void launch_checkpoint(int32_t dtype, void *X, int64_t N, int K, int64_t ldx, int8_t *q,
                       int64_t ldq, uint8_t *exps, int64_t lde, const float *gamma,
                       const float *beta, bool pack, cudaStream_t s) {
    if (dtype == BIGCN_F32)
        launch_type(PackArgs<float>{static_cast<float *>(X), N, K, ldx, q, ldq, exps, lde, gamma,
                                    beta}, pack, s);
    else if (dtype == BIGCN_BF16)
        launch_type(PackArgs<__nv_bfloat16>{static_cast<__nv_bfloat16 *>(X), N, K, ldx, q, ldq, exps,
                                            lde, gamma, beta}, pack, s);
    else
        launch_type(PackArgs<__half>{static_cast<__half *>(X), N, K, ldx, q, ldq, exps, lde, gamma,
                                     beta}, pack, s);
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
    launch_checkpoint(dtype, const_cast<void *>(X), N, K, ldx, q, ldq, exps, lde, nullptr, nullptr,
                      true, as_stream(stream));
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
    launch_checkpoint(dtype, X, N, K, ldx, const_cast<int8_t *>(q), ldq, const_cast<uint8_t *>(exps),
                      lde, gamma, beta, false, as_stream(stream));
    return launch_status();
}
