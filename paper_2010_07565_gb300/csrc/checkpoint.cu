// Activations to 8 bits and back (bigcn_checkpoint_pack, bigcn_checkpoint_unpack): the arithmetic
// is checkpoint.cuh's, a few operations a column; both are bound by memory. 2^20 x 512 bf16: packing
// 255 us (0.95 of a copy's rate), unpacking 267 us (0.90), 398 with gamma and beta.
#include "norm.cuh"

namespace bigcn {
namespace {

constexpr int kCkThreads = 256;

// Both directions lay a row over `tpr` threads (a power of two, 8 to 256) in pieces of 16
// bytes of X, as layer norm does (norm.cuh). A thread takes three or four pieces, J of
// a row by R rows, all loaded before the first is used (eight to unpack: 616 -> 635 us for both at
// 2^20 x 512 bf16); a row longer than tpr J pieces goes over several blocks.
template <int V, int J, int R>
struct Place {
    int64_t i[R];            // rows
    int k0;                  // column of piece 0
    int step;                // columns from one piece to the next
    __device__ __forceinline__ Place(int tpr, unsigned parts) {
        const int t = threadIdx.x & (tpr - 1), rows = kCkThreads / tpr;
        const unsigned set = blockIdx.x / parts, part = blockIdx.x % parts;
#pragma unroll
        for (int r = 0; r < R; ++r) i[r] = (int64_t(set) * R + r) * rows + threadIdx.x / tpr;
        step = tpr * V;
        k0 = int(part) * step * J + t * V;
    }
};

struct CkArgs {
    void *X;                 // read by the packing, written by the unpacking
    int64_t N;
    int K;
    int64_t ldx;
    int8_t *q;
    int64_t ldq;
    uint8_t *exps;
    int64_t lde;
    const float *gamma;
    const float *beta;
    bool aligned;            // gamma and beta to 32 bytes
};

template <typename T, int A, int J, int R>
__global__ void __launch_bounds__(kCkThreads)
pack_kernel(const CkArgs a, const int tpr, const unsigned parts) {
    constexpr int V = kPiece<T>, H = V / 2;
    const Place<V, J, R> at(tpr, parts);
    const int K = a.K, left = K - at.k0;
    Raw<A> w[R][J];
    bool odd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const T *row = static_cast<const T *>(a.X) + at.i[r] * a.ldx + at.k0;
        const bool whole = whole_pieces<A>(row, tpr >= 32);
        odd[r] = odd_pieces<A>(row);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            w[r][j] = raw_zero<A>();
            if (at.i[r] < a.N && left > j * at.step)
                w[r][j] = load_piece<T, A>(row + j * at.step, left - j * at.step, whole, odd[r]);
        }
    }
    // Past K a piece is zeros and so is its q.
    const int kq = (K + 15) / 16 * 16 - at.k0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float2 x[J][H];
        uint32_t own[J], top[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            unpack16<T>(settled<A>(w[r][j], odd[r]), x[j]);
            own[j] = top_bits(x[j]);
        }
        group_tops<32 / V>(own, top);
        if (at.i[r] >= a.N) continue;
        int8_t *q = a.q + at.i[r] * a.ldq + at.k0;
        uint8_t *exps = a.exps + at.i[r] * a.lde;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (j * at.step >= kq) break;
            const uint32_t b = scale_byte(top[j]);
            *reinterpret_cast<QPiece<H> *>(q + j * at.step) = quantise_piece(x[j], b);
            if ((threadIdx.x & (32 / V - 1)) == 0 && j * at.step < left)
                exps[unsigned(at.k0 + j * at.step) / kGroup] = uint8_t(b);
        }
        const int groups = int(checkpoint_groups(K)), t = threadIdx.x & (tpr - 1);
        if (blockIdx.x % parts + 1 == parts && groups + t < (groups + 3) / 4 * 4) exps[groups + t] = 0;
    }
}

// With gamma, beta or both (values_kernel below: without).
template <typename T, int A, int J, int R>
__global__ void __launch_bounds__(kCkThreads)
unpack_kernel(const CkArgs a, const int tpr, const unsigned parts) {
    constexpr int V = kPiece<T>, H = V / 2;
    const Place<V, J, R> at(tpr, parts);
    const int left = a.K - at.k0;
    QPiece<H> w[R][J];
    uint8_t b[R][J];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (at.i[r] < a.N && left > j * at.step) {
                const int k = at.k0 + j * at.step;
                w[r][j] = *reinterpret_cast<const QPiece<H> *>(a.q + at.i[r] * a.ldq + k);
                b[r][j] = a.exps[at.i[r] * a.lde + unsigned(k) / kGroup];
            }
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int n = left - j * at.step;
        if (n <= 0) break;
        const int k = at.k0 + j * at.step;
        float2 g[H], c[H];
        if (a.gamma) load_params(a.gamma + k, a.aligned, n, g);
        if (a.beta) load_params(a.beta + k, a.aligned, n, c);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (at.i[r] >= a.N) continue;
            float2 v[H];
            dequantise_piece<H>(w[r][j], unpack_factor(b[r][j]), v);
#pragma unroll
            for (int e = 0; e < H; ++e)
                v[e] = __ffma2_rn(v[e], a.gamma ? g[e] : both(1.0f), a.beta ? c[e] : both(0.0f));
            T *out = static_cast<T *>(a.X) + at.i[r] * a.ldx + k;
            store_piece<T, A>(out, pack16<T>(v), n, whole_pieces<A>(out, tpr >= 32));
        }
    }
}

// Without gamma and beta: rows as one sequence of pieces, so that every lane has work whatever a row's length
// (232,965 x 602 to bf16 111 -> 80 us, to fp32 173 -> 108; 2^20 x 512 bf16 363 -> 267, 298 with four pieces a
// thread).
template <typename T> constexpr int kValuePieces = sizeof(T) == 4 ? 3 : 2;      // a thread's
template <typename T, int A>
__global__ void __launch_bounds__(kCkThreads)
values_kernel(const CkArgs a, const uint32_t per_row, const uint32_t magic) {
    constexpr int V = kPiece<T>, H = V / 2, kUnits = kValuePieces<T>;
    const PieceWalk<kUnits * kCkThreads> walk(per_row, magic);
    QPiece<H> w[kUnits];
    uint8_t b[kUnits];
    T *to[kUnits];
    int n[kUnits];                // of the piece's columns in the row
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        int64_t row;
        uint32_t piece;
        walk.at(threadIdx.x + u * kCkThreads, row, piece);
        to[u] = static_cast<T *>(a.X) + row * a.ldx + int64_t(piece) * V;
        n[u] = row < a.N ? a.K - int(piece) * V : 0;
        if (n[u] > 0) {
            w[u] = *reinterpret_cast<const QPiece<H> *>(a.q + row * a.ldq + int64_t(piece) * V);
            b[u] = a.exps[row * a.lde + piece / (kGroup / V)];
        }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        if (n[u] <= 0) continue;
        float2 v[H];
        dequantise_piece<H>(w[u], unpack_factor(b[u]), v);
        store_piece<T, A>(to[u], pack16<T>(v), n[u], whole_pieces<A>(to[u], true));
    }
}
template <typename T, int A> void launch_values(const CkArgs &a, cudaStream_t s) {
    const uint32_t per_row = uint32_t(checkpoint_groups(a.K) * (kGroup / kPiece<T>));
    const int64_t block = kValuePieces<T> * kCkThreads;
    values_kernel<T, A><<<unsigned((a.N * int64_t(per_row) + block - 1) / block), kCkThreads, 0, s>>>(
        a, per_row, piece_magic(per_row));
}

template <typename T, int A, int J, int R>
void launch_pieces(const CkArgs &a, bool pack, int tpr, unsigned parts, cudaStream_t s) {
    const int64_t rows = kCkThreads / tpr * R;
    const unsigned blocks = unsigned((a.N + rows - 1) / rows * parts);
    if (pack) pack_kernel<T, A, J, R><<<blocks, kCkThreads, 0, s>>>(a, tpr, parts);
    else unpack_kernel<T, A, J, R><<<blocks, kCkThreads, 0, s>>>(a, tpr, parts);
}

// The fewest threads (8, or more) that hold a row in at most four pieces, else all 256 and
// several blocks a row.
template <typename T, int A>
void launch_checkpoint_rows(const CkArgs &a, bool pack, cudaStream_t s) {
    if (!pack && !a.gamma && !a.beta) return launch_values<T, A>(a, s);
    const int64_t pieces = (int64_t(a.K) + kPiece<T> - 1) / kPiece<T>;
    int tpr = 8;
    while (tpr < kCkThreads && int64_t(tpr) * 4 < pieces) tpr *= 2;
    const int64_t need = (pieces + tpr - 1) / tpr;
    const int J = need < 4 ? int(need) : 4;
    const unsigned parts = unsigned((need + J - 1) / J);
    if (J == 1) launch_pieces<T, A, 1, 4>(a, pack, tpr, parts, s);
    else if (J == 2) launch_pieces<T, A, 2, 2>(a, pack, tpr, parts, s);
    else if (J == 3) launch_pieces<T, A, 3, 1>(a, pack, tpr, parts, s);
    else launch_pieces<T, A, 4, 1>(a, pack, tpr, parts, s);
}

template <typename T>
void launch_type(const CkArgs &a, bool pack, cudaStream_t s) {
    const uint64_t es = sizeof(T);
    const uint64_t where[] = {uint64_t(uintptr_t(a.X)), uint64_t(a.ldx) * es};
    const int A = alignment_of(where, 2);
    if (A == 16) launch_checkpoint_rows<T, 16>(a, pack, s);
    else if (A == 8) launch_checkpoint_rows<T, 8>(a, pack, s);
    else if (A == 4) launch_checkpoint_rows<T, 4>(a, pack, s);
    else launch_checkpoint_rows<T, es == 2 ? 2 : 4>(a, pack, s);
}

void launch_checkpoint(int32_t dtype, void *X, int64_t N, int K, int64_t ldx, int8_t *q,
                       int64_t ldq, uint8_t *exps, int64_t lde, const float *gamma,
                       const float *beta, bool pack, cudaStream_t s) {
    const CkArgs a{X,    N,   K,     ldx,  q, ldq, exps, lde, gamma, beta,
                   aligned_to(gamma, 32) && aligned_to(beta, 32)};
    if (dtype == BIGCN_F32) launch_type<float>(a, pack, s);
    else if (dtype == BIGCN_BF16) launch_type<__nv_bfloat16>(a, pack, s);
    else launch_type<__half>(a, pack, s);
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
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols ||
        ldx < K ||
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
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols ||
        ldx < K ||
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
