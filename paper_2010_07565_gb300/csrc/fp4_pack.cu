// Rows to 4 bits and back, and a matrix's columns to 4-bit rows (bigcn_fp4_pack, bigcn_fp4_unpack,
// bigcn_fp4_pack_columns): the arithmetic is fp4.cuh's; all are bound by memory.
//
// Rows are taken as one sequence of octets (packing) or 16-byte pieces (reading back), each row up to a
// whole group, so that every lane has work whatever a row's length: laid over a power of two
// threads, 602 columns kept 59 of 100 lanes busy. 232,965 x 602 fp32: packing 105 us (131 so; 6.05 TB/s,
// 0.90 of a copy's rate), reading back to bf16 68 us (101; 5.2 TB/s: rows aligned to 4 bytes), to fp32 101
// us; 2^20 x 128 fp32 101 and 56 us. From bf16, 232,965 x 602 76 us (0.69), 2^20 x 256 122 (0.83).
#include "fp4.cuh"
#include "norm.cuh"

namespace bigcn {
namespace {

constexpr int kFp4Threads = 256;

struct Fp4Args {
    void *X;                 // read by the packing, written by the unpacking
    int64_t N;
    int K;
    int64_t ldx;
    uint8_t *q;
    int64_t ldq;
    uint8_t *exps;
    int64_t lde;
};

// Pieces per thread: all asked for before the first is used.
constexpr int kFp4Pieces = 4;

// An octet, 8 columns (P pieces), a lane: a word of codes.
template <typename T, int A>
__global__ void __launch_bounds__(kFp4Threads)
fp4_pack_kernel(const Fp4Args a, const uint32_t per_row, const uint32_t magic) {
    constexpr int V = kPiece<T>, H = V / 2, P = 8 / V, U = kFp4Pieces / P, kLanes = kGroup / 8;
    const PieceWalk<U * kFp4Threads> walk(per_row, magic);
    Raw<A> w[U][P];
    bool odd[U];
    int64_t row[U];
    uint32_t octet[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        walk.at(threadIdx.x + u * kFp4Threads, row[u], octet[u]);
        const int n = a.K - int(octet[u]) * 8;
        const T *x = static_cast<const T *>(a.X) + row[u] * a.ldx + int64_t(octet[u]) * 8;
        const bool whole = whole_pieces<A>(x, true);
        odd[u] = odd_pieces<A>(x);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            w[u][p] = raw_zero<A>();
            if (row[u] < a.N && n > p * V) w[u][p] = load_piece<T, A>(x + p * V, n - p * V, whole, odd[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float2 x[4];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float2 v[H];
            unpack16<T>(settled<A>(w[u][p], odd[u]), v);
#pragma unroll
            for (int e = 0; e < H; ++e) x[p * H + e] = v[e];
        }
        uint32_t own[1] = {top_bits(x)}, top[1];
        group_tops<kLanes>(own, top);
        if (row[u] >= a.N) continue;
        const uint32_t b = fp4_scale_byte(top[0]);
        const float2 f = both(pack_factor(b));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __fmul2_rn(x[e], f);
        const uint32_t c = fp4_codes(x[0].x, x[0].y, x[1].x, x[1].y, x[2].x, x[2].y, x[3].x, x[3].y);
        *reinterpret_cast<uint32_t *>(a.q + row[u] * a.ldq + int64_t(octet[u]) * 4) =
            b == kNanByte ? 0u : c;
        if (octet[u] % kLanes == 0) {
            uint8_t *e = a.exps + row[u] * a.lde + octet[u] / kLanes;
            *e = uint8_t(b);
            if (octet[u] + kLanes == per_row)               // the row's last group: zeros up to a word
                for (uint32_t g = per_row / kLanes; g % 4 != 0; ++g) *++e = 0;
        }
    }
}

// 2^(b - 127), as the tensor core reads the byte.
__device__ __forceinline__ float fp4_factor(uint32_t b) {
    return b == 0u ? __uint_as_float(0x00400000u) : unpack_factor(b);
}

// A piece a lane. (Rows aligned to less than 16 bytes through shared memory, so that a store of fewer bytes a
// lane is a run of memory: 232,965 x 602 to bf16 72 -> 81 us.)
template <typename T, int A>
__global__ void __launch_bounds__(kFp4Threads)
fp4_unpack_kernel(const Fp4Args a, const uint32_t per_row, const uint32_t magic) {
    constexpr int V = kPiece<T>, H = V / 2, kLanes = kGroup / V;
    const PieceWalk<kFp4Pieces * kFp4Threads> walk(per_row, magic);
    uint32_t w[kFp4Pieces];
    uint8_t b[kFp4Pieces];
    T *to[kFp4Pieces];
    int n[kFp4Pieces];                  // of the piece's columns in the row
#pragma unroll
    for (int u = 0; u < kFp4Pieces; ++u) {
        int64_t row;
        uint32_t piece;
        walk.at(threadIdx.x + u * kFp4Threads, row, piece);
        w[u] = 0u;
        b[u] = 0;
        to[u] = static_cast<T *>(a.X) + row * a.ldx + int64_t(piece) * V;
        n[u] = row < a.N ? a.K - int(piece) * V : 0;
        if (row < a.N) {
            const uint8_t *q = a.q + row * a.ldq + int64_t(piece) * (V / 2);
            if constexpr (V == 8) w[u] = *reinterpret_cast<const uint32_t *>(q);
            else w[u] = *reinterpret_cast<const uint16_t *>(q);
            b[u] = a.exps[row * a.lde + piece / kLanes];
        }
    }
#pragma unroll
    for (int u = 0; u < kFp4Pieces; ++u) {
        uint32_t h[4];
        fp4_halves(w[u], h);
        const float2 f = both(fp4_factor(b[u]));
        float2 v[H];
#pragma unroll
        for (int e = 0; e < H; ++e)
            v[e] = __fmul2_rn(__half22float2(*reinterpret_cast<const __half2 *>(&h[e])), f);
        if (n[u] > 0) store_piece<T, A>(to[u], pack16<T>(v), n[u], whole_pieces<A>(to[u], true));
    }
}

template <typename T, int A>
void launch_fp4_rows(const Fp4Args &a, bool pack, cudaStream_t s) {
    const int columns = pack ? 8 : kPiece<T>;               // of a thread's unit
    const uint32_t per_row = uint32_t(checkpoint_groups(a.K) * (kGroup / columns));
    const uint32_t magic = piece_magic(per_row);
    const int64_t block = kFp4Threads * (pack ? kFp4Pieces * kPiece<T> / 8 : kFp4Pieces);
    const unsigned blocks = unsigned((a.N * int64_t(per_row) + block - 1) / block);
    if (pack) fp4_pack_kernel<T, A><<<blocks, kFp4Threads, 0, s>>>(a, per_row, magic);
    else fp4_unpack_kernel<T, A><<<blocks, kFp4Threads, 0, s>>>(a, per_row, magic);
}

template <typename T>
void launch_fp4_type(const Fp4Args &a, bool pack, cudaStream_t s) {
    const uint64_t es = sizeof(T);
    const uint64_t where[] = {uint64_t(uintptr_t(a.X)), uint64_t(a.ldx) * es};
    const int A = alignment_of(where, 2);
    if (A == 16) launch_fp4_rows<T, 16>(a, pack, s);
    else if (A == 8) launch_fp4_rows<T, 8>(a, pack, s);
    else if (A == 4) launch_fp4_rows<T, 4>(a, pack, s);
    else launch_fp4_rows<T, es == 2 ? 2 : 4>(a, pack, s);
}

void launch_fp4(int32_t dtype, const Fp4Args &a, bool pack, cudaStream_t s) {
    if (dtype == BIGCN_F32) launch_fp4_type<float>(a, pack, s);
    else if (dtype == BIGCN_BF16) launch_fp4_type<__nv_bfloat16>(a, pack, s);
    else launch_fp4_type<__half>(a, pack, s);
}

// Columns of W to rows: a warp takes 8 V columns of one group of 32 rows, a lane V neighbouring columns
// (16 bytes) of eight rows, which are one word of codes each; four lanes hold a column and share its
// largest magnitude. The eight warps' groups of a column are 128 bytes of its row, put together in
// shared memory. 8192 x 1024 fp32: 15 us (a column a lane, 32 loads of four bytes: 17), one wave's
// latency; 4096 x 4096 23 us (29); 8192 x 1024 bf16 17 us (25), 4096 x 4096 27: a lane holds 64 values of these, 32
// of fp32, and has the 64 registers of four blocks an SM (132 bytes of spills).
constexpr int kColumnGroups = kFp4Threads / 32;
template <typename T>
__device__ __forceinline__ void load_columns(const T *p, int64_t n, bool wide, float (&v)[kPiece<T>]) {
    if (wide && n >= kPiece<T>) {
        float2 x[kPiece<T> / 2];
        unpack16<T>(*reinterpret_cast<const uint4 *>(p), x);
#pragma unroll
        for (int e = 0; e < kPiece<T> / 2; ++e) v[2 * e] = x[e].x, v[2 * e + 1] = x[e].y;
    } else {
#pragma unroll
        for (int e = 0; e < kPiece<T>; ++e) v[e] = e < n ? to_f32(p[e]) : 0.0f;
    }
}
template <typename T>
__global__ void __launch_bounds__(kFp4Threads, 4)
fp4_columns_kernel(const T *__restrict__ W, int K, int F, int64_t ldw, bool wide, uint8_t *__restrict__ q,
                   int64_t ldq, uint8_t *__restrict__ exps, int64_t lde) {
    constexpr int V = kPiece<T>, kCols = 8 * V;
    __shared__ __align__(16) uint32_t codes[kCols][kColumnGroups * 4 + 4];      // (read 16 bytes at a time)
    __shared__ uint8_t bytes[kCols][kColumnGroups];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int column = lane % 8 * V, octet = lane / 8;
    const int groups = int(checkpoint_groups(K));
    const int g0 = int(blockIdx.x) * kColumnGroups, g = g0 + warp;
    const int64_t k0 = int64_t(g) * kGroup + octet * 8;
    for (int64_t j0 = int64_t(blockIdx.y) * kCols; j0 < F; j0 += int64_t(gridDim.y) * kCols) {
        const int64_t left = F - j0 - column;
        const T *p = W + k0 * ldw + j0 + column;
        float x[8][V];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int c = 0; c < V; ++c) x[e][c] = 0.0f;
            if (k0 + e < K && left > 0) load_columns(p + e * ldw, left, wide, x[e]);
        }
        uint32_t word[V], b[V];
#pragma unroll
        for (int c = 0; c < V; ++c) {
            uint32_t top = 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, abs_bits(x[e][c]));
            top = max(top, __shfl_xor_sync(kFullMask, top, 8));
            top = max(top, __shfl_xor_sync(kFullMask, top, 16));
            b[c] = fp4_scale_byte(top);
            const float f = pack_factor(b[c]);
            word[c] = b[c] == kNanByte
                          ? 0u
                          : fp4_codes(x[0][c] * f, x[1][c] * f, x[2][c] * f, x[3][c] * f, x[4][c] * f,
                                      x[5][c] * f, x[6][c] * f, x[7][c] * f);
        }
        __syncthreads();                    // the previous columns have been stored
#pragma unroll
        for (int c = 0; c < V; ++c) {
            codes[column + c][warp * 4 + octet] = word[c];
            if (octet == 0) bytes[column + c][warp] = g < groups ? uint8_t(b[c]) : uint8_t(0);
        }
        __syncthreads();
        const int u = threadIdx.x % kColumnGroups;
        for (int c = threadIdx.x / kColumnGroups; c < kCols && j0 + c < F; c += kFp4Threads / kColumnGroups) {
            if (g0 + u < groups)
                *reinterpret_cast<uint4 *>(q + (j0 + c) * ldq + int64_t(g0 + u) * 16) =
                    *reinterpret_cast<const uint4 *>(&codes[c][u * 4]);
            if (g0 + u < (groups + 3) / 4 * 4) exps[(j0 + c) * lde + g0 + u] = bytes[c][u];
        }
    }
}

template <typename T>
void launch_columns(const void *W, int K, int F, int64_t ldw, uint8_t *q, int64_t ldq, uint8_t *exps,
                    int64_t lde, cudaStream_t s) {
    const int64_t cols = 8 * kPiece<T>, strips = (int64_t(F) + cols - 1) / cols, groups = checkpoint_groups(K);
    const dim3 grid(unsigned((groups + kColumnGroups - 1) / kColumnGroups),
                    unsigned(strips < 65535 ? strips : 65535));
    const bool wide = (reinterpret_cast<uintptr_t>(W) | uint64_t(ldw) * sizeof(T)) % 16 == 0;
    fp4_columns_kernel<T><<<grid, kFp4Threads, 0, s>>>(static_cast<const T *>(W), K, F, ldw, wide, q, ldq,
                                                       exps, lde);
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" bigcn_status bigcn_fp4_pack(int32_t dtype, const void *X, int64_t N, int32_t K,
                                       int64_t ldx, uint8_t *q, int64_t ldq, uint8_t *exps,
                                       int64_t lde, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols || ldx < K ||
        !fp4_strides_ok(N, K, ldq, lde))
        return BIGCN_ERR_INVALID_ARG;
    if (N > 0 && N > kMaxElems / ldx) return BIGCN_ERR_INVALID_ARG;
    if (N == 0) return BIGCN_OK;
    if (!X || !q || !exps) return BIGCN_ERR_INVALID_ARG;
    if (!aligned_to(X, es) || !checkpoint_aligned(q, exps)) return BIGCN_ERR_MISALIGNED;
    const size_t xb = span_bytes(N, K, ldx, es), qb = fp4_q_span(N, K, ldq),
                 eb = checkpoint_exps_span(N, K, lde);
    if (overlaps(q, qb, X, xb) || overlaps(exps, eb, X, xb) || overlaps(q, qb, exps, eb))
        return BIGCN_ERR_INVALID_ARG;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    launch_fp4(dtype, Fp4Args{const_cast<void *>(X), N, K, ldx, q, ldq, exps, lde}, true,
               as_stream(stream));
    return launch_status();
}

extern "C" bigcn_status bigcn_fp4_unpack(int32_t dtype, const uint8_t *q, int64_t ldq,
                                         const uint8_t *exps, int64_t lde, int64_t N, int32_t K,
                                         void *X, int64_t ldx, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols || ldx < K ||
        !fp4_strides_ok(N, K, ldq, lde))
        return BIGCN_ERR_INVALID_ARG;
    if (N > 0 && N > kMaxElems / ldx) return BIGCN_ERR_INVALID_ARG;
    if (N == 0) return BIGCN_OK;
    if (!X || !q || !exps) return BIGCN_ERR_INVALID_ARG;
    if (!aligned_to(X, es) || !checkpoint_aligned(q, exps)) return BIGCN_ERR_MISALIGNED;
    const size_t xb = span_bytes(N, K, ldx, es);
    if (overlaps(X, xb, q, fp4_q_span(N, K, ldq)) ||
        overlaps(X, xb, exps, checkpoint_exps_span(N, K, lde)))
        return BIGCN_ERR_INVALID_ARG;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    launch_fp4(dtype,
               Fp4Args{X, N, K, ldx, const_cast<uint8_t *>(q), ldq, const_cast<uint8_t *>(exps), lde},
               false, as_stream(stream));
    return launch_status();
}

extern "C" bigcn_status bigcn_fp4_pack_columns(int32_t dtype, const void *W, int32_t K, int32_t F,
                                               int64_t ldw, uint8_t *q, int64_t ldq, uint8_t *exps,
                                               int64_t lde, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || K < 1 || K > kMaxCols || F < 1 || F > kMaxCols || ldw < F ||
        !fp4_strides_ok(F, K, ldq, lde) || int64_t(K) > kMaxElems / ldw)
        return BIGCN_ERR_INVALID_ARG;
    if (!W || !q || !exps) return BIGCN_ERR_INVALID_ARG;
    if (!aligned_to(W, es) || !checkpoint_aligned(q, exps)) return BIGCN_ERR_MISALIGNED;
    const size_t wb = span_bytes(K, F, ldw, es), qb = fp4_q_span(F, K, ldq),
                 eb = checkpoint_exps_span(F, K, lde);
    if (overlaps(q, qb, W, wb) || overlaps(exps, eb, W, wb) || overlaps(q, qb, exps, eb))
        return BIGCN_ERR_INVALID_ARG;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32) launch_columns<float>(W, K, F, ldw, q, ldq, exps, lde, s);
    else if (dtype == BIGCN_BF16) launch_columns<__nv_bfloat16>(W, K, F, ldw, q, ldq, exps, lde, s);
    else launch_columns<__half>(W, K, F, ldw, q, ldq, exps, lde, s);
    return launch_status();
}
