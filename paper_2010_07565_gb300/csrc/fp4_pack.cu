// Rows to 4 bits and back, and a matrix's columns to 4-bit rows (bigcn_fp4_pack, bigcn_fp4_unpack,
// bigcn_fp4_pack_columns): the arithmetic is fp4.cuh's; all are bound by memory.
//
// A thread takes octets, 8 consecutive columns of a row: 32 or 16 bytes of X and one word of codes;
// four neighbouring lanes hold a group and share its largest magnitude by shuffles.
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

// A row lies over `tpr` threads (a power of two, 8 to 256), J octets of it by R rows to a thread,
// all loaded before the first is used; a longer row goes over several blocks (`parts`).
template <int J, int R>
struct Octets {
    int64_t i[R];            // rows
    int k0;                  // column of octet 0
    int step;                // columns from one octet to the next
    __device__ __forceinline__ Octets(int tpr, unsigned parts) {
        const int t = threadIdx.x & (tpr - 1), rows = kFp4Threads / tpr;
        const unsigned set = blockIdx.x / parts, part = blockIdx.x % parts;
#pragma unroll
        for (int r = 0; r < R; ++r) i[r] = (int64_t(set) * R + r) * rows + threadIdx.x / tpr;
        step = tpr * 8;
        k0 = int(part) * step * J + t * 8;
    }
};

template <typename T, int A, int J, int R>
__global__ void __launch_bounds__(kFp4Threads)
fp4_pack_kernel(const Fp4Args a, const int tpr, const unsigned parts) {
    constexpr int V = kPiece<T>, P = 8 / V, H = V / 2;      // P pieces of V elements an octet
    const Octets<J, R> at(tpr, parts);
    const int K = a.K, left = K - at.k0;
    Raw<A> w[R][J][P];
    bool odd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const T *row = static_cast<const T *>(a.X) + at.i[r] * a.ldx + at.k0;
        const bool whole = whole_pieces<A>(row, tpr >= 32);
        odd[r] = odd_pieces<A>(row);
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int n = left - j * at.step - p * V;
                w[r][j][p] = raw_zero<A>();
                if (at.i[r] < a.N && n > 0)
                    w[r][j][p] = load_piece<T, A>(row + j * at.step + p * V, n, whole, odd[r]);
            }
    }
    const int groups = int(checkpoint_groups(K));
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float2 x[J][4];
        uint32_t own[J], top[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float2 v[H];
                unpack16<T>(settled<A>(w[r][j][p], odd[r]), v);
#pragma unroll
                for (int e = 0; e < H; ++e) x[j][p * H + e] = v[e];
            }
            own[j] = top_bits(x[j]);
        }
        group_tops<4>(own, top);
        if (at.i[r] >= a.N) continue;
        uint8_t *q = a.q + at.i[r] * a.ldq;
        uint8_t *exps = a.exps + at.i[r] * a.lde;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int k = at.k0 + j * at.step, g = k / kGroup;
            if (g >= groups) break;
            const uint32_t b = fp4_scale_byte(top[j]);
            const float2 f = both(pack_factor(b));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = __fmul2_rn(x[j][e], f);
            const uint32_t codes = fp4_codes(x[j][0].x, x[j][0].y, x[j][1].x, x[j][1].y, x[j][2].x,
                                             x[j][2].y, x[j][3].x, x[j][3].y);
            *reinterpret_cast<uint32_t *>(q + k / 2) = b == kNanByte ? 0u : codes;
            if ((threadIdx.x & 3) == 0) exps[g] = uint8_t(b);
        }
        const int t = threadIdx.x & (tpr - 1);
        if (blockIdx.x % parts + 1 == parts && groups + t < (groups + 3) / 4 * 4) exps[groups + t] = 0;
    }
}

// 2^(b - 127), as the tensor core reads the byte.
__device__ __forceinline__ float fp4_factor(uint32_t b) {
    return b == 0u ? __uint_as_float(0x00400000u) : unpack_factor(b);
}

template <typename T, int A, int J, int R>
__global__ void __launch_bounds__(kFp4Threads)
fp4_unpack_kernel(const Fp4Args a, const int tpr, const unsigned parts) {
    constexpr int V = kPiece<T>, P = 8 / V, H = V / 2;
    const Octets<J, R> at(tpr, parts);
    const int left = a.K - at.k0;
    uint32_t w[R][J];
    uint8_t b[R][J];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (at.i[r] < a.N && left > j * at.step) {
                const int k = at.k0 + j * at.step;
                w[r][j] = *reinterpret_cast<const uint32_t *>(a.q + at.i[r] * a.ldq + k / 2);
                b[r][j] = a.exps[at.i[r] * a.lde + k / kGroup];
            }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (at.i[r] >= a.N) continue;
        T *row = static_cast<T *>(a.X) + at.i[r] * a.ldx + at.k0;
        const bool whole = whole_pieces<A>(row, tpr >= 32);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (left <= j * at.step) break;
            uint32_t h[4];
            fp4_halves(w[r][j], h);
            const float2 f = both(fp4_factor(b[r][j]));
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int n = left - j * at.step - p * V;
                if (n <= 0) break;
                float2 v[H];
#pragma unroll
                for (int e = 0; e < H; ++e)
                    v[e] = __fmul2_rn(
                        __half22float2(*reinterpret_cast<const __half2 *>(&h[p * H + e])), f);
                store_piece<T, A>(row + j * at.step + p * V, pack16<T>(v), n, whole);
            }
        }
    }
}

template <typename T, int A, int J, int R>
void launch_octets(const Fp4Args &a, bool pack, int tpr, unsigned parts, cudaStream_t s) {
    const int64_t rows = kFp4Threads / tpr * R;
    const unsigned blocks = unsigned((a.N + rows - 1) / rows * parts);
    if (pack) fp4_pack_kernel<T, A, J, R><<<blocks, kFp4Threads, 0, s>>>(a, tpr, parts);
    else fp4_unpack_kernel<T, A, J, R><<<blocks, kFp4Threads, 0, s>>>(a, tpr, parts);
}

// The fewest threads (8, or more) that hold a row in at most two octets, else all 256 and
// several blocks a row.
template <typename T, int A>
void launch_fp4_rows(const Fp4Args &a, bool pack, cudaStream_t s) {
    const int64_t octets = checkpoint_groups(a.K) * 4;
    int tpr = 8;
    while (tpr < kFp4Threads && int64_t(tpr) * 2 < octets) tpr *= 2;
    const int64_t need = (octets + tpr - 1) / tpr;
    const int J = need < 2 ? 1 : 2;
    const unsigned parts = unsigned((need + J - 1) / J);
    if (J == 1) launch_octets<T, A, 1, 2>(a, pack, tpr, parts, s);
    else launch_octets<T, A, 2, 1>(a, pack, tpr, parts, s);
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

// Columns of W to rows: a lane takes a column, a warp 32 consecutive columns of one group of 32 rows
// (whose loads are coalesced); the eight warps' groups of a column are 128 bytes of its row, put
// together in shared memory.
constexpr int kColumnGroups = kFp4Threads / 32;
template <typename T>
__global__ void __launch_bounds__(kFp4Threads)
fp4_columns_kernel(const T *__restrict__ W, int K, int F, int64_t ldw, uint8_t *__restrict__ q,
                   int64_t ldq, uint8_t *__restrict__ exps, int64_t lde) {
    __shared__ uint4 codes[32][kColumnGroups + 1];
    __shared__ uint8_t bytes[32][kColumnGroups];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int groups = int(checkpoint_groups(K));
    const int g0 = int(blockIdx.x) * kColumnGroups, g = g0 + warp;
    for (int64_t j0 = int64_t(blockIdx.y) * 32; j0 < F; j0 += int64_t(gridDim.y) * 32) {
        const int64_t j = j0 + lane;
        float x[32];
        uint32_t top = 0u;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const int64_t k = int64_t(g) * kGroup + e;
            x[e] = j < F && k < K ? to_f32(W[k * ldw + j]) : 0.0f;
            top = max(top, abs_bits(x[e]));
        }
        const uint32_t b = fp4_scale_byte(top);
        const float f = pack_factor(b);
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float *v = x + 8 * e;
            w[e] = b == kNanByte ? 0u
                                 : fp4_codes(v[0] * f, v[1] * f, v[2] * f, v[3] * f, v[4] * f,
                                             v[5] * f, v[6] * f, v[7] * f);
        }
        __syncthreads();                    // the previous columns have been stored
        codes[lane][warp] = make_uint4(w[0], w[1], w[2], w[3]);
        bytes[lane][warp] = g < groups ? uint8_t(b) : uint8_t(0);
        __syncthreads();
        const int c = threadIdx.x / kColumnGroups, u = threadIdx.x % kColumnGroups;
        if (j0 + c < F) {
            if (g0 + u < groups)
                *reinterpret_cast<uint4 *>(q + (j0 + c) * ldq + int64_t(g0 + u) * 16) = codes[c][u];
            if (g0 + u < (groups + 3) / 4 * 4) exps[(j0 + c) * lde + g0 + u] = bytes[c][u];
        }
    }
}

template <typename T>
void launch_columns(const void *W, int K, int F, int64_t ldw, uint8_t *q, int64_t ldq, uint8_t *exps,
                    int64_t lde, cudaStream_t s) {
    const int64_t strips = (int64_t(F) + 31) / 32, groups = checkpoint_groups(K);
    const dim3 grid(unsigned((groups + kColumnGroups - 1) / kColumnGroups),
                    unsigned(strips < 65535 ? strips : 65535));
    fp4_columns_kernel<T><<<grid, kFp4Threads, 0, s>>>(static_cast<const T *>(W), K, F, ldw, q, ldq,
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
