// The weight gradient of a product whose input is kept as a checkpoint
// (bigcn_checkpoint_weight_grad): with the input gamma v + beta,
//
//   dW[k,j] = gamma_k sum_i v_ik dZ_ij + beta_k s_j,   s_j = db_j = sum_i dZ_ij.
//
// The rows are split into chunks whose partial sums a second kernel adds in order, so
// that the result does not depend on scheduling.
#include "checkpoint.cuh"
#include "launch.cuh"

namespace bigcn {
namespace {

constexpr int kGradThreads = 256;
constexpr int kTileK = 64, kTileF = 64, kTileRows = 16;
constexpr int kMaxGradChunks = 64;
constexpr size_t kAlign = 256;

struct GradArgs {
    const int8_t *q;
    int64_t ldq;
    const uint8_t *exps;
    int64_t lde;
    int64_t N;
    int K;
    const void *dZ;
    int F;
    int64_t lddz;
    float *partial;          // chunks x K x F
    float *colsum;           // chunks x F
    int chunks;
};

// A 64 x 64 tile of a chunk's partial product; 4 x 4 outputs a thread. The blocks of
// the first feature tile also sum dZ's columns.
template <typename T>
__global__ void __launch_bounds__(kGradThreads) grad_tile_kernel(const GradArgs a) {
    __shared__ float sv[kTileRows][kTileK];
    __shared__ float sz[kTileRows][kTileF];
    const int k0 = blockIdx.x * kTileK, f0 = blockIdx.y * kTileF, c = blockIdx.z;
    const int64_t r0 = a.N * c / a.chunks, r1 = a.N * (c + 1) / a.chunks;
    const int tk = threadIdx.x / 16, tf = threadIdx.x % 16;
    float acc[4][4] = {};
    float colsum = 0.0f;
    for (int64_t r = r0; r < r1; r += kTileRows) {
        for (int t = threadIdx.x; t < kTileRows * kTileK; t += kGradThreads) {
            const int64_t i = r + t / kTileK;
            const int k = k0 + t % kTileK;
            sv[t / kTileK][t % kTileK] =
                i < r1 && k < a.K
                    ? float(a.q[i * a.ldq + k]) * unpack_factor(a.exps[i * a.lde + k / kGroup])
                    : 0.0f;
        }
        for (int t = threadIdx.x; t < kTileRows * kTileF; t += kGradThreads) {
            const int64_t i = r + t / kTileF;
            const int f = f0 + t % kTileF;
            sz[t / kTileF][t % kTileF] =
                i < r1 && f < a.F ? to_f32(static_cast<const T *>(a.dZ)[i * a.lddz + f]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kTileRows; ++e)
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    acc[p][w] = fmaf(sv[e][tk + 16 * p], sz[e][tf + 16 * w], acc[p][w]);
        if (k0 == 0 && threadIdx.x < kTileF)
            for (int e = 0; e < kTileRows; ++e) colsum += sz[e][threadIdx.x];
        __syncthreads();
    }
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int k = k0 + tk + 16 * p, f = f0 + tf + 16 * w;
            if (k < a.K && f < a.F) a.partial[(int64_t(c) * a.K + k) * a.F + f] = acc[p][w];
        }
    if (k0 == 0 && threadIdx.x < kTileF && f0 + threadIdx.x < a.F)
        a.colsum[int64_t(c) * a.F + f0 + threadIdx.x] = colsum;
}

__global__ void __launch_bounds__(kGradThreads)
grad_sum_kernel(const float *__restrict__ partial, const float *__restrict__ colsum, int chunks,
                int K, int F, const float *__restrict__ gamma, const float *__restrict__ beta,
                float *__restrict__ dW, int64_t lddw, float *__restrict__ db) {
    const int64_t n = int64_t(K) * F;
    for (int64_t t = int64_t(blockIdx.x) * kGradThreads + threadIdx.x; t < n;
         t += int64_t(gridDim.x) * kGradThreads) {
        const int64_t k = t / F, f = t % F;
        float s = 0.0f, cs = 0.0f;
        for (int c = 0; c < chunks; ++c) {
            s += partial[int64_t(c) * n + t];
            cs += colsum[int64_t(c) * F + f];
        }
        dW[k * lddw + f] = fmaf(gamma ? gamma[k] : 1.0f, s, beta ? beta[k] * cs : 0.0f);
        if (db && k == 0) db[f] = cs;
    }
}

int64_t grad_chunks(int64_t N, int K, int F) {
    const int64_t tiles = ((int64_t(K) + kTileK - 1) / kTileK) * ((F + kTileF - 1) / kTileF);
    int64_t c = (1024 + tiles - 1) / tiles;
    if (c > kMaxGradChunks) c = kMaxGradChunks;
    if (c > (N + kTileRows - 1) / kTileRows) c = (N + kTileRows - 1) / kTileRows;
    return c < 1 ? 1 : c;
}

size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

template <typename T>
void launch_grad(const GradArgs &a, cudaStream_t s) {
    grad_tile_kernel<T><<<dim3(unsigned((a.K + kTileK - 1) / kTileK),
                               unsigned((a.F + kTileF - 1) / kTileF), unsigned(a.chunks)),
                          kGradThreads, 0, s>>>(a);
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" size_t bigcn_checkpoint_weight_grad_workspace_bytes(int64_t N, int32_t K, int32_t F) {
    if (N < 0 || N > int64_t(INT32_MAX) || K < 1 || F < 1 ||
        int64_t(K) > kMaxElems / 4096 / F)
        return 0;
    const size_t c = size_t(grad_chunks(N, K, F));
    return round_up(c * size_t(K) * size_t(F) * 4) + round_up(c * size_t(F) * 4);
}

extern "C" bigcn_status bigcn_checkpoint_weight_grad(
    int32_t dtype, const int8_t *q, int64_t ldq, const uint8_t *exps, int64_t lde, int64_t N,
    int32_t K, const float *gamma, const float *beta, const void *dZ, int32_t F, int64_t lddz,
    float *dW, int64_t lddw, float *db, void *workspace, size_t ws_bytes, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || F < 1 || lddz < F || lddw < F)
        return BIGCN_ERR_INVALID_ARG;
    const size_t need = bigcn_checkpoint_weight_grad_workspace_bytes(N, K, F);
    if (need == 0 || int64_t(K) > kMaxElems / lddw || !dW) return BIGCN_ERR_INVALID_ARG;
    if (N > 0 && (!q || !exps || !dZ || !workspace || ws_bytes < need || N > kMaxElems / lddz ||
                  !checkpoint_strides_ok(N, K, ldq, lde)))
        return BIGCN_ERR_INVALID_ARG;
    if ((N > 0 && !checkpoint_aligned(q, exps)) || (gamma && !aligned_to(gamma, 4)) ||
        (beta && !aligned_to(beta, 4)) || (dZ && !aligned_to(dZ, es)) || !aligned_to(dW, 4) ||
        (db && !aligned_to(db, 4)) || (N > 0 && !aligned_to(workspace, kAlign)))
        return BIGCN_ERR_MISALIGNED;
    const void *in[] = {N > 0 ? q : nullptr, N > 0 ? exps : nullptr, gamma, beta, dZ};
    const size_t inb[] = {checkpoint_q_span(N, K, ldq), checkpoint_exps_span(N, K, lde),
                          size_t(K) * 4, size_t(K) * 4, span_bytes(N, F, lddz, es)};
    const void *out[] = {dW, db, N > 0 ? workspace : nullptr};
    const size_t outb[] = {span_bytes(K, F, lddw, 4), size_t(F) * 4, need};
    for (int o = 0; o < 3; ++o) {
        for (int p = 0; p < 5; ++p)
            if (overlaps(out[o], outb[o], in[p], inb[p])) return BIGCN_ERR_INVALID_ARG;
        for (int p = o + 1; p < 3; ++p)
            if (overlaps(out[o], outb[o], out[p], outb[p])) return BIGCN_ERR_INVALID_ARG;
    }
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    if (N == 0) {       // no rows: every sum is 0
        if (cudaMemset2DAsync(dW, size_t(lddw) * 4, 0, size_t(F) * 4, size_t(K), s) != cudaSuccess ||
            (db && cudaMemsetAsync(db, 0, size_t(F) * 4, s) != cudaSuccess)) {
            cudaGetLastError();
            return BIGCN_ERR_CUDA;
        }
        return BIGCN_OK;
    }
    const int chunks = int(grad_chunks(N, K, F));
    float *partial = static_cast<float *>(workspace);
    float *colsum = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                              round_up(size_t(chunks) * size_t(K) * F * 4));
    const GradArgs a{q, ldq, exps, lde, N, K, dZ, F, lddz, partial, colsum, chunks};
    if (dtype == BIGCN_F32) launch_grad<float>(a, s);
    else if (dtype == BIGCN_BF16) launch_grad<__nv_bfloat16>(a, s);
    else launch_grad<__half>(a, s);
    const int64_t blocks = (int64_t(K) * F + kGradThreads - 1) / kGradThreads;
    grad_sum_kernel<<<unsigned(blocks < 4096 ? blocks : 4096), kGradThreads, 0, s>>>(
        partial, colsum, chunks, K, F, gamma, beta, dW, lddw, db);
    return launch_status();
}
