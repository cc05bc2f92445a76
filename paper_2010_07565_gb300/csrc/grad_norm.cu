// The norm of many tensors together and their scaling down to a limit (bigcn_grad_norm,
// bigcn_clip_grad_norm):
//
//   norm = sqrt(sum over all tensors and elements of g^2),   g' = g min(1, max_norm / norm)
//
// Two kernels: the blocks' sums of squares, and the sums' sum with the scaling, for which every
// block adds all blocks' sums itself, in the same order, so that nothing is counted or waited for.
// The tensors' addresses and lengths go as kernel parameters: nothing is copied to the device and
// a captured call holds what it needs.
//
// Sums. A thread adds the squares of 16 or 32 elements in fp32, and those sums in fp64 (whose
// additions are a sixteenth of the work then; all in fp64 they would bound the kernel). Where a sum of squares
// leaves [2^-80, 2^100], by which single squares may have left fp32's range, it is taken again of
// elements scaled by a power of two.
//
// Bound by memory: every element is read for the norm, read again, from L2 where it is still there,
// and written. 48 matrices of 4096 x 1024 bf16 with their vectors: 201 us (the norm alone 67 at 6.0
// TB/s), 1.2 GB at 5.9 TB/s; a copy's rate would take 179 us, 119 if nothing were read twice. A thread's
// loads of the next chunks ahead, in registers or in a ring in shared memory, and a block's
// chunks strided through memory instead of a run of it gave nothing.
#include <algorithm>
#include <cmath>
#include <cstdlib>

#include "norm.cuh"

namespace bigcn {
namespace {

constexpr int kClipThreads = 256;
constexpr int kClipBlocks = 608;        // of a launch: four an SM; the workspace query asks no device
constexpr int kClipTensors = 960;       // of a launch
constexpr int kFewTensors = 24;         // of a call whose table is a small one
constexpr int kClipMost = 1 << 16;      // of a call
constexpr size_t kClipAlign = 256;
constexpr int64_t kClipKept = int64_t(64) << 20;    // bytes, of the tensors' end, that L2 is to keep

// An element range: `count` elements from `in`, to `out` (nullptr: none). Elements are taken by
// their place in 16-byte pieces of memory (of `in`): chunk c of the tensor holds pieces c kChunk
// .. of those that it touches, its first piece the one that its first element lies in.
constexpr int kChunk = 1024;            // pieces: 16 KB
struct ClipTensor {
    const void *in;
    void *out;
    int64_t count;
    int32_t chunk_end;                  // this and the earlier tensors' chunks
    int32_t dtype;
};
// kTensors: a launch's parameters hold its table. The largest takes 2 us longer to pass than the least (six
// tensors of 92,000 fp32: norm 13 -> 11 us, with the scaling 15 -> 13).
template <int kTensors>
struct ClipTable {
    int n;
    int chunks;                         // of all tensors
    ClipTensor t[kTensors];
};
static_assert(sizeof(ClipTable<kClipTensors>) <= 32000, "kernel parameters");

__host__ __device__ constexpr int64_t clip_chunks(uintptr_t address, int64_t count, int es) {
    const int64_t shift = int64_t(address & 15) / es, V = 16 / es;
    return count == 0 ? 0 : ((shift + count + V - 1) / V + kChunk - 1) / kChunk;
}

// The tensor that chunk c lies in.
template <int kTensors>
__device__ __forceinline__ int tensor_of(const ClipTable<kTensors> &table, int c) {
    int lo = 0, hi = table.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (table.t[mid].chunk_end > c) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Pieces of a chunk that a thread has under way at once.
constexpr int kClipAhead = 4;

// The sum of squares of kAhead pieces, in fp64.
template <typename T>
__device__ __forceinline__ double squares(const uint4 (&w)[kClipAhead]) {
    constexpr int H = kPiece<T> / 2;
    auto sum = [&](float f) {
        float2 s = both(0.0f);
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u) {
            float2 v[H];
            unpack16<T>(w[u], v);
#pragma unroll
            for (int e = 0; e < H; ++e) {
                v[e] = __fmul2_rn(v[e], both(f));
                s = __ffma2_rn(v[e], v[e], s);
            }
        }
        return s.x + s.y;
    };
    const float s = sum(1.0f);
    if (s >= 0x1p-80f && s <= 0x1p100f) return double(s);
    uint32_t any = 0u;
#pragma unroll
    for (int u = 0; u < kClipAhead; ++u) any |= w[u].x | w[u].y | w[u].z | w[u].w;
    if (any == 0u) return 0.0;
    // (A NaN goes the second way and stays one.)
    if (s < 0x1p-80f) return double(sum(0x1p100f)) * 0x1p-200;
    return double(sum(0x1p-70f)) * 0x1p140;
}

// A block's chunks: a run of all, so that what it reads last it can scale first.
struct ClipRun {
    int first, end;
    __device__ __forceinline__ explicit ClipRun(int chunks)
        : first(int(int64_t(chunks) * blockIdx.x / gridDim.x)),
          end(int(int64_t(chunks) * (blockIdx.x + 1) / gridDim.x)) {}
};

// Places of a chunk: its pieces begin at `piece`, of which piece q holds elements (piece + q) V -
// shift + 0 .. V - 1 of the tensor, those within [0, count).
// (kKeep: in L2 as usual. What will not be there any more when the scaling comes to it leaves L2 first: 48
// x 4096 x 1024 bf16 210 -> 202 us, by evict-first loads behind the first 64 MB from the end, of each launch where
// a call has more than one. The norm alone does the same: 400 MB behind a buffer that was just written 94 -> 82 us,
// and the same tensors read again 75 and 77, 96 MB 31 -> 30 and 29 -> 25.)
template <typename T, bool kKeep>
__device__ __forceinline__ uint4 load_place(const T *in, int64_t first, int64_t count) {
    constexpr int V = kPiece<T>;
    if (first >= 0 && first + V <= count) {
        if constexpr (kKeep) return *reinterpret_cast<const uint4 *>(in + first);
        uint64_t policy;
        uint4 v;
        asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "l"(in + first), "l"(policy));
        return v;
    }
    if (first >= count) return make_uint4(0u, 0u, 0u, 0u);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (first + e >= 0 && first + e < count) {
            if constexpr (sizeof(T) == 4) w[e] = reinterpret_cast<const uint32_t *>(in)[first + e];
            else w[e / 2] |= uint32_t(reinterpret_cast<const uint16_t *>(in)[first + e]) << (16 * (e % 2));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void store_place(T *out, int64_t first, int64_t count, uint4 v) {
    constexpr int V = kPiece<T>;
    if (first >= count) return;
    if (first >= 0 && first + V <= count && (reinterpret_cast<uintptr_t>(out + first) & 15) == 0) {
        *reinterpret_cast<uint4 *>(out + first) = v;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (first + e >= 0 && first + e < count) {
            if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(out)[first + e] = w[e];
            else reinterpret_cast<uint16_t *>(out)[first + e] = uint16_t(w[e / 2] >> (16 * (e % 2)));
        }
}

template <typename T, bool kKeep>
__device__ __forceinline__ double chunk_squares(const ClipTensor &t, int64_t piece) {
    constexpr int V = kPiece<T>;
    const T *in = static_cast<const T *>(t.in);
    const int64_t shift = int64_t(reinterpret_cast<uintptr_t>(in) & 15) / int(sizeof(T));
    double total = 0.0;
#pragma unroll 1
    for (int q = threadIdx.x; q < kChunk; q += kClipThreads * kClipAhead) {
        uint4 w[kClipAhead];
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u)
            w[u] = load_place<T, kKeep>(in, (piece + q + u * kClipThreads) * V - shift, t.count);
        total += squares<T>(w);
    }
    return total;
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const ClipTensor &t, int64_t piece, float factor) {
    constexpr int V = kPiece<T>, H = V / 2;
    const T *in = static_cast<const T *>(t.in);
    const int64_t shift = int64_t(reinterpret_cast<uintptr_t>(in) & 15) / int(sizeof(T));
#pragma unroll 1
    for (int q = threadIdx.x; q < kChunk; q += kClipThreads * kClipAhead) {
        uint4 w[kClipAhead];
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u)
            w[u] = load_place<T, false>(in, (piece + q + u * kClipThreads) * V - shift, t.count);
#pragma unroll
        for (int u = 0; u < kClipAhead; ++u) {
            if (factor != 1.0f) {       // (1: the bits as they are)
                float2 v[H];
                unpack16<T>(w[u], v);
#pragma unroll
                for (int e = 0; e < H; ++e) v[e] = __fmul2_rn(v[e], both(factor));
                w[u] = pack16<T>(v);
            }
            store_place<T>(static_cast<T *>(t.out), (piece + q + u * kClipThreads) * V - shift, t.count,
                           w[u]);
        }
    }
}

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFullMask, v, o);
    return v;
}
// The block's sum, for thread 0 or, read from part[0] behind a barrier, for all.
__device__ __forceinline__ double block_sum64(double v, double (&part)[kClipThreads / 32]) {
    v = warp_sum64(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kClipThreads / 32; ++w) s += part[w];
    return s;
}

template <int kTensors>
__global__ void __launch_bounds__(kClipThreads)
norm_kernel(const __grid_constant__ ClipTable<kTensors> table, double *__restrict__ partial) {
    __shared__ double part[kClipThreads / 32];
    const ClipRun run(table.chunks);
    double total = 0.0;
    int at = run.first < run.end ? tensor_of(table, run.first) : 0;
    for (int c = run.first; c < run.end; ++c) {
        while (table.t[at].chunk_end <= c) ++at;
        const ClipTensor &t = table.t[at];
        const int64_t piece = int64_t(c - (at > 0 ? table.t[at - 1].chunk_end : 0)) * kChunk;
        auto add = [&](auto keep) {
            if (t.dtype == BIGCN_F32) total += chunk_squares<float, keep.value>(t, piece);
            else if (t.dtype == BIGCN_BF16) total += chunk_squares<__nv_bfloat16, keep.value>(t, piece);
            else total += chunk_squares<__half, keep.value>(t, piece);
        };
        if (int64_t(run.end - c) * int(gridDim.x) * (kChunk * 16) <= kClipKept) add(std::true_type{});
        else add(std::false_type{});
    }
    total = block_sum64(total, part);
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
    allow_dependent_launch();
}

// The blocks' sums, of one launch or several, added in one order by every block.
__device__ __forceinline__ double all_sums(const double *partial, int n,
                                           double (&part)[kClipThreads / 32]) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kClipThreads) s += __ldcg(partial + i);
    return block_sum64(s, part);
}

// The norm, and (nullable) the sum.
__global__ void __launch_bounds__(kClipThreads)
norm_end_kernel(const double *partial, int n, float *norm, double *sum) {
    __shared__ double part[kClipThreads / 32];
    grid_dependency_wait();
    const double s = all_sums(partial, n, part);
    if (threadIdx.x == 0) {
        *norm = float(sqrt(s));
        if (sum) *sum = s;
    }
}

template <int kTensors>
__global__ void __launch_bounds__(kClipThreads)
clip_kernel(const __grid_constant__ ClipTable<kTensors> table, const double *partial, int n,
            double max_norm, float *norm, bool in_place) {
    __shared__ double part[kClipThreads / 32];
    grid_dependency_wait();
    const double root = sqrt(all_sums(partial, n, part));
    const float root32 = float(root);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = root32;
    // A norm that is no number leaves the tensors as they are.
    const bool over = isfinite(root32) && double(root32) > max_norm;
    if (!over && in_place) return;
    const float factor = over ? float(max_norm / root) : 1.0f;
    const ClipRun run(table.chunks);
    int at = run.first < run.end ? tensor_of(table, run.end - 1) : 0;
    for (int c = run.end - 1; c >= run.first; --c) {
        while (at > 0 && table.t[at - 1].chunk_end > c) --at;
        const ClipTensor &t = table.t[at];
        const int64_t piece = int64_t(c - (at > 0 ? table.t[at - 1].chunk_end : 0)) * kChunk;
        if (t.dtype == BIGCN_F32) chunk_scale<float>(t, piece, factor);
        else if (t.dtype == BIGCN_BF16) chunk_scale<__nv_bfloat16>(t, piece, factor);
        else chunk_scale<__half>(t, piece, factor);
    }
}

struct Range {
    uintptr_t begin, end;
};

// Checks a call's tensors; out nullptr: in place or none.
bigcn_status check_tensors(int32_t n, const int32_t *dtypes, const void *const *in,
                           void *const *out, const int64_t *counts, const float *norm,
                           const void *workspace, size_t ws_bytes) {
    if (n < 0 || n > kClipMost || !norm || !workspace || (n > 0 && (!dtypes || !in || !counts)) ||
        ws_bytes < bigcn_grad_norm_workspace_bytes(n))
        return BIGCN_ERR_INVALID_ARG;
    int64_t chunks = 0;
    bool aligned = aligned_to(norm, 4) && aligned_to(workspace, kClipAlign);
    for (int32_t i = 0; i < n; ++i) {
        const size_t es = dtype_bytes(dtypes[i]);
        if (es == 0 || counts[i] < 0 || counts[i] > kMaxElems / 8) return BIGCN_ERR_INVALID_ARG;
        if (counts[i] == 0) continue;
        if (!in[i] || (out && !out[i])) return BIGCN_ERR_INVALID_ARG;
        chunks += clip_chunks(reinterpret_cast<uintptr_t>(in[i]), counts[i], int(es));
        if (chunks > INT32_MAX) return BIGCN_ERR_INVALID_ARG;
        aligned = aligned && aligned_to(in[i], es) && (!out || aligned_to(out[i], es));
    }
    if (!aligned) return BIGCN_ERR_MISALIGNED;
    // Nothing that is written may overlap anything else: sorted, no range reaches the next. (A
    // tensor listed twice counts twice in the norm; to scale it twice is refused.) Tensors that are
    // read only may overlap each other.
    const int64_t most = 2 * int64_t(n) + 2;
    Range *r = static_cast<Range *>(std::malloc(size_t(most) * sizeof(Range)));
    if (!r) return BIGCN_ERR_INVALID_ARG;
    int64_t m = 0;
    auto add = [&](const void *p, size_t bytes) {
        if (bytes > 0) r[m++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes};
    };
    auto apart = [&] {
        const auto less = [](const Range &a, const Range &b) { return a.begin < b.begin; };
        if (!std::is_sorted(r, r + m, less)) std::sort(r, r + m, less);
        for (int64_t i = 1; i < m; ++i)
            if (r[i].begin < r[i - 1].end) return false;
        return true;
    };
    const size_t wsb = bigcn_grad_norm_workspace_bytes(n);
    add(norm, 4);
    add(workspace, wsb);
    bool ok = true;
    if (out) {
        for (int32_t i = 0; i < n; ++i) add(out[i], size_t(counts[i]) * dtype_bytes(dtypes[i]));
        ok = apart();
        // Each read range against the written ones, sorted: the last that begins before its end.
        for (int32_t i = 0; ok && i < n; ++i) {
            const size_t bytes = size_t(counts[i]) * dtype_bytes(dtypes[i]);
            if (bytes == 0 || in[i] == out[i]) continue;
            const uintptr_t begin = reinterpret_cast<uintptr_t>(in[i]), end = begin + bytes;
            const Range *next = std::lower_bound(
                r, r + m, end, [](const Range &a, uintptr_t e) { return a.begin < e; });
            ok = next == r || next[-1].end <= begin;
        }
    } else {
        ok = apart();
        for (int32_t i = 0; ok && i < n; ++i) {
            const size_t bytes = size_t(counts[i]) * dtype_bytes(dtypes[i]);
            ok = !overlaps(in[i], bytes, norm, 4) && !overlaps(in[i], bytes, workspace, wsb);
        }
    }
    std::free(r);
    return ok ? BIGCN_OK : BIGCN_ERR_INVALID_ARG;
}

int clip_grid(int chunks) { return chunks < kClipBlocks ? chunks : kClipBlocks; }

// The tables of a call, one after the other: `launch` gets each.
template <int kTensors, typename Launch>
void each_table(int32_t n, const int32_t *dtypes, const void *const *in, void *const *out,
                const int64_t *counts, Launch launch) {
    ClipTable<kTensors> table;
    int32_t i = 0;
    do {
        table.n = table.chunks = 0;
        for (; i < n && table.n < kTensors; ++i) {
            if (counts[i] == 0) continue;
            table.chunks += int(clip_chunks(reinterpret_cast<uintptr_t>(in[i]), counts[i],
                                            int(dtype_bytes(dtypes[i]))));
            table.t[table.n++] = {in[i], out ? out[i] : nullptr, counts[i], table.chunks, dtypes[i]};
        }
        if (table.n > 0) launch(table);
    } while (i < n);
}

// The sums of squares of all blocks of all launches: how many, from `partial` on.
template <int kTensors>
int launch_sums(int32_t n, const int32_t *dtypes, const void *const *in, const int64_t *counts,
                double *partial, cudaStream_t s) {
    int sums = 0;
    each_table<kTensors>(n, dtypes, in, nullptr, counts, [&](const ClipTable<kTensors> &table) {
        const int grid = clip_grid(table.chunks);
        norm_kernel<kTensors><<<unsigned(grid), kClipThreads, 0, s>>>(table, partial + sums);
        sums += grid;
    });
    return sums;
}

template <int kTensors>
void launch_clip(int32_t n, const int32_t *dtypes, const void *const *in, void *const *out,
                 const int64_t *counts, float max_norm, float *norm, double *partial, cudaStream_t s) {
    int sums = launch_sums<kTensors>(n, dtypes, in, counts, partial, s);
    if (sums == 0 || n > kTensors) {            // several launches' sums are added once for all
        double *sum = partial + sums;
        launch_kernel(norm_end_kernel, dim3(1), dim3(kClipThreads), 0, s, true, dim3(1, 1, 1), partial,
                      sums, norm, sum);
        partial = sum;
        sums = 1;
    }
    bool in_place = true;
    for (int32_t i = 0; i < n; ++i) in_place = in_place && (counts[i] == 0 || in[i] == out[i]);
    bool pdl = true;
    each_table<kTensors>(n, dtypes, in, out, counts, [&](const ClipTable<kTensors> &table) {
        launch_kernel(clip_kernel<kTensors>, dim3(unsigned(clip_grid(table.chunks))), dim3(kClipThreads),
                      0, s, pdl, dim3(1, 1, 1), table, partial, sums, double(max_norm), norm, in_place);
        pdl = false;
    });
}

}  // namespace
}  // namespace bigcn

using namespace bigcn;

extern "C" size_t bigcn_grad_norm_workspace_bytes(int32_t n) {
    if (n < 0 || n > kClipMost) return 0;
    // The blocks' sums of a launch for every kClipTensors tensors, and the sum of those.
    const size_t launches = (size_t(n) + kClipTensors - 1) / kClipTensors;
    return ((launches * kClipBlocks + 1) * sizeof(double) + kClipAlign - 1) / kClipAlign * kClipAlign;
}

extern "C" bigcn_status bigcn_grad_norm(int32_t n, const int32_t *dtypes, const void *const *tensors,
                                        const int64_t *counts, float *norm, void *workspace,
                                        size_t ws_bytes, void *stream) {
    const bigcn_status ok =
        check_tensors(n, dtypes, tensors, nullptr, counts, norm, workspace, ws_bytes);
    if (ok != BIGCN_OK) return ok;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    double *partial = static_cast<double *>(workspace);
    const int sums = n <= kFewTensors ? launch_sums<kFewTensors>(n, dtypes, tensors, counts, partial, s)
                                      : launch_sums<kClipTensors>(n, dtypes, tensors, counts, partial, s);
    launch_kernel(norm_end_kernel, dim3(1), dim3(kClipThreads), 0, s, true, dim3(1, 1, 1), partial, sums,
                  norm, nullptr);
    return launch_status();
}

extern "C" bigcn_status bigcn_clip_grad_norm(int32_t n, const int32_t *dtypes,
                                             const void *const *tensors, void *const *out,
                                             const int64_t *counts, float max_norm, float *norm,
                                             void *workspace, size_t ws_bytes, void *stream) {
    if (!(max_norm >= 0.0f) || (n > 0 && !out)) return BIGCN_ERR_INVALID_ARG;
    const bigcn_status ok = check_tensors(n, dtypes, tensors, out, counts, norm, workspace, ws_bytes);
    if (ok != BIGCN_OK) return ok;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;
    const cudaStream_t s = as_stream(stream);
    double *partial = static_cast<double *>(workspace);
    const auto launch = n <= kFewTensors ? launch_clip<kFewTensors> : launch_clip<kClipTensors>;
    launch(n, dtypes, tensors, out, counts, max_norm, norm, partial, s);
    return launch_status();
}
