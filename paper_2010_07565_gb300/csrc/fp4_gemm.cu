// The product of two matrices of microscaled 4-bit rows (bigcn_fp4_gemm), Z = A B^T + bias, on the
// tensor cores: tcgen05 block-scaled e2m1 x e2m1 with a ue8m0 scale per 32 columns of either
// operand, fp32 accumulators in tensor memory. Codes go by tensor copies from memory into their
// swizzled places (128 bytes, 256 columns, of a row a stage). The scale bytes, four groups to a word,
// go by way of registers to where the tensor core's copy into tensor memory wants them: of 128
// rows, row r at word (r mod 32) 4 + r / 32, so a lane's words of rows lane, lane + 32, ... are 16 bytes.
//
// Roles of a CTA (12 warps), which takes tiles of 128 rows by NT columns in turn: warp 0 copies the
// codes, warps 2 and 3 bring A's and B's scale bytes, 16 groups (two stages) of a row at a time and
// asked for several such units ahead, warp 1 issues the MMAs, warps 4-11 take the sums out, each every
// second 32 columns of the 32 rows that it may read. They meet on mbarriers only:
//   full[stage]   its copies have landed        empty[stage]  its MMAs are done
//   summed[acc]   a tile's MMAs are done        taken[acc]    its sums were taken
#include "fp4.cuh"
#include "launch.cuh"
#include "tc_rows.cuh"
#include "tensor_map.cuh"

namespace bigcn {

__device__ unsigned int g_fp4_timeouts;

namespace {

constexpr int kGemmThreads = 384;
constexpr int kOutWarps = 8;            // that take the sums out
constexpr int kUnit = 16;               // groups whose scale bytes are loaded at a time: two stages'
constexpr int kTmemCols = 512;
constexpr int kScaleChunk = 512;        // bytes: a word of scales of 128 rows
constexpr int kMaxGemmCols = 1 << 15;   // K: at most 512 accumulating MMAs (see the header)

template <int NT>
struct Fp4Shape {
    static constexpr int kA = kUmmaM * 128, kB = NT * 128;
    static constexpr int kChunks = NT > 128 ? NT / 128 : 1;         // of B's scales
    static constexpr int kScales = 2 * (1 + kChunks) * kScaleChunk;
    static constexpr int kStage = kA + kB + kScales;
    static constexpr int kStages = NT >= 256 ? 3 : NT >= 128 ? 5 : NT >= 64 ? 6 : 7;
    static constexpr int kStaging = kOutWarps * 32 * 33 * 4;
    static constexpr int kRowsB = (NT + 31) / 32;                   // rows of B a lane of its scale warp has
    static constexpr int kAheadA = 6, kAheadB = 3;                  // units of scale bytes in flight
    static constexpr int kRings = (kAheadA * 4 + kAheadB * kRowsB) * 512;
    static constexpr int kSmem = 1024 + kStages * kStage + kStaging + kRings;
    static constexpr int kAccs = NT > 128 ? 1 : 2;
    static constexpr int kScaleCols = 8 * (1 + kChunks);            // of tensor memory, a stage
    static_assert(kStage % 1024 == 0, "swizzled tiles start on 1024 bytes");
    static_assert(kSmem <= 227 * 1024 - 1024, "shared memory per CTA");
    static_assert(kAccs * NT + kStages * kScaleCols <= kTmemCols, "tensor memory per CTA");
};

struct Fp4GemmArgs {
    CUtensorMap a_map, b_map;
    const uint8_t *a_exps, *b_exps;
    int64_t lda_e, ldb_e;
    int64_t N;
    int F;
    int groups;              // of 32 columns
    int nt;                  // column tiles
    int64_t tiles;
    const float *bias;       // nullable
    void *Z;
    int64_t ldz;
};

// Instruction descriptor of the block-scaled product: e2m1 x e2m1, both K-major, ue8m0 scales, M =
// 128, N = n; the scales of a 64-column step are bytes id and id + 1 of their words.
__device__ __forceinline__ uint32_t fp4_idesc(int n, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | (uint32_t(n >> 3) << 17) | (1u << 23) |
           (uint32_t(kUmmaM >> 4) << 24) | (id << 29);
}
__device__ __forceinline__ void mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                        uint32_t a_scales, uint32_t b_scales, bool accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %6, 0;\n"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], "
        "p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(a_scales), "r"(b_scales), "r"(accumulate ? 1u : 0u));
}
// 512 bytes, 32 rows of 16, to four columns of tensor memory, the same in each quarter of its lanes.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t saddr) {
    uint64_t d = uint64_t((saddr >> 4) & 0x3FFFu);
    d |= uint64_t(128 >> 4) << 32;              // groups of 8 rows 128 bytes apart, no swizzle
    d |= uint64_t(1) << 46;
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(d));
}

// A warp's 32 rows by 32 columns of sums from shared memory (pitch 33) to Z, with the bias: a row
// at a time in fp32, two in 16 bits, where `pairs` says that two columns are one aligned word.
template <typename T>
__device__ __forceinline__ void store_sums(const float *stage, T *z, int64_t ldz, int rows, int cols,
                                           const float *bias, int lane, bool pairs) {
    if constexpr (sizeof(T) == 4) {
        const float b = bias && lane < cols ? __ldg(bias + lane) : 0.0f;
        T *to = z + lane;
        if (lane >= cols) return;
        if (rows == 32) {
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 16) {
                float v[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) v[r] = stage[(r0 + r) * 33 + lane] + b;
#pragma unroll
                for (int r = 0; r < 16; ++r, to += ldz) *to = v[r];
            }
        } else {
            for (int r = 0; r < rows; ++r, to += ldz) *to = stage[r * 33 + lane] + b;
        }
    } else {
        const int c = 2 * (lane & 15), r0 = lane >> 4;
        const bool first = c < cols, second = c + 1 < cols;
        const float b0 = bias && first ? __ldg(bias + c) : 0.0f;
        const float b1 = bias && second ? __ldg(bias + c + 1) : 0.0f;
        T *to = z + r0 * ldz + c;
        if (!first) return;
#pragma unroll 8
        for (int r = r0; r < 32; r += 2, to += 2 * ldz) {
            if (r >= rows) break;
            const float v0 = stage[r * 33 + c] + b0, v1 = stage[r * 33 + c + 1] + b1;
            if (pairs && second) {
                uint32_t w;
                if constexpr (std::is_same<T, __half>::value) {
                    const __half2 x = __floats2half2_rn(v0, v1);
                    w = *reinterpret_cast<const uint32_t *>(&x);
                } else {
                    const __nv_bfloat162 x = __floats2bfloat162_rn(v0, v1);
                    w = *reinterpret_cast<const uint32_t *>(&x);
                }
                *reinterpret_cast<uint32_t *>(to) = w;
            } else {
                to[0] = from_f32<T>(v0);
                if (second) to[1] = from_f32<T>(v1);
            }
        }
    }
}

// Asks for the scale bytes of unit u (16 groups) of the rows row0 + lane, + 32, ...: four words a row,
// zeros behind the last group and the last row, whatever memory holds there, to `to` + 512 j.
// `wide`: rows aligned to 16 bytes.
template <int R>
__device__ __forceinline__ void copy_unit(uint32_t to, const uint8_t *exps, int64_t ld, int64_t row0,
                                          int64_t rows, int groups, int u, int lane, bool wide) {
    const int left = groups - u * kUnit;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int64_t i = row0 + 32 * j + lane;
        const bool in = i < rows;
        const uint8_t *p = exps + (in ? i * ld + u * kUnit : 0);
        const uint32_t at = to + uint32_t(j * 512);
        if (wide) {
            const uint32_t n = in ? uint32_t(min(left, 16)) : 0u;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(p), "r"(n)
                         : "memory");
        } else {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int n = in ? min(max(left - 4 * h, 0), 4) : 0;
                copy4(at + uint32_t(4 * h), n > 0 ? p + 4 * h : exps, uint32_t(n));
            }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
// Word h of stage `half` of a unit, of rows lane, lane + 32, ...: 16 bytes for each 128 rows.
template <int R>
__device__ __forceinline__ void store_scales(uint32_t to, const uint4 (&w)[R], int half, int lane) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < (R + 3) / 4; ++c) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (4 * c + j < R) {
                    const uint4 &x = w[4 * c + j < R ? 4 * c + j : 0];
                    v[j] = half ? (h ? x.w : x.z) : (h ? x.y : x.x);
                } else {
                    v[j] = 0u;
                }
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                             to + uint32_t((h * ((R + 3) / 4) + c) * kScaleChunk + lane * 16)),
                         "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                         : "memory");
        }
}

// Tile t: its first row and first column.
struct Tile {
    int64_t m0;
    int n0;
    __device__ __forceinline__ Tile(int64_t t, int nt, int NT) {
        if (t >> 32 == 0) {
            const uint32_t m = uint32_t(t) / uint32_t(nt);
            m0 = int64_t(m) * kUmmaM;
            n0 = int(uint32_t(t) - m * uint32_t(nt)) * NT;
        } else {
            m0 = t / nt * kUmmaM;
            n0 = int(t % nt) * NT;
        }
    }
};

// A scale warp's work: R rows a lane, chunks from `offset` of a stage on. Each lane has a ring of its own
// of kAhead units, which it alone fills (by asynchronous copies, kAhead - 1 units ahead) and reads.
template <int NT, int R, int kAhead>
__device__ __forceinline__ void bring_scales(const Fp4GemmArgs &p, bool a, uint32_t base, uint32_t offset,
                                             uint32_t ring,
                                             const uint64_t *empty, const uint64_t *full,
                                             volatile uint32_t *stopv, int stages, int lane) {
    using S = Fp4Shape<NT>;
    const uint8_t *exps = a ? p.a_exps : p.b_exps;
    const int64_t rows = a ? p.N : p.F, ld = a ? p.lda_e : p.ldb_e;
    const bool wide = (reinterpret_cast<uintptr_t>(exps) & 15) == 0 && ld % 16 == 0;
    const int units = (stages + 1) / 2;
    int64_t t_next = blockIdx.x;
    int u_next = 0, slot_next = 0;
    const uint32_t own = ring + uint32_t(lane * 16);
    auto ask = [&] {
        if (t_next < p.tiles) {
            const Tile tile(t_next, p.nt, NT);
            copy_unit<R>(own + uint32_t(slot_next * R * 512), exps, ld, a ? tile.m0 : tile.n0, rows,
                         p.groups, u_next, lane, wide);
            if (++u_next == units) u_next = 0, t_next += gridDim.x;
        } else {
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        if (++slot_next == kAhead) slot_next = 0;
    };
#pragma unroll 1
    for (int i = 0; i < kAhead - 1; ++i) ask();
    int s = 0, u = 0, slot = 0;
    uint32_t parity = 1u;
    for (int64_t t = blockIdx.x; t < p.tiles;) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 2) : "memory");
        uint4 w[R];
#pragma unroll
        for (int j = 0; j < R; ++j)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[j].x), "=r"(w[j].y), "=r"(w[j].z), "=r"(w[j].w)
                         : "r"(own + uint32_t((slot * R + j) * 512))
                         : "memory");
        if (++slot == kAhead) slot = 0;
        ask();
        const int n = min(2, stages - 2 * u);
        if (++u == units) u = 0, t += gridDim.x;
        for (int half = 0; half < n; ++half) {
            if (!__all_sync(kFullMask, wait_unless(smem_addr(&empty[s]), parity, stopv))) {
                *stopv = 1u;
                t = p.tiles;
                break;
            }
            store_scales<R>(base + uint32_t(s * S::kStage) + offset, w, half, lane);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&full[s]));
            if (++s == S::kStages) s = 0, parity ^= 1u;
        }
    }
    // What is still in flight lands before the shared memory is given up.
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int NT>
__global__ void __launch_bounds__(kGemmThreads, 1)
fp4_gemm_kernel(const __grid_constant__ Fp4GemmArgs p) {
    using S = Fp4Shape<NT>;
    constexpr int kStages = S::kStages;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], summed[S::kAccs], taken[S::kAccs],
        done;
    __shared__ uint32_t tmem_base, stop;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;

    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_addr(&tmem_base)),
                     "r"(kTmemCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&full[s]), 3);          // both scale warps; the boxes' bytes
            mbar_init(smem_addr(&empty[s]), 1);
        }
        for (int b = 0; b < S::kAccs; ++b) {
            mbar_init(smem_addr(&summed[b]), 1);
            mbar_init(smem_addr(&taken[b]), kOutWarps);
        }
        mbar_init(smem_addr(&done), 1);
        stop = 0u;
        mbar_fence_init();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    volatile uint32_t *const stopv = &stop;
    const int stages = (p.groups + 7) / 8;              // of a tile
    const uint32_t rings = base + uint32_t(kStages * S::kStage + S::kStaging);

    if (warp == 0) {
        // Copies into the ring of stages.
        int s = 0, issued = 0;
        uint32_t parity = 1u;
        bool ok = true;
        for (int64_t t = blockIdx.x; ok && t < p.tiles; t += gridDim.x) {
            const Tile tile(t, p.nt, NT);
            for (int st = 0; st < stages; ++st) {
                if (!__all_sync(kFullMask, wait_unless(smem_addr(&empty[s]), parity, stopv))) {
                    *stopv = 1u;
                    ok = false;
                    break;
                }
                const uint32_t at = base + uint32_t(s * S::kStage), bar = smem_addr(&full[s]);
                if (elect_one()) {
                    mbar_expect(bar, S::kA + S::kB);
                    tma_load(at, &p.a_map, st * 128, int(tile.m0), bar);
                    tma_load(at + S::kA, &p.b_map, st * 128, tile.n0, bar);
                }
                __syncwarp();
                ++issued;
                if (++s == kStages) s = 0, parity ^= 1u;
            }
        }
        // What is still in flight lands before the shared memory is given up.
        for (int it = issued > kStages ? issued - kStages : 0; it < issued; ++it)
            mbar_wait(smem_addr(&full[it % kStages]), uint32_t(it / kStages) & 1u);
    } else if (warp == 2) {
        bring_scales<NT, 4, S::kAheadA>(p, true, base, S::kA + S::kB, rings, empty, full, stopv, stages, lane);
    } else if (warp == 3) {
        bring_scales<NT, S::kRowsB, S::kAheadB>(p, false, base, S::kA + S::kB + 2 * kScaleChunk,
                                                rings + S::kAheadA * 4 * 512, empty, full, stopv, stages,
                                                lane);
    } else if (warp == 1) {
        // The warp stays together, one lane issues.
        int s = 0, b = 0;
        uint32_t parity = 0u, acc_parity = 1u;
        bool any = false, ok = true;
        for (int64_t t = blockIdx.x; ok && t < p.tiles; t += gridDim.x) {
            const int n = (min(NT, p.F - Tile(t, p.nt, NT).n0) + 31) / 32 * 32;
            const uint32_t acc = tmem + uint32_t(b * NT);
            ok = __all_sync(kFullMask, wait_unless(smem_addr(&taken[b]), acc_parity, stopv));
            for (int st = 0; ok && st < stages; ++st) {
                ok = __all_sync(kFullMask, wait_unless(smem_addr(&full[s]), parity, stopv));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = base + uint32_t(s * S::kStage);
                const uint32_t scales = at + S::kA + S::kB;
                // A stage has columns of tensor memory of its own: its MMAs have ended when it is
                // filled again.
                const uint32_t sa = tmem + uint32_t(S::kAccs * NT + s * S::kScaleCols), sb = sa + 8;
                const uint64_t da = sw128_desc(at), db = sw128_desc(at + S::kA);
                const int steps = min(4, (p.groups - st * 8 + 1) / 2);
                if (elect_one()) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        copy_scales(sa + uint32_t(4 * h), scales + uint32_t(h * kScaleChunk));
#pragma unroll
                        for (int c = 0; c < S::kChunks; ++c)
                            copy_scales(sb + uint32_t(4 * (h * S::kChunks + c)),
                                        scales + uint32_t((2 + h * S::kChunks + c) * kScaleChunk));
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k >= steps) break;
                        mma_fp4(acc, da + uint32_t(2 * k), db + uint32_t(2 * k),
                                fp4_idesc(n, uint32_t(k % 2) * 2u), sa + uint32_t(4 * (k / 2)),
                                sb + uint32_t(4 * S::kChunks * (k / 2)), st > 0 || k > 0);
                    }
                    mma_commit(smem_addr(&empty[s]));
                    if (st == stages - 1) mma_commit(smem_addr(&summed[b]));
                }
                __syncwarp();
                any = true;
                if (++s == kStages) s = 0, parity ^= 1u;
            }
            if (++b == S::kAccs) b = 0, acc_parity ^= 1u;
        }
        if (!ok) *stopv = 1u;
        if (elect_one()) {
            if (any) mma_commit(smem_addr(&done));
            else mbar_arrive(smem_addr(&done));
        }
        __syncwarp();
    } else {
        // Sums out, a warp the 32 lanes of tensor memory that it may read, every second 32 columns.
        // Tiles whose waits ran out are NaN.
        const int quad = warp & 3, half = (warp - 4) >> 2;
        float *const stage = reinterpret_cast<float *>(smem_raw + (base - raw) + kStages * S::kStage) +
                             (warp - 4) * 32 * 33;
        const bool pairs = sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(p.Z) & 3) == 0 &&
                           p.ldz % 2 == 0;
        int b = 0;
        uint32_t parity = 0u;
        bool ok = true;
        for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
            const Tile tile(t, p.nt, NT);
            const int64_t row0 = tile.m0 + 32 * quad;
            const int cols = min(NT, p.F - tile.n0);
            const int rows = int(min(int64_t(32), max(int64_t(0), p.N - row0)));
            if (ok) {
                ok = __all_sync(kFullMask, wait_unless(smem_addr(&summed[b]), parity, stopv));
                if (!ok) *stopv = 1u;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + (uint32_t(32 * quad) << 16) + uint32_t(b * NT);
            T *z = static_cast<T *>(p.Z) + row0 * p.ldz + tile.n0;
            const float *bias = p.bias ? p.bias + tile.n0 : nullptr;
#pragma unroll 1
            for (int c = 32 * half; c < cols; c += 64) {
                uint32_t v[32];
                tmem_ld32(acc + uint32_t(c), v);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    stage[lane * 33 + e] = __uint_as_float(ok ? v[e] : 0x7FC00000u);
                __syncwarp();
                store_sums<T>(stage, z + c, p.ldz, rows, cols - c, bias ? bias + c : nullptr, lane, pairs);
                __syncwarp();
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&taken[b]));
            if (++b == S::kAccs) b = 0, parity ^= 1u;
        }
    }

    // Every MMA has ended once `done` completes.
    const bool ended = mbar_wait(smem_addr(&done), 0u);
    if (__syncthreads_or(!ended || *stopv != 0u) && tid == 0) atomicAdd(&g_fp4_timeouts, 1u);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                     "r"(kTmemCols));
}

template <typename T, int NT>
void launch_nt(const Fp4GemmArgs &p, unsigned grid, cudaStream_t s) {
    using S = Fp4Shape<NT>;
    cudaFuncSetAttribute(fp4_gemm_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    fp4_gemm_kernel<T, NT><<<grid, kGemmThreads, S::kSmem, s>>>(p);
}

template <typename T>
void launch_gemm(const Fp4GemmArgs &p, int NT, unsigned grid, cudaStream_t s) {
    if (NT == 256) launch_nt<T, 256>(p, grid, s);
    else if (NT == 128) launch_nt<T, 128>(p, grid, s);
    else if (NT == 64) launch_nt<T, 64>(p, grid, s);
    else launch_nt<T, 32>(p, grid, s);
}

}  // namespace

uint32_t take_fp4_timeouts() {
    unsigned int n = 0;
    const unsigned int zero = 0;
    if (cudaMemcpyFromSymbol(&n, g_fp4_timeouts, sizeof(n)) != cudaSuccess ||
        cudaMemcpyToSymbol(g_fp4_timeouts, &zero, sizeof(zero)) != cudaSuccess) {
        cudaGetLastError();
        return ~0u;
    }
    return n;
}

}  // namespace bigcn

using namespace bigcn;

extern "C" bigcn_status bigcn_fp4_gemm(int32_t dtype, const uint8_t *aq, int64_t ldaq,
                                       const uint8_t *a_exps, int64_t ldae, int64_t N,
                                       const uint8_t *bq, int64_t ldbq, const uint8_t *b_exps,
                                       int64_t ldbe, int32_t F, int32_t K, const float *bias, void *Z,
                                       int64_t ldz, void *stream) {
    const size_t es = dtype_bytes(dtype);
    if (es == 0 || N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxGemmCols || F < 1 ||
        F > kMaxCols || ldz < F || !fp4_strides_ok(N, K, ldaq, ldae) ||
        !fp4_strides_ok(F, K, ldbq, ldbe) || (N > 0 && N > kMaxElems / ldz))
        return BIGCN_ERR_INVALID_ARG;
    if (N == 0) return BIGCN_OK;
    if (!aq || !a_exps || !bq || !b_exps || !Z) return BIGCN_ERR_INVALID_ARG;
    if (!checkpoint_aligned(aq, a_exps) || !checkpoint_aligned(bq, b_exps) || !aligned_to(Z, es) ||
        (bias && !aligned_to(bias, 4)))
        return BIGCN_ERR_MISALIGNED;
    const void *in[] = {aq, a_exps, bq, b_exps, bias};
    const size_t inb[] = {fp4_q_span(N, K, ldaq), checkpoint_exps_span(N, K, ldae),
                          fp4_q_span(F, K, ldbq), checkpoint_exps_span(F, K, ldbe), size_t(F) * 4};
    for (int p = 0; p < 5; ++p)
        if (overlaps(Z, span_bytes(N, F, ldz, es), in[p], inb[p])) return BIGCN_ERR_INVALID_ARG;
    DeviceInfo dev;
    const bigcn_status st = current_device(&dev);
    if (st != BIGCN_OK) return st;

    const int64_t mt = (N + kUmmaM - 1) / kUmmaM;
    // Tiles of 256 columns read A once for twice as many, but leave no room for a second accumulator:
    // only where the MMAs of a tile are long beside taking its sums out.
    int NT = F > 128 && K > 2048 ? 256 : F > 64 ? 128 : F > 32 ? 64 : 32;
    while (NT > 32 && mt * ((F + NT - 1) / NT) * 2 <= dev.sm_count) NT /= 2;
    Fp4GemmArgs p;
    p.groups = int(checkpoint_groups(K));
    const int64_t width = int64_t(p.groups) * 16;
    if (!encode_map(&p.a_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, aq, width, N, N > 1 ? ldaq : width, 128,
                    kUmmaM, true) ||
        !encode_map(&p.b_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, bq, width, F, F > 1 ? ldbq : width, 128,
                    NT, true))
        return BIGCN_ERR_CUDA;
    p.a_exps = a_exps;
    p.b_exps = b_exps;
    p.lda_e = ldae;
    p.ldb_e = ldbe;
    p.N = N;
    p.F = F;
    p.nt = (F + NT - 1) / NT;
    p.tiles = mt * p.nt;
    p.bias = bias;
    p.Z = Z;
    p.ldz = ldz;
    const unsigned grid = unsigned(p.tiles < dev.sm_count ? p.tiles : dev.sm_count);
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32) launch_gemm<float>(p, NT, grid, s);
    else if (dtype == BIGCN_BF16) launch_gemm<__nv_bfloat16>(p, NT, grid, s);
    else launch_gemm<__half>(p, NT, grid, s);
    return launch_status();
}
