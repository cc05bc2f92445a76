// The product of two matrices of microscaled 4-bit rows (bigcn_fp4_gemm), Z = A B^T + bias, on the
// tensor cores: tcgen05 block-scaled e2m1 x e2m1 with a ue8m0 scale per 32 columns of either
// operand, fp32 accumulators in tensor memory. Codes go by tensor copies from memory into their
// swizzled places (128 bytes, 256 columns, of a row a stage). The scale bytes, four groups to a word,
// go to tensor memory as the MMAs read them: of 128 rows, row r's word in column r / 32 and in lane r
// mod 32 of each quarter of the lanes, written by a warp of each quarter.
//
// Roles of a CTA (16 warps), which takes tiles of 128 rows by NT columns in turn: warp 0 copies the
// codes; warps 2 and 3 ask for A's and B's scale bytes, a unit of 16 groups (two stages) of a row at a
// time and several units ahead; warps 12-15 put them into tensor memory; warp 1 issues the MMAs; warps
// 4-11 take the sums out, each kBatch columns at a time of the 32 rows that it may read. They
// meet on mbarriers only:
//   full[stage]    its codes have landed         empty[stage]    its MMAs are done
//   loaded[slot]   a unit's scale bytes landed   freed[slot]     they were read
//   filled[unit]   they are in tensor memory     used[unit]      the unit's MMAs are done
//   summed[acc]    a tile's MMAs are done        taken[acc]      its sums were taken
// (By way of shared memory, places filled by the threads that had asked for the bytes, each unit cost 1500
// cycles: the fence before the tensor core's own copy waits for all that its thread still has under way.)
#include "fp4.cuh"
#include "launch.cuh"
#include "tc_rows.cuh"
#include "tensor_map.cuh"

namespace bigcn {

__device__ unsigned int g_fp4_timeouts;

namespace {

constexpr int kOutWarps = 8;            // that take the sums out
constexpr int kUnit = 16;               // groups whose scale bytes are brought at a time: two stages'
constexpr int kUnits = 4;               // of scale bytes in tensor memory
constexpr int kSlots = 6;               // units of scale bytes on their way or in shared memory
constexpr int kTmemCols = 512;
constexpr int kGemmThreads = 512;
constexpr int kMaxGemmCols = 1 << 15;   // K: at most 512 accumulating MMAs (see the header)

template <int NT>
struct Fp4Shape {
    static constexpr int kA = kUmmaM * 128, kB = NT * 128;
    static constexpr int kStage = kA + kB;
    static constexpr int kStages = NT >= 256 ? 3 : NT >= 128 ? 4 : NT >= 64 ? 5 : 6;
    static constexpr int kRowsB = NT / 32;                          // a lane of B's scales has
    static constexpr int kChunks = NT > 128 ? NT / 128 : 1;         // of 128 rows of B
    static constexpr int kSlot = (4 + kRowsB) * 512;                // 16 bytes of each row
    static constexpr int kScaleCols = 16 * (1 + kChunks);           // of tensor memory, a unit
    // Columns that a warp stages at a time, and words from one staged row to the next: accesses of 4, 8
    // and 16 bytes of a lane's row, or of a row by neighbouring lanes, then fall into different banks.
    static constexpr int kBatch = NT >= 256 ? 32 : NT >= 64 ? 64 : 32;
    static constexpr int kPitch = kBatch + 4;
    static constexpr int kStaging = kOutWarps * 32 * kPitch * 4;
    static constexpr int kSmem = 1024 + kStages * kStage + kStaging + kSlots * kSlot;
    static constexpr int kAccs = NT > 128 ? 1 : 2;
    static_assert(kStage % 1024 == 0, "swizzled tiles start on 1024 bytes");
    static_assert(kSmem <= 227 * 1024 - 1024, "shared memory per CTA");
    static_assert(kAccs * NT + kUnits * kScaleCols <= kTmemCols, "tensor memory per CTA");
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
    int vec;                 // bytes that Z and its rows are aligned to, at most 16
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
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

// A warp's rows of sums, kBatch columns from shared memory to Z, with the bias: VB bytes of a row a lane
// (Z's rows are aligned to them), neighbouring lanes along the row.
template <typename T, int kBatch, int VB>
__device__ __forceinline__ void store_sums(const float *stage, T *z, int64_t ldz, int rows, int cols,
                                           const float *bias, int lane) {
    constexpr int kPitch = kBatch + 4, kCols = VB / int(sizeof(T));
    constexpr int kLanes = kBatch / kCols < 32 ? kBatch / kCols : 32;       // of a row
    constexpr int kParts = kBatch / kCols / kLanes, kRows = 32 / kLanes;
    const int r0 = lane / kLanes, c0 = lane % kLanes * kCols;
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
        const int c = c0 + part * kLanes * kCols, n = cols - c;
        if (n <= 0) continue;
        float b[kCols];
#pragma unroll
        for (int e = 0; e < kCols; ++e) b[e] = bias && e < n ? __ldg(bias + c + e) : 0.0f;
        const float *from = stage + r0 * kPitch + c;
        T *to = z + r0 * ldz + c;
        constexpr int kAtOnce = kCols >= 4 ? 4 : 8;
#pragma unroll 1
        for (int r = r0; r < rows; r += kAtOnce * kRows) {
            float v[kAtOnce][kCols];
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                const float *f = from + q * kRows * kPitch;
                if constexpr (kCols % 4 == 0) {
#pragma unroll
                    for (int e = 0; e < kCols; e += 4)
                        *reinterpret_cast<float4 *>(&v[q][e]) = *reinterpret_cast<const float4 *>(f + e);
                } else if constexpr (kCols == 2) {
                    *reinterpret_cast<float2 *>(&v[q][0]) = *reinterpret_cast<const float2 *>(f);
                } else {
                    v[q][0] = *f;
                }
            }
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                if (r + q * kRows >= rows) break;
                T out[kCols];
#pragma unroll
                for (int e = 0; e < kCols; ++e) out[e] = from_f32<T>(v[q][e] + b[e]);
                if (n >= kCols) {
                    if constexpr (VB == 16)
                        *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(out);
                    else if constexpr (VB == 8)
                        *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(out);
                    else if constexpr (VB == 4)
                        *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(out);
                    else *to = out[0];
                } else {
#pragma unroll
                    for (int e = 0; e < kCols; ++e)
                        if (e < n) to[e] = out[e];
                }
                to += kRows * ldz;
            }
            from += kAtOnce * kRows * kPitch;
        }
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

// A's or B's scale warp: 16 bytes of R rows a lane, unit after unit, into its part of the ring of slots.
// One lane arrives for all once a unit has landed, kLag units behind what is asked for.
template <int NT, int R>
__device__ __forceinline__ void ask_scales(const Fp4GemmArgs &p, bool a, uint32_t slots,
                                           const uint64_t *freed, const uint64_t *loaded,
                                           volatile uint32_t *stopv, int lane) {
    const uint8_t *const exps = a ? p.a_exps : p.b_exps;
    const int64_t rows = a ? p.N : p.F, ld = a ? p.lda_e : p.ldb_e;
    const bool wide = (reinterpret_cast<uintptr_t>(exps) & 15) == 0 && ld % 16 == 0;
    const int units = (p.groups + kUnit - 1) / kUnit;
    constexpr int kLag = kSlots - 2;
    int slot = 0, asked = 0;
    uint32_t parity = 1u;
    bool ok = true;
    auto landed = [&](int n) {              // the n-th unit of all
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&loaded[n % kSlots]));
    };
    for (int64_t t = blockIdx.x; ok && t < p.tiles; t += gridDim.x) {
        const Tile tile(t, p.nt, NT);
        const uint8_t *row[R];
        bool in[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t i = (a ? tile.m0 : tile.n0) + 32 * j + lane;
            in[j] = i < rows;
            row[j] = exps + (in[j] ? i * ld : 0);
        }
        for (int u = 0; u < units; ++u) {
            ok = __all_sync(kFullMask, wait_unless(smem_addr(&freed[slot]), parity, stopv));
            if (!ok) {
                *stopv = 1u;
                break;
            }
            const int left = p.groups - u * kUnit;
            const uint32_t to = slots + uint32_t(slot * Fp4Shape<NT>::kSlot + lane * 16);
#pragma unroll
            for (int j = 0; j < R; ++j) {
                // (Zeros behind the last group and the last row, whatever memory holds there; the
                // words behind the last group's are never used.)
                const uint8_t *from = row[j] + u * kUnit;
                if (wide) {
                    const uint32_t n = in[j] ? uint32_t(min(left, kUnit)) : 0u;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + uint32_t(j * 512)),
                                 "l"(from), "r"(n)
                                 : "memory");
                } else {
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (left > 4 * h)
                            copy4(to + uint32_t(j * 512 + 4 * h), from + 4 * h,
                                  in[j] ? uint32_t(min(left - 4 * h, 4)) : 0u);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (asked >= kLag) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kLag) : "memory");
                landed(asked - kLag);
            }
            ++asked;
            if (++slot == kSlots) slot = 0, parity ^= 1u;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    for (int n = asked > kLag ? asked - kLag : 0; n < asked; ++n) landed(n);
}

// A placing warp: a unit's words to tensor memory, in the quarter of its lanes that the warp may write.
// Word h of 128 rows is four columns; A's and B's of a word lie together.
template <int NT>
__device__ __forceinline__ void place_scales(const Fp4GemmArgs &p, uint32_t slots, uint32_t tmem,
                                             const uint64_t *freed, const uint64_t *loaded,
                                             const uint64_t *used, const uint64_t *filled,
                                             volatile uint32_t *stopv, int lane) {
    using S = Fp4Shape<NT>;
    const int units = (p.groups + kUnit - 1) / kUnit;
    int slot = 0, q = 0;
    uint32_t slot_parity = 0u, parity = 1u;
    for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x)
        for (int u = 0; u < units; ++u) {
            const bool go = wait_unless(smem_addr(&loaded[slot]), slot_parity, stopv) &&
                            wait_unless(smem_addr(&used[q]), parity, stopv);
            if (!__all_sync(kFullMask, go)) {
                *stopv = 1u;
                return;
            }
            uint32_t v[S::kScaleCols];
#pragma unroll
            for (int j = 0; j < 4 * (1 + S::kChunks); ++j) {
                uint32_t w[4] = {0u, 0u, 0u, 0u};
                if (j < 4 + S::kRowsB)
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                 : "r"(slots + uint32_t(slot * S::kSlot + j * 512 + lane * 16))
                                 : "memory");
#pragma unroll
                for (int h = 0; h < 4; ++h) v[h * 4 * (1 + S::kChunks) + j] = w[h];
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t to = tmem + uint32_t(q * S::kScaleCols);
#pragma unroll
            for (int c = 0; c < S::kScaleCols; c += 16) tmem_st16(to + uint32_t(c), v + c);
            tmem_wait_st();
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_addr(&filled[q]));
                mbar_arrive(smem_addr(&freed[slot]));
            }
            if (++slot == kSlots) slot = 0, slot_parity ^= 1u;
            if (++q == kUnits) q = 0, parity ^= 1u;
        }
}

template <typename T, int NT>
__global__ void __launch_bounds__(kGemmThreads, 1)
fp4_gemm_kernel(const __grid_constant__ Fp4GemmArgs p) {
    using S = Fp4Shape<NT>;
    constexpr int kStages = S::kStages;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], loaded[kSlots], freed[kSlots],
        filled[kUnits], used[kUnits], summed[S::kAccs], taken[S::kAccs], done;
    __shared__ uint32_t tmem_base, stop;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    const uint32_t staging = base + uint32_t(kStages * S::kStage);
    const uint32_t slots = staging + uint32_t(S::kStaging);

    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_addr(&tmem_base)),
                     "r"(kTmemCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&full[s]), 1);
            mbar_init(smem_addr(&empty[s]), 1);
        }
        for (int q = 0; q < kSlots; ++q) {
            mbar_init(smem_addr(&loaded[q]), 2);            // both scale warps
            mbar_init(smem_addr(&freed[q]), 4);
        }
        for (int q = 0; q < kUnits; ++q) {
            mbar_init(smem_addr(&filled[q]), 4);
            mbar_init(smem_addr(&used[q]), 1);
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
        ask_scales<NT, 4>(p, true, slots, freed, loaded, stopv, lane);
    } else if (warp == 3) {
        ask_scales<NT, S::kRowsB>(p, false, slots + 4 * 512, freed, loaded, stopv, lane);
    } else if (warp >= 12) {
        place_scales<NT>(p, slots, tmem + (uint32_t(32 * (warp & 3)) << 16) + S::kAccs * NT, freed, loaded,
                         used, filled, stopv, lane);
    } else if (warp == 1) {
        // One thread issues. A stage of 256 columns takes the tensor core 256 or 512 cycles; this loop
        // has to stay below that, at four cycles and more an instruction.
        if (elect_one()) {
            const uint32_t full0 = smem_addr(full), empty0 = smem_addr(empty);
            const uint32_t filled0 = smem_addr(filled), used0 = smem_addr(used);
            const uint32_t scales0 = tmem + uint32_t(S::kAccs * NT);
            const uint64_t desc0 = sw128_desc(base);
            uint32_t s = 0, b = 0, q = 0, parity = 0u, acc_parity = 1u, unit_parity = 0u;
            bool ok = true;
            for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
                const int n = (min(NT, p.F - (p.nt == 1 ? 0 : Tile(t, p.nt, NT).n0)) + 31) / 32 * 32;
                const uint32_t idesc = fp4_idesc(n, 0u), idesc2 = fp4_idesc(n, 2u);
                const uint32_t acc = tmem + b * NT;
                ok = wait_unless(smem_addr(&taken[b]), acc_parity, stopv);
                if (!ok) break;
                uint32_t word = 0u;             // the stage's scales, in tensor memory
                bool more = false;              // (the first MMA starts the sum)
                for (int left = p.groups, odd = 0; left > 0; left -= 8, odd ^= 1) {
                    if (odd) {
                        word += 8 * (1 + S::kChunks);
                    } else {
                        ok = wait_unless(filled0 + 8 * q, unit_parity, stopv);
                        word = scales0 + q * S::kScaleCols;
                    }
                    ok = ok && wait_unless(full0 + 8 * s, parity, stopv);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = desc0 + s * (S::kStage / 16), db = da + S::kA / 16;
                    constexpr uint32_t kNext = 4 * (1 + S::kChunks), kB = 4;
                    mma_fp4(acc, da, db, idesc, word, word + kB, more);
                    more = true;
                    if (left > 2) mma_fp4(acc, da + 2, db + 2, idesc2, word, word + kB, true);
                    if (left > 4) mma_fp4(acc, da + 4, db + 4, idesc, word + kNext, word + kNext + kB, true);
                    if (left > 6) mma_fp4(acc, da + 6, db + 6, idesc2, word + kNext, word + kNext + kB, true);
                    mma_commit(empty0 + 8 * s);
                    if (++s == kStages) s = 0, parity ^= 1u;
                    if (odd || left <= 8) {
                        mma_commit(used0 + 8 * q);
                        if (++q == kUnits) q = 0, unit_parity ^= 1u;
                    }
                }
                if (!ok) break;
                mma_commit(smem_addr(&summed[b]));
                if (++b == S::kAccs) b = 0, acc_parity ^= 1u;
            }
            if (!ok) *stopv = 1u;
            mma_commit(smem_addr(&done));
        }
        __syncwarp();
    } else {
        // Sums out, a warp the 32 lanes of tensor memory that it may read, every second kBatch columns.
        // Tiles whose waits ran out are NaN.
        constexpr int kBatch = S::kBatch, kPitch = S::kPitch;
        const int quad = warp & 3, half = (warp - 4) >> 2;
        float *const stage = reinterpret_cast<float *>(smem_raw + (staging - raw)) +
                             (warp - 4) * 32 * kPitch;
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
            for (int c = kBatch * half; c < cols; c += 2 * kBatch) {
#pragma unroll
                for (int h = 0; h < kBatch; h += 32) {
                    if (c + h >= cols) break;
                    uint32_t v[32];
                    tmem_ld32(acc + uint32_t(c + h), v);
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<uint4 *>(stage + lane * kPitch + h + e) =
                            ok ? make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3])
                               : make_uint4(0x7FC00000u, 0x7FC00000u, 0x7FC00000u, 0x7FC00000u);
                }
                if (c + 2 * kBatch >= cols) {       // the warp's last of this tile
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&taken[b]));
                }
                __syncwarp();
                const float *bc = bias ? bias + c : nullptr;
                if (p.vec == 16) store_sums<T, kBatch, 16>(stage, z + c, p.ldz, rows, cols - c, bc, lane);
                else if (p.vec == 8) store_sums<T, kBatch, 8>(stage, z + c, p.ldz, rows, cols - c, bc, lane);
                else if (p.vec == 4) store_sums<T, kBatch, 4>(stage, z + c, p.ldz, rows, cols - c, bc, lane);
                else if constexpr (sizeof(T) == 2)
                    store_sums<T, kBatch, 2>(stage, z + c, p.ldz, rows, cols - c, bc, lane);
                __syncwarp();
            }
            if (kBatch * half >= cols) {            // no columns of this tile
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&taken[b]));
            }
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
    const uint64_t where = uint64_t(uintptr_t(Z)) | uint64_t(N > 1 ? ldz : 0) * es | 16;
    p.vec = int(where & (~where + 1));
    const unsigned grid = unsigned(p.tiles < dev.sm_count ? p.tiles : dev.sm_count);
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32) launch_gemm<float>(p, NT, grid, s);
    else if (dtype == BIGCN_BF16) launch_gemm<__nv_bfloat16>(p, NT, grid, s);
    else launch_gemm<__half>(p, NT, grid, s);
    return launch_status();
}
