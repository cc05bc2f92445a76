// The product of two matrices of microscaled 4-bit rows (bigcn_fp4_gemm), Z = A B^T + bias, on the
// tensor cores: tcgen05 block-scaled e2m1 x e2m1 with a ue8m0 scale per 32 columns of either
// operand, fp32 accumulators in tensor memory. Codes go by tensor copies from memory into their
// swizzled places (128 bytes, 256 columns, of a row a stage). The scale bytes, four groups to a word,
// go to tensor memory as the MMAs read them: of 128 rows, row r's word in column r / 32 and in lane r
// mod 32 of each quarter of the lanes, written by a warp of each quarter.
//
// Roles of a CTA (16 or 24 warps), which takes tiles of 128 rows by NT columns in turn: warp 0 copies the
// codes; warps 2 and 3 ask for A's and B's scale bytes, a unit of 16 groups (two stages) of a row at a
// time and several units ahead; warps 4-7 put them into tensor memory; warp 1 issues the MMAs; the others
// take the sums out, kBatch columns at a time of the 32 rows that a warp may read. They meet on
// mbarriers:
//   ready[stage]   its codes and scales are there    free[stage]   its MMAs are done
//   loaded[slot]   a unit's scale bytes landed       read[slot]    they were read
//   summed[acc]    a tile's MMAs are done            taken[acc]    its sums were taken
// The thread that issues is the one to spare: about 50 cycles an MMA, and at first 575 a stage beside them
// for its waits, commits and arithmetic, of the 512 that a stage's MMAs take the tensor core with 256
// columns; 700 with barriers of their own for A, B and the scales. So one barrier says that a stage is
// there, one that it is free, and nothing is divided or recomputed for it. (Scale bytes by way of shared memory
// and the tensor core's own copy took as long, with one proxy fence and four more copies a unit.)
//
// What bounds it (L2 flushed before each call; floors at a copy's 6754 GB/s):
//   232,965 x 602 x 128 fp32: 38 us of 28.7. Start and end of 12 tiles a CTA; B stays in shared memory
//     (46 us when it was copied for every tile).
//   232,965 x 128 x 602 fp32: 117 us of 85. Stores: Z's rows are aligned to 8 bytes, a store of 256 bytes
//     touches three lines, L1 at 83 %. x 604: 107, x 640: 103, x 601 (4 bytes a lane): 195.
//   2^17 x 8192 x 256 bf16: 132 us of 95. A's copies are 128 bytes of rows 4 KB apart, and a stage's boxes and
//     MMAs wait for each other 40 % of the issuing thread's time; sums are taken out while nothing is
//     multiplied, 10 to 16 us of all. More of A on its way did not help (six stages of A beside three of
//     B 159, boxes of two stages at a time 165, prefetches to L2 by a warp of their own 148, all for 142). The
//     16-bit sums held there spill 12 bytes a thread.
#include "fp4.cuh"
#include "launch.cuh"
#include "tc_rows.cuh"
#include "tensor_map.cuh"

namespace bigcn {

__device__ unsigned int g_fp4_timeouts;

namespace {

constexpr int kUnit = 16;               // groups whose scale bytes are brought at a time: two stages'
constexpr int kTmemCols = 512;
constexpr int kMaxGemmCols = 1 << 15;   // K: at most 512 accumulating MMAs (see the header)

// kOnce: a CTA's columns are always the same and B's stages, at most kHeld, stay in shared memory.
template <int NT, bool kOnce>
struct Fp4Shape {
    static constexpr int kA = kUmmaM * 128, kB = NT * 128;
    static constexpr int kHeld = kOnce ? 3 : 0;
    static constexpr int kStage = kOnce ? kA : kA + kB;
    static constexpr int kStages = NT >= 256 ? 4 : kOnce ? 5 : NT >= 128 ? 4 : 5;
    static constexpr int kRowsB = NT / 32;                          // a lane of B's scales has
    static constexpr int kChunks = NT > 128 ? NT / 128 : 1;         // of 128 rows of B
    static constexpr int kSlots = NT >= 256 ? 2 : 6;                // units on their way or in shared memory
    static constexpr int kSlot = (4 + kRowsB) * 512;                // 16 bytes of each row
    static constexpr int kScaleCols = 8 * (1 + kChunks);            // of tensor memory, a stage
    // Warps that take the sums out. With kPair two of them, of the same quarter of the lanes, stage 64 columns
    // together, half each, and store half the rows each: longer runs of a row at a time, and twice the
    // warps to wait on memory.
    static constexpr int kOutWarps = NT == 64 || NT == 128 ? 16 : 8;
    static constexpr bool kPair = kOutWarps == 16;
    static constexpr int kThreads = (8 + kOutWarps) * 32;
    // Columns that are staged at a time, and words from one staged row to the next: accesses of 4, 8
    // and 16 bytes of a lane's row, or of a row by neighbouring lanes, then fall into different banks.
    static constexpr int kBatch = NT >= 256 ? 16 : NT >= 64 ? 64 : 32;
    static constexpr int kPitch = kBatch + 4;
    static constexpr int kStaging = 8 * 32 * kPitch * 4;
    static constexpr int kSmem = 1024 + kStages * kStage + kHeld * kB + kStaging + kSlots * kSlot;
    static constexpr int kAccs = NT > 128 ? 1 : 2;
    static_assert(kA % 1024 == 0 && kB % 1024 == 0, "swizzled tiles start on 1024 bytes");
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
    uint32_t mt;             // row tiles
    uint32_t step_m, step_n; // from a CTA's tile to its next
    const float *bias;       // nullable
    void *Z;
    int64_t ldz;
    int vec;                 // bytes that Z and its rows are aligned to, at most 32
    bool direct;             // 16-bit sums, or those of 256 columns, go straight to Z (store_direct)
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
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

template <typename T, int kCols>
__device__ __forceinline__ void load_staged(const float *f, float (&v)[kCols]) {
    if constexpr (kCols % 4 == 0) {
#pragma unroll
        for (int e = 0; e < kCols; e += 4)
            *reinterpret_cast<float4 *>(&v[e]) = *reinterpret_cast<const float4 *>(f + e);
    } else if constexpr (kCols == 2) {
        *reinterpret_cast<float2 *>(&v[0]) = *reinterpret_cast<const float2 *>(f);
    } else {
        v[0] = *f;
    }
}
template <typename T, int kCols>
__device__ __forceinline__ void store_staged(T *to, const float (&v)[kCols], const float (&b)[kCols]) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (kCols == 4)
            *reinterpret_cast<float4 *>(to) =
                make_float4(v[0] + b[0], v[1] + b[1], v[2] + b[2], v[3] + b[3]);
        else if constexpr (kCols == 2)
            *reinterpret_cast<float2 *>(to) = make_float2(v[0] + b[0], v[1] + b[1]);
        else *to = v[0] + b[0];
    } else if constexpr (kCols == 1) {
        *to = from_f32<T>(v[0] + b[0]);
    } else {
        uint32_t w[kCols / 2];
#pragma unroll
        for (int e = 0; e < kCols; e += 2) {
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 x = __floats2half2_rn(v[e] + b[e], v[e + 1] + b[e + 1]);
                w[e / 2] = *reinterpret_cast<const uint32_t *>(&x);
            } else {
                const __nv_bfloat162 x = __floats2bfloat162_rn(v[e] + b[e], v[e + 1] + b[e + 1]);
                w[e / 2] = *reinterpret_cast<const uint32_t *>(&x);
            }
        }
        if constexpr (kCols == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (kCols == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(to) = w[0];
    }
}
// kStore rows of sums, kBatch columns from shared memory to Z, with the bias: VB bytes of a row a lane (Z's
// rows are aligned to them), neighbouring lanes along the row.
template <typename T, int kBatch, int kStore, int VB>
__device__ __forceinline__ void store_sums(const float *stage, T *z, int64_t ldz, int rows, int cols,
                                           const float *bias, int lane) {
    constexpr int kPitch = kBatch + 4, kCols = VB / int(sizeof(T));
    constexpr int kLanes = kBatch / kCols < 32 ? kBatch / kCols : 32;       // of a row
    constexpr int kParts = kBatch / kCols / kLanes, kRows = 32 / kLanes, kTurns = kStore / kRows;
    // (Few rows at once: the roles' code together is more than the instruction caches like. Sixteen rows of two
    // columns 123 to 126 us, eight 122, four and two 117, 232,965 x 128 x 602 fp32.)
    constexpr int kMost = kCols >= 4 && kCols < 8 ? 8 : 4, kAtOnce = kTurns < kMost ? kTurns : kMost;
    static_assert(kTurns > 0 && kTurns % kAtOnce == 0, "whole turns");
    const int r0 = lane / kLanes, c0 = lane % kLanes * kCols;
    const int64_t step = kRows * ldz;
#pragma unroll 1
    for (int part = 0; part < kParts; ++part) {
        const int c = c0 + part * kLanes * kCols, n = cols - c;
        float b[kCols];
#pragma unroll
        for (int e = 0; e < kCols; ++e) b[e] = bias && e < n ? __ldg(bias + c + e) : 0.0f;
        const float *from = stage + r0 * kPitch + c;
        T *to = z + r0 * ldz + c;
        if (n >= kCols) {
#pragma unroll 1
            for (int r = r0; r < rows; r += kAtOnce * kRows, from += kAtOnce * kRows * kPitch) {
                float v[kAtOnce][kCols];
#pragma unroll
                for (int q = 0; q < kAtOnce; ++q) load_staged<T>(from + q * kRows * kPitch, v[q]);
#pragma unroll
                for (int q = 0; q < kAtOnce; ++q, to += step)
                    if (r + q * kRows < rows) store_staged<T>(to, v[q], b);
            }
        } else {
#pragma unroll 1
            for (int e = 0; e < n; ++e)
                for (int r = r0; r < rows; r += kRows)
                    to[(r - r0) * ldz + e] = from_f32<T>(from[(r - r0) * kPitch + e] +
                                                         (bias ? __ldg(bias + c + e) : 0.0f));
        }
    }
}

// 32 columns of sums, a row a lane, straight to Z's rows where these are aligned to 32 bytes: whole sectors,
// each lane's own. `stage`: 32 floats, for the bias.
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]),
                 "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
// The columns' biases, each lane's own in `bias`, to 32 sums of a row.
__device__ __forceinline__ void add_bias(uint32_t (&v)[32], float bias, float *stage, int lane) {
    __syncwarp();
    stage[lane] = bias;
    __syncwarp();
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        const float4 b = *reinterpret_cast<const float4 *>(stage + e);
        v[e] = __float_as_uint(__uint_as_float(v[e]) + b.x);
        v[e + 1] = __float_as_uint(__uint_as_float(v[e + 1]) + b.y);
        v[e + 2] = __float_as_uint(__uint_as_float(v[e + 2]) + b.z);
        v[e + 3] = __float_as_uint(__uint_as_float(v[e + 3]) + b.w);
    }
}
// 32 sums as the words that they are in Z.
template <typename T> constexpr int kWordsOut = 32 * int(sizeof(T)) / 4;
template <typename T>
__device__ __forceinline__ void pack_sums(const uint32_t (&v)[32], uint32_t (&w)[kWordsOut<T>]) {
#pragma unroll
    for (int e = 0; e < kWordsOut<T>; ++e) {
        if constexpr (sizeof(T) == 4) {
            w[e] = v[e];
        } else {
            const float x = __uint_as_float(v[2 * e]), y = __uint_as_float(v[2 * e + 1]);
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(x, y);
                w[e] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
                w[e] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
}
template <typename T>
__device__ __forceinline__ void store_direct(const uint32_t (&w)[kWordsOut<T>], T *row, int cols) {
    constexpr int kCols = 32 / int(sizeof(T));          // of 32 bytes
#pragma unroll
    for (int c = 0; c < 32; c += kCols) {
        constexpr int kPer = 4 / int(sizeof(T));        // columns of a word
        if (c + kCols <= cols) {
            uint32_t x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = w[c / kPer + e];
            store32(row + c, x);
        } else {
#pragma unroll
            for (int e = 0; e < kCols; ++e)
                if (c + e < cols) {
                    if constexpr (sizeof(T) == 4)
                        reinterpret_cast<uint32_t *>(row)[c + e] = w[c + e];
                    else
                        reinterpret_cast<uint16_t *>(row)[c + e] =
                            uint16_t(w[(c + e) / 2] >> (16 * (e % 2)));
                }
        }
    }
}

// A CTA's tiles, blockIdx.x, + gridDim.x, ...: m and n in tiles. (A division a tile costs each role 300
// cycles and more.)
struct Tiles {
    uint32_t m, n;
    __device__ __forceinline__ explicit Tiles(const Fp4GemmArgs &p)
        : m(blockIdx.x / uint32_t(p.nt)), n(blockIdx.x % uint32_t(p.nt)) {}
    __device__ __forceinline__ bool more(const Fp4GemmArgs &p) const { return m < p.mt; }
    __device__ __forceinline__ void next(const Fp4GemmArgs &p) {
        m += p.step_m;
        n += p.step_n;
        if (n >= uint32_t(p.nt)) n -= uint32_t(p.nt), ++m;
    }
    __device__ __forceinline__ int64_t m0() const { return int64_t(m) * kUmmaM; }
};

// A's or B's scale warp: 16 bytes of R rows a lane, unit after unit, into its part of the ring of slots.
// One lane arrives for all once a unit has landed, kLag units behind what is asked for.
template <int NT, int kSlots, int R>
__device__ __forceinline__ void ask_scales(const Fp4GemmArgs &p, bool a, uint32_t slots,
                                           const uint64_t *read, const uint64_t *loaded,
                                           volatile uint32_t *stopv, int lane) {
    const uint8_t *const exps = a ? p.a_exps : p.b_exps;
    const int64_t rows = a ? p.N : p.F, ld = a ? p.lda_e : p.ldb_e;
    const bool wide = (reinterpret_cast<uintptr_t>(exps) & 15) == 0 && ld % 16 == 0;
    const int units = (p.groups + kUnit - 1) / kUnit;
    constexpr int kSlot = (4 + NT / 32) * 512, kLag = kSlots > 2 ? kSlots - 2 : 1;
    int slot = 0, asked = 0;
    uint32_t parity = 1u;
    bool ok = true;
    auto landed = [&](int n) {              // the n-th unit of all
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&loaded[n % kSlots]));
    };
    for (Tiles t(p); ok && t.more(p); t.next(p)) {
        const uint8_t *row[R];
        bool in[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int64_t i = (a ? t.m0() : int64_t(t.n) * NT) + 32 * j + lane;
            in[j] = i < rows;
            row[j] = exps + (in[j] ? i * ld : 0);
        }
        for (int u = 0; u < units; ++u) {
            ok = __all_sync(kFullMask, wait_unless(smem_addr(&read[slot]), parity, stopv));
            if (!ok) {
                *stopv = 1u;
                break;
            }
            const int left = p.groups - u * kUnit;
            const uint32_t to = slots + uint32_t(slot * kSlot + lane * 16);
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

// A placing warp: the scale words of a unit's stages to tensor memory, in the quarter of its lanes that the
// warp may write. Word h of 128 rows is four columns; A's and B's of a word lie together.
template <int NT, bool kOnce>
__device__ __forceinline__ void place_scales(const Fp4GemmArgs &p, uint32_t slots, uint32_t tmem,
                                             const uint64_t *read, const uint64_t *loaded,
                                             const uint64_t *free, const uint64_t *ready,
                                             volatile uint32_t *stopv, int stages, int lane) {
    using S = Fp4Shape<NT, kOnce>;
    constexpr int kCols = 4 * (1 + S::kChunks);         // of a word
    int slot = 0, s = 0;
    uint32_t slot_parity = 0u, parity = 1u;
    for (Tiles t(p); t.more(p); t.next(p))
        for (int st = 0; st < stages; st += 2) {
            if (!__all_sync(kFullMask, wait_unless(smem_addr(&loaded[slot]), slot_parity, stopv))) {
                *stopv = 1u;
                return;
            }
            uint32_t v[4 * kCols];
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
                uint32_t w[4] = {0u, 0u, 0u, 0u};
                if (j < 4 + S::kRowsB)
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                 : "r"(slots + uint32_t(slot * S::kSlot + j * 512 + lane * 16))
                                 : "memory");
#pragma unroll
                for (int h = 0; h < 4; ++h) v[h * kCols + j] = w[h];
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&read[slot]));
            if (++slot == S::kSlots) slot = 0, slot_parity ^= 1u;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (st + half >= stages) break;
                if (!__all_sync(kFullMask, wait_unless(smem_addr(&free[s]), parity, stopv))) {
                    *stopv = 1u;
                    return;
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t to = tmem + uint32_t(s * S::kScaleCols);
#pragma unroll
                for (int c = 0; c < S::kScaleCols; c += 8)
                    tmem_st8(to + uint32_t(c), v + half * S::kScaleCols + c);
                tmem_wait_st();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&ready[s]));
                if (++s == S::kStages) s = 0, parity ^= 1u;
            }
        }
}

template <typename T, int NT, bool kOnce>
__global__ void __launch_bounds__(Fp4Shape<NT, kOnce>::kThreads, 1)
fp4_gemm_kernel(const __grid_constant__ Fp4GemmArgs p) {
    using S = Fp4Shape<NT, kOnce>;
    constexpr int kStages = S::kStages, kSlots = S::kSlots;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t ready[kStages], free[kStages], loaded[kSlots], read[kSlots],
        summed[S::kAccs], taken[S::kAccs], done;
    __shared__ uint32_t tmem_base, stop;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    const uint32_t held = base + uint32_t(kStages * S::kStage), staging = held + uint32_t(S::kHeld * S::kB);
    const uint32_t slots = staging + uint32_t(S::kStaging);

    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_addr(&tmem_base)),
                     "r"(kTmemCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&ready[s]), 5);             // the boxes' bytes, the placing warps
            mbar_init(smem_addr(&free[s]), 1);
        }
        for (int q = 0; q < kSlots; ++q) {
            mbar_init(smem_addr(&loaded[q]), 2);            // both scale warps
            mbar_init(smem_addr(&read[q]), 4);
        }
        for (int b = 0; b < S::kAccs; ++b) {
            mbar_init(smem_addr(&summed[b]), 1);
            mbar_init(smem_addr(&taken[b]), S::kOutWarps);
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
        bool bring_b = true;
        for (Tiles t(p); ok && t.more(p); t.next(p)) {
            for (int st = 0; st < stages; ++st) {
                if (!__all_sync(kFullMask, wait_unless(smem_addr(&free[s]), parity, stopv))) {
                    *stopv = 1u;
                    ok = false;
                    break;
                }
                const uint32_t at = base + uint32_t(s * S::kStage), bar = smem_addr(&ready[s]);
                if (elect_one()) {
                    mbar_expect(bar, bring_b ? S::kA + S::kB : S::kA);
                    tma_load(at, &p.a_map, st * 128, int(t.m0()), bar);
                    if (bring_b)
                        tma_load(kOnce ? held + uint32_t(st * S::kB) : at + S::kA, &p.b_map, st * 128,
                                 int(t.n) * NT, bar);
                }
                __syncwarp();
                ++issued;
                if (++s == kStages) s = 0, parity ^= 1u;
            }
            if (kOnce) bring_b = false;
        }
        // What is still in flight lands before the shared memory is given up.
        for (int it = issued > kStages ? issued - kStages : 0; it < issued; ++it)
            mbar_wait(smem_addr(&ready[it % kStages]), uint32_t(it / kStages) & 1u);
    } else if (warp == 2) {
        ask_scales<NT, kSlots, 4>(p, true, slots, read, loaded, stopv, lane);
    } else if (warp == 3) {
        ask_scales<NT, kSlots, S::kRowsB>(p, false, slots + 4 * 512, read, loaded, stopv, lane);
    } else if (warp >= 4 && warp < 8) {
        place_scales<NT, kOnce>(p, slots, tmem + (uint32_t(32 * (warp & 3)) << 16) + S::kAccs * NT, read,
                                loaded, free, ready, stopv, stages, lane);
    } else if (warp == 1) {
        // One thread issues. A stage of 256 columns takes the tensor core 256 or 512 cycles; this loop
        // has to stay below that, at four cycles and more an instruction.
        if (elect_one()) {
            const uint32_t ready0 = smem_addr(ready), free0 = smem_addr(free);
            const uint32_t scales0 = tmem + uint32_t(S::kAccs * NT);
            const uint64_t desc0 = sw128_desc(base), desc_held = sw128_desc(held);
            uint32_t s = 0, b = 0, parity = 0u, acc_parity = 1u;
            bool ok = true;
            // Columns of the last tile, rounded up to what an MMA takes.
            const uint32_t whole = fp4_idesc(NT, 0u);
            const uint32_t last = fp4_idesc((p.F - (p.nt - 1) * NT + 31) / 32 * 32, 0u);
            for (Tiles t(p); t.more(p); t.next(p)) {
                const uint32_t idesc = t.n + 1 == uint32_t(p.nt) ? last : whole;
                const uint32_t idesc2 = idesc | fp4_idesc(0, 2u);
                const uint32_t acc = tmem + b * NT;
                ok = wait_unless(smem_addr(&taken[b]), acc_parity, stopv);
                bool more = false;              // (the first MMA starts the sum)
                uint64_t db = desc_held;
                for (int left = p.groups; ok && left > 0; left -= 8) {
                    ok = wait_unless(ready0 + 8 * s, parity, stopv);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = desc0 + s * (S::kStage / 16);
                    if (!kOnce) db = da + S::kA / 16;
                    const uint32_t sa = scales0 + s * S::kScaleCols, sb = sa + 4;
                    constexpr uint32_t kNext = 4 * (1 + S::kChunks);
                    mma_fp4(acc, da, db, idesc, sa, sb, more);
                    more = true;
                    if (left > 2) mma_fp4(acc, da + 2, db + 2, idesc2, sa, sb, true);
                    if (left > 4) mma_fp4(acc, da + 4, db + 4, idesc, sa + kNext, sb + kNext, true);
                    if (left > 6) mma_fp4(acc, da + 6, db + 6, idesc2, sa + kNext, sb + kNext, true);
                    mma_commit(free0 + 8 * s);
                    if (++s == kStages) s = 0, parity ^= 1u;
                    if (kOnce) db += S::kB / 16;
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
        // Sums out, a warp the 32 lanes of tensor memory that it may read, every second batch of columns.
        // Tiles whose waits ran out are NaN.
        constexpr int kBatch = S::kBatch, kPitch = S::kPitch;
        constexpr int kLoad = kBatch / (S::kPair ? 2 : 1), kStore = S::kPair ? 16 : 32;
        constexpr int kWidth = S::kPair ? kLoad : 32;       // columns of a direct store
        const int quad = warp & 3, out = (warp - 8) >> 2;
        const int half = S::kPair ? out >> 1 : out, mate = S::kPair ? out & 1 : 0;
        float *const stage = reinterpret_cast<float *>(smem_raw + (staging - raw)) +
                             (quad + 4 * half) * 32 * kPitch;
        auto meet = [&] {                                   // with the other warp of the pair
            if constexpr (S::kPair)
                asm volatile("bar.sync %0, 64;" ::"r"(1 + quad + 4 * half) : "memory");
            else __syncwarp();
        };
        int b = 0;
        uint32_t parity = 0u;
        bool ok = true;
        for (Tiles t(p); t.more(p); t.next(p)) {
            const int64_t row0 = t.m0() + 32 * quad;
            const int n0 = int(t.n) * NT, cols = min(NT, p.F - n0);
            const int rows = int(min(int64_t(32), max(int64_t(0), p.N - row0)));
            const float *bias = p.bias ? p.bias + n0 : nullptr;
            // Straight stores: parts of 32 columns, kStep apart; the biases of several come while the MMAs
            // are on their way.
            constexpr bool kDirect = sizeof(T) == 2 || NT >= 256;
            constexpr int kStep = S::kOutWarps / 4 * kWidth, kParts = NT > kStep ? NT / kStep : 1;
            const int c0 = kWidth * (S::kPair ? out : half);
            float own[kParts];
            auto load_own = [&] {
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    const int c = c0 + q * kStep + lane;
                    own[q] = bias && c < cols ? __ldg(bias + c) : 0.0f;
                }
            };
            if (kDirect && kParts > 1 && p.direct) load_own();
            if (ok) {
                ok = __all_sync(kFullMask, wait_unless(smem_addr(&summed[b]), parity, stopv));
                if (!ok) *stopv = 1u;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + (uint32_t(32 * quad) << 16) + uint32_t(b * NT);
            T *z = static_cast<T *>(p.Z) + row0 * p.ldz + n0;
            auto taken_out = [&] {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&taken[b]));
            };
            if (kDirect && p.direct) {
                // With one accumulator 16-bit sums are held until it has been given back (with the biases loaded
                // ahead 2^17 x 8192 x 256 bf16 142 -> 136 us).
                constexpr bool kHold = S::kAccs == 1 && sizeof(T) == 2;
                if (kParts == 1) load_own();
                T *row = z + lane * p.ldz;
                uint32_t w[kHold ? kParts : 1][kWordsOut<T>];
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    const int c = c0 + q * kStep;
                    if (c >= cols) break;
                    uint32_t v[32];
                    tmem_ld32(acc + uint32_t(c), v);
                    if (!ok)
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0x7FC00000u;
                    if (bias) add_bias(v, own[q], stage + 36 * mate, lane);
                    pack_sums<T>(v, w[kHold ? q : 0]);
                    if (!kHold && lane < rows) store_direct<T>(w[0], row + c, cols - c);
                }
                taken_out();
                if constexpr (kHold) {
#pragma unroll
                    for (int q = 0; q < kParts; ++q) {
                        const int c = c0 + q * kStep;
                        if (c < cols && lane < rows) store_direct<T>(w[q], row + c, cols - c);
                    }
                }
            } else {
#pragma unroll 1
                for (int c = kBatch * half; c < cols; c += 2 * kBatch) {
                    const int h = kLoad * mate;
                    if (c + h < cols) {
                        uint32_t v[kLoad];
                        if constexpr (kLoad == 32) tmem_ld32(acc + uint32_t(c + h), v);
                        else tmem_ld16(acc + uint32_t(c + h), v);
                        uint4 *const to = reinterpret_cast<uint4 *>(stage + lane * kPitch + h);
#pragma unroll
                        for (int e = 0; e < kLoad / 4; ++e)
                            to[e] = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                        if (!ok)
                            for (int e = 0; e < kLoad; ++e)
                                stage[lane * kPitch + h + e] = __uint_as_float(0x7FC00000u);
                    }
                    if (c + 2 * kBatch >= cols) taken_out();        // the warp's last of this tile
                    meet();
                    const float *bc = bias ? bias + c : nullptr;
                    const float *from = stage + kStore * mate * kPitch;
                    T *zc = z + kStore * mate * p.ldz + c;
                    const int nr = min(kStore, rows - kStore * mate), nc = cols - c;
                    if (p.vec >= 16) store_sums<T, kBatch, kStore, 16>(from, zc, p.ldz, nr, nc, bc, lane);
                    else if (p.vec == 8) store_sums<T, kBatch, kStore, 8>(from, zc, p.ldz, nr, nc, bc, lane);
                    else if (p.vec == 4) store_sums<T, kBatch, kStore, 4>(from, zc, p.ldz, nr, nc, bc, lane);
                    else if constexpr (sizeof(T) == 2)
                        store_sums<T, kBatch, kStore, 2>(from, zc, p.ldz, nr, nc, bc, lane);
                    meet();
                }
                if (kBatch * half >= cols) taken_out();             // no columns of this tile
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

template <typename T, int NT, bool kOnce>
void launch_nt(const Fp4GemmArgs &p, unsigned grid, cudaStream_t s) {
    using S = Fp4Shape<NT, kOnce>;
    cudaFuncSetAttribute(fp4_gemm_kernel<T, NT, kOnce>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         S::kSmem);
    fp4_gemm_kernel<T, NT, kOnce><<<grid, S::kThreads, S::kSmem, s>>>(p);
}

template <typename T>
void launch_gemm(const Fp4GemmArgs &p, int NT, unsigned grid, cudaStream_t s) {
    const bool once = p.nt == 1 && p.groups <= 8 * Fp4Shape<128, true>::kHeld && p.mt > grid;
    if (NT == 256) launch_nt<T, 256, false>(p, grid, s);
    else if (NT == 128 && once) launch_nt<T, 128, true>(p, grid, s);
    else if (NT == 128) launch_nt<T, 128, false>(p, grid, s);
    else if (NT == 64 && once) launch_nt<T, 64, true>(p, grid, s);
    else if (NT == 64) launch_nt<T, 64, false>(p, grid, s);
    else launch_nt<T, 32, false>(p, grid, s);
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
    // Tiles of 256 columns read A once for twice as many, but leave no room for a second accumulator: only
    // where a tile's MMAs are long beside taking its sums out, and the last tile is more than half full
    // (2^17 rows, 256 columns of bf16: K = 8192 132 us, by 128 columns 167; K = 4096 79 and 95; K = 2080 72 and
    // 70; K = 1024 fp32 52 and 44; 219,247 x 2106 x 274 fp16 193 and 154).
    int NT = F > 128 && K > 2048 && (F + 127) / 128 % 2 == 0 ? 256 : F > 64 ? 128 : F > 32 ? 64 : 32;
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
    p.mt = uint32_t(mt);
    const int64_t tiles = mt * p.nt;
    p.bias = bias;
    p.Z = Z;
    p.ldz = ldz;
    const uint64_t where = uint64_t(uintptr_t(Z)) | uint64_t(N > 1 ? ldz : 0) * es | 32;
    p.vec = int(where & (~where + 1));
    p.direct = p.vec == 32;
    const unsigned grid = unsigned(tiles < dev.sm_count ? tiles : dev.sm_count);
    p.step_m = grid / uint32_t(p.nt);
    p.step_n = grid % uint32_t(p.nt);
    const cudaStream_t s = as_stream(stream);
    if (dtype == BIGCN_F32) launch_gemm<float>(p, NT, grid, s);
    else if (dtype == BIGCN_BF16) launch_gemm<__nv_bfloat16>(p, NT, grid, s);
    else launch_gemm<__half>(p, NT, grid, s);
    return launch_status();
}
