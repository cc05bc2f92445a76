// The weight gradient of a product whose input is kept as a checkpoint
// (bigcn_checkpoint_weight_grad): with the input gamma v + beta,
//
//   dW[k,j] = gamma_k sum_i v_ik dZ_ij + beta_k s_j,   s_j = db_j = sum_i dZ_ij.
//
// The sum over the rows i runs on the tensor cores (tcgen05, bf16 operands, fp32
// accumulators), and nothing is rounded on the way in: v = q 2^e has 7 significant bits
// and is a bf16; dZ is one bf16 part (bf16), two (fp16: 8 + 3 bits) or three (fp32: 8 + 8 + 8
// bits, exact above 2^-110, within 2^-134 below).
//
// Operands. M = 128 features a tile, N = the columns, the contraction over 32 or 64 rows a
// stage. Both matrices are row-major, i.e. their features and columns lie along memory
// rows, and the tensor core takes them that way (MN-major), so nothing is transposed: a
// bf16 dZ goes by tensor copies from memory into its swizzled place; q (and an fp32 or
// fp16 dZ) by tensor copies into a ring of raw slots, from which the workers expand it.
//
// Roles of a CTA (608 threads): warps 0-15, the workers, turn raw slots into operand
// stages, in two teams that take every second stage each (one's latencies pass under the
// other's instructions), and take the running sums. Warp 16 copies, warp 17 issues the MMAs, warp
// 18 copies the scale bytes (with the boxes in one warp: 336 us for 299 at 2^20 x 512 x 256 bf16).
// They meet on mbarriers only:
//   loaded[slot]   a slot's copies have landed         freed[slot]   it may be refilled
//   filled[stage]  a team has written a stage          used[stage]   its MMAs are done
//                    (where dZ is copied as an operand, freed[slot] says both)
//   summed         a block's MMAs are done             drained       its sums were taken
//
// Running sums. The tensor core truncates when it accumulates (measured: 2.0e-8 of the
// result per accumulating MMA, always towards 0; 1080 MMAs gave 2.2e-5), so an accumulator
// takes kDrain stages, 48 or 64 MMAs (about 1e-6), and is then added, in fp32, to the running sums:
// 256 accumulator columns of tensor memory and 256 of sums. (Sums in registers, with two
// accumulators in turn, left room for 8 worker warps: 236 us at 232,965 x 602 x 128 fp32, the
// workers' instructions at 1.7 a cycle being the limit.)
//
// Split. A CTA holds 256 / NT feature tiles (`mt` of them, fewer in small calls), so that
// dZ is read and split into parts once for that many; the rows are split so that the grid is
// about one CTA per SM (kGradCtas), a last group of fewer tiles into fewer runs. A second kernel
// adds the runs in order, sums s_j, and applies gamma and beta. The columns of dZ are summed by
// the CTA that has them in shared memory anyway: of the groups of feature tiles that read the
// same rows, group g takes the g-th 64 columns.
//
// What bounds it (cycles and times of one kernel by ncu, at 1.92 to 1.94 GHz; the call's by events):
//   fp32 dZ (232,965 x 602 x 128, 32 rows a stage: 122 us, 883 TFLOP/s of the three parts' products):
//     this kernel 118 us, 229,000 cycles for a CTA's 135 stages, its start and its end: 1700 a
//     stage, in which shared memory moves 184 KB (48 copied and read, 40 of operands written, 96 read
//     by the MMAs), 108 bytes a cycle of the 128 it has; the tensor pipe is active in 41 %. A
//     kept in the tensor core's collector for the three parts changed nothing (131 us both ways
//     then). The second kernel reads 17 MB of sums: 11 us alone, partly under the first's end.
//   bf16 dZ (2^20 x 512 x 256, 64 rows a stage: 276 us, 995 TFLOP/s): this kernel 263 us, 504,000
//     cycles for 432 stages: 1170 a stage, tensor pipe 44 %, shared memory 120 KB (940 cycles). A
//     slot's way through copy, expansion and MMA takes four times that, and four slots fit; dZ is read
//     by four groups of tiles, three times of four from L2. The second kernel: 11 us alone.
//   small calls (2708 x 1433 x 64 fp32: 14.3 us): this kernel's and the second's latencies (10.7 and
//     8.0 us alone).
//   rows of dZ that are no multiple of 16 bytes (the workers load it, an element a lane): 232,965 x
//     602 x 41 111 us in fp32 and 182 in bf16, 2708 x 1433 x 7 as long as x 64.
#include "checkpoint.cuh"
#include "checkpoint_runs.cuh"
#include "launch.cuh"
#include "tc_rows.cuh"
#include "tensor_map.cuh"

namespace bigcn {

__device__ unsigned int g_grad_timeouts;

namespace {

constexpr int kGradCtas = 152;          // SMs of a GB300; the workspace query asks no device
constexpr int kWorkers = 512;
constexpr int kWorkerWarps = kWorkers / 32;
constexpr int kTeams = 2;               // of workers, which take stages in turn
constexpr int kTeamWarps = kWorkerWarps / kTeams;
constexpr int kCopyWarp = kWorkerWarps, kMmaWarp = kWorkerWarps + 1, kScaleWarp = kWorkerWarps + 2;
constexpr int kGradThreads = kWorkers + 96;
constexpr int kAccCols = 256;           // accumulator columns; as many of running sums
constexpr size_t kAlign = 256;
constexpr int kSmemMost = 227 * 1024 - 1024 - 5120;   // less alignment and static memory

__host__ __device__ constexpr int round_up_to(int x, int a) { return (x + a - 1) / a * a; }

// Shared memory of a variant: NT columns, PARTS bf16 parts of dZ, kTma: dZ comes by tensor
// copies (else its rows are not 16-byte aligned and the workers load it).
template <int NT, int PARTS, bool kTma>
struct GradShape {
    static constexpr int kTiles = kAccCols / NT;
    static constexpr bool kDirect = kTma && PARTS == 1;     // copied as an operand
    // Rows of a stage: 64 where the stages' B needs no room of its own, which halves what the
    // workers spend on barriers.
    static constexpr int kRows = kDirect ? 64 : 32;
    static constexpr int kAtom = kRows * 128;
    static constexpr int kElem = PARTS == 3 ? 4 : 2;
    static constexpr int kSlotZ = kTma ? kRows * NT * kElem : 0;
    static constexpr int kSlotQ = kTiles * kRows * 128;
    static constexpr int kSlot = round_up_to(kSlotZ + kSlotQ + kTiles * kRows * 4, 1024);
    static constexpr int kOpA = kTiles * 2 * kAtom;
    static constexpr int kPart = NT / 64 * kAtom;
    static constexpr int kOp = kOpA + (kDirect ? 0 : PARTS * kPart);
    static constexpr int kStages = 3 * (kOp + kSlot) <= kSmemMost ? 3 : 2;
    static constexpr int kFit = (kSmemMost - kStages * kOp) / kSlot;
    static constexpr int kSlots = kFit < 8 ? kFit : 8;
    static constexpr int kSmem = 1024 + kStages * kOp + kSlots * kSlot;
    // 48 (64 where there are no parts) accumulating MMAs, kRows / 16 per stage and part, between
    // two drains.
    static constexpr int kDrain = kDirect ? 16 : PARTS == 1 ? 24 : PARTS == 2 ? 12 : 8;
    static_assert(kSlots >= kTeams && kStages >= kTeams && kSlots >= kStages, "shared memory per CTA");
};

struct GradParams {
    CUtensorMap q_map;       // K rounded up to 16 bytes x N
    CUtensorMap z_map;       // F x N of dZ (kTma), or
    bool z_atoms;            // 64 x N x F / 64: all atoms of a stage are one box
    const uint8_t *exps;
    int64_t lde;
    int64_t N;
    const void *dZ;
    int64_t lddz;
    int F;
    int64_t stages;          // of kRows rows
    int nt;                  // column tiles
    int64_t tiles;           // feature tiles
    int mt;                  // feature tiles of a group
    int64_t groups;
    int parts_full, parts_last;      // runs of rows of a group, of the last group
    float *partial;          // [nt][tiles][parts_full][NT][128]
    float *colsum;           // [parts_full][nt * NT]
};

template <typename T> __device__ __forceinline__ float dz_at(const GradParams &p, int64_t i, int j) {
    return i < p.N && j < p.F ? to_f32(static_cast<const T *>(p.dZ)[i * p.lddz + j]) : 0.0f;
}

// Four int8 to bf16 pairs, exactly: 0x43qq is 128 + (q & 127), or 256 + q with q's sign bit
// cleared, so that subtracting 0x43(q & 128), 128 or 256, leaves q; times 2^e.
__device__ __forceinline__ void expand4(uint32_t w, __nv_bfloat162 factor, uint32_t &lo,
                                        uint32_t &hi) {
    const uint32_t x[2] = {__byte_perm(w, 0x43434343u, 0x4140), __byte_perm(w, 0x43434343u, 0x4342)};
    uint32_t r[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t a = x[h] & 0xFF7FFF7Fu, b = x[h] & 0xFF80FF80u;
        const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a),
                                                 *reinterpret_cast<const __nv_bfloat162 *>(&b)),
                                         factor);
        r[h] = *reinterpret_cast<const uint32_t *>(&v);
    }
    lo = r[0];
    hi = r[1];
}

// 2^(b - 127) in both halves, as unpack_factor.
__device__ __forceinline__ __nv_bfloat162 bf16_factor(uint32_t b) {
    const uint32_t f2 = b == kNanByte ? 0x7FC07FC0u : b * 0x00800080u;
    return *reinterpret_cast<const __nv_bfloat162 *>(&f2);
}

template <int PARTS>
__device__ __forceinline__ void parts_of(float v0, float v1, uint32_t (&out)[3]) {
    if constexpr (PARTS == 1) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(v0, v1);     // bf16 already: exact
        out[0] = *reinterpret_cast<const uint32_t *>(&v);
    } else {
        bf16_parts(v0, v1, out[0], out[1], out[2]);     // of 11 bits the third part is 0
    }
}

__device__ __forceinline__ float2 bf16_pair(uint32_t u) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
}

template <typename T, int NT, int PARTS, bool kTma>
__global__ void __launch_bounds__(kGradThreads, 1)
grad_rows_kernel(const __grid_constant__ GradParams p) {
    using S = GradShape<NT, PARTS, kTma>;
    constexpr int kSlots = S::kSlots, kStages = S::kStages, kDrain = S::kDrain, kRows = S::kRows;
    constexpr int kAtom = S::kAtom;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t loaded[kSlots], freed[kSlots], filled[kStages], used[kStages],
        summed, drained, done;
    __shared__ float colpart[kWorkerWarps][64];
    __shared__ uint32_t tmem_base, stop;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    unsigned char *const mem = smem_raw + (base - raw);
    constexpr int kSlot0 = kStages * S::kOp;            // slots follow the stages

    // This CTA's group of feature tiles, run of rows and columns.
    const int ny = blockIdx.x % p.nt;
    const int64_t r = blockIdx.x / p.nt, full = (p.groups - 1) * p.parts_full;
    const int64_t group = r < full ? r % (p.groups - 1) : p.groups - 1;
    const int run = int(r < full ? r / (p.groups - 1) : r - full);
    const int runs = r < full ? p.parts_full : p.parts_last;
    const int64_t tile0 = group * p.mt;
    const int mt = int(min(int64_t(p.mt), p.tiles - tile0));
    const int64_t st0 = p.stages * run / runs;
    const int n = int(p.stages * (run + 1) / runs - st0);
    const int n0 = ny * NT, cols = min(NT, p.F - n0), atoms = (cols + 63) / 64;
    const bool sums_cols = group < atoms;               // of the columns n0 + 64 group ..
    const int own = sums_cols ? int(group) : -1;

    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_addr(&tmem_base)),
                     "r"(2 * kAccCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(smem_addr(&loaded[s]), 33);       // the scale warp's lanes; boxes' bytes
            mbar_init(smem_addr(&freed[s]), S::kDirect ? 1 : kTeamWarps);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&filled[s]), kTeamWarps);
            mbar_init(smem_addr(&used[s]), 1);
        }
        mbar_init(smem_addr(&summed), 1);
        mbar_init(smem_addr(&drained), kWorkerWarps);
        mbar_init(smem_addr(&done), 1);
        stop = 0u;
        mbar_fence_init();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    volatile uint32_t *const stopv = &stop;

    float colsum[4] = {0.0f, 0.0f, 0.0f, 0.0f};

    if (warp == kCopyWarp || warp == kScaleWarp) {
        const int boxes = p.z_atoms ? NT / 64 : atoms;
        const uint32_t bytes = uint32_t(mt * kRows * 128 + (kTma ? boxes * kRows * 64 * S::kElem : 0));
        int issued = 0, s = 0;
        uint32_t slot = base + uint32_t(kSlot0), parity = 1u;
        int64_t row = st0 * kRows;
        for (int st = 0; st < n; ++st, row += kRows) {
            const bool go = st < kSlots || wait_unless(smem_addr(&freed[s]), parity, stopv);
            if (!__all_sync(kFullMask, go)) {
                *stopv = 1u;
                break;
            }
            const uint32_t bar = smem_addr(&loaded[s]);
            if (warp == kScaleWarp) {
                // Scale bytes: lane = row, four groups (128 features) a copy.
#pragma unroll
                for (int h = 0; h < kRows / 32; ++h) {
                    const int64_t i = row + 32 * h + lane;
                    const bool in = i < p.N;
                    const uint8_t *e = p.exps + (in ? i * p.lde + tile0 * 4 : 0);
                    for (int t = 0; t < mt; ++t)
                        copy4(slot + uint32_t(S::kSlotZ + S::kSlotQ + (t * kRows + 32 * h + lane) * 4),
                              in ? e + t * 4 : e, in ? 4u : 0u);
                }
                copies_arrive(bar);
            } else if (elect_one()) {
                mbar_expect(bar, bytes);
                if constexpr (kTma) {
                    if (p.z_atoms) tma_load_3d(slot, &p.z_map, 0, int(row), n0 / 64, bar);
                    else for (int a = 0; a < atoms; ++a)
                        tma_load(slot + uint32_t(a * kRows * 64 * S::kElem), &p.z_map, n0 + 64 * a,
                                 int(row), bar);
                }
                for (int t = 0; t < mt; ++t)
                    tma_load(slot + uint32_t(S::kSlotZ + t * kRows * 128), &p.q_map,
                             int(tile0 + t) * 128, int(row), bar);
            }
            issued = st + 1;
            slot += S::kSlot;
            if (++s == kSlots) s = 0, slot = base + uint32_t(kSlot0), parity ^= 1u;
            __syncwarp();
        }
        // What is still in flight lands before the shared memory is given up.
        for (int st = max(0, issued - kSlots); st < issued; ++st)
            mbar_wait(smem_addr(&loaded[st % kSlots]), uint32_t(st / kSlots) & 1u);
    } else if (warp == kMmaWarp) {
        // The warp stays together (its addresses are uniform then), one lane issues.
        const uint32_t idesc = atom_idesc(round_up_to(cols, 16));
        bool any = false;
        int s = 0, o = 0, at = 0;           // slot, stage, place in the block of kDrain
        uint32_t op_parity = 0u, drain_parity = 1u;
        for (int st = 0; st < n; ++st) {
            // (What the workers have filled they have seen loaded.)
            bool go = wait_unless(smem_addr(&filled[o]), op_parity, stopv);
            if (at == 0 && st > 0) go = go && wait_unless(smem_addr(&drained), drain_parity, stopv);
            if (!__all_sync(kFullMask, go)) {
                *stopv = 1u;
                break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t a0 = atom_desc<kRows>(base + uint32_t(o * S::kOp));
            const uint64_t b0 = atom_desc<kRows>(
                base + uint32_t(S::kDirect ? kSlot0 + s * S::kSlot : o * S::kOp + S::kOpA));
            const bool last = at + 1 == kDrain || st == n - 1;
            if (elect_one()) {
#pragma unroll 1
                for (int t = 0; t < mt; ++t)
#pragma unroll
                    for (int k = 0; k < kRows / 16; ++k)
#pragma unroll
                        for (int part = 0; part < PARTS; ++part)
                            mma_rows(tmem + uint32_t(t * NT),
                                     a0 + uint32_t((t * 2 * kAtom + k * 2048) >> 4),
                                     b0 + uint32_t((part * S::kPart + k * 2048) >> 4), idesc,
                                     at > 0 || k > 0 || part > 0);
                mma_commit(S::kDirect ? smem_addr(&freed[s]) : smem_addr(&used[o]));
                if (last) mma_commit(smem_addr(&summed));
            }
            any = true;
            if (++at == kDrain) at = 0, drain_parity ^= 1u;
            if (++s == kSlots) s = 0;
            if (++o == kStages) o = 0, op_parity ^= 1u;
        }
        if (elect_one()) {
            if (any) mma_commit(smem_addr(&done));
            else mbar_arrive(smem_addr(&done));
        }
        __syncwarp();
    } else {
        // Worker of the team that takes every second stage: of 16 rows in turn row `row`, 8
        // features 8 c .. of each tile, 4 columns 4 c .. of each atom. Loaded without tensor
        // copies, dZ is taken four rows a warp, a column per lane, the team's next stage ahead.
        const int team = warp / kTeamWarps, tw = warp % kTeamWarps;
        const int row = (tid >> 4) & 15, c = tid & 15;
        const int quad = warp & 3, quarter = warp >> 2;
        constexpr int kLoadCols = kTma ? 1 : NT / 32;
        float z[kLoadCols][4];
        auto load = [&](int st) {
            if constexpr (!kTma) {
                const int64_t i = (st0 + st) * kRows + 4 * tw;
#pragma unroll
                for (int q = 0; q < kLoadCols; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        z[q][e] = st < n && n0 + 32 * q < p.F ? dz_at<T>(p, i + e, n0 + 32 * q + lane)
                                                              : 0.0f;
            }
        };
        // Adds the accumulators of block b to the running sums: this warp's lanes, 64 columns.
        auto drain = [&](int b) -> bool {
            const bool go = wait_unless(smem_addr(&summed), uint32_t(b) & 1u, stopv);
            if (!__all_sync(kFullMask, go)) return false;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = tmem + (uint32_t(32 * quad) << 16) + uint32_t(64 * quarter);
#pragma unroll 1
            for (int w = 0; w < 2; ++w) {
                if (64 * quarter + 32 * w >= mt * NT) break;
                uint32_t acc[32], sum[32];
                tmem_ld32(at + uint32_t(32 * w), acc);
                if (b > 0) {
                    tmem_ld32(at + uint32_t(kAccCols + 32 * w), sum);
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        acc[j] = __float_as_uint(__uint_as_float(sum[j]) + __uint_as_float(acc[j]));
                }
                tmem_st32(at + uint32_t(kAccCols + 32 * w), acc);
            }
            tmem_wait_st();
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&drained));
            return true;
        };
        int taken = 0, next_drain = kDrain;         // blocks drained, the next one's end
        bool ok = true;
        load(team);
        // Slot and stage of st, and the parities of their phases.
        int s = team % kSlots, o = team % kStages;
        uint32_t sp = uint32_t(team / kSlots) & 1u, op_parity = uint32_t(team / kStages) & 1u;
        const uint32_t a_at = uint32_t((c >> 3) * kAtom) + atom_offset(row, c & 7);
        const uint32_t b_at = atom_offset(row, c >> 1) + (c & 1) * 8;
#pragma unroll 1
        for (int st = team; st < n; st += kTeams) {
            // A block is drained a stage after its end: its MMAs are done by then, and the
            // next one's first stage is filled or under way.
            if (st > next_drain) {
                ok = drain(taken);
                if (!ok) break;
                ++taken;
                next_drain += kDrain;
            }
            // (A stage's first use waits for the phase before the first, which is complete.)
            bool go = wait_unless(smem_addr(&loaded[s]), sp, stopv);
            if constexpr (S::kDirect) {
                // The slot of the stage's last use: freed by the same MMAs. (Its next phase is
                // st's own or later: kSlots >= kStages.)
                const int last = st - kStages;
                if (last >= 0)
                    go = go && wait_unless(smem_addr(&freed[last % kSlots]),
                                           uint32_t(last / kSlots) & 1u, stopv);
            } else {
                go = go && wait_unless(smem_addr(&used[o]), op_parity ^ 1u, stopv);
            }
            ok = __all_sync(kFullMask, go);
            if (!ok) break;
            const unsigned char *slot = mem + kSlot0 + s * S::kSlot;
            unsigned char *op = mem + o * S::kOp;
            // A: 8 features of a row to a 16-byte chunk. (16 rows on, a chunk is 2048 bytes on:
            // the swizzle repeats every 8.)
#pragma unroll
            for (int t = 0; t < S::kTiles; ++t) {
                if (t >= mt) break;
                const unsigned char *sq = slot + S::kSlotZ + t * kRows * 128 + row * 128 + c * 8;
                const unsigned char *se =
                    slot + S::kSlotZ + S::kSlotQ + (t * kRows + row) * 4 + (c >> 2);
                unsigned char *dst = op + 2 * t * kAtom + a_at;
#pragma unroll
                for (int h = 0; h < kRows / 16; ++h) {
                    const uint2 q = *reinterpret_cast<const uint2 *>(sq + h * 2048);
                    const __nv_bfloat162 f = bf16_factor(se[h * 64]);
                    uint4 v;
                    expand4(q.x, f, v.x, v.y);
                    expand4(q.y, f, v.z, v.w);
                    *reinterpret_cast<uint4 *>(dst + h * 2048) = v;
                }
            }
            // B: dZ's parts, and its columns' sums.
            if constexpr (S::kDirect) {
                if (sums_cols)
#pragma unroll
                    for (int h = 0; h < kRows / 16; ++h) {
                        const uint2 u =
                            *reinterpret_cast<const uint2 *>(slot + own * kAtom + b_at + h * 2048);
                        const float2 f0 = bf16_pair(u.x), f1 = bf16_pair(u.y);
                        colsum[0] += f0.x;
                        colsum[1] += f0.y;
                        colsum[2] += f1.x;
                        colsum[3] += f1.y;
                    }
            } else if constexpr (kTma) {
#pragma unroll
                for (int a = 0; a < NT / 64; ++a) {
                    if (a >= atoms) break;
#pragma unroll
                    for (int h = 0; h < kRows / 16; ++h) {
                        float v[4];
                        if constexpr (PARTS == 3) {
                            const float4 x = *reinterpret_cast<const float4 *>(
                                slot + (a * kRows + row) * 256 + c * 16 + h * 4096);
                            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
                        } else {
                            const uint2 u = *reinterpret_cast<const uint2 *>(
                                slot + (a * kRows + row) * 128 + c * 8 + h * 2048);
                            const float2 f0 = __half22float2(*reinterpret_cast<const __half2 *>(&u.x));
                            const float2 f1 = __half22float2(*reinterpret_cast<const __half2 *>(&u.y));
                            v[0] = f0.x, v[1] = f0.y, v[2] = f1.x, v[3] = f1.y;
                        }
                        if (a == own)
#pragma unroll
                            for (int e = 0; e < 4; ++e) colsum[e] += v[e];
                        uint32_t x[3], y[3];
                        parts_of<PARTS>(v[0], v[1], x);
                        parts_of<PARTS>(v[2], v[3], y);
                        unsigned char *dst = op + S::kOpA + a * kAtom + b_at + h * 2048;
#pragma unroll
                        for (int q = 0; q < PARTS; ++q)
                            *reinterpret_cast<uint2 *>(dst + q * S::kPart) = make_uint2(x[q], y[q]);
                    }
                }
            } else {
#pragma unroll
                for (int q = 0; q < kLoadCols; ++q) {
                    if (q / 2 >= atoms) break;
                    if (q / 2 == own)
                        colsum[q % 2] += (z[q][0] + z[q][1]) + (z[q][2] + z[q][3]);
                    // Neighbouring lanes exchange a row's value: the even one writes the pair of
                    // columns of rows 0 and 2, the odd one of rows 1 and 3.
                    const bool odd = lane & 1;
                    const int col = 32 * (q % 2) + (lane & ~1);
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const float got =
                            __shfl_xor_sync(kFullMask, odd ? z[q][e] : z[q][e + 1], 1);
                        uint32_t part[3];
                        parts_of<PARTS>(odd ? got : z[q][e], odd ? z[q][e + 1] : got, part);
                        unsigned char *dst = op + S::kOpA + (q / 2) * kAtom +
                                             atom_offset(4 * tw + e + (odd ? 1 : 0), col >> 3) +
                                             (col & 7) * 2;
#pragma unroll
                        for (int w = 0; w < PARTS; ++w)
                            *reinterpret_cast<uint32_t *>(dst + w * S::kPart) = part[w];
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (!S::kDirect) mbar_arrive(smem_addr(&freed[s]));
                mbar_arrive(smem_addr(&filled[o]));
            }
            load(st + kTeams);
            s += kTeams;
            if (s >= kSlots) s -= kSlots, sp ^= 1u;
            o += kTeams;
            if (o >= kStages) o -= kStages, op_parity ^= 1u;
        }
        for (; ok && taken * kDrain < n; ++taken) ok = drain(taken);
        if (!ok) *stopv = 1u;
    }

    // Every MMA has ended once `done` completes. A CTA whose waits ran out leaves NaN for its sums.
    const bool ended = mbar_wait(smem_addr(&done), 0u);
    const bool ok = __syncthreads_and(ended && *stopv == 0u) != 0;
    float *const own_colsum = p.colsum + int64_t(run) * p.nt * NT + n0 + 64 * own;
    const int own_cols = sums_cols ? min(64, cols - 64 * own) : 0;
    allow_dependent_launch();
    if (!ok) {
        if (tid == 0) atomicAdd(&g_grad_timeouts, 1u);
        abandon_run(p.partial, p.tiles, p.parts_full, NT, ny, tile0, mt, run, own_colsum, own_cols);
    }
    if (ok && warp < kWorkerWarps) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int quad = warp & 3, quarter = warp >> 2, f = 32 * quad + lane;
#pragma unroll 1
        for (int w = 0; w < 2; ++w) {
            const int at = 64 * quarter + 32 * w, t = at / NT, col = at % NT;
            if (t >= mt) break;
            uint32_t sum[32];
            tmem_ld32(tmem + (uint32_t(32 * quad) << 16) + uint32_t(kAccCols + at), sum);
            float *dst = run_sums(p.partial, p.tiles, p.parts_full, NT, ny, tile0 + t, run) + col * 128 + f;
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (col + j < cols) dst[j * 128] = __uint_as_float(sum[j]);
        }
        if (sums_cols) {
            // Rows of a warp, then the warps in order.
            if constexpr (kTma) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    colsum[e] += __shfl_xor_sync(kFullMask, colsum[e], 16);
                    if (lane < 16) colpart[warp][4 * lane + e] = colsum[e];
                }
            } else {
                colpart[warp][lane] = colsum[0];
                colpart[warp][32 + lane] = colsum[1];
            }
            asm volatile("bar.sync 1, 512;" ::: "memory");
            if (tid < own_cols) {
                float t = 0.0f;
                for (int w = 0; w < kWorkerWarps; ++w) t += colpart[w][tid];
                own_colsum[tid] = t;
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == kMmaWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                     "r"(2 * kAccCols));
}

// How a call is cut into CTAs.
struct GradPlan {
    int NT, nt, mt, parts_full, parts_last;
    int64_t tiles, groups;
    size_t partial_bytes, colsum_bytes;
};

// NT: the widest tile that F fills and for which there are as many groups of feature tiles
// as 64-column atoms to sum (each sums one); at most `most`. mt: all the tiles that fit
// unless runs of rows get shorter than 256, where fewer tiles and longer runs mean
// less to add up: 2708 x 1433 x 64, fp32. A stage costs a CTA about mt + 3 (the workers' time:
// a tile of A, against dZ's parts and the barriers), by which the last group's runs are longer.
GradPlan grad_plan(int64_t N, int K, int F, int most) {
    GradPlan g;
    g.tiles = (int64_t(K) + 127) / 128;
    g.NT = 64;
    for (int NT = 128; NT <= most; NT *= 2)
        if (F > NT / 2 && (g.tiles + kAccCols / NT - 1) / (kAccCols / NT) >= NT / 64) g.NT = NT;
    g.nt = int((int64_t(F) + g.NT - 1) / g.NT);
    const int64_t longest = N / 128 > 1 ? N / 128 : 1;             // runs of 128 rows or more
    auto cut = [&](int mt) {
        g.mt = mt;
        g.groups = (g.tiles + mt - 1) / mt;
        const int rest = int(g.tiles - (g.groups - 1) * mt);
        const int64_t cost = (g.groups - 1) * (mt + 3) + rest + 3;
        auto runs = [&](int tiles) {
            int64_t s = int64_t(kGradCtas / g.nt) * (tiles + 3) / cost;
            s = s < longest ? s : longest;
            return int(s > 1 ? s : 1);
        };
        g.parts_last = runs(rest);
        g.parts_full = g.groups > 1 ? runs(mt) : g.parts_last;
    };
    int mt = kAccCols / g.NT;
    if (mt > g.tiles) mt = int(g.tiles);
    for (cut(mt); mt > 1 && N / g.parts_full < 256; cut(mt)) mt = (mt + 1) / 2;
    g.partial_bytes = size_t(g.nt) * size_t(g.tiles) * size_t(g.parts_full) * size_t(g.NT) * 128 * 4;
    g.colsum_bytes = size_t(g.parts_full) * size_t(g.nt) * size_t(g.NT) * 4;
    return g;
}

size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
size_t plan_bytes(const GradPlan &g) { return round_up(g.partial_bytes) + round_up(g.colsum_bytes); }

// dZ's widest tile: loaded by the workers it is kept in registers a stage ahead, 128
// columns of it.
constexpr int kMostTma = 256, kMostLoaded = 128;

template <typename T, int NT, int PARTS, bool kTma>
void launch_rows(const GradParams &p, unsigned grid, cudaStream_t s) {
    using S = GradShape<NT, PARTS, kTma>;
    cudaFuncSetAttribute(grad_rows_kernel<T, NT, PARTS, kTma>,
                         cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    grad_rows_kernel<T, NT, PARTS, kTma><<<grid, kGradThreads, S::kSmem, s>>>(p);
}

template <typename T, int PARTS>
void launch_type(const GradParams &p, int NT, bool tma, unsigned grid, cudaStream_t s) {
    if (tma && NT == 256) launch_rows<T, 256, PARTS, true>(p, grid, s);
    else if (tma && NT == 128) launch_rows<T, 128, PARTS, true>(p, grid, s);
    else if (tma) launch_rows<T, 64, PARTS, true>(p, grid, s);
    else if (NT == 128) launch_rows<T, 128, PARTS, false>(p, grid, s);
    else launch_rows<T, 64, PARTS, false>(p, grid, s);
}

}  // namespace

uint32_t take_grad_timeouts() {
    unsigned int n = 0;
    const unsigned int zero = 0;
    if (cudaMemcpyFromSymbol(&n, g_grad_timeouts, sizeof(n)) != cudaSuccess ||
        cudaMemcpyToSymbol(g_grad_timeouts, &zero, sizeof(zero)) != cudaSuccess) {
        cudaGetLastError();
        return ~0u;
    }
    return n;
}

}  // namespace bigcn

using namespace bigcn;

extern "C" size_t bigcn_checkpoint_weight_grad_workspace_bytes(int64_t N, int32_t K, int32_t F) {
    if (N < 0 || N > int64_t(INT32_MAX) || K < 1 || K > kMaxCols || F < 1 || F > kMaxCols ||
        int64_t(K) > kMaxElems / (1 << 20) / F)
        return 0;
    const size_t a = plan_bytes(grad_plan(N, K, F, kMostTma));
    const size_t b = plan_bytes(grad_plan(N, K, F, kMostLoaded));
    return a > b ? a : b;
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

    GradParams p;
    const CUtensorMapDataType type = dtype == BIGCN_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : dtype == BIGCN_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                           : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    // Tensor copies want rows that start on 16-byte boundaries. A bf16 dZ is copied as an operand,
    // in stages of 64 rows (GradShape); all atoms of a stage at once where F is a multiple of 64
    // (behind a last partial atom the box would read past the rows' end).
    const int64_t zrow = lddz * int64_t(es);
    const bool direct = dtype == BIGCN_BF16;
    const int most = aligned_to(dZ, 16) && zrow % 16 == 0 ? kMostTma : kMostLoaded;
    p.z_atoms = F % 64 == 0;
    const bool tma =
        most == kMostTma &&
        (p.z_atoms ? encode_map(&p.z_map, type, dZ, 64, N, zrow, 64, direct ? 64 : 32, direct, F / 64,
                            64 * int64_t(es), grad_plan(N, K, F, most).NT / 64)
                   : encode_map(&p.z_map, type, dZ, F, N, zrow, 64, direct ? 64 : 32, direct));
    const int rows = tma && direct ? 64 : 32;
    const int64_t width = (int64_t(K) + 15) / 16 * 16;
    if (!encode_map(&p.q_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, q, width, N, N > 1 ? ldq : width, 128, rows,
                false))
        return BIGCN_ERR_CUDA;
    p.stages = (N + rows - 1) / rows;
    const GradPlan g = grad_plan(N, K, F, tma ? kMostTma : kMostLoaded);
    p.exps = exps;
    p.lde = lde;
    p.N = N;
    p.dZ = dZ;
    p.lddz = lddz;
    p.F = F;
    p.nt = g.nt;
    p.tiles = g.tiles;
    p.mt = g.mt;
    p.groups = g.groups;
    p.parts_full = g.parts_full;
    p.parts_last = g.parts_last;
    p.partial = static_cast<float *>(workspace);
    p.colsum = reinterpret_cast<float *>(static_cast<char *>(workspace) + round_up(g.partial_bytes));
    const int64_t grid = ((g.groups - 1) * g.parts_full + g.parts_last) * g.nt;
    if (dtype == BIGCN_F32) launch_type<float, 3>(p, g.NT, tma, unsigned(grid), s);
    else if (dtype == BIGCN_BF16) launch_type<__nv_bfloat16, 1>(p, g.NT, tma, unsigned(grid), s);
    else launch_type<__half, 2>(p, g.NT, tma, unsigned(grid), s);
    const GradSumParams sum{p.partial, p.colsum, g.tiles, g.groups, g.parts_full, g.parts_last,
                            g.mt,      g.NT,     g.nt * g.NT, K, F, gamma, beta, dW, lddw, db};
    launch_kernel(grad_sum_kernel, dim3(unsigned(g.tiles * ((F + 3) / 4))), dim3(kSumThreads), 0, s,
                  true, dim3(1, 1, 1), sum);
    return launch_status();
}
