// tcgen05 building blocks for contractions over rows (A^T B with row-major A and B):
// bf16 operands kept as they lie in memory, features along the 128-byte swizzled rows
// (MN-major), a contraction row after the other; tensor copies into them; waits that end
// when another role of the CTA has given up.
#pragma once

#include <cuda.h>

#include <cstdint>

#include "async.cuh"
#include "tc.cuh"

namespace bigcn {

// A tile is built of atoms of 64 columns (128 bytes) by the contraction rows of a stage, one
// atom after the other; within an atom 8 rows of 128 bytes make a swizzle unit.

// Byte offset of the 16-byte chunk c (8 columns) of row r in an atom.
__device__ __forceinline__ uint32_t atom_offset(int r, int c) {
    return uint32_t(r * 128 + ((c ^ (r & 7)) << 4));
}

// Shared-memory matrix descriptor, MN-major, 128B swizzle: atoms of kRows rows one after the
// other along the columns (leading byte offset), groups of 8 rows 1024 bytes apart along the
// contraction (stride byte offset), descriptor version 1.
template <int kRows> __device__ __forceinline__ uint64_t atom_desc(uint32_t saddr) {
    uint64_t d = uint64_t((saddr >> 4) & 0x3FFFu);
    d |= uint64_t((kRows * 128) >> 4) << 16;
    d |= uint64_t(1024 >> 4) << 32;
    d |= uint64_t(1) << 46;
    d |= uint64_t(2) << 61;
    return d;
}

// Instruction descriptor: BF16 x BF16 -> F32, both MN-major, M = 128, N = n.
__device__ __forceinline__ uint32_t atom_idesc(int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | (uint32_t(n >> 3) << 17) |
           (uint32_t(kUmmaM >> 4) << 24);
}

__device__ __forceinline__ void mma_rows(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc,
                                         bool accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u));
}

// True for one lane of a warp that is together, always the same one.
__device__ __forceinline__ bool elect_one() {
    uint32_t on;
    asm volatile(
        "{\n.reg .pred p;\n"
        "elect.sync _|p, 0xffffffff;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(on));
    return on != 0;
}

__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
        : "memory");
}

// 32 columns of this warp's lanes, loaded when it returns (one statement with the wait, so that
// nothing that uses them is moved between).
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
          "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Two values as three bf16 parts each, in pairs: the upper halves of v, of what is left
// (exact), and what is left then, 8 bits of the 24 each: together v, but where the last part's
// bits pass below bf16's least subnormal, 2^-133 (|v| < 2^-110), within 2^-134. A NaN or an
// infinity leaves a NaN in the middle part.
__device__ __forceinline__ void bf16_parts(float v0, float v1, uint32_t &hi, uint32_t &mid,
                                           uint32_t &lo) {
    const uint32_t u0 = __float_as_uint(v0), u1 = __float_as_uint(v1);
    const float r0 = v0 - __uint_as_float(u0 & 0xFFFF0000u);
    const float r1 = v1 - __uint_as_float(u1 & 0xFFFF0000u);
    const uint32_t w0 = __float_as_uint(r0), w1 = __float_as_uint(r1);
    hi = __byte_perm(u0, u1, 0x7632);
    mid = __byte_perm(w0, w1, 0x7632);
    const __nv_bfloat162 l = __floats2bfloat162_rn(r0 - __uint_as_float(w0 & 0xFFFF0000u),
                                                   r1 - __uint_as_float(w1 & 0xFFFF0000u));
    lo = *reinterpret_cast<const uint32_t *>(&l);
}

// A box of a two-dimensional tensor at (x, y) into shared memory; counts its bytes on bar.
// x times the element size is a multiple of 16.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y,
                                         uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], "
        "[%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z,
                                            uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], "
        "[%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
}

// Four bytes from memory to shared memory, zeros where `bytes` is 0; and this thread's
// arrival on bar once all its earlier such copies have landed (at once where it made none), one of
// those that the barrier was initialised for.
__device__ __forceinline__ void copy4(uint32_t dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ void copies_arrive(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// mbar_wait that also ends once another role of the CTA has set *stop; false then, or
// after kWaitLimit polls.
__device__ __forceinline__ bool wait_unless(uint32_t bar, uint32_t parity,
                                            const volatile uint32_t *stop) {
    for (uint32_t it = 0; it < kWaitLimit; ++it) {
        uint32_t done;
        asm volatile(
            "{\n.reg .pred p;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
            "selp.u32 %0, 1, 0, p;\n}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
        if (done) return true;
        if (*stop) return false;
    }
    return false;
}

}  // namespace bigcn
