// Rows in microscaled 4-bit floating point: groups of 32 columns, v = m 2^(b - 127) with m an
// e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign) and b one byte per group, the least b >= 1 by which
// the group's largest magnitude rounds to at most 6. Two codes a byte, the even column in the low
// half; a group is 16 bytes. A group with a NaN or an infinity has b = 255 and codes 0: its values
// are NaN, to the tensor core (whose scale type, ue8m0, has that NaN) as to the unpacking.
//
// A power of two as scale makes the packing exact but for the one rounding to e2m1: v 2^(127 - b)
// is exact (or below 2^-126, which rounds to 0 either way), and the conversion rounds to nearest
// even as the definition asks.
#pragma once

#include "checkpoint.cuh"

namespace bigcn {

// The scale byte from the bits of the largest magnitude: with amax = 1.f 2^(x - 127), the byte
// x - 2 brings it to [4, 8); from 7 on (f >= 0x600000), where it would round to 8, x - 1.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax_bits) {
    const int b = int((amax_bits + 0x200000u) >> 23) - 2;
    return amax_bits >= 0x7F800000u ? kNanByte : uint32_t(max(b, 1));
}

// Eight values as they are scaled already to a word of codes, value 0 in the low bits.
__device__ __forceinline__ uint32_t fp4_codes(float v0, float v1, float v2, float v3, float v4,
                                              float v5, float v6, float v7) {
    uint32_t r;
    asm("{\n.reg .b8 a, b, c, d;\n"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        "mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(r)
        : "f"(v0), "f"(v1), "f"(v2), "f"(v3), "f"(v4), "f"(v5), "f"(v6), "f"(v7));
    return r;
}

// A word of codes to eight halves (exact), in pairs.
__device__ __forceinline__ void fp4_halves(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n.reg .b8 a, b, c, d;\n"
        "mov.b32 {a, b, c, d}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}

// The checks that every call with 4-bit rows makes of them.
inline bool fp4_strides_ok(int64_t N, int32_t K, int64_t ldq, int64_t lde) {
    return ldq >= checkpoint_groups(K) * 16 && ldq % 16 == 0 && lde >= checkpoint_groups(K) &&
           lde % 4 == 0 && (N == 0 || (N <= kMaxElems / ldq && N <= kMaxElems / lde));
}
inline size_t fp4_q_span(int64_t N, int32_t K, int64_t ldq) {
    return span_bytes(N, checkpoint_groups(K) * 16, ldq, 1);
}

}  // namespace bigcn
