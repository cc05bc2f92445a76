// Activations kept in 8 bits, and the element types of the row-wise operators.
//
// A checkpoint holds a row in groups of 32 columns: v = q 2^(b - 127) with q an
// int8 in [-127, 127] and b one byte per group, the least b >= 1 by which the
// group's largest magnitude rounds to at most 127. A power of two rather than
// amax / 127 costs at most one of the 8 bits and buys three things: a byte per
// scale, a division-free packing whose result does not depend on rounding, and
// values of 7 significant bits, exact in bf16 and so exact as an operand of the
// tensor cores. A group with a NaN or an infinity has b = 255 and q = 0; its values are NaN.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "bigcn_internal.cuh"

namespace bigcn {

constexpr int kGroup = 32;              // columns per scale
constexpr uint32_t kNanByte = 255;
constexpr int kMaxCols = 1 << 30;       // of a row: 32-bit column indices step past its end

__host__ __device__ constexpr int64_t checkpoint_groups(int64_t K) {
    return (K + kGroup - 1) / kGroup;
}

// The scale byte of a group from the bits of its largest magnitude (the integer
// maximum of |v|'s bits, by which a NaN is larger than an infinity). With
// amax = 1.f 2^(x - 127), amax 2^(133 - x) lies in [64, 128) and rounds to 128
// from 127.5 on (f >= 0x7F0000), where the step is doubled: adding 0x10000 carries
// into the exponent just there.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
    const int b = int((amax_bits + 0x10000u) >> 23) - 6;
    return amax_bits >= 0x7F800000u ? kNanByte : uint32_t(max(b, 1));
}

// 2^(127 - b), which scales a group's values to [-127.5, 127.5). (An infinity for a NaN
// group, whose q are written 0 without it.)
__device__ __forceinline__ float pack_factor(uint32_t b) {
    return __uint_as_float(0x7F000000u - (b << 23));
}

// 2^(b - 127), NaN for a NaN group.
__device__ __forceinline__ float unpack_factor(uint32_t b) {
    return __uint_as_float(b == kNanByte ? 0x7FC00000u : b << 23);
}

// v times a group's factor to int8, rounded to nearest even, in the low byte: v f + 1.5 2^23,
// rounded once, has the two's complement of the nearest integer in its low bits (v f is exact,
// the factor a power of two). One multiply-add instead of a conversion, which has an eighth of
// its rate.
__device__ __forceinline__ uint32_t q_low(float v, float f) {
    return __float_as_uint(fmaf(v, f, 12582912.0f));
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) {
    return __bfloat162float(v);
}

// Results are rounded to the tensor's type once, to nearest even.
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
    return __float2bfloat16_rn(v);
}

inline size_t dtype_bytes(int32_t dtype) {
    return dtype == BIGCN_F32 ? 4 : dtype == BIGCN_BF16 || dtype == BIGCN_F16 ? 2 : 0;
}

// The checks that every call with a checkpoint makes of it (q and exps not NULL).
inline bool checkpoint_strides_ok(int64_t N, int32_t K, int64_t ldq, int64_t lde) {
    return ldq >= K && ldq % 16 == 0 && lde >= checkpoint_groups(K) && lde % 4 == 0 &&
           (N == 0 || (N <= kMaxElems / ldq && N <= kMaxElems / lde));
}
inline bool checkpoint_aligned(const void *q, const void *exps) {
    return aligned_to(q, 16) && aligned_to(exps, 4);
}
// Bytes that a call may touch: rows of round_up(K, 16) bytes and round_up(groups, 4).
inline size_t checkpoint_q_span(int64_t N, int32_t K, int64_t ldq) {
    return span_bytes(N, (int64_t(K) + 15) / 16 * 16, ldq, 1);
}
inline size_t checkpoint_exps_span(int64_t N, int32_t K, int64_t lde) {
    return span_bytes(N, (checkpoint_groups(K) + 3) / 4 * 4, lde, 1);
}

}  // namespace bigcn
