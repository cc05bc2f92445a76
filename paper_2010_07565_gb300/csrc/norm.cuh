// What the row-wise kernels of layer norm and the checkpoints share: how a row is laid over
// threads, 16 bytes of columns at a time, packed arithmetic, sums over a row's threads.
//
// A row lies in the registers of `tpr` threads (a power of two), J pieces of V elements each
// (16 bytes: 4 fp32 or 8 16-bit columns): piece j of thread t holds columns (j tpr + t) V ..
// + V - 1, whatever the rows' alignment, so that a group of 32 columns lies in 32 / V lanes. Rows
// that are aligned to A < 16 bytes only are read and written in 16 / A accesses a piece, which
// share their sectors in L1.
//
// These kernels are bound by memory only if they issue few instructions (16 an element and
// SM cycle at 5 bytes an element fill all issue slots): elements go through packed fp32
// arithmetic in pairs, and maxima of two groups share a word.
#pragma once

#include <type_traits>

#include "checkpoint.cuh"
#include "launch.cuh"

namespace bigcn {

constexpr int kRowThreads = 256;        // threads of a block, or of a row where that is more
constexpr int kMostRowThreads = 512;

template <typename T> constexpr int kPiece = 16 / int(sizeof(T));      // V

// ---- 16 bytes of a row --------------------------------------------------------------------
// Rows aligned to 8 bytes lie at 0 or 8 of 16, each row at the same for all its pieces: `whole`,
// by which its pieces are one access or two, is a branch that the row's threads take together
// (232,965 x 602 fp32, rows at 0 and 8 in turn: forward and its checkpoint read back 355 -> 309 us,
// backward 305 -> 247). Not
// so where a warp holds several rows, which would part (90,863 x 55 columns: 37 -> 51 us), and not
// by the four places of rows aligned to 4 bytes, whose code is too long (100,000 x 601 fp32:
// backward 132 -> 310 us).
template <int A> __device__ __forceinline__ bool whole_pieces(const void *row, bool together) {
    return A == 8 && together && (reinterpret_cast<uintptr_t>(row) & 15) == 0;
}

// 16 bytes as they were read. A piece of a row that is aligned to 2 bytes may start 2 bytes past a
// word (`odd`): it is read as the three words between and a half at each end, and joined by
// settled(), later: a use behind each load would wait for it (100,000 x 601 bf16: backward from
// the checkpoint 238 -> 203 us, from its input 323 -> 245).
struct OddPiece {
    uint4 w;                 // odd: three words and the half before them
    uint32_t end;            // odd: the half behind them
};
template <int A> using Raw = typename std::conditional<A == 2, OddPiece, uint4>::type;
template <int A> __device__ __forceinline__ Raw<A> raw_zero() {
    if constexpr (A == 2) return {make_uint4(0u, 0u, 0u, 0u), 0u};
    else return make_uint4(0u, 0u, 0u, 0u);
}
template <int A> __device__ __forceinline__ bool odd_pieces(const void *row) {
    return A == 2 && (reinterpret_cast<uintptr_t>(row) & 2) != 0;
}
template <int A> __device__ __forceinline__ Raw<A> load16(const void *p, bool whole, bool odd) {
    if constexpr (A == 16) {
        return *static_cast<const uint4 *>(p);
    } else if constexpr (A == 8) {
        if (whole) return *static_cast<const uint4 *>(p);
        const uint2 *q = static_cast<const uint2 *>(p);
        const uint2 a = q[0], b = q[1];
        return make_uint4(a.x, a.y, b.x, b.y);
    } else if constexpr (A == 4) {
        const uint32_t *q = static_cast<const uint32_t *>(p);
        return make_uint4(q[0], q[1], q[2], q[3]);
    } else {
        if (!odd) return {load16<4>(p, false, false), 0u};
        const uint16_t *h = static_cast<const uint16_t *>(p);
        const uint32_t *q = reinterpret_cast<const uint32_t *>(h + 1);
        return {make_uint4(q[0], q[1], q[2], h[0]), h[7]};
    }
}
template <int A> __device__ __forceinline__ uint4 settled(const Raw<A> &r, bool odd) {
    if constexpr (A == 2) {
        if (!odd) return r.w;
        return make_uint4(__byte_perm(r.w.w, r.w.x, 0x5410), __byte_perm(r.w.x, r.w.y, 0x5432),
                          __byte_perm(r.w.y, r.w.z, 0x5432), __byte_perm(r.w.z, r.end, 0x5432));
    } else {
        return r;
    }
}
template <int A> __device__ __forceinline__ void store16(void *p, uint4 v, bool whole) {
    if constexpr (A == 16) {
        *static_cast<uint4 *>(p) = v;
    } else if constexpr (A == 8) {
        if (whole) {
            store16<16>(p, v, true);
        } else {
            static_cast<uint2 *>(p)[0] = make_uint2(v.x, v.y);
            static_cast<uint2 *>(p)[1] = make_uint2(v.z, v.w);
        }
    } else if constexpr (A == 4) {
        uint32_t *q = static_cast<uint32_t *>(p);
        q[0] = v.x;
        q[1] = v.y;
        q[2] = v.z;
        q[3] = v.w;
    } else {
        if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
            store16<4>(p, v, false);
            return;
        }
        uint16_t *h = static_cast<uint16_t *>(p);
        uint32_t *q = reinterpret_cast<uint32_t *>(h + 1);
        h[0] = uint16_t(v.x);
        q[0] = __byte_perm(v.x, v.y, 0x5432);
        q[1] = __byte_perm(v.y, v.z, 0x5432);
        q[2] = __byte_perm(v.z, v.w, 0x5432);
        h[7] = uint16_t(v.w >> 16);
    }
}

// The first n < V elements of a piece (zeros behind them), and their store. 16-bit columns at p, a multiple
// of 4, come as words and a last half, each into the register that it stays in: with an element a load the
// joins stood behind the loads and waited for each (400,000 x 500 fp16: backward 504 us, x 504 275).
template <typename T> __device__ __forceinline__ uint4 load_some(const T *p, int n) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
            if (e < n) w[e] = reinterpret_cast<const uint32_t *>(p)[e];
        } else {
            if (2 * e + 1 < n) w[e] = reinterpret_cast<const uint32_t *>(p)[e];
            else if (2 * e < n) w[e] = reinterpret_cast<const uint16_t *>(p)[2 * e];
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T> __device__ __forceinline__ void store_some(T *p, uint4 v, int n) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) reinterpret_cast<uint32_t *>(p)[e] = w[e];
    } else if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (2 * e + 1 < n) reinterpret_cast<uint32_t *>(p)[e] = w[e];
            else if (2 * e < n) reinterpret_cast<uint16_t *>(p)[2 * e] = uint16_t(w[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) reinterpret_cast<uint16_t *>(p)[e] = uint16_t(w[e / 2] >> (16 * (e % 2)));
    }
}
template <typename T, int A>
__device__ __forceinline__ Raw<A> load_piece(const T *p, int n, bool whole, bool odd) {
    if (n >= kPiece<T>) return load16<A>(p, whole, odd);
    if constexpr (A == 2) {
        if (odd) {          // the first half, then words, and a half where n is even
            const uint4 v = load_some(p + 1, n - 1);
            return {make_uint4(v.x, v.y, v.z, reinterpret_cast<const uint16_t *>(p)[0]), 0u};
        }
        return {load_some(p, n), 0u};
    } else {
        return load_some(p, n);
    }
}
template <typename T, int A>
__device__ __forceinline__ void store_piece(T *p, uint4 v, int n, bool whole) {
    if (n >= kPiece<T>) store16<A>(p, v, whole);
    else store_some(p, v, n);
}

// ---- pairs of fp32 ------------------------------------------------------------------------
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

template <typename T>
__device__ __forceinline__ void unpack16(uint4 w, float2 (&v)[kPiece<T> / 2]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            v[e] = make_float2(__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (std::is_same<T, __half>::value)
                v[e] = __half22float2(*reinterpret_cast<const __half2 *>(&u[e]));
            else v[e] = make_float2(__uint_as_float(u[e] << 16), __uint_as_float(u[e] & 0xFFFF0000u));
        }
    }
}
// Rounded to T once, to nearest even.
template <typename T>
__device__ __forceinline__ uint4 pack16(const float2 (&v)[kPiece<T> / 2]) {
    uint32_t u[4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            u[2 * e] = __float_as_uint(v[e].x);
            u[2 * e + 1] = __float_as_uint(v[e].y);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(v[e].x, v[e].y);
                u[e] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[e].x, v[e].y);
                u[e] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// Zeros in the elements of a piece from n on.
template <int H> __device__ __forceinline__ void clear_from(float2 (&v)[H], int n) {
#pragma unroll
    for (int e = 0; e < H; ++e) {
        v[e].x = 2 * e < n ? v[e].x : 0.0f;
        v[e].y = 2 * e + 1 < n ? v[e].y : 0.0f;
    }
}

// V entries of gamma or beta at p, of which n lie in the row; `aligned`: p to 32 bytes. Eight are
// one load of 32 bytes: two of 16, 32 bytes apart between lanes, take twice the L1 cycles
// (8191 x 8192 fp16: L1 at 82 %, 70 us). Loaded anew for every use: the compiler would keep
// them across a loop over rows in registers that it then spills.
template <int H>
__device__ __forceinline__ void load_params(const float *p, bool aligned, int n, float2 (&v)[H]) {
    if (aligned && n >= 2 * H) {
        if constexpr (H == 4)
            asm volatile("ld.global.nc.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(v[0].x), "=f"(v[0].y), "=f"(v[1].x), "=f"(v[1].y), "=f"(v[2].x),
                           "=f"(v[2].y), "=f"(v[3].x), "=f"(v[3].y)
                         : "l"(p));
        else
            asm volatile("ld.global.nc.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(v[0].x), "=f"(v[0].y), "=f"(v[1].x), "=f"(v[1].y)
                         : "l"(p));
    } else {
#pragma unroll
        for (int e = 0; e < H; ++e) {
            v[e].x = 2 * e < n ? __ldg(p + 2 * e) : 0.0f;
            v[e].y = 2 * e + 1 < n ? __ldg(p + 2 * e + 1) : 0.0f;
        }
    }
}

// What stands in for a gamma or a beta that is not given, read with a stride of 0.
static __device__ __align__(32) const float kOnes[8] = {1, 1, 1, 1, 1, 1, 1, 1};
static __device__ __align__(32) const float kZeros[8] = {0, 0, 0, 0, 0, 0, 0, 0};

// The largest magnitude of a piece as bits (a NaN is larger than an infinity).
template <int H> __device__ __forceinline__ uint32_t top_bits(const float2 (&v)[H]) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < H; ++e)
        asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(v[e].x), "f"(v[e].y));
    return __float_as_uint(m);
}

// Largest magnitudes of the groups of 32 columns that this lane's pieces belong to (kLanes
// neighbouring lanes each), two to a word: a scale byte needs the upper 16 bits only.
template <int kLanes, int J>
__device__ __forceinline__ void group_tops(const uint32_t (&own)[J], uint32_t (&top)[J]) {
#pragma unroll
    for (int j = 0; j < J; j += 2) {
        uint32_t w = __byte_perm(own[j], j + 1 < J ? own[j + 1 < J ? j + 1 : j] : 0u, 0x7632);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1)
            w = __vmaxu2(w, __shfl_xor_sync(kFullMask, w, o));
        top[j] = w << 16;
        if (j + 1 < J) top[j + 1 < J ? j + 1 : j] = w & 0xFFFF0000u;
    }
}

// A piece to int8 and back (checkpoint.cuh has the rounding): V bytes as one word or two.
template <int H> using QPiece = typename std::conditional<H == 4, uint2, uint32_t>::type;
__device__ __forceinline__ uint32_t quantise4(float2 a, float2 b, float f) {
    const float2 x = __ffma2_rn(a, both(f), both(12582912.0f));
    const float2 y = __ffma2_rn(b, both(f), both(12582912.0f));
    return __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040),
                       __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
}
// By the group's scale byte; zeros in a NaN group, whose last columns may lie behind the row.
template <int H> __device__ __forceinline__ QPiece<H> quantise_piece(const float2 (&v)[H], uint32_t b) {
    const float f = pack_factor(b);
    const uint32_t keep = b == kNanByte ? 0u : ~0u;
    if constexpr (H == 2) return quantise4(v[0], v[1], f) & keep;
    else return make_uint2(quantise4(v[0], v[1], f) & keep, quantise4(v[2], v[3], f) & keep);
}
__device__ __forceinline__ void dequantise4(uint32_t w, float f, float2 &a, float2 &b) {
    const uint32_t u = w ^ 0x80808080u;
    float m[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        m[e] = __uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440u + uint32_t(e)));
    a = __fmul2_rn(__fadd2_rn(make_float2(m[0], m[1]), both(-8388736.0f)), both(f));
    b = __fmul2_rn(__fadd2_rn(make_float2(m[2], m[3]), both(-8388736.0f)), both(f));
}
template <int H> __device__ __forceinline__ void dequantise_piece(QPiece<H> w, float f, float2 (&v)[H]) {
    if constexpr (H == 2) {
        dequantise4(w, f, v[0], v[1]);
    } else {
        dequantise4(w.x, f, v[0], v[1]);
        dequantise4(w.y, f, v[2], v[3]);
    }
}

// ---- layouts ------------------------------------------------------------------------------
// Pieces of a thread that are compiled, by V. The least that holds a row is taken, so a
// thread's pieces before the next smaller option are all within the row.
constexpr int kOptions[2][7] = {{1, 2, 3, 4, 5, 6, 8}, {1, 2, 3, 4, 0, 0, 0}};
__host__ __device__ constexpr int full_pieces(int V, int J) {
    int full = 0;
    for (int q = 0; q < 7; ++q)
        if (kOptions[V == 8][q] > 0 && kOptions[V == 8][q] < J) full = kOptions[V == 8][q];
    return full;
}

// tpr threads a row, J pieces a thread; J == 0: rows that no layout holds in registers.
struct RowLayout {
    int tpr, J;
};

// The fewest threads (8 or more, so that a group of 32 columns lies in one row's lanes) that
// hold a row of K, with at most `most` elements each, `warp_most` where they are a warp; and then
// more threads while the rows do not fill the card (each has less to do then).
inline RowLayout row_layout(int64_t N, int K, int V, int most, int warp_most, const DeviceInfo &dev) {
    const int *options = kOptions[V == 8];
    const int64_t pieces = (int64_t(K) + V - 1) / V;
    auto fit = [&](int threads) {
        const int64_t need = (pieces + threads - 1) / threads;
        for (int q = 0; q < 7 && options[q] > 0; ++q)
            if (options[q] >= need)
                return options[q] * V <= (threads == 32 ? warp_most : most) ? options[q] : 0;
        return 0;
    };
    int tpr = 8;
    while (fit(tpr) == 0 && tpr < kMostRowThreads) tpr *= 2;
    while (tpr < kRowThreads && tpr < pieces && N * tpr < int64_t(dev.sm_count) * 2 * kRowThreads)
        tpr *= 2;
    return {tpr, fit(tpr)};
}

// Rows as one sequence of pieces (or octets), per_row of them a row, whole groups: piece kBlock blockIdx.x +
// i of all is piece `k` of row `row`. `magic` is piece_magic(per_row).
template <int kBlock>
struct PieceWalk {
    int64_t row0;
    uint32_t r0, per_row, magic;
    __device__ __forceinline__ PieceWalk(uint32_t per, uint32_t mag) : per_row(per), magic(mag) {
        const uint64_t first = uint64_t(blockIdx.x) * kBlock;
        if (first >> 32 == 0) {
            row0 = uint32_t(first) / per;
            r0 = uint32_t(first) - uint32_t(row0) * per;
        } else {
            row0 = int64_t(first / per);
            r0 = uint32_t(first - uint64_t(row0) * per);
        }
    }
    // (Below kBlock pieces a row the product with floor(2^32 / per_row) + 1 has the quotient in its
    // upper half: r0 + i < 2 kBlock, and its excess, at most per_row for each 2^32, stays below one.)
    __device__ __forceinline__ void at(uint32_t i, int64_t &row, uint32_t &k) const {
        const uint32_t t = r0 + i;
        const uint32_t q = per_row > kBlock ? uint32_t(t >= per_row) : __umulhi(t, magic);
        row = row0 + q;
        k = t - q * per_row;
    }
};

inline uint32_t piece_magic(uint32_t per_row) { return uint32_t((uint64_t(1) << 32) / per_row + 1); }

// The alignment in bytes, at most 16, of everything in `addresses` (pointers and byte strides).
inline int alignment_of(const uint64_t *addresses, int n) {
    uint64_t all = 16;
    for (int q = 0; q < n; ++q) all |= addresses[q];
    return int(all & (~all + 1));
}

// ---- sums over a row's threads ------------------------------------------------------------
// The same value for all of them. kWarp: the row is one warp; else `red` holds a float per warp
// and sum (unused where a row is within a warp), and every thread of the block calls it.
template <bool kWarp, int kN>
__device__ __forceinline__ void row_sum(float (&v)[kN], int tpr, float (*red)[kMostRowThreads / 32]) {
    if constexpr (kWarp) {
#pragma unroll
        for (int n = 0; n < kN; ++n) v[n] = warp_sum(v[n]);
        return;
    }
    for (int o = min(tpr, 32) >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < kN; ++n) v[n] += __shfl_xor_sync(kFullMask, v[n], o);
    if (tpr <= 32) return;
    const int warp = threadIdx.x >> 5, warps = tpr >> 5, first = warp & ~(warps - 1);
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < kN; ++n) red[n][warp] = v[n];
    __syncthreads();
    // Every warp adds the row's warps alike, a power of two of them, in a few instructions a value.
#pragma unroll
    for (int n = 0; n < kN; ++n) v[n] = red[n][first + (threadIdx.x & (warps - 1))];
    for (int o = warps >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int n = 0; n < kN; ++n) v[n] += __shfl_xor_sync(kFullMask, v[n], o);
}

// A thread's sums over its share (columns threadIdx.x, + kRowThreads, ...) of a row of any length: in fp32 for kRun
// terms, whose sums are added in fp64 (one running fp32 sum over 2^24 equal columns is off by 3e-4 of itself). A
// share of at most kRun terms is a plain fp32 sum. term(k, sums) adds column k's.
constexpr int kRun = 256;
// kPlain: rows of one share by a plain loop (4096 x 16400 fp32, RMS backward from the input 304 -> 259 us, from the
// checkpoint 316 -> 214); the forward passes take longer so (RMS, 4096 x 16400: 374 -> 437). kFour: longer rows four
// terms at a time, as the compiler would not (64 x 70001 fp32, layer norm's 238 -> 101 and 181 -> 160; a 16-bit
// layer's checkpoint, without, 195 -> 138 by the RMS norm and 195 -> 162, though 4096 x 16400 152 -> 154 and 169).
template <bool kPlain, bool kFour, int kN, typename Term>
__device__ __forceinline__ void share_sums(int K, float (&v)[kN], Term term) {
    constexpr int kShares = kRowThreads * kRun;
    if (kPlain && K <= kShares) {
#pragma unroll
        for (int n = 0; n < kN; ++n) v[n] = 0.0f;
        for (int k = threadIdx.x; k < K; k += kRowThreads) term(k, v);
        return;
    }
    double all[kN] = {};
    for (int first = threadIdx.x; first < K; first += kShares) {
        float run[kN] = {};
        const int end = min(K, first + kShares);
        if constexpr (kFour) {
#pragma unroll 4
            for (int k = first; k < end; k += kRowThreads) term(k, run);
        } else {
            for (int k = first; k < end; k += kRowThreads) term(k, run);
        }
#pragma unroll
        for (int n = 0; n < kN; ++n) all[n] += double(run[n]);
    }
#pragma unroll
    for (int n = 0; n < kN; ++n) v[n] = float(all[n]);
}

// Sums of a block of kRowThreads, the same for every thread; warps added in order.
template <int kN>
__device__ __forceinline__ void block_sum(float (&v)[kN]) {
    constexpr int kWarps = kRowThreads / 32;
    __shared__ float part[kN][kWarps];
#pragma unroll
    for (int n = 0; n < kN; ++n) v[n] = warp_sum(v[n]);
    __syncthreads();                    // the previous sums have been read
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int n = 0; n < kN; ++n) part[n][threadIdx.x >> 5] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        v[n] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v[n] += part[n][w];
    }
}

}  // namespace bigcn
