// act8.h -- the 8-bit checkpoint of an activation matrix [rows][C].
//
// Groups of 32 successive channels of a row (the last group of a row may be
// shorter) share a power-of-two step.  With amax the group's largest
// magnitude, s is the biased exponent of the smallest power of two 2^(s-127)
// for which rint(amax * 2^(133-s)) <= 127, kept within [7, 254]; a value is
// stored as code = rint(x * 2^(133-s)) and stands for code * 2^(s-133).  Codes
// have 7 magnitude bits, so that value is exact in bfloat16 and float32 (s >= 7
// keeps every nonzero one a normal number): decoding never rounds.  Rounding to half
// a step, of a step in (amax / 127.5, amax / 63.75] or 2^-126, is the only loss.
// s = 255 marks a group that holds an infinity or a NaN: all of it decodes to
// NaN, so a diverged activation is not hidden by its checkpoint.  Its codes are 0, or
// with ACT8_DECIDES the values' signs (0 for NaN): ReLU decisions x > 0 are read from
// the codes, or from the values that they stand for with an infinite step
// (infinities of x's sign, NaN for 0), since a NaN decides nothing.  The largest
// float32 magnitudes (from 1.9921875 * 2^127 on) would need s = 255; they take
// 254 and saturate at code 127, up to a step off.
//
// Buffer: codes [rows][pitch], pitch = C rounded up to 16 (padding codes 0), then
// the exponents [rows][ceil(C / 32)], both bytes.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "act.h"

namespace lpp {

constexpr int kAct8Group = 32;
__host__ __device__ inline int act8_pitch(int C) { return (C + 15) & ~15; }
__host__ __device__ inline int act8_groups(int C) { return (C + kAct8Group - 1) / kAct8Group; }
inline long act8_bytes(long rows, int C) { return rows * ((long)act8_pitch(C) + act8_groups(C)); }

// exponent byte from the bit pattern of the group's largest magnitude: adding
// 2^-7 of the leading bit carries into the exponent exactly where rint of the
// mantissa in 64ths would reach 128
__device__ __forceinline__ uint32_t act8_exp(uint32_t amax) {
    const uint32_t s = min(max((amax + 0x10000u) >> 23, 7u), 254u);
    return amax >= 0x7f800000u ? 255u : s;
}
// steps per unit of a group with exponent s, 2^(133-s)
__device__ __forceinline__ float act8_inv(uint32_t s) { return __uint_as_float((260u - s) << 23); }
// value of one step, 2^(s-133), for 255 the float with the bits bad (NaN)
__device__ __forceinline__ float act8_step(uint32_t s, uint32_t bad = 0x7fc00000u) {
    return __uint_as_float(s == 255u ? bad : (s - 6u) << 23);
}
// four codes, one a byte.  Adding 1.5 * 2^23 rounds to an integer (ties to even)
// and leaves it in two's complement in the low byte.  keep_sign: a nonzero value
// under half a step takes +-1 instead of 0.
__device__ __forceinline__ uint32_t act8_code4(const float* x, float inv, bool keep_sign) {
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float r = __builtin_amdgcn_fmed3f(x[j] * inv, -127.f, 127.f);
        if (keep_sign && x[j] != 0.f && fabsf(r) <= 0.5f) r = copysignf(1.f, x[j]);
        b[j] = __float_as_uint(r + 12582912.f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
    return lo | hi;
}
// the signs of four values as codes, 0 for NaN
__device__ __forceinline__ uint32_t act8_sign4(const float* x) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w |= (x[j] > 0.f ? 1u : x[j] < 0.f ? 255u : 0u) << (8 * j);
    return w;
}
// the four values of four codes (signed bytes, converted one by one)
__device__ __forceinline__ void act8_val4(uint32_t w, float step, float* v) {
    v[0] = (float)(int8_t)w * step;
    v[1] = (float)(int8_t)(w >> 8) * step;
    v[2] = (float)(int8_t)(w >> 16) * step;
    v[3] = (float)(int8_t)(w >> 24) * step;
}

// the largest of a value over L (2, 4 or 8) neighbouring lanes, those that hold a
// group's channels, through the lane permutes of the VALU (no LDS)
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    static_assert(L == 2 || L == 4 || L == 8, "lanes of a group");
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    if constexpr (L > 2)
        v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));   // lane ^ 2
    if constexpr (L > 4)
        v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));   // mirrored in 8 lanes
    return v;
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Output tensors of this size on are stored past the L2 caches (8 x 4 MB), where they
// would only displace what the kernel still reads: RMS norm of 131072 x 128 bf16, 38.4
// -> 33.8 us, unpacking to 100352 x 256, 12.5 -> 11.9.
constexpr long kStreamBytes = 32l << 20;

// 16 bytes at any element address (global memory takes vector accesses unaligned)
typedef uint32_t u4any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// A chunk: V = 16 / sizeof(T) successive values of a row, as they lie in memory.
// Loading and conversion are apart, so that a thread's loads are all under way before
// the first is waited for.
template <typename T>
__device__ __forceinline__ void chunk_values(u4 w, float* v) {
    constexpr int V = 16 / (int)sizeof(T);
#pragma unroll
    for (int j = 0; j < V; ++j)
        v[j] = sizeof(T) == 4 ? __uint_as_float(w[j])
                              : __uint_as_float((j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
}
// Rows of a matrix whose length is no multiple of V end in a chunk that runs into the
// next row; in the last ones (tail_rows) it would end behind the matrix.
template <typename T>
inline long tail_rows(long rows, int C, long ld) {
    constexpr int V = 16 / (int)sizeof(T);
    const long over = (C + V - 1) / V * V - C, dist = rows > 1 ? ld : over;
    return over ? std::min(rows, (over + dist - 1) / dist) : 0;
}
// the chunk at p of which n values exist; exact: none behind them may be touched.  The
// rest of the result is anything (chunk_mask) where exact is not set.
template <typename T>
__device__ __forceinline__ u4 ld_chunk(const T* p, int n, bool exact) {
    constexpr int V = 16 / (int)sizeof(T);
    if (!exact) return *(const u4any*)p;
    u4 w = u4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (j >= n) continue;
        if constexpr (sizeof(T) == 4) w[j] = ((const uint32_t*)p)[j];
        else w[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
    }
    return w;
}
// zeros in place of the values from the n-th on
template <typename T>
__device__ __forceinline__ u4 chunk_mask(u4 w, int n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) w[k] = k < n ? w[k] : 0u;
        else w[k] = 2 * k + 1 < n ? w[k] : 2 * k < n ? w[k] & 0xffffu : 0u;
    }
    return w;
}
// STREAM: a tensor that the caches will not hold until it is read (kStreamBytes)
template <bool STREAM = false, typename T>
__device__ __forceinline__ void st_chunk(T* p, int n, const float* v) {
    constexpr int V = 16 / (int)sizeof(T);
    if (n >= V) {
        u4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            w[k] = sizeof(T) == 4 ? __float_as_uint(v[k]) : pack_bf16x2(v[(2 * k) % V], v[(2 * k + 1) % V]);
        if (STREAM) __builtin_nontemporal_store(w, (u4any*)p);
        else *(u4any*)p = w;
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < n) st1(p, j, v[j]);
    }
}

// n / d for n < 2^31 and 2 <= d: with L = ceil(log2 d) and m = ceil(2^(31+L) / d),
// n m / 2^(31+L) exceeds n / d by less than n d / (d 2^(31+L)) < 1 / d
struct FastDiv {
    unsigned m, sh;
};
inline FastDiv fast_div(unsigned d) {
    unsigned L = 1;
    while ((1ull << L) < d) ++L;
    return FastDiv{(unsigned)(((1ull << (31 + L)) + d - 1) / d), L - 1};
}
__device__ __forceinline__ unsigned div_by(unsigned n, FastDiv f) { return __umulhi(n, f.m) >> f.sh; }

}  // namespace lpp
