// groupnorm.h -- what the group norm's kernels share (groupnorm.hip, groupnorm_whole.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "act8.h"
#include "kernels.h"

namespace lpp {

// 1 / (1 + e^-z): e^-z = 2^t (1 + r ln 2) with t = -z log2 e rounded and r what that lost,
// so that large |z| cost no accuracy; the reciprocal is the unit's, off by one unit in the
// last place.  |z| under 2^126: beyond, t would be infinite and r NaN.
__device__ __forceinline__ float sigmoid(float z) {
    const float t = z * -1.44269504f, r = __builtin_fmaf(z, -1.44269504f, -t) + z * -1.9259630e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    return __builtin_amdgcn_rcpf(__builtin_fmaf(e, __builtin_fmaf(r, 0.693147181f, 1.f), 1.f));
}
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if (ACT == ACT_RELU) return fmaxf(z, 0.f);      // (0 for NaN)
    // (from 128 on the sigmoid is 1, from -128 on 0; a NaN stays one through the other factor)
    if (ACT == ACT_SILU) return z * sigmoid(__builtin_amdgcn_fmed3f(z, -128.f, 128.f));
    return z;
}
// dy * act'(z)
template <int ACT>
__device__ __forceinline__ float act_grad(float dy, float z) {
    if (ACT == ACT_RELU) return z > 0.f ? dy : 0.f;
    if (ACT == ACT_SILU) {
        // (the same for the derivative, 1 and 0 there; a NaN stays one)
        z = __builtin_elementwise_maximum(__builtin_elementwise_minimum(z, 128.f), -128.f);
        const float s = sigmoid(z);
        return dy * (s * (1.f + z * (1.f - s)));
    }
    return dy;
}

// 2^-e with 2^(e - 1) <= n < 2^e: sums of n values are taken of the values times it, an exact
// factor, so that they are as small as the values
__device__ __forceinline__ float sum_scale(float n) {
    return __uint_as_float((253u << 23) - (__float_as_uint(n) & 0x7f800000u));
}

// lanes (a power of two, one wave at most) that a workgroup has for each of n items
__device__ __forceinline__ int item_lanes(int threads, int n) {
    int l = 6;
    while (l > 0 && (n << l) > threads) --l;
    return l;
}

// Sums of V channels over the lanes of a wave that share them (lane distance 2^lw and up);
// each exchange halves the channels that a lane goes on with.  v[0 .. n) are the sums of
// channels first .. first + n - 1 afterwards.
template <int V>
__device__ __forceinline__ void fold(float* v, int lw, int& first, int& n) {
    const int lane = threadIdx.x & 63;
    int d = 1 << lw;
    first = 0;
    n = V;
#pragma unroll
    for (int h = V / 2; h >= 1; h /= 2) {
        if (d >= 64) return;
        const bool up = (lane & d) != 0;
#pragma unroll
        for (int j = 0; j < h; ++j) {
            const float keep = up ? v[j + h] : v[j], send = up ? v[j] : v[j + h];
            v[j] = keep + __shfl_xor(send, d);
        }
        first += up ? h : 0;
        n = h;
        d <<= 1;
    }
    for (; d < 64; d <<= 1) v[0] += __shfl_xor(v[0], d);
}

// first row whose last chunk must not be read past its values (chunks from channel 0 on)
inline long exact_row(int dt, long rows, int C, long ld) {
    return rows - (dt == DT_BF16 ? tail_rows<bf16>(rows, C, ld) : tail_rows<float>(rows, C, ld));
}

// the same where a chunk may begin at any channel, so that up to V - 1 values lie behind it
inline long exact_row_any(int dt, long rows, long ld) {
    const long over = dt == DT_BF16 ? 7 : 3, dist = rows > 1 ? ld : over;
    return rows - std::min(rows, (over + dist - 1) / dist);
}

}  // namespace lpp
