// rowred.h -- reductions over the threads that share a row.
#pragma once
#include <hip/hip_runtime.h>

namespace lpp {

// v + its value on a lane that DPP control CTRL names
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// sum over the TPR threads of a row; all of them get it.  TPR <= 64: lanes of one
// wave, through VALU lane permutes (quad, half-row and row mirrors, then swaps of 16-
// and 32-lane halves).  Above: the wave sums meet in LDS (two slots in turn, so that one
// barrier a sum is enough).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* slots, int& turn) {
    v = dpp_add<0xB1>(v);
    if constexpr (TPR > 2) v = dpp_add<0x4E>(v);
    if constexpr (TPR > 4) v = dpp_add<0x141>(v);
    if constexpr (TPR > 8) v = dpp_add<0x140>(v);
    if constexpr (TPR > 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (TPR > 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float* s = slots + turn * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += s[w];
    }
    return v;
}

// two sums at once: one barrier for both (slots: 4 * TPR / 64 of them)
template <int TPR>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* slots, int& turn) {
    int none = 0;
    a = row_sum<(TPR < 64 ? TPR : 64)>(a, slots, none);
    b = row_sum<(TPR < 64 ? TPR : 64)>(b, slots, none);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float* s = slots + turn * 2 * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
            s[2 * (threadIdx.x >> 6)] = a;
            s[2 * (threadIdx.x >> 6) + 1] = b;
        }
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            a += s[2 * w];
            b += s[2 * w + 1];
        }
    }
}

// LDS of a row between its TPR threads.  Up to 64 they are lanes of one wave, whose LDS
// accesses are in order: only the compiler has to keep them so.  Rows of a workgroup may take
// different branches then.
template <int TPR>
__device__ __forceinline__ void row_sync() {
    if constexpr (TPR > 64) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// the largest of v and its value on a lane that DPP control CTRL names
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
    return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true)));
}

// the largest of a value over the TPR threads of a row (a NaN only where all are), as row_sum
template <int TPR>
__device__ __forceinline__ float row_max(float v, float* slots, int& turn) {
    v = dpp_max<0xB1>(v);
    if constexpr (TPR > 2) v = dpp_max<0x4E>(v);
    if constexpr (TPR > 4) v = dpp_max<0x141>(v);
    if constexpr (TPR > 8) v = dpp_max<0x140>(v);
    if constexpr (TPR > 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if constexpr (TPR > 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float* s = slots + turn * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = fmaxf(v, s[w]);
    }
    return v;
}

}  // namespace lpp
