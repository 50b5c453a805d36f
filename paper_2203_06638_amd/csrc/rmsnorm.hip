// rmsnorm.hip -- root-mean-square norm over the channels of each row of a matrix
// [rows][C], after a residual addition if there is one, and its gradient.
//
//   h = x (+ res, rounded to the storage type), rstd = 1 / sqrt(mean_c h^2 + eps),
//   y = h * rstd * gamma
//   g = dy * gamma, dx = rstd * (g - h * rstd^2 * mean_c(g h)) (+ dres),
//   dgamma = sum over rows of dy * h * rstd
//
// Sums and statistics are float32.  No sums cross workgroups in the forward pass.
#include <algorithm>

#include "act8.h"
#include "kernels.h"
#include "launch.h"

#ifndef RMSWGS
#define RMSWGS 2048
#endif
#ifndef RMSPARTS
#define RMSPARTS 1024
#endif
namespace lpp {

// sum over the TPR threads of a row; all of them get it.  TPR <= 64: lanes of one
// wave.  Above: the wave sums meet in LDS (two slots in turn, so that one barrier
// a sum is enough).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* slots, int& turn) {
#pragma unroll
    for (int d = 1; d < (TPR < 64 ? TPR : 64); d *= 2) v += __shfl_xor(v, d, 64);
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

// A row's C channels are cut into chunks of V = 16 / sizeof(T); thread t of the
// row's TPR threads holds chunks t, t + TPR, ... (NC of them) in registers, so that
// the row is read once, and its 32-channel groups lie in neighbouring lanes.
// Workgroups walk over the rows and keep gamma in registers.
template <typename T, int TPR, int NC>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void rmsnorm_k(RmsArgs p) {
    constexpr int V = 16 / (int)sizeof(T), L = kAct8Group / V;
    constexpr int TB = TPR > 256 ? TPR : 256, RB = TB / TPR;   // threads, rows of a workgroup
    __shared__ float slots[2 * (TB / 64)];
    int turn = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    float gam[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int ch = (c * TPR + t) * V + j;
            gam[c][j] = ch < p.C ? p.gamma[ch] : 0.f;
        }
    const long step = (long)gridDim.x * RB;
    // (every thread of a workgroup takes the same number of turns: barriers)
    for (long r0 = (long)blockIdx.x * RB; r0 < p.rows; r0 += step) {
        const long r = r0 + rl;
        const bool ok = r < p.rows;
        float h[NC][V];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V;
            ld_chunk((const T*)p.x + r * p.ldx + ch, ok ? p.C - ch : 0, h[c]);
        }
        if (p.res) {
            float e[NC][V];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int ch = (c * TPR + t) * V;
                ld_chunk((const T*)p.res + r * p.ldres + ch, ok ? p.C - ch : 0, e[c]);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int ch = (c * TPR + t) * V;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[c][j] += e[c][j];
                    if constexpr (sizeof(T) == 2) h[c][j] = from_bf16(to_bf16(h[c][j]));
                }
                if (p.h) st_chunk((T*)p.h + r * p.ldh + ch, ok ? p.C - ch : 0, h[c]);
            }
        }
        float ss = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) ss = __builtin_fmaf(h[c][j], h[c][j], ss);
        const float rstd = 1.f / sqrtf(row_sum<TPR>(ss, slots, turn) / (float)p.C + p.eps);
        if (ok && t == 0 && p.rstd) p.rstd[r] = rstd;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) h[c][j] = h[c][j] * rstd * gam[c][j];
            if (p.y) st_chunk((T*)p.y + r * p.ldy + ch, ok ? p.C - ch : 0, h[c]);
            if (p.q) {
                uint32_t m = 0;
#pragma unroll
                for (int j = 0; j < V; ++j) m = max(m, ch + j < p.C ? abs_bits(h[c][j]) : 0u);
                const uint32_t s = act8_exp(group_max<L>(m));
                uint32_t w[V / 4];
#pragma unroll
                for (int k = 0; k < V / 4; ++k)
                    w[k] = s == 255u ? 0u : act8_code4(h[c] + 4 * k, act8_inv(s), p.keep_sign);
                if (ok && ch < p.pitch) {
                    uint8_t* o = p.q + r * p.pitch + ch;
                    if constexpr (V == 8) *(uint2*)o = uint2{w[0], w[1]};
                    else *(uint32_t*)o = w[0];
                }
                if (ok && ch < p.C && t % L == 0) p.exps[r * p.G + ch / kAct8Group] = (uint8_t)s;
            }
        }
    }
}

// v, added to what is there with acc
template <typename T>
__device__ __forceinline__ void st_sum(T* p, int n, const float* v, bool acc) {
    constexpr int V = 16 / (int)sizeof(T);
    float e[V];
    if (acc) {
        ld_chunk(p, n, e);
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] += v[j];
        v = e;
    }
    st_chunk(p, n, v);
}

// The gradient.  dgamma: every thread sums its channels over the rows it walks
// over, the workgroup's row lanes meet in LDS, and each workgroup writes one row of
// partials [workgroup][stride], summed in a fixed order by launch_part_sums.
template <typename T, int TPR, int NC>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void rmsnorm_bwd_k(RmsBwdArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int TB = TPR > 256 ? TPR : 256, RB = TB / TPR;
    __shared__ float slots[2 * (TB / 64)];
    __shared__ float sums[RB > 1 ? TB * V : 1];
    int turn = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    float gam[NC][V], dg[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int ch = (c * TPR + t) * V + j;
            gam[c][j] = ch < p.C ? p.gamma[ch] : 0.f;
            dg[c][j] = 0.f;
        }
    const long step = (long)gridDim.x * RB;
    for (long r0 = (long)blockIdx.x * RB; r0 < p.rows; r0 += step) {
        const long r = r0 + rl;
        const bool ok = r < p.rows;
        float dy[NC][V], h[NC][V], res[NC][V];
        const float rstd = ok ? p.rstd[r] : 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V;
            const int n = ok ? p.C - ch : 0;
            ld_chunk((const T*)p.dy + r * p.lddy + ch, n, dy[c]);
            if (p.dres) ld_chunk((const T*)p.dres + r * p.lddres + ch, n, res[c]);
            if (p.h) {
                ld_chunk((const T*)p.h + r * p.ldh + ch, n, h[c]);
            } else {
                uint32_t w[V / 4], s = 7u;
#pragma unroll
                for (int k = 0; k < V / 4; ++k) w[k] = 0u;
                if (n > 0) {
                    const uint8_t* o = p.q + r * p.pitch + ch;
                    if constexpr (V == 8) {
                        const uint2 u = *(const uint2*)o;
                        w[0] = u.x;
                        w[1] = u.y;
                    } else {
                        w[0] = *(const uint32_t*)o;
                    }
                    s = p.exps[r * p.G + ch / kAct8Group];
                }
#pragma unroll
                for (int k = 0; k < V / 4; ++k) act8_val4(w[k], act8_step(s), h[c] + 4 * k);
                // (padding channels of a NaN group)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (j >= n) h[c][j] = 0.f;
            }
        }
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) s = __builtin_fmaf(dy[c][j] * gam[c][j], h[c][j], s);
        const float k = row_sum<TPR>(s, slots, turn) / (float)p.C * (rstd * rstd);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V;
            const int n = ok ? p.C - ch : 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                dg[c][j] = __builtin_fmaf(dy[c][j], h[c][j] * rstd, dg[c][j]);
                dy[c][j] = rstd * (dy[c][j] * gam[c][j] - h[c][j] * k);
            }
            if (p.dres) {
#pragma unroll
                for (int j = 0; j < V; ++j) dy[c][j] += res[c][j];
            }
            if (p.dx) st_sum((T*)p.dx + r * p.lddx + ch, n, dy[c], p.acc1);
            if (p.dx2) st_sum((T*)p.dx2 + r * p.lddx + ch, n, dy[c], p.acc2);
        }
    }
    if (!p.part) return;
    float* out = p.part + (long)blockIdx.x * p.pstride;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if constexpr (RB > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j) sums[threadIdx.x * V + j] = dg[c][j];
            __syncthreads();
            for (int e = threadIdx.x; e < TPR * V; e += TB) {
                float a = 0.f;
                for (int w = 0; w < RB; ++w) a += sums[w * TPR * V + e];
                const int ch = c * TPR * V + e;
                if (ch < p.C) out[ch] = a;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int ch = (c * TPR + t) * V + j;
                if (ch < p.C) out[ch] = dg[c][j];
            }
        }
    }
}

// threads of a row and chunks of a thread for rows of `chunks` chunks
struct RowShape { int tpr, nc; };
static RowShape row_shape(int chunks) {
    for (int tpr : {8, 16, 32, 64})
        if (chunks <= tpr) return {tpr, 1};
    for (int nc : {2, 4})
        if (chunks <= 64 * nc) return {64, nc};
    for (int nc : {2, 4})
        if (chunks <= 256 * nc) return {256, nc};
    for (int nc : {2, 4})
        if (chunks <= 1024 * nc) return {1024, nc};
    return {0, 0};
}
static int row_chunks(int dt, int C) {
    const int V = dt == DT_BF16 ? 8 : 4;
    return (C + V - 1) / V;
}

template <bool BWD, typename T, int TPR, int NC, typename P>
static void rms_launch(const P& p, int wgs, hipStream_t st) {
    const dim3 grid((unsigned)wgs), block(TPR > 256 ? TPR : 256);
    if constexpr (BWD) launch((rmsnorm_bwd_k<T, TPR, NC>), grid, block, 0, st, p);
    else launch((rmsnorm_k<T, TPR, NC>), grid, block, 0, st, p);
}

template <bool BWD, typename T, typename P>
static hipError_t rms_dispatch(const P& p, RowShape s, int wgs, hipStream_t st) {
    switch (s.tpr * 16 + s.nc) {
    case 8 * 16 + 1: rms_launch<BWD, T, 8, 1>(p, wgs, st); break;
    case 16 * 16 + 1: rms_launch<BWD, T, 16, 1>(p, wgs, st); break;
    case 32 * 16 + 1: rms_launch<BWD, T, 32, 1>(p, wgs, st); break;
    case 64 * 16 + 1: rms_launch<BWD, T, 64, 1>(p, wgs, st); break;
    case 64 * 16 + 2: rms_launch<BWD, T, 64, 2>(p, wgs, st); break;
    case 64 * 16 + 4: rms_launch<BWD, T, 64, 4>(p, wgs, st); break;
    case 256 * 16 + 2: rms_launch<BWD, T, 256, 2>(p, wgs, st); break;
    case 256 * 16 + 4: rms_launch<BWD, T, 256, 4>(p, wgs, st); break;
    case 1024 * 16 + 2: rms_launch<BWD, T, 1024, 2>(p, wgs, st); break;
    case 1024 * 16 + 4:
        // (rows of kRmsMaxC bf16 channels are 2 chunks a thread)
        if constexpr (sizeof(T) == 4) {
            rms_launch<BWD, T, 1024, 4>(p, wgs, st);
            break;
        }
        return hipErrorInvalidValue;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_rmsnorm(int dt, RmsArgs p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    p.pitch = act8_pitch(p.C);
    p.G = act8_groups(p.C);
    p.exps = p.q ? p.q + p.rows * p.pitch : nullptr;
    const RowShape s = row_shape(row_chunks(dt, p.C));
    if (!s.tpr) return hipErrorInvalidValue;
    const int rb = std::max(256, s.tpr) / s.tpr;
    const int wgs = (int)std::min(s.tpr > 256 ? 512l : (long)RMSWGS, (p.rows + rb - 1) / rb);
    return dt == DT_BF16 ? rms_dispatch<false, bf16>(p, s, wgs, st) : rms_dispatch<false, float>(p, s, wgs, st);
}

int rmsnorm_bwd_parts(long rows, int C) {
    const RowShape s = row_shape((C + 3) / 4);
    const int rb = std::max(256, s.tpr) / std::max(1, s.tpr);
    return (int)std::max(1l, std::min((long)RMSPARTS, (rows + 2 * rb - 1) / (2 * rb)));
}

hipError_t launch_rmsnorm_bwd(int dt, RmsBwdArgs p, hipStream_t st) {
    if (p.rows <= 0 && !p.part) return hipSuccess;
    p.pitch = act8_pitch(p.C);
    p.G = act8_groups(p.C);
    p.exps = p.q ? p.q + p.rows * p.pitch : nullptr;
    p.pstride = (p.C + 3) / 4 * 4;
    const RowShape s = row_shape(row_chunks(dt, p.C));
    if (!s.tpr) return hipErrorInvalidValue;
    const int wgs = rmsnorm_bwd_parts(p.rows, p.C);
    return dt == DT_BF16 ? rms_dispatch<true, bf16>(p, s, wgs, st) : rms_dispatch<true, float>(p, s, wgs, st);
}

}  // namespace lpp
