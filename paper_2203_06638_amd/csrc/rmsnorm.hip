// rmsnorm.hip -- root-mean-square norm over the channels of each row of a matrix
// [rows][C], after a residual addition if there is one, and its gradient.
//
//   h = x (+ res, rounded to the storage type), rstd = 1 / sqrt(mean_c h^2 + eps),
//   y = h * rstd * gamma
//   g = dy * gamma, u = h * rstd, dx = rstd * (g - u * mean_c(g u)) (+ dres),
//   dgamma = sum over rows of dy * u
//
// Sums and statistics are float32.  No sums cross workgroups in the forward pass.
#include <algorithm>

#include "act8.h"
#include "kernels.h"
#include "launch.h"
#include "rowred.h"

namespace lpp {

// a thread's gammas: V from channel ch on, 0 past the row
template <int V>
__device__ __forceinline__ void ld_gamma(const float* gamma, int ch, int C, float* v) {
#pragma unroll
    for (int k = 0; k < V; k += 4) {
        const int n = C - (ch + k);
        chunk_values<float>(
            chunk_mask<float>(ld_chunk(gamma + (n > 0 ? ch + k : 0), n, (n > 0 && n < 4) || C < 4), n), v + k);
    }
}

// A row's C channels are cut into chunks of V = 16 / sizeof(T); thread t of the
// row's TPR threads holds chunks t, t + TPR, ... (NC of them) in registers, so that
// the row is read once, and its 32-channel groups lie in neighbouring lanes.
// Workgroups walk over the rows and keep gamma in registers.
template <typename T, int TPR, int NC, bool ST>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void rmsnorm_k(RmsArgs p) {
    // lanes of a 32-channel group (rows of 2 or 4 lanes are one group)
    constexpr int V = 16 / (int)sizeof(T), L = kAct8Group / V < TPR ? kAct8Group / V : TPR;
    constexpr int TB = TPR > 256 ? TPR : 256, RB = TB / TPR;   // threads, rows of a workgroup
    __shared__ float slots[2 * (TB / 64)];
    int turn = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    float gam[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c) ld_gamma<V>(p.gamma, (c * TPR + t) * V, p.C, gam[c]);
    const long step = (long)gridDim.x * RB;
    // (every thread of a workgroup takes the same number of turns: barriers)
    for (long r0 = (long)blockIdx.x * RB; r0 < p.rows; r0 += step) {
        const bool ok = r0 + rl < p.rows;
        const long r = min(r0 + rl, p.rows - 1);
        const bool exact = r >= p.exact;
        u4 xw[NC], ew[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V, n = p.C - ch, at = n > 0 ? ch : 0;
            xw[c] = ld_chunk((const T*)p.x + r * p.ldx + at, n, exact);
            if (p.res) ew[c] = ld_chunk((const T*)p.res + r * p.ldres + at, n, exact);
        }
        float h[NC][V];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V, n = p.C - ch;
            chunk_values<T>(chunk_mask<T>(xw[c], n), h[c]);
            if (p.res) {
                float e[V];
                chunk_values<T>(chunk_mask<T>(ew[c], n), e);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    h[c][j] += e[j];
                    if constexpr (sizeof(T) == 2) h[c][j] = from_bf16(to_bf16(h[c][j]));
                }
                if (p.h) st_chunk<ST>((T*)p.h + r * p.ldh + ch, ok ? n : 0, h[c]);
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
            if (p.y) st_chunk<ST>((T*)p.y + r * p.ldy + ch, ok ? p.C - ch : 0, h[c]);
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

// whether a thread's next row is loaded while it works on one (short rows, whose raw
// chunks fit the registers beside it: with it 512 workgroups do as well as 1024)
template <typename T, int TPR, int NC>
constexpr bool kAhead = TPR <= 64 && NC * 16 / (int)sizeof(T) <= 16;

// v, added to what is there with acc
template <typename T>
__device__ __forceinline__ void st_sum(T* p, int n, const float* v, bool acc) {
    constexpr int V = 16 / (int)sizeof(T);
    float e[V];
    if (acc) {
        if (n <= 0) return;
        chunk_values<T>(ld_chunk(p, n, n < V), e);
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
    constexpr int W = TB / 64, TW = TPR < 64 ? TPR : 64;   // waves; threads of one whose sums differ by channel
    __shared__ __attribute__((aligned(16))) float sums[RB > 1 ? W * TW * NC * V : 1];
    int turn = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    float gam[NC][V], dg[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        ld_gamma<V>(p.gamma, (c * TPR + t) * V, p.C, gam[c]);
#pragma unroll
        for (int j = 0; j < V; ++j) dg[c][j] = 0.f;
    }
    const long step = (long)gridDim.x * RB;
    u4 yw[NC], hw[NC], ew[NC];
    uint32_t hs[NC];
    float rs;
    auto load = [&](long r0) {
        const long r = min(r0 + rl, p.rows - 1);
        const bool exact = r >= p.exact;
        rs = p.rstd[r];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V, n = p.C - ch, at = n > 0 ? ch : 0;
            yw[c] = ld_chunk((const T*)p.dy + r * p.lddy + at, n, exact);
            if (p.dres) ew[c] = ld_chunk((const T*)p.dres + r * p.lddres + at, n, exact);
            if (p.h) {
                hw[c] = ld_chunk((const T*)p.h + r * p.ldh + at, n, exact);
            } else {
                const uint8_t* o = p.q + r * p.pitch + at;
                if constexpr (V == 8) {
                    const uint2 u = *(const uint2*)o;
                    hw[c][0] = u.x;
                    hw[c][1] = u.y;
                } else {
                    hw[c][0] = *(const uint32_t*)o;
                }
                hs[c] = p.exps[r * p.G + at / kAct8Group];
            }
        }
    };
    if (kAhead<T, TPR, NC> && p.rows > 0) load((long)blockIdx.x * RB);
    for (long r0 = (long)blockIdx.x * RB; r0 < p.rows; r0 += step) {
        const bool ok = r0 + rl < p.rows;
        const long r = min(r0 + rl, p.rows - 1);
        if (!kAhead<T, TPR, NC>) load(r0);
        const float rstd = ok ? rs : 0.f;
        float dy[NC][V], h[NC][V];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int n = ok ? p.C - (c * TPR + t) * V : 0;
            chunk_values<T>(chunk_mask<T>(yw[c], n), dy[c]);
            if (p.h) {
                chunk_values<T>(chunk_mask<T>(hw[c], n), h[c]);
            } else {
#pragma unroll
                for (int k = 0; k < V / 4; ++k) act8_val4(hw[c][k], act8_step(hs[c]), h[c] + 4 * k);
                // (padding channels of a NaN group, and chunks past the row)
#pragma unroll
                for (int j = 0; j < V; ++j) h[c][j] = j < n ? h[c][j] : 0.f;
            }
        }
        float e[NC][V];
        if (p.dres) {
#pragma unroll
            for (int c = 0; c < NC; ++c) chunk_values<T>(ew[c], e[c]);
        }
        if (kAhead<T, TPR, NC>) load(r0 + step);
        // (h from here on is u: rstd^2 need not be a float32 number)
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                h[c][j] *= rstd;
                s = __builtin_fmaf(dy[c][j] * gam[c][j], h[c][j], s);
            }
        const float k = row_sum<TPR>(s, slots, turn) / (float)p.C;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = (c * TPR + t) * V;
            const int n = ok ? p.C - ch : 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                dg[c][j] = __builtin_fmaf(dy[c][j], h[c][j], dg[c][j]);
                dy[c][j] = rstd * (dy[c][j] * gam[c][j] - h[c][j] * k);
            }
            if (p.dres) {
#pragma unroll
                for (int j = 0; j < V; ++j) dy[c][j] += e[c][j];
            }
            if (p.dx) st_sum((T*)p.dx + r * p.lddx + ch, n, dy[c], p.acc1);
            if (p.dx2) st_sum((T*)p.dx2 + r * p.lddx + ch, n, dy[c], p.acc2);
        }
    }
    if (!p.part) return;
    float* out = p.part + (long)blockIdx.x * p.pstride;
    if constexpr (RB > 1) {
        // rows of a wave through lane swaps, waves through LDS
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
#pragma unroll
                for (int d = TW; d < 64; d *= 2) dg[c][j] += __shfl_xor(dg[c][j], d, 64);
                if (lane < TW) sums[((wave * NC + c) * TW + lane) * V + j] = dg[c][j];
            }
        __syncthreads();
        for (int ch = threadIdx.x; ch < p.C; ch += TB) {
            float a = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) a += sums[w * (NC * TW * V) + ch];
            out[ch] = a;
        }
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const int ch = (c * TPR + t) * V + k;
                st_chunk(out + ch, p.C - ch, dg[c] + k);
            }
    }
}

// threads of a row and chunks of a thread: a wave to a row up to 2048 channels (32 a
// lane in registers), so that rows need no barrier; 16 channels at least, which a
// checkpoint's padding fills up to (1067994 x 8 bf16, gradient: 26 us, 67 with 8 lanes).
// The gradient's 32 channels a lane (1025 to 2048) take 390 registers in float32 and 306
// in bf16, so one wave a SIMD with nothing loaded ahead: 1000 x 2048 float32, 12.6 us of
// which the bytes need 5.2.  8 a lane take 78 and 102: six and four waves.
struct RowShape { int tpr, nc; };
static RowShape row_shape(int dt, int C) {
    const int V = dt == DT_BF16 ? 8 : 4, chunks = (C + V - 1) / V;
    for (int tpr : {2, 4, 8, 16, 32, 64})
        if (chunks <= tpr && tpr * V >= 16) return {tpr, 1};
    for (int nc : {2, 4, 8})
        if (chunks <= 64 * nc && nc * V <= 32) return {64, nc};
    for (int nc : {2, 4})
        if (chunks <= 256 * nc) return {256, nc};
    for (int nc : {2, 4})
        if (chunks <= 1024 * nc) return {1024, nc};
    return {0, 0};
}

template <bool BWD, typename T, int TPR, int NC, typename P>
static void rms_launch(const P& p, int wgs, hipStream_t st) {
    const dim3 grid((unsigned)wgs), block(TPR > 256 ? TPR : 256);
    if constexpr (BWD) launch((rmsnorm_bwd_k<T, TPR, NC>), grid, block, 0, st, p);
    else if (p.rows * p.C * (long)sizeof(T) >= kStreamBytes)
        launch((rmsnorm_k<T, TPR, NC, true>), grid, block, 0, st, p);
    else
        launch((rmsnorm_k<T, TPR, NC, false>), grid, block, 0, st, p);
}

template <bool BWD, typename T, typename P>
static hipError_t rms_dispatch(const P& p, RowShape s, int wgs, hipStream_t st) {
    switch (s.tpr * 16 + s.nc) {
    case 2 * 16 + 1:
        if constexpr (sizeof(T) == 2) rms_launch<BWD, T, 2, 1>(p, wgs, st);
        else return hipErrorInvalidValue;   // (8 channels of float32)
        break;
    case 4 * 16 + 1: rms_launch<BWD, T, 4, 1>(p, wgs, st); break;
    case 8 * 16 + 1: rms_launch<BWD, T, 8, 1>(p, wgs, st); break;
    case 16 * 16 + 1: rms_launch<BWD, T, 16, 1>(p, wgs, st); break;
    case 32 * 16 + 1: rms_launch<BWD, T, 32, 1>(p, wgs, st); break;
    case 64 * 16 + 1: rms_launch<BWD, T, 64, 1>(p, wgs, st); break;
    case 64 * 16 + 2: rms_launch<BWD, T, 64, 2>(p, wgs, st); break;
    case 64 * 16 + 4: rms_launch<BWD, T, 64, 4>(p, wgs, st); break;
    case 64 * 16 + 8:
        if constexpr (sizeof(T) == 4) rms_launch<BWD, T, 64, 8>(p, wgs, st);
        else return hipErrorInvalidValue;   // (row_shape: 4 chunks of bf16 a lane)
        break;
    case 256 * 16 + 2:
        if constexpr (sizeof(T) == 2) rms_launch<BWD, T, 256, 2>(p, wgs, st);
        else return hipErrorInvalidValue;   // (row_shape: a wave to a row)
        break;
    case 256 * 16 + 4: rms_launch<BWD, T, 256, 4>(p, wgs, st); break;
    case 1024 * 16 + 2: rms_launch<BWD, T, 1024, 2>(p, wgs, st); break;
    case 1024 * 16 + 4:
        if constexpr (sizeof(T) == 4) rms_launch<BWD, T, 1024, 4>(p, wgs, st);
        else return hipErrorInvalidValue;   // (kRmsMaxC bf16 channels are 2 chunks a thread)
        break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

// Workgroups, which walk over the rows.  Forward, 131072 x 128 bf16 with residual, output
// and checkpoint: 512 31.6 us, 1024 26.6, 2048 29.  Backward, where each also leaves a
// row of partials to be summed: 384 30.3 + 4.4 us, 512 26.1 + 3.9, 1024 26.0 + 4.9.
constexpr long kRmsWgs = 1024, kRmsBwdWgs = 512;

// the first row whose last chunk must not be read past its values
static long exact_row(int dt, long rows, int C, long ld) {
    return rows - (dt == DT_BF16 ? tail_rows<bf16>(rows, C, ld) : tail_rows<float>(rows, C, ld));
}

hipError_t launch_rmsnorm(int dt, RmsArgs p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    p.pitch = act8_pitch(p.C);
    p.G = act8_groups(p.C);
    p.exps = p.q ? p.q + p.rows * p.pitch : nullptr;
    p.exact = exact_row(dt, p.rows, p.C, std::min(p.ldx, p.res ? p.ldres : p.ldx));
    const RowShape s = row_shape(dt, p.C);
    if (!s.tpr) return hipErrorInvalidValue;
    const int rb = std::max(256, s.tpr) / s.tpr;
    const int wgs = (int)std::min(kRmsWgs, (p.rows + rb - 1) / rb);
    return dt == DT_BF16 ? rms_dispatch<false, bf16>(p, s, wgs, st) : rms_dispatch<false, float>(p, s, wgs, st);
}

int rmsnorm_bwd_parts(long rows, int C) {
    const RowShape s = row_shape(DT_F32, C);
    const int rb = std::max(256, s.tpr) / std::max(1, s.tpr);   // rows that a workgroup takes at once
    // (few rows: one workgroup; up to four turns of short rows cost less than a sum, a turn
    // 0.6 us and the sum 2.5; a turn of 2048 channels takes 3 us)
    const long turns = s.nc > 1 ? 1 : 4;
    return rows <= turns * rb ? 1 : (int)std::min(kRmsBwdWgs, (rows + rb - 1) / rb);
}

hipError_t launch_rmsnorm_bwd(int dt, RmsBwdArgs p, hipStream_t st) {
    if (p.rows <= 0 && !p.part) return hipSuccess;
    p.pitch = act8_pitch(p.C);
    p.G = act8_groups(p.C);
    p.exps = p.q ? p.q + p.rows * p.pitch : nullptr;
    p.exact = exact_row(dt, p.rows, p.C, std::min({p.lddy, p.h ? p.ldh : p.lddy, p.dres ? p.lddres : p.lddy}));
    p.pstride = (p.C + 3) / 4 * 4;
    const RowShape s = row_shape(dt, p.C);
    if (!s.tpr) return hipErrorInvalidValue;
    const int wgs = rmsnorm_bwd_parts(p.rows, p.C);
    return dt == DT_BF16 ? rms_dispatch<true, bf16>(p, s, wgs, st) : rms_dispatch<true, float>(p, s, wgs, st);
}

}  // namespace lpp
