// act8.hip -- 8-bit activation checkpoints (act8.h): packing, unpacking, and the
// weight gradient of a 1x1 conv or linear layer read from one.
#include <algorithm>
#include <type_traits>

#include "act8.h"
#include "kernels.h"
#include "launch.h"
#include "ldstile.h"

namespace lpp {

// ---------------------------------------------------------------- pack, unpack
//
// One pass; bound by HBM (e + 33/32 bytes a value).  A lane takes V = 16 /
// sizeof(T) successive channels (a chunk), so that a wave's loads are whole
// cache lines and the 32 / V lanes of a group are neighbours: the group's
// maximum takes two or three lane permutes.  Rows are cut into whole groups,
// so the lanes of a ragged last group idle.  A thread takes kPackU chunks, all
// loads first.
constexpr int kPackU = 4;

struct PackGeom {
    unsigned n;        // chunks: rows x cpr
    unsigned cpr;      // chunks per row, whole groups
    FastDiv div;       // by cpr
    int C, pitch, G;
    long ld;
};

template <bool A, typename T>
__global__ __launch_bounds__(256) void act8_pack_k(const T* __restrict__ x, PackGeom g, uint8_t* __restrict__ codes,
                                                   uint8_t* __restrict__ exps, int keep_sign) {
    constexpr int V = 16 / (int)sizeof(T), L = kAct8Group / V;
    const unsigned i0 = blockIdx.x * (256u * kPackU) + threadIdx.x;
    unsigned row[kPackU];
    int ch[kPackU];
    float v[kPackU][V];
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        const unsigned i = i0 + u * 256u;
        row[u] = div_by(i, g.div);
        ch[u] = (int)(i - row[u] * g.cpr) * V;
        ld_chunk<A>(x + (long)row[u] * g.ld + ch[u], i < g.n ? g.C - ch[u] : 0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        const unsigned i = i0 + u * 256u;
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) m = max(m, abs_bits(v[u][j]));
        const uint32_t s = act8_exp(group_max<L>(m));
        uint32_t w[V / 4];
#pragma unroll
        for (int k = 0; k < V / 4; ++k)
            w[k] = s == 255u ? 0u : act8_code4(v[u] + 4 * k, act8_inv(s), keep_sign != 0);
        if (i >= g.n) continue;
        if (ch[u] < g.pitch) {
            uint8_t* p = codes + (long)row[u] * g.pitch + ch[u];
            if constexpr (V == 8) *(uint2*)p = uint2{w[0], w[1]};
            else *(uint32_t*)p = w[0];
        }
        if (threadIdx.x % L == 0) exps[(long)row[u] * g.G + ch[u] / kAct8Group] = (uint8_t)s;
    }
}

template <bool A, typename T>
__global__ __launch_bounds__(256) void act8_unpack_k(const uint8_t* __restrict__ codes,
                                                     const uint8_t* __restrict__ exps, PackGeom g,
                                                     T* __restrict__ x) {
    constexpr int V = 16 / (int)sizeof(T);
    const unsigned i0 = blockIdx.x * (256u * kPackU) + threadIdx.x;
    unsigned row[kPackU];
    int ch[kPackU], n[kPackU];
    uint32_t s[kPackU], w[kPackU][V / 4];
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        const unsigned i = i0 + u * 256u;
        row[u] = div_by(i, g.div);
        ch[u] = (int)(i - row[u] * g.cpr) * V;
        n[u] = i < g.n ? g.C - ch[u] : 0;
        s[u] = 7u;
        if (n[u] > 0) {
            const uint8_t* p = codes + (long)row[u] * g.pitch + ch[u];
            if constexpr (V == 8) {
                const uint2 q = *(const uint2*)p;
                w[u][0] = q.x;
                w[u][1] = q.y;
            } else {
                w[u][0] = *(const uint32_t*)p;
            }
            s[u] = exps[(long)row[u] * g.G + ch[u] / kAct8Group];
        }
    }
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        if (n[u] <= 0) continue;
        float v[V];
#pragma unroll
        for (int k = 0; k < V / 4; ++k) act8_val4(w[u][k], act8_step(s[u]), v + 4 * k);
        st_chunk<A>(x + (long)row[u] * g.ld + ch[u], n[u], v);
    }
}

// whether 16-byte accesses at p + row * ld + (multiple of 16 bytes) are aligned
template <typename T>
static bool rows_aligned(const T* p, long ld, long rows) {
    return ((uintptr_t)p & 15) == 0 && (rows <= 1 || ld * (long)sizeof(T) % 16 == 0);
}

// f(first row, geometry, workgroups) over runs of rows of less than 2^31 chunks
template <typename T, typename F>
static hipError_t for_row_runs(long rows, int C, long ld, F f) {
    constexpr int V = 16 / (int)sizeof(T);
    PackGeom g{};
    g.G = act8_groups(C);
    g.cpr = (unsigned)g.G * (kAct8Group / V);
    g.div = fast_div(g.cpr);
    g.C = C;
    g.pitch = act8_pitch(C);
    g.ld = ld;
    // (the threads behind the last chunk divide their index too)
    const long run = ((1l << 31) - 256 * kPackU) / g.cpr;
    for (long r0 = 0; r0 < rows; r0 += run) {
        g.n = (unsigned)(std::min(run, rows - r0) * g.cpr);
        f(r0, g, dim3((g.n + 256 * kPackU - 1) / (256 * kPackU)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
static hipError_t pack_rows(const T* x, long ld, long rows, int C, bool keep_sign, uint8_t* q, hipStream_t st) {
    const bool al = rows_aligned(x, ld, rows);
    uint8_t* exps = q + rows * act8_pitch(C);
    return for_row_runs<T>(rows, C, ld, [&](long r0, const PackGeom& g, dim3 grid) {
        uint8_t* c = q + r0 * g.pitch;
        uint8_t* e = exps + r0 * g.G;
        if (al) launch((act8_pack_k<true, T>), grid, dim3(256), 0, st, x + r0 * ld, g, c, e, (int)keep_sign);
        else launch((act8_pack_k<false, T>), grid, dim3(256), 0, st, x + r0 * ld, g, c, e, (int)keep_sign);
    });
}

template <typename T>
static hipError_t unpack_rows(const uint8_t* q, long rows, int C, T* x, long ld, hipStream_t st) {
    const bool al = rows_aligned(x, ld, rows);
    const uint8_t* exps = q + rows * act8_pitch(C);
    return for_row_runs<T>(rows, C, ld, [&](long r0, const PackGeom& g, dim3 grid) {
        const uint8_t* c = q + r0 * g.pitch;
        const uint8_t* e = exps + r0 * g.G;
        if (al) launch((act8_unpack_k<true, T>), grid, dim3(256), 0, st, c, e, g, x + r0 * ld);
        else launch((act8_unpack_k<false, T>), grid, dim3(256), 0, st, c, e, g, x + r0 * ld);
    });
}

hipError_t launch_act8_pack(int dt, const void* x, long ld, long rows, int C, bool keep_sign, uint8_t* q,
                            hipStream_t st) {
    return dt == DT_BF16 ? pack_rows((const bf16*)x, ld, rows, C, keep_sign, q, st)
                         : pack_rows((const float*)x, ld, rows, C, keep_sign, q, st);
}

hipError_t launch_act8_unpack(int dt, const uint8_t* q, long rows, int C, void* x, long ld, hipStream_t st) {
    return dt == DT_BF16 ? unpack_rows(q, rows, C, (bf16*)x, ld, st) : unpack_rows(q, rows, C, (float*)x, ld, st);
}

// ---------------------------------------------------------------- weight gradient
//
// dW[o][i] = sum over rows of dY[row][o] * X[row][i], X the values of a checkpoint.
// A matrix product whose reduction runs over the rows, the slow dimension of both
// operands in memory: each K-step of 32 rows goes into LDS as it lies (rows of
// channels, bf16) and the MFMA operands are read with the LDS transpose read.
// Codes become bf16 on the way into LDS, exactly (act8.h).  A float32 dY is cut
// into three bf16 terms of 8 significant bits each, which add up to it exactly, and
// multiplied three times: the products are exact and the sums float32, as with
// float32 operands, at the bf16 MFMA's rate / 3 (five times the float32 one's).
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ s4v lds_tr16(const bf16* p) {
    typedef __attribute__((address_space(3))) s4v lds_s4v;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v*)(uintptr_t)(unsigned)(uintptr_t)(
        const __attribute__((address_space(3))) bf16*)p);
}

struct WgGeom {
    long rows, rps;      // rows; rows of a split
    int O, I, pitch, G;
    long ld;             // elements between rows of dY
    long pstride;        // floats between the partials of two splits
};

template <typename T, int BO, int BI, bool A>
__global__ __launch_bounds__(256) void act8_wgrad_k(const T* __restrict__ dY, const uint8_t* __restrict__ codes,
                                                    const uint8_t* __restrict__ exps, float* __restrict__ part,
                                                    WgGeom g) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;       // bf16 terms of dY
    constexpr int TM = BO / 32, TN = BI / 32;        // 16x16 blocks per wave; waves 2 x 2
    constexpr int WA = BO / 8, WB = BI / 8;          // chunks of 8 channels per LDS row
    constexpr int CA = BO / 64;                      // dY chunks of a thread per K-step
    constexpr int CB = BI / 64;                      // X chunks (8 codes each)
    constexpr int SA = 32 * BO, STEP = NP * SA + 32 * BI;
    __shared__ __attribute__((aligned(16))) bf16 lds[2 * STEP];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave & 1, wn = wave >> 1;
    const int i0 = blockIdx.x * BI, o0 = blockIdx.y * BO;
    const long r_lo = (long)blockIdx.z * g.rps, r_hi = min(g.rows, r_lo + g.rps);
    const int nk = (int)((r_hi - r_lo + 31) / 32);
    const int trow = tid >> 3, tc = tid & 7;         // 8 threads a row

    float a[CA][8];
    uint32_t b[CB][2], bs[CB];
    auto load = [&](int kk) {
        const long r = r_lo + (long)kk * 32 + trow;
        const bool ok = r < r_hi;
#pragma unroll
        for (int c = 0; c < CA; ++c) {
            const int o = o0 + (c * 8 + tc) * 8;
            const int n = ok ? g.O - o : 0;
            if constexpr (sizeof(T) == 4) {
                ld_chunk<A>(dY + r * g.ld + o, n, a[c]);
                ld_chunk<A>(dY + r * g.ld + o + 4, n - 4, a[c] + 4);
            } else {
                ld_chunk<A>(dY + r * g.ld + o, n, a[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            const int i = i0 + (tc * CB + c) * 8;
            const bool in = ok && i < g.pitch;
            const uint2 q = in ? *(const uint2*)(codes + r * g.pitch + i) : uint2{0u, 0u};
            b[c][0] = q.x;
            b[c][1] = q.y;
            // (a chunk of padding channels only has no group of its own)
            bs[c] = in ? exps[r * g.G + min(i / kAct8Group, g.G - 1)] : 7u;
        }
    };
    auto put = [&](int buf) {
        bf16* As = lds + buf * STEP;
        bf16* Bs = As + NP * SA;
#pragma unroll
        for (int c = 0; c < CA; ++c) {
            bf16* p = As + trow * BO + wg_chunk<WA>(c * 8 + tc, trow) * 8;
            uint32_t w[NP][4];
            if constexpr (NP == 1) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[0][k] = (__float_as_uint(a[c][2 * k]) >> 16) | (__float_as_uint(a[c][2 * k + 1]) & 0xffff0000u);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x0 = a[c][2 * k], x1 = a[c][2 * k + 1];
#pragma unroll
                    for (int t = 0; t < NP; ++t) {
                        const uint32_t h0 = __float_as_uint(x0) & 0xffff0000u, h1 = __float_as_uint(x1) & 0xffff0000u;
                        w[t][k] = __builtin_amdgcn_perm(h1, h0, 0x07060302u);
                        if (t + 1 < NP) {
                            // an infinity or NaN is its first term alone
                            const bool f0 = (h0 & 0x7f800000u) != 0x7f800000u, f1 = (h1 & 0x7f800000u) != 0x7f800000u;
                            x0 = f0 ? x0 - __uint_as_float(h0) : 0.f;
                            x1 = f1 ? x1 - __uint_as_float(h1) : 0.f;
                        }
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < NP; ++t) *(uint4*)(p + t * SA) = uint4{w[t][0], w[t][1], w[t][2], w[t][3]};
        }
#pragma unroll
        for (int c = 0; c < CB; ++c) {
            float v[8];
            const float step = act8_step(bs[c]);
            act8_val4(b[c][0], step, v);
            act8_val4(b[c][1], step, v + 4);
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = __builtin_amdgcn_perm(__float_as_uint(v[2 * k + 1]), __float_as_uint(v[2 * k]), 0x07060302u);
            *(uint4*)(Bs + trow * BI + wg_chunk<WB>(tc * CB + c, trow) * 8) = uint4{w[0], w[1], w[2], w[3]};
        }
    };
    const int fs = lane & 15, fg = lane >> 4;
    auto frag = [&](const bf16* base, int c16, auto w) {
        constexpr int W = decltype(w)::value;
        s4v h[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int row = 8 * fg + 4 * k + (fs >> 2);
            const int ch = c16 + 4 * (fs & 3);
            h[k] = lds_tr16(base + row * (8 * W) + wg_chunk<W>(ch >> 3, row) * 8 + (ch & 7));
        }
        return __builtin_bit_cast(bf8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };

    f4 acc[TM][TN];
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y) acc[x][y] = f4{0.f, 0.f, 0.f, 0.f};
    if (nk > 0) {
        load(0);
        put(0);
        if (nk > 1) load(1);
    }
    for (int kk = 0; kk < nk; ++kk) {
        __syncthreads();
        if (kk + 1 < nk) put((kk + 1) & 1);
        if (kk + 2 < nk) load(kk + 2);
        const bf16* As = lds + (kk & 1) * STEP;
        const bf16* Bs = As + NP * SA;
        bf8 fb[TN];
#pragma unroll
        for (int y = 0; y < TN; ++y) fb[y] = frag(Bs, (wn * TN + y) * 16, std::integral_constant<int, WB>{});
#pragma unroll
        for (int t = 0; t < NP; ++t)
#pragma unroll
            for (int x = 0; x < TM; ++x) {
                const bf8 fa = frag(As + t * SA, (wm * TM + x) * 16, std::integral_constant<int, WA>{});
#pragma unroll
                for (int y = 0; y < TN; ++y)
                    acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa, fb[y], acc[x][y], 0, 0, 0);
            }
    }
    float* out = part + (long)blockIdx.z * g.pstride;
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            const int i = i0 + (wn * TN + y) * 16 + (lane & 15);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int o = o0 + (wm * TM + x) * 16 + (lane >> 4) * 4 + k;
                if (o < g.O && i < g.I) out[(long)o * g.I + i] = acc[x][y][k];
            }
        }
}

Act8WgPlan act8_wgrad_plan(long rows, int O, int I) {
    Act8WgPlan p{};
    p.bo = O > 64 ? 128 : 64;
    p.bi = I > 64 ? 128 : 64;
    const long tiles = (long)((O + p.bo - 1) / p.bo) * ((I + p.bi - 1) / p.bi);
    long splits = (512 + tiles - 1) / tiles;
    const long most = std::max(1l, (rows + 255) / 256);
    if (splits > most) splits = most;
    p.rps = std::max(32l, ((rows + splits - 1) / splits + 31) / 32 * 32);
    p.splits = (int)std::max(1l, (rows + p.rps - 1) / p.rps);
    p.part_floats = ((long)O * I + 3) / 4 * 4;
    return p;
}

template <typename T, int BO, int BI>
static void wgrad_tile(bool al, dim3 grid, const T* dY, const uint8_t* q, const uint8_t* exps, float* part,
                       const WgGeom& g, hipStream_t st) {
    if (al) launch((act8_wgrad_k<T, BO, BI, true>), grid, dim3(256), 0, st, dY, q, exps, part, g);
    else launch((act8_wgrad_k<T, BO, BI, false>), grid, dim3(256), 0, st, dY, q, exps, part, g);
}

template <typename T>
static hipError_t wgrad_parts(const T* dY, long ld, const uint8_t* q, long rows, int O, int I, float* part,
                              const Act8WgPlan& p, hipStream_t st) {
    const WgGeom g{rows, p.rps, O, I, act8_pitch(I), act8_groups(I), ld, p.part_floats};
    const uint8_t* exps = q + rows * g.pitch;
    const bool al = rows_aligned(dY, ld, rows);
    const dim3 grid((unsigned)((I + p.bi - 1) / p.bi), (unsigned)((O + p.bo - 1) / p.bo), (unsigned)p.splits);
    if (p.bo == 128 && p.bi == 128) wgrad_tile<T, 128, 128>(al, grid, dY, q, exps, part, g, st);
    else if (p.bo == 128) wgrad_tile<T, 128, 64>(al, grid, dY, q, exps, part, g, st);
    else if (p.bi == 128) wgrad_tile<T, 64, 128>(al, grid, dY, q, exps, part, g, st);
    else wgrad_tile<T, 64, 64>(al, grid, dY, q, exps, part, g, st);
    return hipGetLastError();
}

hipError_t launch_act8_wgrad_part(int dt, const void* dY, long ld, const uint8_t* q, long rows, int O, int I,
                                  float* part, const Act8WgPlan& p, hipStream_t st) {
    return dt == DT_BF16 ? wgrad_parts((const bf16*)dY, ld, q, rows, O, I, part, p, st)
                         : wgrad_parts((const float*)dY, ld, q, rows, O, I, part, p, st);
}

hipError_t launch_act8_wgrad(int dt, const void* dY, long ld, const uint8_t* q, long rows, int O, int I, float* dw,
                             float* ws, hipStream_t st) {
    const Act8WgPlan p = act8_wgrad_plan(rows, O, I);
    hipError_t e = launch_act8_wgrad_part(dt, dY, ld, q, rows, O, I, p.splits > 1 ? ws : dw, p, st);
    if (e == hipSuccess && p.splits > 1) e = launch_part_sums(ws, p.splits, (int)((long)O * I), dw, st);
    return e;
}

}  // namespace lpp
