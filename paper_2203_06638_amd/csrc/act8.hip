// act8.hip -- 8-bit activation checkpoints (act8.h): packing, unpacking, and the
// weight gradient of a 1x1 conv or linear layer read from one.
#include <algorithm>
#include <cmath>
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
// so the lanes of a ragged last group idle; rows of half a group or less take half
// the lanes.  A thread takes kPackU chunks, all loads first.
constexpr int kPackU = 4;

struct PackGeom {
    unsigned n;        // chunks: rows x cpr
    unsigned cpr;      // lanes per row
    FastDiv div;       // by cpr
    int C, pitch, G;
    unsigned exact;    // first of the rows whose last chunk must not be read past its values
    long ld;
};

// lanes that hold a group of rows of C values, padding codes included
template <typename T>
static int lanes_of(int C) {
    return (C <= 16 ? 16 : kAct8Group) * (int)sizeof(T) / 16;
}

// DECIDES: ACT8_DECIDES (a branch that costs the other modes 8%: 54675 x 90 float32
// 7.6 -> 8.2 us)
template <typename T, int L, bool DECIDES>
__global__ __launch_bounds__(256) void act8_pack_k(const T* __restrict__ x, PackGeom g, uint8_t* __restrict__ codes,
                                                   uint8_t* __restrict__ exps, int keep_sign) {
    constexpr int V = 16 / (int)sizeof(T);
    const unsigned i0 = blockIdx.x * (256u * kPackU) + threadIdx.x;
    unsigned row[kPackU];
    int ch[kPackU], n[kPackU];
    u4 w[kPackU];
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        const unsigned i = min(i0 + u * 256u, g.n - 1);
        row[u] = div_by(i, g.div);
        ch[u] = (int)(i - row[u] * g.cpr) * V;
        n[u] = g.C - ch[u];
        w[u] = ld_chunk(x + (long)row[u] * g.ld + (n[u] > 0 ? ch[u] : 0), n[u], row[u] >= g.exact);
    }
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        float v[V];
        chunk_values<T>(chunk_mask<T>(w[u], n[u]), v);
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) m = max(m, abs_bits(v[j]));
        const uint32_t s = act8_exp(group_max<L>(m));
        uint32_t w[V / 4];
#pragma unroll
        for (int k = 0; k < V / 4; ++k)
            w[k] = s == 255u ? 0u : act8_code4(v + 4 * k, act8_inv(s), DECIDES || keep_sign != 0);
        if (DECIDES && s == 255u) {
#pragma unroll
            for (int k = 0; k < V / 4; ++k) w[k] = act8_sign4(v + 4 * k);
        }
        if (i0 + u * 256u >= g.n) continue;
        if (ch[u] < g.pitch) {
            uint8_t* p = codes + (long)row[u] * g.pitch + ch[u];
            if constexpr (V == 8) *(uint2*)p = uint2{w[0], w[1]};
            else *(uint32_t*)p = w[0];
        }
        if (threadIdx.x % L == 0) exps[(long)row[u] * g.G + ch[u] / kAct8Group] = (uint8_t)s;
    }
}

template <typename T, bool ST>
__global__ __launch_bounds__(256) void act8_unpack_k(const uint8_t* __restrict__ codes,
                                                     const uint8_t* __restrict__ exps, PackGeom g, uint32_t bad,
                                                     T* __restrict__ x) {
    constexpr int V = 16 / (int)sizeof(T);
    const unsigned i0 = blockIdx.x * (256u * kPackU) + threadIdx.x;
    unsigned row[kPackU];
    int ch[kPackU], n[kPackU];
    uint32_t s[kPackU], w[kPackU][V / 4];
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        const unsigned i = min(i0 + u * 256u, g.n - 1);
        row[u] = div_by(i, g.div);
        ch[u] = (int)(i - row[u] * g.cpr) * V;
        n[u] = i0 + u * 256u < g.n ? g.C - ch[u] : 0;
        const int c = ch[u] < g.pitch ? ch[u] : 0;
        const uint8_t* p = codes + (long)row[u] * g.pitch + c;
        if constexpr (V == 8) {
            const uint2 q = *(const uint2*)p;
            w[u][0] = q.x;
            w[u][1] = q.y;
        } else {
            w[u][0] = *(const uint32_t*)p;
        }
        s[u] = exps[(long)row[u] * g.G + min(c / kAct8Group, g.G - 1)];
    }
#pragma unroll
    for (int u = 0; u < kPackU; ++u) {
        if (n[u] <= 0) continue;
        float v[V];
#pragma unroll
        for (int k = 0; k < V / 4; ++k) act8_val4(w[u][k], act8_step(s[u], bad), v + 4 * k);
        st_chunk<ST>(x + (long)row[u] * g.ld + ch[u], n[u], v);
    }
}

// f(first row, geometry, workgroups) over runs of rows of less than 2^31 chunks
template <typename T, typename F>
static hipError_t for_row_runs(long rows, int C, long ld, F f) {
    PackGeom g{};
    g.G = act8_groups(C);
    g.cpr = (unsigned)(g.G * lanes_of<T>(C));
    g.div = fast_div(g.cpr);
    g.C = C;
    g.pitch = act8_pitch(C);
    g.ld = ld;
    // (the threads behind the last chunk divide their index too)
    const long run = ((1l << 31) - 256 * kPackU) / g.cpr;
    for (long r0 = 0; r0 < rows; r0 += run) {
        const long left = std::min(run, rows - r0);
        g.n = (unsigned)(left * g.cpr);
        g.exact = (unsigned)std::clamp(rows - tail_rows<T>(rows, C, ld) - r0, 0l, left);
        f(r0, g, dim3((g.n + 256 * kPackU - 1) / (256 * kPackU)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
static hipError_t pack_rows(const T* x, long ld, long rows, int C, Act8Mode mode, uint8_t* q, hipStream_t st) {
    uint8_t* exps = q + rows * act8_pitch(C);
    return for_row_runs<T>(rows, C, ld, [&](long r0, const PackGeom& g, dim3 grid) {
        uint8_t* c = q + r0 * g.pitch;
        uint8_t* e = exps + r0 * g.G;
        constexpr int L = (int)sizeof(T);   // half a group's lanes
        const T* xr = x + r0 * ld;
        const int keep = mode != ACT8_NEAREST;
        if (mode == ACT8_DECIDES) {
            if (C <= 16) launch((act8_pack_k<T, L, true>), grid, dim3(256), 0, st, xr, g, c, e, keep);
            else launch((act8_pack_k<T, 2 * L, true>), grid, dim3(256), 0, st, xr, g, c, e, keep);
        } else {
            if (C <= 16) launch((act8_pack_k<T, L, false>), grid, dim3(256), 0, st, xr, g, c, e, keep);
            else launch((act8_pack_k<T, 2 * L, false>), grid, dim3(256), 0, st, xr, g, c, e, keep);
        }
    });
}

template <typename T>
static hipError_t unpack_rows(const uint8_t* q, long rows, int C, T* x, long ld, bool decides, hipStream_t st) {
    const uint8_t* exps = q + rows * act8_pitch(C);
    const uint32_t bad = decides ? 0x7f800000u : 0x7fc00000u;   // infinity, NaN
    return for_row_runs<T>(rows, C, ld, [&](long r0, const PackGeom& g, dim3 grid) {
        const uint8_t* c = q + r0 * g.pitch;
        const uint8_t* e = exps + r0 * g.G;
        if (rows * C * (long)sizeof(T) >= kStreamBytes)
            launch((act8_unpack_k<T, true>), grid, dim3(256), 0, st, c, e, g, bad, x + r0 * ld);
        else
            launch((act8_unpack_k<T, false>), grid, dim3(256), 0, st, c, e, g, bad, x + r0 * ld);
    });
}

hipError_t launch_act8_pack(int dt, const void* x, long ld, long rows, int C, Act8Mode mode, uint8_t* q,
                            hipStream_t st) {
    return dt == DT_BF16 ? pack_rows((const bf16*)x, ld, rows, C, mode, q, st)
                         : pack_rows((const float*)x, ld, rows, C, mode, q, st);
}

hipError_t launch_act8_unpack(int dt, const uint8_t* q, long rows, int C, void* x, long ld, bool decides,
                              hipStream_t st) {
    return dt == DT_BF16 ? unpack_rows(q, rows, C, (bf16*)x, ld, decides, st)
                         : unpack_rows(q, rows, C, (float*)x, ld, decides, st);
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
    int itiles, tiles;   // tiles along I, in all
    int splits;
    int tail;            // the last rows, which the steps leave out
};

// Eight waves of 32 x 64 (or 16 x 64, 32 x 32, 16 x 32) results, two workgroups of them
// to a compute unit.  Every step's loads are issued kWgAhead steps ahead into
// registers, without a branch around them, which would make the compiler wait for all
// of them: rows past the split's end are read from its last row and met with X = 0,
// chunks wholly past O or I are chunk 0 (they only reach results that are not
// stored), and so is what a chunk that crosses O takes from the next row.  The last
// rows of dY, where such a chunk would end behind the matrix, are added at the end.
// Measured, 2 steps ahead against 4: 1024 x 1024 over 100352 rows 297 and 302 us
// (bf16), 592 and 899 (float32, whose registers then spill).
constexpr int kWgAhead = 2;
constexpr int kWgThreads = 512;

template <typename T, int BO, int BI>
__global__ __launch_bounds__(kWgThreads, 4) void act8_wgrad_k(const T* __restrict__ dY,
                                                              const uint8_t* __restrict__ codes,
                                                              const uint8_t* __restrict__ exps,
                                                              float* __restrict__ part, WgGeom g) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1;       // bf16 terms of dY
    constexpr int TM = BO / 64, TN = BI / 32;        // 16x16 blocks per wave; waves 4 x 2
    constexpr int WA = BO / 8, WB = BI / 8;          // chunks of 8 channels per LDS row
    constexpr int QA = NP == 3 ? 2 : 1;              // 16-byte loads of a dY chunk
    constexpr int SA = 32 * BO, STEP = NP * SA + 32 * BI;
    constexpr int D = kWgAhead;
    static_assert(D % 2 == 0, "LDS buffers alternate");
    __shared__ __attribute__((aligned(16))) bf16 lds[2 * STEP];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave & 3, wn = wave >> 2;
    int tile, split;
    if (g.splits % 8 == 0) {
        // the tiles of a split, which read the same rows, on one of the 8 XCDs
        // (workgroups go round the XCDs by their index): 300 x 300 over 131072 rows
        // bf16 65 us, 100 without.  Where the XCDs' shares would differ it costs more
        // than it saves (25088 rows in 28 splits: 31 us, 28 without).
        const int x = blockIdx.x % 8, k = blockIdx.x / 8;
        tile = k % g.tiles;
        split = k / g.tiles * 8 + x;
    } else {
        tile = blockIdx.x % g.tiles;
        split = blockIdx.x / g.tiles;
    }
    const int i0 = tile % g.itiles * BI, o0 = tile / g.itiles * BO;
    const long r_lo = (long)split * g.rps;
    const int nr = (int)(min(g.rows - g.tail, r_lo + g.rps) - r_lo);   // rows of this split, but for the tail
    const int nk = (nr + 32 * D - 1) / (32 * D) * D;
    // 16 threads a row, a chunk of each operand per K-step (narrow tiles: half of them)
    const int trow = tid >> 4, tc = tid & 15;
    const int ac = tc % WA, bc = tc % WB;
    const int a_c = o0 + ac * 8 < g.O ? o0 + ac * 8 : 0;
    const int b_c = i0 + bc * 8 < g.pitch ? i0 + bc * 8 : 0;
    // (a chunk of padding codes only has no group of its own)
    const int e_c = min(b_c / kAct8Group, g.G - 1);
    // byte offsets from the first row of a step, which is the same for all threads
    uint32_t a_off, b_off, e_off;
    auto offsets = [&](int t) {
        a_off = ((uint32_t)t * (uint32_t)g.ld + (uint32_t)a_c) * (uint32_t)sizeof(T);
        b_off = (uint32_t)t * (uint32_t)g.pitch + (uint32_t)b_c;
        e_off = (uint32_t)t * (uint32_t)g.G + (uint32_t)e_c;
    };

    struct Stage {
        u4 a[QA];
        uint2 b;
        uint32_t e;
    };
    Stage sg[D];
    auto load = [&](Stage& s, int kk) {
        const int first = min(kk * 32, nr - 1), last = nr - 1 - first;
        if (last < 31) offsets(min(trow, last));     // (the last steps)
        const long r = r_lo + first;
        const T* p = (const T*)((const char*)(dY + r * g.ld) + a_off);
#pragma unroll
        for (int q = 0; q < QA; ++q) s.a[q] = *(const u4any*)(p + 4 * q);
        s.b = *(const uint2*)(codes + r * g.pitch + b_off);
        s.e = (exps + r * g.G)[e_off];
    };
    // The fast form takes dY as finite: a not finite value becomes NaN in its lower
    // terms, and meets X = 0 in rows past the end.  Either makes results NaN, and a
    // workgroup that ends with one that is not finite forms all of them again with the
    // CAREFUL form, where such a value is its first term alone.
    auto put = [&](const Stage& s, int kk, int buf, auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        bf16* As = lds + buf * STEP;
        bf16* Bs = As + NP * SA;
        const bool row = kk * 32 + trow < nr;
        if (WA == 16 || tc < WA) {
            bf16* p = As + trow * BO + wg_chunk<WA>(ac, trow) * 8;
            uint32_t x[QA * 4];
#pragma unroll
            for (int k = 0; k < QA * 4; ++k) {
                x[k] = s.a[k / 4][k % 4];
                if (CAREFUL) x[k] = row ? x[k] : 0u;
                // (a NaN whose upper half alone would be an infinity)
                if (CAREFUL && NP > 1 && (x[k] & 0x7fffffffu) > 0x7f800000u) x[k] |= 0x400000u;
            }
            if constexpr (NP == 1) {
                *(u4*)p = u4{x[0], x[1], x[2], x[3]};
            } else {
#pragma unroll
                for (int t = 0; t < NP; ++t) {
                    u4 w;
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = __builtin_amdgcn_perm(x[2 * k + 1], x[2 * k], 0x07060302u);
                    *(u4*)(p + t * SA) = w;
                    if (t + 1 < NP) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float d = __uint_as_float(x[k]) - __uint_as_float(x[k] & 0xffff0000u);
                            x[k] = CAREFUL && (x[k] & 0x7f800000u) == 0x7f800000u ? 0u : __float_as_uint(d);
                        }
                    }
                }
            }
        }
        if (WB == 16 || tc < WB) {
            const float step = row ? act8_step(s.e) : 0.f;
            float v[8];
            act8_val4(s.b.x, step, v);
            act8_val4(s.b.y, step, v + 4);
            u4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = __builtin_amdgcn_perm(__float_as_uint(v[2 * k + 1]), __float_as_uint(v[2 * k]), 0x07060302u);
            *(u4*)(Bs + trow * BI + wg_chunk<WB>(bc, trow) * 8) = w;
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
    auto product = [&](auto careful) {
#pragma unroll
        for (int x = 0; x < TM; ++x)
#pragma unroll
            for (int y = 0; y < TN; ++y) acc[x][y] = f4{0.f, 0.f, 0.f, 0.f};
        if (nr <= 0) return;
        offsets(trow);
#pragma unroll
        for (int s = 0; s < D; ++s) load(sg[s], s);
        put(sg[0], 0, 0, careful);
        load(sg[0], D);
        for (int kk = 0; kk < nk; kk += D) {
#pragma unroll
            for (int s = 0; s < D; ++s) {
                __syncthreads();
                const bf16* As = lds + (s & 1) * STEP;
                const bf16* Bs = As + NP * SA;
                bf8 fa[NP][TM], fb[TN];
#pragma unroll
                for (int y = 0; y < TN; ++y) fb[y] = frag(Bs, (wn * TN + y) * 16, std::integral_constant<int, WB>{});
#pragma unroll
                for (int t = 0; t < NP; ++t)
#pragma unroll
                    for (int x = 0; x < TM; ++x)
                        fa[t][x] = frag(As + t * SA, (wm * TM + x) * 16, std::integral_constant<int, WA>{});
                // the next step's operands go into the other buffer while this one is multiplied
                const int nx = (s + 1) % D;
                put(sg[nx], kk + s + 1, (s + 1) & 1, careful);
                load(sg[nx], kk + s + 1 + D);
#pragma unroll
                for (int t = 0; t < NP; ++t)
#pragma unroll
                    for (int x = 0; x < TM; ++x)
#pragma unroll
                        for (int y = 0; y < TN; ++y)
                            acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[t][x], fb[y], acc[x][y], 0, 0, 0);
            }
        }
        __syncthreads();
    };
    product(std::false_type{});
    bool bad = false;
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y)
#pragma unroll
            for (int k = 0; k < 4; ++k) bad |= abs_bits(acc[x][y][k]) >= 0x7f800000u;
    if (__syncthreads_or(bad)) product(std::true_type{});
    if (split + 1 == g.splits)
        for (long r = g.rows - g.tail; r < g.rows; ++r) {
            float d[TM][4], x[TN];
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    d[m][k] = ld1(dY + r * g.ld, min(o0 + (wm * TM + m) * 16 + (lane >> 4) * 4 + k, g.O - 1));
#pragma unroll
            for (int y = 0; y < TN; ++y) {
                const int i = min(i0 + (wn * TN + y) * 16 + (lane & 15), g.I - 1);
                x[y] = (float)(int8_t)codes[r * g.pitch + i] * act8_step(exps[r * g.G + i / kAct8Group]);
            }
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int y = 0; y < TN; ++y)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[m][y][k] = __builtin_fmaf(d[m][k], x[y], acc[m][y][k]);
        }
    float* out = part + (long)split * g.pstride;
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

// Splits.  A step of a workgroup costs about 0.4 us (bf16 with two workgroups a compute
// unit; float32 0.75, or 1.2 with one: the rule takes both types alike) and a split's
// partials O I 8 bytes of traffic at 4 TB/s: rows / S / 32 steps and S partials
// together are least at S^2 = 6500 rows / (O I) (half or twice that: within 5%).  Never
// more than two workgroups a compute unit, and one where that leaves a split fewer than
// 1536 rows (one against two: 128 x 512 over 131072 rows 41.6 and 44.3 us with the sum,
// 1024 x 1024 over 100352 rows 356 and 297).  Up to 400 rows a sum of partials costs more
// than it saves (64 x 64, 256 rows: 6.7 us in one run, 8.9 in four and a sum for bf16, 7.5
// and 10.1 for float32; 640 rows: 9.6 and 8.9, 13.3 and 10.2; 333 x 100 x 36 float32 10.6
// in one, 6.4 + 3.8 in several and a sum, whose launch it saves).
Act8WgPlan act8_wgrad_plan(long rows, int O, int I) {
    Act8WgPlan p{};
    p.bo = O > 64 ? 128 : 64;
    p.bi = I > 64 ? 128 : 64;
    const long tiles = (long)((O + p.bo - 1) / p.bo) * ((I + p.bi - 1) / p.bi);
    long splits = (long)std::sqrt(6500.0 * rows / ((double)O * I));
    const long two = 512 / tiles;
    splits = std::min(splits, two > 0 && rows / two >= 1536 ? two : 256 / tiles);
    if (splits >= 16) splits = splits / 8 * 8;   // (for the XCDs)
    splits = rows <= 400 ? 1 : std::max(1l, std::min(splits, rows / 64));
    p.rps = std::max(32l, ((rows + splits - 1) / splits + 31) / 32 * 32);
    p.splits = (int)std::max(1l, (rows + p.rps - 1) / p.rps);
    p.part_floats = ((long)O * I + 3) / 4 * 4;
    return p;
}

template <typename T>
static hipError_t wgrad_parts(const T* dY, long ld, const uint8_t* q, long rows, int O, int I, float* part,
                              const Act8WgPlan& p, hipStream_t st) {
    const int it = (I + p.bi - 1) / p.bi, ot = (O + p.bo - 1) / p.bo;
    // rows from whose last chunk 8 channels on would lie behind the matrix
    const long over = (O + 7) / 8 * 8 - O, dist = rows > 1 ? ld : over;
    const long tail = over ? std::min(rows, (over + dist - 1) / dist) : 0;
    const WgGeom g{rows, p.rps, O, I, act8_pitch(I), act8_groups(I), ld, p.part_floats, it, it * ot, p.splits,
                   (int)tail};
    const uint8_t* exps = q + rows * g.pitch;
    const dim3 grid((unsigned)(g.tiles * p.splits)), block(kWgThreads);
    if (p.bo == 128 && p.bi == 128) launch((act8_wgrad_k<T, 128, 128>), grid, block, 0, st, dY, q, exps, part, g);
    else if (p.bo == 128) launch((act8_wgrad_k<T, 128, 64>), grid, block, 0, st, dY, q, exps, part, g);
    else if (p.bi == 128) launch((act8_wgrad_k<T, 64, 128>), grid, block, 0, st, dY, q, exps, part, g);
    else launch((act8_wgrad_k<T, 64, 64>), grid, block, 0, st, dY, q, exps, part, g);
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
