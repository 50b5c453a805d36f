// groupnorm.hip -- group norm of a channels-last activation with an activation
// function behind it, and its gradient.
//
// An activation is [images][pixels][C]; a group is cg = C / G successive channels of
// one image, M = pixels * cg values.
//
//   mean, var over the group's M values, rstd = 1 / sqrt(var + eps),
//   u = (x - mean) * rstd, z = u * gamma + beta, y = act(z)
//   dz = dy * act'(z), dbeta = sum dz, dgamma = sum dz * u (over images and pixels),
//   dx = rstd * (dz * gamma - (s1 + u * s2)) (+ dres),
//   s1 = mean over the group of dz * gamma, s2 = of dz * gamma * u
//
// z is the same expression in both directions, so that a ReLU's gradient decides as the
// forward pass did.  Statistics and sums are float32: means and sums of squared deviations of parts are
// merged (never sums of squares of the values), everything in a fixed order.
//
// This file's kernels spread an image over the chip: partial sums, then a second pass over the
// data, which takes part of it from the caches.  Maps that a workgroup's registers hold take
// groupnorm_whole.hip, which reads them once.  Both do about 8 operations a value forward, 16
// backward, so that the bytes set the floor; how near they come is said at each kernel.
#include <algorithm>

#include "act8.h"
#include "groupnorm.h"
#include "kernels.h"
#include "launch.h"

namespace lpp {

namespace {

constexpr int TB = 256;              // threads of a workgroup
constexpr int kWaves = TB / 64;
constexpr int U = 4;                 // rows that a thread has under way at once

// count, mean and sum of squared deviations of a set of values; a merge takes the sums
// of both and what their means differ by
struct Moments {
    float n, mean, m2;
};
__device__ __forceinline__ void merge(Moments& a, float n, float mean, float m2) {
    const float sum = a.n + n, f = sum > 0.f ? n / sum : 0.f, d = mean - a.mean;
    // (an empty side has no mean: a.n * f is 0 then, before a square could overflow)
    a.m2 += m2 + a.n * f * d * d;
    a.mean += d * f;
    a.n = sum;
}

// A workgroup's part of an activation: a split of an image's rows, a slab of its
// channels.  W = 2^lw lanes take a row's chunks of V channels, the others further rows.
template <int V>
struct Place {
    long image, r0, r1;
    int slab, split, rl, RL, ch, n, c0, c1, g0, np;
    __device__ __forceinline__ Place(const GnShape& s, unsigned b) {
        const unsigned per = (unsigned)(s.slabs * s.splits), i = b / per, k = b - i * per;
        image = i;
        slab = (int)(k / (unsigned)s.splits);
        split = (int)k - slab * s.splits;
        r0 = image * s.pixels + split * s.rps;
        r1 = min(r0 + s.rps, (image + 1) * s.pixels);
        const int t = threadIdx.x;
        RL = TB >> s.lw;
        rl = t >> s.lw;
        const int w = t & ((1 << s.lw) - 1);
        c0 = slab * (V << s.lw);
        c1 = min(s.C, c0 + (V << s.lw));
        ch = c0 + w * V;
        n = s.C - ch;                 // channels of the thread's chunk (none: an idle lane, which loads channel 0)
        if (n <= 0) ch = 0;
        g0 = c0 / s.cg;
        np = (c1 - 1) / s.cg - g0 + 1;   // groups that the slab meets
    }
};
// slabs that group g lies in
template <int V>
__device__ __forceinline__ int first_slab(const GnShape& s, int g) { return g * s.cg / (V << s.lw); }
template <int V>
__device__ __forceinline__ int last_slab(const GnShape& s, int g) { return ((g + 1) * s.cg - 1) / (V << s.lw); }

// f(q, l, ll) for the groups of a workgroup's slab, 2^ll lanes to each, l the thread's.  A group that lies
// in other slabs too has a whole wave in each of them, so that its parts are merged in one order
// everywhere: it has one mean and one rstd, the stored ones.  (The slab's other groups share all
// threads.)
template <int V, class F>
__device__ __forceinline__ void each_group(const GnShape& s, const Place<V>& at, F f) {
    const int t = threadIdx.x, wave = t >> 6;
    const bool before = at.c0 != at.g0 * s.cg, behind = at.c1 != (at.g0 + at.np) * s.cg;
    const int ll = item_lanes(TB, at.np), first = before, last = at.np - behind;
    for (int q = first + (t >> ll); q < last; q += TB >> ll) f(q, t & ((1 << ll) - 1), ll);
    const int q = wave == 0 ? 0 : at.np - 1;
    if ((wave == 0 && before) || (wave == 1 && behind && !(before && at.np == 1))) f(q, t & 63, 6);
}

// f(split, slab, part) for every 2^ll-th of a group's parts, l the first: slabs sa .. sa + ns - 1 of
// every split.  Four loads are under way at once.
template <class F>
__device__ __forceinline__ void each_part(const GnShape& s, const float2* ws, long image, int g, int sa, int ns, int l,
                                          int ll, F f) {
    const float2* in = ws + image * s.splits * s.parts + g + sa;
    const int total = ns * s.splits;
    for (int e0 = l; e0 < total; e0 += 4 << ll) {
        float2 m[4];
        int split[4], slab[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = min(e0 + (u << ll), total - 1);
            split[u] = ns == 1 ? e : e / ns;
            slab[u] = e - split[u] * ns;
            m[u] = in[(long)split[u] * s.parts + slab[u]];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (e0 + (u << ll) < total) f(split[u], sa + slab[u], m[u]);
    }
}

// ---- forward -----------------------------------------------------------------

// Mean and squared deviations of every part (a group's channels in a slab, a split of
// the rows), into ws [image][split][part] as pairs; part = group + slab.  A thread sums
// each of its channels about the first value that it reads.  Four loads a thread are under way
// at once (U); with gn_apply_k 16 x 3136 x 256 bf16 takes 26.8 us (16.1 at a large copy's rate if the
// data were read once).
template <typename T>
__global__ __launch_bounds__(TB) void gn_stats_k(GnArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float sm[2][kWaves][64 * V];
    __shared__ float scnt[kWaves];
    const Place<V> at(p.s, blockIdx.x);
    const T* x = (const T*)p.x + at.ch;
    float k[V], s[V], ss[V];
    const long lead = min(at.r0 + at.rl, at.r1 - 1);
    chunk_values<T>(ld_chunk(x + lead * p.ldx, at.n, lead >= p.exact), k);
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = ss[j] = 0.f;
    const long mine = at.r1 - at.r0 - at.rl;
    float cnt = mine > 0 ? (float)((mine - 1) / at.RL + 1) : 0.f;
    const float scale = sum_scale(cnt);
    auto add = [&](u4 w) {
        float v[V];
        chunk_values<T>(w, v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = v[j] - k[j];
            s[j] = __builtin_fmaf(d, scale, s[j]);
            ss[j] = __builtin_fmaf(d, d, ss[j]);
        }
    };
    const long whole = min(at.r1, p.exact);
    long r = at.r0 + at.rl;
    for (; r + (U - 1) * at.RL < whole; r += U * at.RL) {
        u4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = ld_chunk(x + (r + u * at.RL) * p.ldx, at.n, false);
#pragma unroll
        for (int u = 0; u < U; ++u) add(w[u]);
    }
    for (; r < at.r1; r += at.RL) add(ld_chunk(x + r * p.ldx, at.n, r >= p.exact));
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float e = cnt > 0.f ? s[j] / (cnt * scale) : 0.f;
        s[j] = cnt > 0.f ? k[j] + e : 0.f;
        // (an infinite sum stays one; rounding leaves nothing below 0)
        const float m2 = ss[j] == INFINITY ? ss[j] : ss[j] - e * (e * cnt);
        ss[j] = m2 < 0.f ? 0.f : m2;
    }
    // the wave's rows: each merge halves the channels that a lane goes on with (as fold)
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
    int d = 1 << p.s.lw, first = 0, n = V;
#pragma unroll
    for (int h = V / 2; h >= 1; h /= 2) {
        if (d >= 64) continue;
        const bool up = (lane & d) != 0;
        const float oc = __shfl_xor(cnt, d);
#pragma unroll
        for (int j = 0; j < h; ++j) {
            Moments m{cnt, up ? s[j + h] : s[j], up ? ss[j + h] : ss[j]};
            const float mean = __shfl_xor(up ? s[j] : s[j + h], d), m2 = __shfl_xor(up ? ss[j] : ss[j + h], d);
            merge(m, oc, mean, m2);
            s[j] = m.mean;
            ss[j] = m.m2;
        }
        cnt += oc;
        first += up ? h : 0;
        n = h;
        d <<= 1;
    }
    const int apart = d;       // lanes from here on repeat the channels of the lower ones
    for (; d < 64; d <<= 1) {
        Moments m{cnt, s[0], ss[0]};
        const float oc = __shfl_xor(cnt, d), mean = __shfl_xor(s[0], d), m2 = __shfl_xor(ss[0], d);
        merge(m, oc, mean, m2);
        s[0] = m.mean;
        ss[0] = m.m2;
        cnt = m.n;
    }
    if (lane < apart) {
        const int c = (t & ((1 << p.s.lw) - 1)) * V + first;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < n) {
                sm[0][wave][c + j] = s[j];
                sm[1][wave][c + j] = ss[j];
            }
        if (lane == 0) scnt[wave] = cnt;
    }
    __syncthreads();
    const int ll = item_lanes(TB, at.np), l = t & ((1 << ll) - 1);
    float2* out = (float2*)p.ws + (at.image * p.s.splits + at.split) * p.s.parts;
    for (int q = t >> ll; q < at.np; q += TB >> ll) {
        const int g = at.g0 + q;
        const int lo = max(g * p.s.cg, at.c0) - at.c0, hi = min((g + 1) * p.s.cg, at.c1) - at.c0;
        Moments a{0.f, 0.f, 0.f};
        for (int e = l; e < (hi - lo) * kWaves; e += 1 << ll) {
            const int c = lo + e / kWaves, w = e % kWaves;
            merge(a, scnt[w], sm[0][w][c], sm[1][w][c]);
        }
        for (int d = 1; d < 1 << ll; d <<= 1) {
            const float n = __shfl_xor(a.n, d), mean = __shfl_xor(a.mean, d), m2 = __shfl_xor(a.m2, d);
            merge(a, n, mean, m2);
        }
        if (l == 0) out[g + at.slab] = float2{a.mean, a.m2};
    }
}

// Mean and rstd of the slab's groups from their parts, then y.  Every workgroup merges its groups'
// parts by itself (some KB from the L2): one launch less than a kernel in between.
template <typename T, int ACT, bool ST>
__global__ __launch_bounds__(TB) void gn_apply_k(GnArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float smean[64 * V], srstd[64 * V];
    const Place<V> at(p.s, blockIdx.x);
    each_group(p.s, at, [&](int q, int l, int ll) {
        const int g = at.g0 + q, sa = first_slab<V>(p.s, g), ns = last_slab<V>(p.s, g) - sa + 1;
        Moments a{0.f, 0.f, 0.f};
        each_part(p.s, (const float2*)p.ws, at.image, g, sa, ns, l, ll, [&](int split, int slab, float2 m) {
            const int lo = max(g * p.s.cg, slab * (V << p.s.lw)), hi = min((g + 1) * p.s.cg, (slab + 1) * (V << p.s.lw));
            const long rows = min((split + 1) * p.s.rps, p.s.pixels) - split * p.s.rps;
            merge(a, (float)rows * (float)(hi - lo), m.x, m.y);
        });
        for (int d = 1; d < 1 << ll; d <<= 1) {
            const float n = __shfl_xor(a.n, d), mean = __shfl_xor(a.mean, d), m2 = __shfl_xor(a.m2, d);
            merge(a, n, mean, m2);
        }
        if (l == 0) {
            const float rstd = 1.f / sqrtf(a.m2 / ((float)p.s.pixels * (float)p.s.cg) + p.eps);
            smean[q] = a.mean;
            srstd[q] = rstd;
            if (at.split == 0 && sa == at.slab) {
                if (p.mean) p.mean[at.image * p.s.G + g] = a.mean;
                if (p.rstd) p.rstd[at.image * p.s.G + g] = rstd;
            }
        }
    });
    __syncthreads();
    float mu[V], rs[V], ga[V], be[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = min(at.ch + j, p.s.C - 1), q = c / p.s.cg - at.g0;
        const bool has = j < at.n;
        mu[j] = has ? smean[q] : 0.f;
        rs[j] = has ? srstd[q] : 0.f;
        ga[j] = p.gamma[c];
        be[j] = p.beta[c];
    }
    const T* x = (const T*)p.x + at.ch;
    T* y = (T*)p.y + at.ch;
    auto put = [&](u4 w, long r) {
        float v[V];
        chunk_values<T>(w, v);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = act_value<ACT>(__builtin_fmaf((v[j] - mu[j]) * rs[j], ga[j], be[j]));
        st_chunk<ST>(y + r * p.ldy, at.n, v);
    };
    const long whole = min(at.r1, p.exact);
    long r = at.r0 + at.rl;
    for (; r + (U - 1) * at.RL < whole; r += U * at.RL) {
        u4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = ld_chunk(x + (r + u * at.RL) * p.ldx, at.n, false);
#pragma unroll
        for (int u = 0; u < U; ++u) put(w[u], r + u * at.RL);
    }
    for (; r < at.r1; r += at.RL) put(ld_chunk(x + r * p.ldx, at.n, r >= p.exact), r);
}

// ---- gradient ------------------------------------------------------------------

// A thread's channels: what z and u take of x
template <int V>
struct Channels {
    float mu[V], rs[V], ga[V], be[V];
    __device__ __forceinline__ void load(const GnBwdArgs& p, const Place<V>& at) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = min(at.ch + j, p.s.C - 1);
            const long g = at.image * p.s.G + c / p.s.cg;
            mu[j] = p.mean[g];
            rs[j] = p.rstd[g];
            ga[j] = p.gamma[c];
            be[j] = p.beta[c];
        }
    }
};

// Sums over a split's rows of dz and dz * u: for every channel, into ws behind the
// parts' [image][split][2][cp], and gamma times them for every part.  (32 x 784 x 250 float32: 13.4 us,
// 50 MB at 3.7 TB/s.)
template <typename T, int ACT>
__global__ __launch_bounds__(TB) void gn_bwd_sums_k(GnBwdArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float sm[2][kWaves][64 * V];
    const Place<V> at(p.s, blockIdx.x);
    const T *x = (const T*)p.x + at.ch, *dy = (const T*)p.dy + at.ch;
    Channels<V> k;
    k.load(p, at);
    float a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = b[j] = 0.f;
    auto add = [&](u4 xw, u4 yw) {
        float v[V], g[V];
        chunk_values<T>(xw, v);
        chunk_values<T>(yw, g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float u = (v[j] - k.mu[j]) * k.rs[j];
            const float dz = act_grad<ACT>(g[j], __builtin_fmaf(u, k.ga[j], k.be[j]));
            a[j] += dz;
            b[j] = __builtin_fmaf(dz, u, b[j]);
        }
    };
    const long whole = min(at.r1, p.exact);
    long r = at.r0 + at.rl;
    for (; r + (U - 1) * at.RL < whole; r += U * at.RL) {
        u4 xw[U], yw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            xw[u] = ld_chunk(x + (r + u * at.RL) * p.ldx, at.n, false);
            yw[u] = ld_chunk(dy + (r + u * at.RL) * p.lddy, at.n, false);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) add(xw[u], yw[u]);
    }
    for (; r < at.r1; r += at.RL) add(ld_chunk(x + r * p.ldx, at.n, r >= p.exact), ld_chunk(dy + r * p.lddy, at.n, r >= p.exact));
    const int t = threadIdx.x, wave = t >> 6;
    int first, n;
    fold<V>(a, p.s.lw, first, n);
    fold<V>(b, p.s.lw, first, n);
    {
        const int c = (t & ((1 << p.s.lw) - 1)) * V + first;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < n) {
                sm[0][wave][c + j] = a[j];
                sm[1][wave][c + j] = b[j];
            }
    }
    __syncthreads();
    const long row = at.image * p.s.splits + at.split;
    float* out = p.ws + p.s.sums + row * 2 * p.s.cp;
    for (int c = t; c < at.c1 - at.c0; c += TB) {
        float sa = sm[0][0][c], sb = sm[1][0][c];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            sa += sm[0][w][c];
            sb += sm[1][w][c];
        }
        out[at.c0 + c] = sa;
        out[p.s.cp + at.c0 + c] = sb;
        const float g = p.gamma[at.c0 + c];
        sm[0][0][c] = sa * g;
        sm[1][0][c] = sb * g;
    }
    __syncthreads();
    const int ll = item_lanes(TB, at.np), l = t & ((1 << ll) - 1);
    float2* part = (float2*)p.ws + row * p.s.parts;
    for (int q = t >> ll; q < at.np; q += TB >> ll) {
        const int g = at.g0 + q;
        const int lo = max(g * p.s.cg, at.c0) - at.c0, hi = min((g + 1) * p.s.cg, at.c1) - at.c0;
        float sa = 0.f, sb = 0.f;
        for (int c = lo + l; c < hi; c += 1 << ll) {
            sa += sm[0][0][c];
            sb += sm[1][0][c];
        }
        for (int d = 1; d < 1 << ll; d <<= 1) {
            sa += __shfl_xor(sa, d);
            sb += __shfl_xor(sb, d);
        }
        if (l == 0) part[g + at.slab] = float2{sa, sb};
    }
}

// dgamma and dbeta: kColumns columns of the channels' sums a workgroup, 32 threads to four
// columns, over all images and splits.  No atomics, so that the order is fixed; a launch of its
// own takes 3.9 us for 128 images of 128 channels: latency.
constexpr int kColumns = TB / 32 * 4;
__device__ void gn_columns(const GnBwdArgs& p, int block, float* sm) {
    const int t = threadIdx.x, q = t % (kColumns / 4), l = t / (kColumns / 4), col = block * kColumns + q * 4;
    const float* in = p.ws + p.s.sums + col;
    f4 a = f4{0.f, 0.f, 0.f, 0.f};
    if (col < 2 * p.s.cp) {
#pragma unroll 4
        for (long r = l; r < p.s.rows_ws; r += 32) a += *(const f4*)(in + r * 2 * p.s.cp);
    }
    *(f4*)(sm + l * kColumns + q * 4) = a;
    __syncthreads();
    const int c = block * kColumns + t;
    if (t < kColumns && c < 2 * p.s.cp) {
        float v = sm[t];
#pragma unroll
        for (int k = 1; k < 32; ++k) v += sm[k * kColumns + t];
        if (c < p.s.C) {
            if (p.dbeta) p.dbeta[c] = v;
        } else if (c >= p.s.cp && c < p.s.cp + p.s.C) {
            if (p.dgamma) p.dgamma[c - p.s.cp] = v;
        }
    }
}

__global__ __launch_bounds__(TB) void gn_columns_k(GnBwdArgs p) {
    __shared__ __attribute__((aligned(16))) float sm[1024];
    gn_columns(p, blockIdx.x, sm);
}

// dx; the first `extra` workgroups sum dgamma and dbeta beside it.  Four waves a SIMD in float32: the 784
// workgroups of 32 x 784 x 250 with a residual then run at once (19.2 us, 100 MB at 5.2 TB/s; 21.9 with
// three); bf16's registers would spill.  With gn_bwd_sums_k 32 x 3136 x 256 bf16 takes 61.9 us
// (30 at a large copy's rate if x and dy were read once).
template <typename T, int ACT, bool ST>
__global__ __launch_bounds__(TB, sizeof(T) == 4 ? 4 : 3) void gn_bwd_apply_k(GnBwdArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) float sm[2 * 64 * V > 1024 ? 2 * 64 * V : 1024];
    if ((int)blockIdx.x < p.extra) {
        gn_columns(p, blockIdx.x, sm);
        return;
    }
    const Place<V> at(p.s, blockIdx.x - p.extra);
    float *s1 = sm, *s2 = sm + 64 * V;
    const float size = (float)p.s.pixels * (float)p.s.cg;
    each_group(p.s, at, [&](int q, int l, int ll) {
        const int g = at.g0 + q, sa = first_slab<V>(p.s, g), ns = last_slab<V>(p.s, g) - sa + 1;
        float a = 0.f, b = 0.f;
        each_part(p.s, (const float2*)p.ws, at.image, g, sa, ns, l, ll, [&](int, int, float2 m) {
            a += m.x;
            b += m.y;
        });
        for (int d = 1; d < 1 << ll; d <<= 1) {
            a += __shfl_xor(a, d);
            b += __shfl_xor(b, d);
        }
        if (l == 0) {
            s1[q] = a / size;
            s2[q] = b / size;
        }
    });
    Channels<V> k;
    k.load(p, at);
    __syncthreads();
    float m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int q = min(at.ch + j, p.s.C - 1) / p.s.cg - at.g0;
        m1[j] = j < at.n ? s1[q] : 0.f;
        m2[j] = j < at.n ? s2[q] : 0.f;
    }
    const T *x = (const T*)p.x + at.ch, *dy = (const T*)p.dy + at.ch, *dres = (const T*)p.dres + at.ch;
    T* dx = (T*)p.dx + at.ch;
    auto put = [&](u4 xw, u4 yw, u4 ew, long r) {
        float v[V], g[V], e[V];
        chunk_values<T>(xw, v);
        chunk_values<T>(yw, g);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float u = (v[j] - k.mu[j]) * k.rs[j];
            const float dz = act_grad<ACT>(g[j], __builtin_fmaf(u, k.ga[j], k.be[j]));
            v[j] = k.rs[j] * (dz * k.ga[j] - (m1[j] + u * m2[j]));
        }
        if (p.dres) {
            chunk_values<T>(ew, e);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] += e[j];
        }
        st_chunk<ST>(dx + r * p.lddx, at.n, v);
    };
    const long whole = min(at.r1, p.exact);
    long r = at.r0 + at.rl;
    for (; r + (U - 1) * at.RL < whole; r += U * at.RL) {
        u4 xw[U], yw[U], ew[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            xw[u] = ld_chunk(x + (r + u * at.RL) * p.ldx, at.n, false);
            yw[u] = ld_chunk(dy + (r + u * at.RL) * p.lddy, at.n, false);
            if (p.dres) ew[u] = ld_chunk(dres + (r + u * at.RL) * p.lddres, at.n, false);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) put(xw[u], yw[u], ew[u], r + u * at.RL);
    }
    for (; r < at.r1; r += at.RL) {
        u4 ew = u4{0u, 0u, 0u, 0u};
        if (p.dres) ew = ld_chunk(dres + r * p.lddres, at.n, r >= p.exact);
        put(ld_chunk(x + r * p.ldx, at.n, r >= p.exact), ld_chunk(dy + r * p.lddy, at.n, r >= p.exact), ew, r);
    }
}

// Slabs of at most 64 chunks; as many splits of an image's rows as give about eight
// workgroups a compute unit, with eight rows a thread at least and at most about a
// thousand (whose sums are float32).
GnShape gn_shape(int V, long images, long pixels, int C, int G) {
    GnShape s{};
    s.images = images;
    s.pixels = pixels;
    s.C = C;
    s.G = G;
    s.cg = C / G;
    const int chunks = (C + V - 1) / V;
    while (s.lw < 6 && (1 << s.lw) < chunks) ++s.lw;
    s.slabs = (C + (V << s.lw) - 1) / (V << s.lw);
    const long RL = TB >> s.lw, wgs = std::max(1L, images * s.slabs);
    long splits = std::min((2048 + wgs - 1) / wgs, std::max(1L, pixels / (RL * 8)));
    splits = std::max(splits, (pixels + RL * 1024 - 1) / (RL * 1024));
    s.rps = (pixels + splits - 1) / splits;
    s.splits = (int)((pixels + s.rps - 1) / s.rps);
    s.parts = G + s.slabs - 1;
    s.cp = (C + 3) / 4 * 4;
    s.rows_ws = images * s.splits;
    s.sums = (s.rows_ws * s.parts * 2 + 3) / 4 * 4;
    return s;
}

// workgroups that sum dgamma and dbeta, a multiple of the 8 XCDs
int column_wgs(const GnShape& s) { return ((2 * s.cp + kColumns - 1) / kColumns + 7) / 8 * 8; }

template <typename T, int ACT>
void gn_launch(const GnArgs& p, unsigned wgs, hipStream_t st) {
    launch((gn_stats_k<T>), dim3(wgs), dim3(TB), 0, st, p);
    if (p.s.images * p.s.pixels * p.s.C * (long)sizeof(T) >= kStreamBytes)
        launch((gn_apply_k<T, ACT, true>), dim3(wgs), dim3(TB), 0, st, p);
    else
        launch((gn_apply_k<T, ACT, false>), dim3(wgs), dim3(TB), 0, st, p);
}
template <typename T, int ACT>
void gn_bwd_launch(GnBwdArgs p, unsigned wgs, hipStream_t st) {
    if (wgs) launch((gn_bwd_sums_k<T, ACT>), dim3(wgs), dim3(TB), 0, st, p);
    // (workgroups with the same rows go to the same XCD in both kernels)
    p.extra = p.dgamma || p.dbeta ? column_wgs(p.s) : 0;
    const unsigned grid = p.extra + (p.dx ? wgs : 0);
    if (grid == 0) return;
    if (p.s.images * p.s.pixels * p.s.C * (long)sizeof(T) >= kStreamBytes)
        launch((gn_bwd_apply_k<T, ACT, true>), dim3(grid), dim3(TB), 0, st, p);
    else
        launch((gn_bwd_apply_k<T, ACT, false>), dim3(grid), dim3(TB), 0, st, p);
}

}  // namespace

long groupnorm_threads(long images, long pixels, int C, int G) {
    long most = 0;
    for (int V : {4, 8}) {
        const GnShape s = gn_shape(V, images, pixels, C, G);
        most = std::max(most, images * s.slabs * s.splits + column_wgs(s));
    }
    return most * TB;
}
long groupnorm_ws(long images, long pixels, int C, int G) {
    long most = 0;
    for (int V : {4, 8}) {
        const GnShape s = gn_shape(V, images, pixels, C, G);
        most = std::max(most, s.rows_ws * s.parts * 2);
    }
    return most;
}
long groupnorm_bwd_ws(long images, long pixels, int C, int G) {
    long most = 0;
    for (int V : {4, 8}) {
        const GnShape s = gn_shape(V, images, pixels, C, G);
        most = std::max(most, s.sums + s.rows_ws * 2 * s.cp);
    }
    return most;
}

hipError_t launch_groupnorm(int dt, GnArgs p, long images, long pixels, int C, int G, hipStream_t st) {
    if (images <= 0) return hipSuccess;
    p.exact = exact_row(dt, images * pixels, C, p.ldx);
    const GnWhole whole = groupnorm_whole(dt == DT_BF16 ? 8 : 4, images, pixels, C, G, std::max(p.ldx, p.ldy), false);
    if (whole.threads) {
        if (whole.slots > 2 || C % 8) p.exact = exact_row_any(dt, images * pixels, p.ldx);
        return launch_groupnorm_whole(dt, p, whole, st);
    }
    p.s = gn_shape(dt == DT_BF16 ? 8 : 4, images, pixels, C, G);
    const unsigned wgs = (unsigned)(images * p.s.slabs * p.s.splits);
    if (dt == DT_BF16) {
        if (p.act == ACT_RELU) gn_launch<bf16, ACT_RELU>(p, wgs, st);
        else if (p.act == ACT_SILU) gn_launch<bf16, ACT_SILU>(p, wgs, st);
        else gn_launch<bf16, ACT_NONE>(p, wgs, st);
    } else {
        if (p.act == ACT_RELU) gn_launch<float, ACT_RELU>(p, wgs, st);
        else if (p.act == ACT_SILU) gn_launch<float, ACT_SILU>(p, wgs, st);
        else gn_launch<float, ACT_NONE>(p, wgs, st);
    }
    return hipGetLastError();
}

hipError_t launch_groupnorm_bwd(int dt, GnBwdArgs p, long images, long pixels, int C, int G, hipStream_t st) {
    p.s = gn_shape(dt == DT_BF16 ? 8 : 4, images, pixels, C, G);
    p.exact = exact_row(dt, images * pixels, C, std::min({p.lddy, p.ldx, p.dres ? p.lddres : p.ldx}));
    const GnWhole whole = groupnorm_whole(dt == DT_BF16 ? 8 : 4, images, pixels, C, G,
                                          std::max({p.lddy, p.ldx, p.dres ? p.lddres : 0, p.dx ? p.lddx : 0}), true);
    if (images > 0 && whole.threads) {
        if (whole.slots > 2 || C % 8)
            p.exact = exact_row_any(dt, images * pixels, std::min({p.lddy, p.ldx, p.dres ? p.lddres : p.ldx}));
        p.s.rows_ws = images;
        p.s.sums = 0;
        if (images == 1) p.ws = nullptr;
        hipError_t e = launch_groupnorm_whole_bwd(dt, p, whole, st);
        if (e == hipSuccess && p.ws && (p.dgamma || p.dbeta)) {
            launch(gn_columns_k, dim3((unsigned)((2 * p.s.cp + kColumns - 1) / kColumns)), dim3(TB), 0, st, p);
            e = hipGetLastError();
        }
        return e;
    }
    const unsigned wgs = (unsigned)(images * p.s.slabs * p.s.splits);
    if (dt == DT_BF16) {
        if (p.act == ACT_RELU) gn_bwd_launch<bf16, ACT_RELU>(p, wgs, st);
        else if (p.act == ACT_SILU) gn_bwd_launch<bf16, ACT_SILU>(p, wgs, st);
        else gn_bwd_launch<bf16, ACT_NONE>(p, wgs, st);
    } else {
        if (p.act == ACT_RELU) gn_bwd_launch<float, ACT_RELU>(p, wgs, st);
        else if (p.act == ACT_SILU) gn_bwd_launch<float, ACT_SILU>(p, wgs, st);
        else gn_bwd_launch<float, ACT_NONE>(p, wgs, st);
    }
    return hipGetLastError();
}

}  // namespace lpp
