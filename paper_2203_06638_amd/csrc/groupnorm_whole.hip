// groupnorm_whole.hip -- group norm, and its gradient, of maps that fit the registers of a
// workgroup: it takes whole groups of one image (a slab of channels, all pixels) and reads them
// once.
//
// Formulas: groupnorm.hip.  W = 2^lw lanes take a row's chunks of V channels, the others
// further rows, so that a thread's channels are the same in all of its NC chunks.  A chunk
// has S slots of channels with the same statistics: one (cg a multiple of V), V / cg of them, or
// V (any cg).
#include <algorithm>
#include <type_traits>

#include "act8.h"
#include "groupnorm.h"
#include "kernels.h"
#include "launch.h"

namespace lpp {

namespace {

// Converted values are not to be kept from one pass over the chunks to the next: twice the
// registers.
template <int NC>
__device__ __forceinline__ void keep_packed(u4* w) {
#pragma unroll
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(w[c]));
}

// A workgroup's slab: images outermost, the slabs of an image on neighbouring places of
// one XCD (workgroups go to the 8 XCDs in turn), which share cache lines.
template <int V, int TB>
struct Slab {
    long image, r0;
    int ch, n, g0, np, rl, RL, w;
    __device__ __forceinline__ Slab(const GnWhole& s) {
        const unsigned b = blockIdx.x, at = (b & 7u) * s.per_xcd + (b >> 3);
        const unsigned i = at / (unsigned)s.slabs;
        image = i;
        r0 = image * s.pixels;
        g0 = (int)(at - i * (unsigned)s.slabs) * s.gps;
        np = min(s.gps, s.G - g0);
        RL = TB >> s.lw;
        rl = threadIdx.x >> s.lw;
        w = threadIdx.x & ((1 << s.lw) - 1);
        ch = g0 * s.cg + w * V;
        n = np * s.cg - w * V;   // channels of the thread's chunk (none: an idle lane)
        if (n <= 0) ch = g0 * s.cg;
    }
};

// The row of a thread's chunk c: a uniform address, and the thread's own offset in it, which fits
// 32 bits (kWholeLd).  Threads without a row in the last round take its first.
template <typename T, int V, int TB>
__device__ __forceinline__ T* row_of(T* m, long ld, const Slab<V, TB>& at, long pixels, int c) {
    const int pix = c * at.RL;
    char* base = (char*)(m + (at.r0 + pix) * ld);
    const uint32_t off = (uint32_t)((pix + at.rl < pixels ? at.rl : 0) * (int)ld + at.ch) * (uint32_t)sizeof(T);
    return (T*)(base + off);
}
// A matrix's chunks; exact: the first row of which nothing behind the last value may be read.
template <typename T, int V, int TB, int NC>
__device__ __forceinline__ void load_slab(T* m, long ld, const Slab<V, TB>& at, long pixels, long exact, u4* w) {
    if (at.r0 + pixels <= exact) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (c * at.RL < pixels) w[c] = ld_chunk(row_of(m, ld, at, pixels, c), at.n, false);
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (c * at.RL < pixels)
                w[c] = ld_chunk(row_of(m, ld, at, pixels, c), at.n,
                                at.r0 + c * at.RL + (c * at.RL + at.rl < pixels ? at.rl : 0) >= exact);
    }
}

// The waves' sums of each channel into sm[k][wave][channel] (a barrier is left to the caller).
template <int V, int TB, int N>
__device__ __forceinline__ void wave_sums(float (*v)[V], int lw, int w, float* sm) {
    const int wave = threadIdx.x >> 6, row = V << lw;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        int first, n;
        fold<V>(v[k], lw, first, n);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < n) sm[(k * (TB / 64) + wave) * row + w * V + first + j] = v[k][j];
    }
}
// out[k][group] = sum of in[k][e][channel], e < E (a power of two), over the group's channels
template <int TB, int N, int E>
__device__ __forceinline__ void channel_sums(const float* in, int row, int cg, int np, float* out) {
    const int t = threadIdx.x, ll = item_lanes(TB, np), l = t & ((1 << ll) - 1);
    for (int q = t >> ll; q < np; q += TB >> ll) {
        float a[N];
#pragma unroll
        for (int k = 0; k < N; ++k) a[k] = 0.f;
        for (int i = l; i < cg * E; i += 1 << ll) {
            const int e = i & (E - 1), c = i / E;
#pragma unroll
            for (int k = 0; k < N; ++k) a[k] += in[(k * E + e) * row + q * cg + c];
        }
        for (int d = 1; d < 1 << ll; d <<= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) a[k] += __shfl_xor(a[k], d);
        if (l == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) out[k * row + q] = a[k];
    }
}

// The groups of the thread's V channels, counted within the slab.
template <int V>
__device__ __forceinline__ void slab_groups(int w, int cg, int np, int* q) {
    int left = w * V / cg;
    q[0] = min(left, np - 1);
    left = (left + 1) * cg - w * V;      // channels of that group from the thread's first on
#pragma unroll
    for (int j = 1; j < V; ++j) {
        const bool next = --left == 0;
        q[j] = min(q[j - 1] + next, np - 1);
        left = next ? cg : left;
    }
}

// v[k][slot] becomes the sum over the workgroup of the slot's group.
//   S < V: one barrier; each thread adds up what its groups' waves and chunks (cpg) left.
//   S = V (any cg): by channel first, then by group, two barriers.
// sm: floats that no earlier sum still uses, whole_lds of them.
template <int V, int TB, int S, int N>
__device__ __forceinline__ void group_sums(float (*v)[S], const GnWhole& s, int w, int np, const int* q, float* sm) {
    const int row = S << s.lw;
    if constexpr (S < V) {
        const int wave = threadIdx.x >> 6, cpg = S == 1 ? s.cg / V : 1;
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int j = 0; j < S; ++j) {
                for (int d = 1 << s.lw; d < 64; d <<= 1) v[k][j] += __shfl_xor(v[k][j], d);
                sm[(k * (TB / 64) + wave) * row + w * S + j] = v[k][j];
            }
        __syncthreads();
        const int first = w / cpg * cpg;      // the group's chunks
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int j = 0; j < S; ++j) {
                float a = 0.f;
                for (int c = first; c < first + cpg; ++c)
#pragma unroll
                    for (int i = 0; i < TB / 64; ++i) a += sm[(k * (TB / 64) + i) * row + c * S + j];
                v[k][j] = a;
            }
    } else {
        wave_sums<V, TB, N>(v, s.lw, w, sm);
        __syncthreads();
        float* out = sm + N * (TB / 64) * row;
        channel_sums<TB, N, TB / 64>(sm, row, s.cg, np, out);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int j = 0; j < S; ++j) v[k][j] = out[k * row + q[j]];
    }
}
// floats of N sums
constexpr int whole_lds(int TB, int slots, int lw, int N) { return N * (TB / 64 + 1) * (slots << lw); }

// The mean comes from the values' sum, then once more from that of the deviations, whose
// squares give the variance: rounding of large means stays out of both.
// x is read once and y written once, so the bytes set the floor.  A workgroup loads, sums and writes in
// turn, all of them in step where they run in one round, and is about 70% of that time issuing
// vector instructions: conversions, masks, and in every thread the divisions and the root of its
// slots' statistics.  32 x 3136 x 256 bf16 24.7 us (4.2 TB/s; with inputs that no cache holds 33.3), 75 x
// 729 x 90 of 96 float32, SiLU, 225 workgroups, 8 chunks a thread of which 5.7 are used, 18.3 (2.1 TB/s),
// one 64 x 64 map 4.4 (latency of its barriers).
// 128 registers: four waves a SIMD, so that one workgroup of 1024 threads, or several small ones,
// fill a compute unit.  Runs of 32 bytes of a row a workgroup instead of 64: 53 us.
template <typename T, int TB, int NC, int S, bool ST>
__global__ __launch_bounds__(TB, 4) void gn_whole_k(GnArgs p, GnWhole s) {
    constexpr int V = 16 / (int)sizeof(T), Q = V / S;      // channels of a slot
    extern __shared__ float lds[];
    if ((blockIdx.x & 7u) * s.per_xcd + (blockIdx.x >> 3) >= s.wgs) return;
    const Slab<V, TB> at(s);
    u4 w[NC] = {};
    load_slab<const T, V, TB, NC>((const T*)p.x, p.ldx, at, s.pixels, p.exact, w);
    float ga[V], be[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = min(at.ch + j, s.G * s.cg - 1);
        ga[j] = p.gamma[c];
        be[j] = p.beta[c];
    }
    int q[V];
    if (S == V) slab_groups<V>(at.w, s.cg, at.np, q);
    const float size = (float)s.pixels * (float)s.cg, scale = sum_scale(size), scaled = size * scale;
    float v[2][S];
#pragma unroll
    for (int j = 0; j < S; ++j) v[0][j] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        __builtin_amdgcn_sched_barrier(0);     // (one chunk at a time: registers)
        float f[V];
        chunk_values<T>(w[c], f);
        if (c * at.RL + at.rl < s.pixels)
#pragma unroll
            for (int j = 0; j < V; ++j) v[0][j / Q] = __builtin_fmaf(f[j], scale, v[0][j / Q]);
    }
    if (S == V)
#pragma unroll
        for (int j = 0; j < S; ++j) v[0][j] = j < at.n ? v[0][j] : 0.f;
    group_sums<V, TB, S, 1>(v, s, at.w, at.np, q, lds);
    keep_packed<NC>(w);
    float mu[S];
#pragma unroll
    for (int j = 0; j < S; ++j) {
        mu[j] = v[0][j] / scaled;
        v[0][j] = v[1][j] = 0.f;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        __builtin_amdgcn_sched_barrier(0);     // (one chunk at a time: registers)
        float f[V];
        chunk_values<T>(w[c], f);
        if (c * at.RL + at.rl < s.pixels)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = f[j] - mu[j / Q];
                v[0][j / Q] = __builtin_fmaf(d, scale, v[0][j / Q]);
                v[1][j / Q] = __builtin_fmaf(d, d, v[1][j / Q]);
            }
    }
    if (S == V)
#pragma unroll
        for (int j = 0; j < S; ++j) v[0][j] = j < at.n ? v[0][j] : 0.f, v[1][j] = j < at.n ? v[1][j] : 0.f;
    group_sums<V, TB, S, 2>(v, s, at.w, at.np, q, lds + whole_lds(TB, S, s.lw, 1));
    keep_packed<NC>(w);
    float rs[S];
#pragma unroll
    for (int j = 0; j < S; ++j) {
        const float e = v[0][j] / scaled;
        const float var = v[1][j] == INFINITY ? v[1][j] : v[1][j] / size - e * e;
        rs[j] = 1.f / sqrtf((var < 0.f ? 0.f : var) + p.eps);
        mu[j] += e;
        // (the thread with the group's first channel; a slab's last chunk may end before its slots do)
        const int c = at.w * V + j * Q, own = S == V ? q[j] : c / s.cg;
        if (at.n > j * Q && at.rl == 0 && c == own * s.cg) {
            const long g = at.image * s.G + at.g0 + own;
            if (p.mean) p.mean[g] = mu[j];
            if (p.rstd) p.rstd[g] = rs[j];
        }
    }
    auto put = [&](auto act) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (c * at.RL >= s.pixels) break;
            __builtin_amdgcn_sched_barrier(0);
            float f[V];
            chunk_values<T>(w[c], f);
#pragma unroll
            for (int j = 0; j < V; ++j)
                f[j] = act_value<decltype(act)::value>(__builtin_fmaf((f[j] - mu[j / Q]) * rs[j / Q], ga[j], be[j]));
            st_chunk<ST>(row_of((T*)p.y, p.ldy, at, s.pixels, c), c * at.RL + at.rl < s.pixels ? at.n : 0, f);
        }
    };
    if (p.act == ACT_RELU) put(std::integral_constant<int, ACT_RELU>());
    else if (p.act == ACT_SILU) put(std::integral_constant<int, ACT_SILU>());
    else put(std::integral_constant<int, ACT_NONE>());
}

// The gradient: the channels' sums of dz and dz * u over the image go to ws [image][2][cp], or,
// of a single image, to dbeta and dgamma themselves.  x and dy stay in registers, which halves the
// maps that fit: 128 x 1024 x 128 bf16 in 32 groups 22.4 us (4.5 TB/s, vector units 73% busy; the two
// kernels of groupnorm.hip 40), 8 x 64 x 64 float32 5.0 (latency).
template <typename T, int TB, int NC, int S, bool ST>
__global__ __launch_bounds__(TB, 4) void gn_whole_bwd_k(GnBwdArgs p, GnWhole s) {
    constexpr int V = 16 / (int)sizeof(T), Q = V / S;
    extern __shared__ float lds[];
    if ((blockIdx.x & 7u) * s.per_xcd + (blockIdx.x >> 3) >= s.wgs) return;
    const Slab<V, TB> at(s);
    u4 xw[NC] = {}, yw[NC] = {};
    load_slab<const T, V, TB, NC>((const T*)p.x, p.ldx, at, s.pixels, p.exact, xw);
    load_slab<const T, V, TB, NC>((const T*)p.dy, p.lddy, at, s.pixels, p.exact, yw);
    int q[V];
    if (S == V) slab_groups<V>(at.w, s.cg, at.np, q);
    float mu[S], rs[S], ga[V], be[V], v[2][V];
#pragma unroll
    for (int j = 0; j < S; ++j) {
        const int own = S == V ? q[j] : min((at.w * V + j * Q) / s.cg, at.np - 1);
        mu[j] = p.mean[at.image * s.G + at.g0 + own];
        rs[j] = p.rstd[at.image * s.G + at.g0 + own];
        if (S < V) q[j] = own;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = min(at.ch + j, s.G * s.cg - 1);
        ga[j] = p.gamma[c];
        be[j] = p.beta[c];
        v[0][j] = v[1][j] = 0.f;
    }
    auto sums = [&](auto act) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            __builtin_amdgcn_sched_barrier(0);
            float f[V], g[V];
            chunk_values<T>(xw[c], f);
            chunk_values<T>(yw[c], g);
            if (c * at.RL + at.rl < s.pixels)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float u = (f[j] - mu[j / Q]) * rs[j / Q];
                    const float dz = act_grad<decltype(act)::value>(g[j], __builtin_fmaf(u, ga[j], be[j]));
                    v[0][j] += dz;
                    v[1][j] = __builtin_fmaf(dz, u, v[1][j]);
                }
        }
    };
    if (p.act == ACT_RELU) sums(std::integral_constant<int, ACT_RELU>());
    else if (p.act == ACT_SILU) sums(std::integral_constant<int, ACT_SILU>());
    else sums(std::integral_constant<int, ACT_NONE>());
    const int row = V << s.lw, t = threadIdx.x;
    float *sm = lds, *ch = lds + 2 * (TB / 64) * row, *out = ch + 2 * row;
    wave_sums<V, TB, 2>(v, s.lw, at.w, sm);
    __syncthreads();
    const int width = at.np * s.cg, c0 = at.g0 * s.cg;
    for (int i = t; i < 2 * row; i += TB) {
        const int k = i >= row, c = i - k * row;
        if (c >= width) continue;
        float a = 0.f;
#pragma unroll
        for (int e = 0; e < TB / 64; ++e) a += sm[(k * (TB / 64) + e) * row + c];
        if (p.ws) p.ws[(at.image * 2 + k) * p.s.cp + c0 + c] = a;
        else if (k ? p.dgamma : p.dbeta) (k ? p.dgamma : p.dbeta)[c0 + c] = a;
        ch[i] = a * p.gamma[c0 + c];
    }
    if (!p.dx) return;
    __syncthreads();
    channel_sums<TB, 2, 1>(ch, row, s.cg, at.np, out);
    __syncthreads();
    keep_packed<NC>(xw);
    keep_packed<NC>(yw);
    const float size = (float)s.pixels * (float)s.cg;
    float m1[S], m2[S];
#pragma unroll
    for (int j = 0; j < S; ++j) {
        m1[j] = out[q[j]] / size;
        m2[j] = out[row + q[j]] / size;
    }
    auto put = [&](auto act) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (c * at.RL >= s.pixels) break;
            __builtin_amdgcn_sched_barrier(0);
            float f[V], g[V];
            chunk_values<T>(xw[c], f);
            chunk_values<T>(yw[c], g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float u = (f[j] - mu[j / Q]) * rs[j / Q];
                const float dz = act_grad<decltype(act)::value>(g[j], __builtin_fmaf(u, ga[j], be[j]));
                f[j] = rs[j / Q] * (dz * ga[j] - (m1[j / Q] + u * m2[j / Q]));
            }
            if (p.dres) {
                float e[V];
                const long r = at.r0 + c * at.RL + at.rl;
                chunk_values<T>(ld_chunk(row_of((const T*)p.dres, p.lddres, at, s.pixels, c), at.n, r >= p.exact), e);
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] += e[j];
            }
            st_chunk<ST>(row_of((T*)p.dx, p.lddx, at, s.pixels, c), c * at.RL + at.rl < s.pixels ? at.n : 0, f);
        }
    };
    if (p.act == ACT_RELU) put(std::integral_constant<int, ACT_RELU>());
    else if (p.act == ACT_SILU) put(std::integral_constant<int, ACT_SILU>());
    else put(std::integral_constant<int, ACT_NONE>());
}

template <typename T, int TB, int NC, int S>
void whole_launch(const GnArgs& p, const GnWhole& s, hipStream_t st) {
    const unsigned lds = sizeof(float) * (whole_lds(TB, S, s.lw, 1) + whole_lds(TB, S, s.lw, 2));
    const dim3 grid(8 * s.per_xcd);
    // 8 chunks are streamed: 60 x 480 x 512 float32 32.6 us, 29.8 streamed, 128 x 500 x 512 60.3 and 59.4,
    // as bf16 38.0 and 38.2.  13 are not: 128 x 3136 x 256 bf16 114 us, 123 streamed, one buffer of 32
    // images again and again 23.8 and 27.6 (but with inputs that no cache holds 33.4 and 31.5, 64 x 784 x 512
    // float32 48.8 and 47.0).
    if (NC == 8 && s.images * s.pixels * (long)s.G * s.cg * (long)sizeof(T) >= kStreamBytes)
        launch((gn_whole_k<T, TB, NC, S, NC == 8>), grid, dim3(TB), lds, st, p, s);
    else
        launch((gn_whole_k<T, TB, NC, S, false>), grid, dim3(TB), lds, st, p, s);
}
template <typename T, int TB, int NC, int S>
void whole_launch(const GnBwdArgs& p, const GnWhole& s, hipStream_t st) {
    const unsigned lds = sizeof(float) * ((16 / sizeof(T)) << s.lw) * (2 * (TB / 64) + 4);
    const dim3 grid(8 * s.per_xcd);
    if (NC >= 4 && s.images * s.pixels * (long)s.G * s.cg * (long)sizeof(T) >= kStreamBytes)
        launch((gn_whole_bwd_k<T, TB, NC, S, NC >= 4>), grid, dim3(TB), lds, st, p, s);
    else
        launch((gn_whole_bwd_k<T, TB, NC, S, false>), grid, dim3(TB), lds, st, p, s);
}
// (bf16 channels with statistics of their own, gradient: the registers of 8 chunks would spill)
template <typename T, int S>
constexpr int kBwdChunks = S == 8 && sizeof(T) == 2 ? 4 : 8;
template <typename T, int S>
hipError_t whole_dispatch(const GnArgs& p, const GnWhole& s, hipStream_t st) {
    switch (s.threads * 32 + s.nc) {
    case 256 * 32 + 1: whole_launch<T, 256, 1, S>(p, s, st); break;
    case 256 * 32 + 2: whole_launch<T, 256, 2, S>(p, s, st); break;
    case 256 * 32 + 4: whole_launch<T, 256, 4, S>(p, s, st); break;
    case 256 * 32 + 8: whole_launch<T, 256, 8, S>(p, s, st); break;
    case 256 * 32 + 13: whole_launch<T, 256, 13, S>(p, s, st); break;
    case 512 * 32 + 4: whole_launch<T, 512, 4, S>(p, s, st); break;
    case 512 * 32 + 8: whole_launch<T, 512, 8, S>(p, s, st); break;
    case 512 * 32 + 13: whole_launch<T, 512, 13, S>(p, s, st); break;
    case 1024 * 32 + 2: whole_launch<T, 1024, 2, S>(p, s, st); break;
    case 1024 * 32 + 4: whole_launch<T, 1024, 4, S>(p, s, st); break;
    case 1024 * 32 + 8: whole_launch<T, 1024, 8, S>(p, s, st); break;
    case 1024 * 32 + 13: whole_launch<T, 1024, 13, S>(p, s, st); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
template <typename T, int S>
hipError_t whole_dispatch(const GnBwdArgs& p, const GnWhole& s, hipStream_t st) {
    switch (s.threads * 32 + s.nc) {
    case 256 * 32 + 1: whole_launch<T, 256, 1, S>(p, s, st); break;
    case 256 * 32 + 2: whole_launch<T, 256, 2, S>(p, s, st); break;
    case 256 * 32 + 4: whole_launch<T, 256, 4, S>(p, s, st); break;
    case 256 * 32 + 8:
        if constexpr (kBwdChunks<T, S> >= 8) whole_launch<T, 256, 8, S>(p, s, st);
        else return hipErrorInvalidValue;   // (groupnorm_whole leaves these to the other kernels)
        break;
    case 512 * 32 + 4: whole_launch<T, 512, 4, S>(p, s, st); break;
    case 512 * 32 + 8:
        if constexpr (kBwdChunks<T, S> >= 8) whole_launch<T, 512, 8, S>(p, s, st);
        else return hipErrorInvalidValue;   // (groupnorm_whole leaves these to the other kernels)
        break;
    case 1024 * 32 + 2: whole_launch<T, 1024, 2, S>(p, s, st); break;
    case 1024 * 32 + 4: whole_launch<T, 1024, 4, S>(p, s, st); break;
    case 1024 * 32 + 8:
        if constexpr (kBwdChunks<T, S> >= 8) whole_launch<T, 1024, 8, S>(p, s, st);
        else return hipErrorInvalidValue;   // (groupnorm_whole leaves these to the other kernels)
        break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
template <typename T, typename P>
hipError_t whole_slots(const P& p, const GnWhole& s, hipStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    return s.slots == 1   ? whole_dispatch<T, 1>(p, s, st)
           : s.slots == 2 ? whole_dispatch<T, 2>(p, s, st)
                          : whole_dispatch<T, V>(p, s, st);
}

}  // namespace

struct WholeSize {
    int threads, nc;
};
constexpr WholeSize kWholeFwd[] = {{256, 1}, {256, 2}, {256, 4}, {256, 8}, {256, 13}, {512, 4}, {512, 8}, {512, 13}, {1024, 2}, {1024, 4}, {1024, 8}, {1024, 13}};
constexpr WholeSize kWholeBwd[] = {{256, 1}, {256, 2}, {256, 4}, {256, 8}, {512, 4}, {512, 8}, {1024, 2}, {1024, 4}, {1024, 8}};
// the first size from `threads` on that holds `pixels` rows of 2^lw chunks
static const WholeSize* whole_size(bool bwd, long pixels, int lw, int threads) {
    auto find = [&](const WholeSize* z, int n) -> const WholeSize* {
        for (int i = 0; i < n; ++i)
            if (z[i].threads >= threads && pixels <= (long)(z[i].threads >> lw) * z[i].nc) return z + i;
        return nullptr;
    };
    return bwd ? find(kWholeBwd, sizeof kWholeBwd / sizeof *kWholeBwd) : find(kWholeFwd, sizeof kWholeFwd / sizeof *kWholeFwd);
}

// Slabs of as few groups as give 64-byte runs of a row (or all its channels), or of more
// if that leaves fewer lanes idle, in the smallest workgroup whose registers hold them; in a larger one
// where the chip would not be full.
GnWhole groupnorm_whole(int V, long images, long pixels, int C, int G, long ld, bool bwd) {
    GnWhole s{};
    if (ld > kWholeLd) return s;
    s.images = images;
    s.pixels = pixels;
    s.G = G;
    s.cg = C / G;
    s.slots = s.cg % V == 0 ? 1 : s.cg * 2 == V ? 2 : V;
    const int least = std::min(G, (4 * V + s.cg - 1) / s.cg);
    double best = 0;
    const WholeSize* size = nullptr;
    for (int gps = least; gps <= std::min(G, 3 * least); ++gps) {
        const int chunks = (gps * s.cg + V - 1) / V;
        int lw = 0;
        while ((1 << lw) < chunks) ++lw;
        if (lw > 6) break;
        const double used = (double)gps * s.cg / (V << lw);
        const WholeSize* z = used > best * 1.1 ? whole_size(bwd, pixels, lw, 256) : nullptr;
        if (!z) continue;
        best = used;
        s.gps = gps;
        s.lw = lw;
        size = z;
    }
    if (!size) return s;
    // small maps: not more workgroups than keep the chip busy
    while (images * ((G + s.gps - 1) / s.gps) > 1024 && s.gps < G && s.lw < 6) {
        const int gps = std::min(G, 2 * s.gps), chunks = (gps * s.cg + V - 1) / V;
        int lw = s.lw;
        while ((1 << lw) < chunks) ++lw;
        const WholeSize* z = lw > 6 ? nullptr : whole_size(bwd, pixels, lw, 256);
        if (!z || z->threads > 512) break;
        s.gps = gps;
        s.lw = lw;
        size = z;
    }
    s.slabs = (G + s.gps - 1) / s.gps;
    const long wgs = images * s.slabs;
    if (wgs >= (1L << 30)) return s;
    s.wgs = (unsigned)wgs;
    s.per_xcd = (s.wgs + 7) / 8;
    while (size->threads < 1024 && wgs * size->threads < 256 * 1024 && pixels > size->threads >> s.lw)
        size = whole_size(bwd, pixels, s.lw, 2 * size->threads);
    // Two kernels that spread an image over the chip do better where a few workgroups have much
    // to compute each (3136 x 256 bf16, 4 images: 16.0 us against 14.5, 16 images: 20.1 against
    // 26.8), and where the last of few rounds is nearly empty (784 x 250 float32 in groups of 25,
    // 32 images, gradient, 320 workgroups: 41 us against 35).
    const long slots = 256 * (1024 / size->threads), rounds = (wgs + slots - 1) / slots;
    if (size->nc > 8 && wgs < 96) return s;
    if (bwd && s.slots == 8 && size->nc > kBwdChunks<bf16, 8>) return s;
    if (size->nc >= 8 && wgs > slots && wgs < 0.7 * rounds * slots) return s;
    if (8L * s.per_xcd * size->threads > kLaunchThreads) return s;
    s.threads = size->threads;
    s.nc = size->nc;
    return s;
}

hipError_t launch_groupnorm_whole(int dt, const GnArgs& p, const GnWhole& s, hipStream_t st) {
    return dt == DT_BF16 ? whole_slots<bf16>(p, s, st) : whole_slots<float>(p, s, st);
}
hipError_t launch_groupnorm_whole_bwd(int dt, const GnBwdArgs& p, const GnWhole& s, hipStream_t st) {
    return dt == DT_BF16 ? whole_slots<bf16>(p, s, st) : whole_slots<float>(p, s, st);
}

}  // namespace lpp
