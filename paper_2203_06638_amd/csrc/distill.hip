// distill.hip -- what is kept of a teacher's answers, and a student's loss against it.
//
// Top logits of a row z[C]: its k largest values in descending order with their
// classes (equal values: the lowest class first; a NaN is above everything), and
//   rest = log of the sum of exp(z / T) over the other classes.
//
// Distillation.  The teacher's probabilities are p = softmax over {v_i / T} of its list
// and, where it is given, rest, which stands for all classes that are not listed.  The
// student's are q = softmax(z / T) at the listed classes and the sum of the others',
//   soft = sum p log(p / q),  hard = -log softmax(z)[label],
//   loss = weight * ((1 - alpha) * hard + alpha * T^2 * soft),
//   d soft / dz_j = (q_j - p_j) / T,   p_j = q_j p_rest / q_rest for a class that is not listed.
//
// Sums are float32 in a fixed order.  exp(x) is taken as 2^(x log2 e) of x <= 0, whose
// relative error grows with |x| while its share of a sum falls as e^x.
#include <algorithm>
#include <type_traits>

#include "act8.h"
#include "kernels.h"
#include "launch.h"
#include "rowred.h"

namespace lpp {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// A thread's chunks of a row: NC of them, chunk c at value (c * TPR + t) * V of the piece
// [c0, c1) of classes.  Values behind the end are -inf.
template <typename T, int TPR, int NC>
struct RowValues {
    static constexpr int V = 16 / (int)sizeof(T);
    u4 w[NC];
    __device__ __forceinline__ void load(const T* row, int c0, int c1, int t, bool exact) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = c0 + (c * TPR + t) * V, n = c1 - ch;
            w[c] = ld_chunk(row + (n > 0 ? ch : c0), n, exact);
        }
    }
    __device__ __forceinline__ void get(int c, int c0, int c1, int t, float* v) const {
        const int n = c1 - (c0 + (c * TPR + t) * V);
        chunk_values<T>(w[c], v);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = j < n ? v[j] : -INFINITY;
    }
};

// ---- distillation ------------------------------------------------------------

// LDS of a row: the list (classes, teacher's values and then probabilities, student's
// logits; the label behind it), and a bit for each class of the piece that is listed
__host__ __device__ inline int distill_lds(int k, int values) { return 3 * (k + 1) + (values + 31) / 32; }

constexpr int kListPitch = kDistillMaxK + 4;   // floats of a row's list in the workspace

enum DistillMode { WHOLE, PIECE_SUMS, PIECE_GRAD };

// WHOLE: a row to TPR threads, in their registers, so that z is read once.  PIECE_SUMS: a
// workgroup takes a piece of a row and leaves its largest value and its three sums;
// PIECE_GRAD: the loss, and the gradient of its piece, from all pieces' sums.
template <typename T, int TPR, int NC, int MODE, bool ST>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void distill_k(DistillArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int TB = TPR > 256 ? TPR : 256, RB = TB / TPR;
    __shared__ float slots[2 * (TB / 64)];
    extern __shared__ float lds[];
    int turn = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    long r = MODE == WHOLE ? (long)blockIdx.x * RB + rl : blockIdx.x / p.grid_pieces;
    const bool ok = r < p.rows;
    if (!ok) r = p.rows - 1;
    const int piece = MODE == WHOLE ? 0 : (int)(blockIdx.x - r * p.grid_pieces);
    const int c0 = piece * p.piece, c1 = min(p.C, c0 + p.piece);
    const StepArgs* step = p.step;
    const int k = step ? step->k : p.k;
    const float alpha = step ? step->alpha : p.alpha, temp = step ? step->temperature : p.temp;
    const float* values = step ? step->values : p.values;
    const int* index = step ? step->index : p.index;
    const float* rests = step ? step->rest : p.rest;
    const int* labels = step ? step->labels : p.labels;
    const float w = p.weight ? p.weight[r] : 1.f;
    const bool use1 = labels && alpha < 1.f, useT = alpha > 0.f, tail = rests && useT;
    const float iT = 1.f / temp, e1 = kLog2e, eT = kLog2e * iT;
    const T* z = (const T*)p.z + r * p.ldz;

    RowValues<T, TPR, NC> x;
    x.load(z, c0, c1, t, r >= p.exact);

    // the list; entry k is the label
    float* at = lds + rl * distill_lds(p.lds_k, TPR * NC * V);
    int* cls = (int*)at;
    float *pr = at + (k + 1), *zc = at + 2 * (k + 1);
    uint32_t* mask = (uint32_t*)(at + 3 * (k + 1));
    for (int e = t; e <= k; e += TPR) {
        int c = e < k ? (useT ? index[r * k + e] : -1) : (use1 ? labels[r] : -1);
        if ((unsigned)c >= (unsigned)p.C) c = -1;
        cls[e] = c;
        pr[e] = e < k && c >= 0 ? values[r * k + e] * iT : -INFINITY;
        // (dz may be z: the pieces' workgroups keep z at the listed classes for each other)
        float* kept = p.ws + 4 * p.rows * p.pieces + r * kListPitch;
        if (MODE == PIECE_GRAD) zc[e] = c >= 0 ? kept[e] : 0.f;
        else zc[e] = c >= 0 ? ld1(z, c) : 0.f;
        if (MODE == PIECE_SUMS && c >= c0 && c < c1) kept[e] = zc[e];
    }
    if (MODE != PIECE_GRAD && tail) {
        for (int e = t; e < (TPR * NC * V + 31) / 32; e += TPR) mask[e] = 0u;
        row_sync<TPR>();
        for (int e = t; e < k; e += TPR) {
            const int c = cls[e] - c0;
            if (cls[e] >= 0 && c >= 0 && c < c1 - c0) atomicOr(&mask[c >> 5], 1u << (c & 31));
        }
    }
    row_sync<TPR>();

    // largest value, and the sums of exp(z - m), exp((z - m) / T) and the latter's over
    // the classes that are not listed
    float m, s1 = 0.f, sT = 0.f, so = 0.f;
    if (MODE == PIECE_GRAD) {
        const f4* all = (const f4*)p.ws + r * p.pieces;
        m = -INFINITY;
        for (int e = t; e < p.pieces; e += TPR) m = fmaxf(m, all[e][0]);
        m = row_max<TPR>(m, slots, turn);
        for (int e = t; e < p.pieces; e += TPR) {
            const f4 s = all[e];
            s1 += s[1] * pow2((s[0] - m) * e1);
            sT += s[2] * pow2((s[0] - m) * eT);
            so += s[3] * pow2((s[0] - m) * eT);
        }
    } else {
        m = -INFINITY;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float v[V];
            x.get(c, c0, c1, t, v);
#pragma unroll
            for (int j = 0; j < V; ++j) m = fmaxf(m, v[j]);
        }
        m = row_max<TPR>(m, slots, turn);
        // (a piece of nothing but -inf: sums of 0)
        const float base = MODE == PIECE_SUMS && m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float v[V];
            x.get(c, c0, c1, t, v);
            const int i = (c * TPR + t) * V;
            const uint32_t listed = tail ? mask[i >> 5] >> (i & 31) : 0u;
            const int n = c1 - c0 - i;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = v[j] - base;
                if (use1) s1 += j < n ? pow2(d * e1) : 0.f;
                const float e = j < n ? pow2(d * eT) : 0.f;
                sT += e;
                so += (listed >> j) & 1u ? 0.f : e;
            }
        }
    }
    s1 = row_sum<TPR>(s1, slots, turn);
    sT = row_sum<TPR>(sT, slots, turn);
    so = row_sum<TPR>(so, slots, turn);
    if (MODE == PIECE_SUMS) {
        if (t == 0) ((f4*)p.ws)[r * p.pieces + piece] = f4{m, s1, sT, so};
        return;
    }

    // the teacher's probabilities
    const float rest = tail ? rests[r] : -INFINITY;
    float tm = rest;
    for (int e = t; e < k; e += TPR) tm = fmaxf(tm, pr[e]);
    tm = row_max<TPR>(tm, slots, turn);
    float ts = 0.f;
    bool bad = rest != rest;      // (row_max drops a NaN)
    for (int e = t; e < k; e += TPR) {
        bad |= pr[e] != pr[e];
        ts += cls[e] >= 0 && tm > -INFINITY ? pow2((pr[e] - tm) * kLog2e) : 0.f;
    }
    ts = row_sum<TPR>(bad ? NAN : ts, slots, turn) + (rest > -INFINITY ? pow2((rest - tm) * kLog2e) : 0.f);
    // (a list without an entry, or of -inf alone, says nothing)
    const bool some = useT && !(tm == -INFINITY && ts == ts);
    const float lt = logf(ts), lq = logf(sT);
    for (int e = t; e < k; e += TPR) {
        const float d = pr[e] - tm;
        // (log p where the row sums need it: pr holds p from here on, zc of an entry stays)
        pr[e] = cls[e] >= 0 && some ? pow2(d * kLog2e) / ts : 0.f;
    }
    row_sync<TPR>();

    float soft = 0.f, sp = 0.f, sq = 0.f;
    for (int e = t; e < k; e += TPR) {
        const int c = cls[e];
        if (c < 0 || !some) continue;
        bool first = true;
        for (int o = 0; o < e; ++o) first &= cls[o] != c;
        const float pe = pr[e], u = (zc[e] - m) * iT - lq, q = pow2(u * kLog2e);
        const float d = (values[r * k + e] * iT - tm) - lt - u;
        sp += pe;
        if (first) sq += q;
        if (tail) {
            // both sides' probabilities add up to 1: p log(p / q) - p + q in place of
            // p log(p / q) keeps the sum exact where p is near q
            if (pe > 0.f) soft += !first ? pe * d - pe : d > -1.f ? pe * (d + expm1f(-d)) : pe * d - pe + q;
            else if (pe != pe) soft = pe;
            else if (first) soft += q;
        } else if (pe != 0.f) {
            soft += pe * d;
        }
    }
    soft = row_sum<TPR>(soft, slots, turn);
    float others = 1.f / sT;      // what gT times exp((z - m) / T) of a class that is not listed has
    if (tail) {
        sp = row_sum<TPR>(sp, slots, turn);
        sq = row_sum<TPR>(sq, slots, turn);
        const float q = so / sT, pe = some ? (rest > -INFINITY ? pow2((rest - tm) * kLog2e) / ts : 0.f) : 0.f;
        if (some) {
            const float d = (rest - tm) - lt - logf(q);
            if (pe > 0.f) soft += d > -1.f ? pe * (d + expm1f(-d)) : pe * d - pe + q;
            else soft += q;
        }
        // q - p of the rest is p - q of the list, which is the smaller and so the more
        // exact of the two where the rest is large
        others = so != 0.f ? (pe > 0.5f ? sp - sq : q - pe) / so : 0.f;
    }
    const int y = cls[k];
    const float a1 = use1 ? 1.f - alpha : 0.f, aT = some ? alpha * temp : 0.f;
    if (t == 0 && ok && piece == 0) {
        float l = 0.f;
        if (y >= 0 && use1) l += a1 * (logf(s1) - (zc[k] - m));
        if (some) l += aT * temp * soft;
        p.loss[r] = w != 0.f ? w * l : 0.f;
    }
    if (!p.dz) return;
    const float g1 = y >= 0 && use1 ? p.scale * w * a1 : 0.f, gT = p.scale * w * aT;
    const bool live = w != 0.f && (g1 != 0.f || gT != 0.f);   // (a row without a loss has no gradient, whatever it holds)
    const float k1 = g1 != 0.f ? g1 / s1 : 0.f, kT = gT != 0.f ? gT * others : 0.f;
    T* dz = (T*)p.dz + r * p.lddz;
    // (dz may be z: what the list needs of z was read above, before a barrier)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float v[V];
        x.get(c, c0, c1, t, v);
        const int ch = c0 + (c * TPR + t) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = v[j] - m;
            float g = 0.f;
            if (use1) g = k1 * pow2(d * e1);
            if (useT) g = __builtin_fmaf(kT, pow2(d * eT), g);
            v[j] = live ? g : 0.f;
        }
        if (ok) st_chunk<ST>(dz + ch, c1 - ch, v);
    }
    row_sync<TPR>();
    for (int e = t; e <= k; e += TPR) {
        const int c = cls[e];
        if (c < c0 || c >= c1 || !ok || !live) continue;
        float pe = 0.f;
        bool listed = false;
        for (int o = 0; o < k; ++o)
            if (cls[o] == c) {
                pe += pr[o];
                listed = true;
            }
        const float d = zc[e] - m, q = pow2(d * eT);
        float g = g1 != 0.f ? g1 * (pow2(d * e1) / s1 - (c == y ? 1.f : 0.f)) : 0.f;
        if (gT != 0.f) g += listed || !tail ? gT * (q / sT - pe) : kT * q;
        st1(dz, c, g);
    }
}

// ---- top logits --------------------------------------------------------------

typedef unsigned long long u64;

// A value and its class as one number: larger for larger values (NaN above all, -0 as 0),
// and for the lower class of equal ones.  0 is no element's.
__device__ __forceinline__ u64 rank_key(float v, int c) {
    const uint32_t b = __float_as_uint(v + 0.f);
    const uint32_t k = v != v ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
    return (u64)k << 32 | (uint32_t)~c;
}
__device__ __forceinline__ float key_value(u64 key) {
    const uint32_t k = (uint32_t)(key >> 32);
    return k == 0xffffffffu ? NAN : __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ u64 shfl_xor64(u64 v, int d) {
    return (u64)(uint32_t)__shfl_xor((int)(v >> 32), d) << 32 | (uint32_t)__shfl_xor((int)v, d);
}
// the largest over the TPR threads of a row (TPR > 64: two barriers)
template <int TPR>
__device__ __forceinline__ u64 row_max64(u64 v, u64* slots) {
    for (int d = 1; d < 64 && d < TPR; d *= 2) {
        const u64 o = shfl_xor64(v, d);
        v = o > v ? o : v;
    }
    if constexpr (TPR > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
        __syncthreads();
        v = slots[0];
        for (int w = 1; w < TPR / 64; ++w) v = slots[w] > v ? slots[w] : v;
    }
    return v;
}

// candidates that a row's LDS holds; a row of so few values has all of them there
template <int TPR>
constexpr int kCandidates = TPR <= 16 ? 128 : TPR <= 64 ? 256 : 1024;

// The k largest of the keys that TPR threads hold; each(f) calls f(key) for those of a
// thread.  emit(i, key) takes the i-th; returns the k-th, 0 where there are fewer keys.
//
// The k-th largest of the threads' own maxima is a bound that at least k keys reach, and
// few more: T threads with random values leave about T ln(T / (T - k)).  Those go to LDS,
// where each is placed by counting the larger ones.  Values laid out against the
// threads can leave too many; then the k largest are taken one by one.
template <int TPR, class Each, class Emit>
__device__ __forceinline__ u64 top_keys(int k, int t, u64* cand, int* count, u64* border, u64* slots, Each each,
                                        Emit emit) {
    constexpr int N = kCandidates<TPR>;
    u64 best = 0;
    each([&](u64 key) { best = key > best ? key : best; });
    if (t == 0) *count = 0, *border = 0;
    u64 bound = 0;
    if (k < TPR) {
        cand[t] = best;
        row_sync<TPR>();
        int larger = 0;
        for (int o = 0; o < TPR; ++o) larger += cand[o] > best;
        if (larger == k - 1 && best) *border = best;     // (keys differ: one thread, or none)
        row_sync<TPR>();
        bound = *border;
    }
    row_sync<TPR>();
    if (best >= bound)
        each([&](u64 key) {
            if (key < bound || !key) return;
            const int i = atomicAdd(count, 1);
            if (i < N) cand[i] = key;
        });
    if (t == 0) *border = 0;
    row_sync<TPR>();
    const int m = *count;
    if (m <= N) {
        for (int i = t; i < m; i += TPR) {
            const u64 key = cand[i];
            int larger = 0;
            for (int o = 0; o < m; ++o) larger += cand[o] > key;
            if (larger < k) emit(larger, key);
            if (larger == k - 1) *border = key;
        }
        row_sync<TPR>();
        return *border;
    }
    u64 last = 0;
    for (int i = 0; i < k; ++i) {
        const u64 top = row_max64<TPR>(best, slots);
        if (best == top) {
            if (top) emit(i, top);
            best = 0;
            each([&](u64 key) {
                if (key < top && key > best) best = key;
            });
        }
        last = top;
    }
    return last;
}

// log of the sum of exp(z / T) from its largest value m and the sum of exp((z - base) / T),
// base m where that is finite
__device__ __forceinline__ float rest_base(float m) { return fabsf(m) == INFINITY ? 0.f : m; }

// WHOLE: a row to TPR threads.  PIECE_SUMS: a workgroup takes a piece of a row and leaves
// the piece's k largest keys, the largest of the others and their sum.
template <typename T, int TPR, int NC, int MODE>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void top_logits_k(TopArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int TB = TPR > 256 ? TPR : 256, RB = TB / TPR;
    __shared__ u64 cands[RB][kCandidates<TPR>], borders[RB], slots[TB / 64];
    __shared__ int counts[RB];
    __shared__ float fslots[2 * (TB / 64)];
    int turn = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    long r = MODE == WHOLE ? (long)blockIdx.x * RB + rl : blockIdx.x / p.pieces;
    const bool ok = r < p.rows;
    if (!ok) r = p.rows - 1;
    const int piece = MODE == WHOLE ? 0 : (int)(blockIdx.x - r * p.pieces);
    const int c0 = piece * p.piece, c1 = min(p.C, c0 + p.piece);
    RowValues<T, TPR, NC> x;
    x.load((const T*)p.z + r * p.ldz, c0, c1, t, r >= p.exact);
    auto each = [&](auto f) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float v[V];
            x.get(c, c0, c1, t, v);
            const int ch = c0 + (c * TPR + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (ch + j < c1) f(rank_key(v[j], ch + j));
        }
    };
    u64* keys = MODE == WHOLE ? nullptr : (u64*)p.ws + (r * p.pieces + piece) * p.k;
    if (MODE == PIECE_SUMS)
        for (int i = c1 - c0 + t; i < p.k; i += TPR) keys[i] = 0;
    const u64 border = top_keys<TPR>(p.k, t, cands[rl], &counts[rl], &borders[rl], slots, each, [&](int i, u64 key) {
        if (!ok) return;
        if (MODE == WHOLE) {
            p.values[r * p.k + i] = key_value(key);
            p.index[r * p.k + i] = (int)~(uint32_t)key;
        } else {
            keys[i] = key;
        }
    });
    if (!p.rest) return;
    const float eT = kLog2e / p.temp;
    float m = -INFINITY, s = 0.f;
    each([&](u64 key) {
        if (key < border) m = fmaxf(m, key_value(key));
    });
    m = row_max<TPR>(m, fslots, turn);
    const float base = rest_base(m);
    each([&](u64 key) {
        if (key < border) s += pow2((key_value(key) - base) * eT);
    });
    s = row_sum<TPR>(s, fslots, turn);
    if (t || !ok) return;
    if (MODE == WHOLE) p.rest[r] = base / p.temp + logf(s);
    else ((float2*)((u64*)p.ws + p.rows * p.pieces * p.k))[r * p.pieces + piece] = float2{m, s};
}

// A row's answer from its pieces'.
__global__ __launch_bounds__(256) void top_merge_k(TopArgs p) {
    __shared__ u64 cand[kCandidates<256>], border_s, slots[4];
    __shared__ int count;
    __shared__ float fslots[8];
    int turn = 0;
    const int t = threadIdx.x;
    const long r = blockIdx.x;
    const u64* keys = (const u64*)p.ws + r * p.pieces * p.k;
    const long n = (long)p.pieces * p.k;
    auto each = [&](auto f) {
        for (long i = t; i < n; i += 256)
            if (keys[i]) f(keys[i]);
    };
    const u64 border = top_keys<256>(p.k, t, cand, &count, &border_s, slots, each, [&](int i, u64 key) {
        p.values[r * p.k + i] = key_value(key);
        p.index[r * p.k + i] = (int)~(uint32_t)key;
    });
    if (!p.rest) return;
    const float2* part = (const float2*)((const u64*)p.ws + p.rows * p.pieces * p.k) + r * p.pieces;
    const float eT = kLog2e / p.temp;
    float m = -INFINITY, s = 0.f;
    each([&](u64 key) {
        if (key < border) m = fmaxf(m, key_value(key));
    });
    for (int i = t; i < p.pieces; i += 256) m = fmaxf(m, part[i].x);
    m = row_max<256>(m, fslots, turn);
    const float base = rest_base(m);
    each([&](u64 key) {
        if (key < border) s += pow2((key_value(key) - base) * eT);
    });
    for (int i = t; i < p.pieces; i += 256) s += part[i].y * pow2((rest_base(part[i].x) - base) * eT);
    s = row_sum<256>(s, fslots, turn);
    if (t == 0) p.rest[r] = base / p.temp + logf(s);
}

// ---- plans -------------------------------------------------------------------

// Threads of a row and chunks of a thread; rows of more than kWholeChunks chunks are cut
// into pieces of at most kPieceChunks.
struct RowPlan {
    int tpr, nc;
    int pieces, piece;    // piece: classes
};
constexpr int kPieceChunks = 256 * 8;
RowPlan row_plan(int V, int C, int k) {
    const int chunks = (C + V - 1) / V;
    if (chunks <= 16 && k < 16) return {16, 1, 1, C};
    if (k <= 32)
        for (int nc : {1, 2, 4})
            if (chunks <= 64 * nc) return {64, nc, 1, C};
    for (int nc : {2, 4, 8})
        if (chunks <= 256 * nc) return {256, nc, 1, C};
    const int pieces = (chunks + kPieceChunks - 1) / kPieceChunks;
    const int per = (chunks + pieces - 1) / pieces;
    return {256, 8, (chunks + per - 1) / per, per * V};
}

long exact_row(int dt, long rows, int C, long ld) {
    return rows - (dt == DT_BF16 ? tail_rows<bf16>(rows, C, ld) : tail_rows<float>(rows, C, ld));
}

template <typename T, int TPR, int NC, int MODE, typename P>
void row_launch(const P& p, long wgs, hipStream_t st) {
    const dim3 grid((unsigned)wgs), block(TPR > 256 ? TPR : 256);
    constexpr int V = 16 / (int)sizeof(T), RB = TPR > 256 ? 1 : 256 / TPR;
    if constexpr (std::is_same<P, DistillArgs>::value) {
        const unsigned lds = sizeof(float) * RB * distill_lds(p.lds_k, TPR * NC * V);
        if (p.dz && p.rows * p.C * (long)sizeof(T) >= kStreamBytes)
            launch((distill_k<T, TPR, NC, MODE, true>), grid, block, lds, st, p);
        else
            launch((distill_k<T, TPR, NC, MODE, false>), grid, block, lds, st, p);
    } else {
        launch((top_logits_k<T, TPR, NC, MODE>), grid, block, 0, st, p);
    }
}

template <typename T, typename P>
hipError_t whole_rows(const P& p, RowPlan s, hipStream_t st) {
    const long wgs = (p.rows + (s.tpr < 256 ? 256 / s.tpr : 1) - 1) / (s.tpr < 256 ? 256 / s.tpr : 1);
    switch (s.tpr * 16 + s.nc) {
    case 16 * 16 + 1: row_launch<T, 16, 1, WHOLE>(p, wgs, st); break;
    case 64 * 16 + 1: row_launch<T, 64, 1, WHOLE>(p, wgs, st); break;
    case 64 * 16 + 2: row_launch<T, 64, 2, WHOLE>(p, wgs, st); break;
    case 64 * 16 + 4: row_launch<T, 64, 4, WHOLE>(p, wgs, st); break;
    case 256 * 16 + 2: row_launch<T, 256, 2, WHOLE>(p, wgs, st); break;
    case 256 * 16 + 4: row_launch<T, 256, 4, WHOLE>(p, wgs, st); break;
    case 256 * 16 + 8: row_launch<T, 256, 8, WHOLE>(p, wgs, st); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <typename T>
hipError_t top_rows(TopArgs p, RowPlan s, hipStream_t st) {
    if (s.pieces == 1) return whole_rows<T>(p, s, st);
    row_launch<T, 256, 8, PIECE_SUMS>(p, p.rows * p.pieces, st);
    launch(top_merge_k, dim3((unsigned)p.rows), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t distill_rows(DistillArgs p, RowPlan s, hipStream_t st) {
    if (s.pieces == 1) return whole_rows<T>(p, s, st);
    p.grid_pieces = s.pieces;
    row_launch<T, 256, 8, PIECE_SUMS>(p, p.rows * s.pieces, st);
    p.grid_pieces = p.dz ? s.pieces : 1;
    row_launch<T, 256, 8, PIECE_GRAD>(p, p.rows * p.grid_pieces, st);
    return hipGetLastError();
}

}  // namespace

long top_logits_wgs(long rows, int C, int k) {
    return rows * std::max(row_plan(4, C, k).pieces, row_plan(8, C, k).pieces);
}
long top_logits_ws(long rows, int C, int k) {
    const long pieces = std::max(row_plan(4, C, k).pieces, row_plan(8, C, k).pieces);
    return pieces > 1 ? rows * pieces * (2L * k + 2) : 0;
}
long distill_ws(long rows, int C) {
    const long pieces = std::max(row_plan(4, C, 1).pieces, row_plan(8, C, 1).pieces);
    return pieces > 1 ? rows * (4 * pieces + kListPitch) : 0;
}

hipError_t launch_top_logits(int dt, TopArgs p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    const RowPlan s = row_plan(dt == DT_BF16 ? 8 : 4, p.C, p.k);
    p.exact = exact_row(dt, p.rows, p.C, p.ldz);
    p.pieces = s.pieces;
    p.piece = s.piece;
    return dt == DT_BF16 ? top_rows<bf16>(p, s, st) : top_rows<float>(p, s, st);
}

hipError_t launch_distill(int dt, DistillArgs p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    const RowPlan s = row_plan(dt == DT_BF16 ? 8 : 4, p.C, 1);
    p.exact = exact_row(dt, p.rows, p.C, p.ldz);
    p.pieces = s.pieces;
    p.piece = s.piece;
    p.lds_k = p.step ? kDistillMaxK : p.k;
    return dt == DT_BF16 ? distill_rows<bf16>(p, s, st) : distill_rows<float>(p, s, st);
}

}  // namespace lpp
