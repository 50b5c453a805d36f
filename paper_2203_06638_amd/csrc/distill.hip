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
// [c0, c1) of classes.
template <typename T, int TPR, int NC>
struct RowChunks {
    static constexpr int V = 16 / (int)sizeof(T);
    u4 w[NC];
    __device__ __forceinline__ void load(const T* row, int c0, int c1, int t, bool exact) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int ch = c0 + (c * TPR + t) * V, n = c1 - ch;
            w[c] = ld_chunk(row + (n > 0 ? ch : c0), n, exact);
        }
    }
    // Converted values are not to be kept from one pass over the chunks to the next: twice the
    // registers, and half the workgroups.
    __device__ __forceinline__ void again() {
#pragma unroll
        for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(w[c]));
    }
    // value j of chunk c
    __device__ __forceinline__ float one(int c, int j) const {
        const int i = sizeof(T) == 4 ? j : j >> 1;
        const uint32_t word = i & 2 ? (i & 1 ? w[c].w : w[c].z) : (i & 1 ? w[c].y : w[c].x);
        return __uint_as_float(sizeof(T) == 4 ? word : j & 1 ? word & 0xffff0000u : word << 16);
    }
    // the values of chunk c, -inf behind the end
    __device__ __forceinline__ void get(int c, int c0, int c1, int t, float* v) const {
        const int n = c1 - (c0 + (c * TPR + t) * V);
        chunk_values<T>(w[c], v);
        if (n >= V) return;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = j < n ? v[j] : -INFINITY;
    }
};
// the larger of two, NaN if one is
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

enum RowMode { WHOLE, PIECE_SUMS, PIECE_GRAD };
// What a row's gradient takes: exp(z / T) alone (or exp(z) alone); both; or both with T = 2 or T = 4,
// where exp(z) is a power of the other.
enum RowExps { ONE_EXP, TWO_EXPS, SQUARE, FOURTH };

// ---- distillation ------------------------------------------------------------

// LDS of a row: the list (classes, teacher's values and then probabilities, student's
// logits, whether a class is listed before; the label behind it), three results
// and the largest listed logit, and a bit for each class of the piece that is listed
__host__ __device__ inline int distill_lds(int k, int values) { return 4 * (k + 1) + 4 + (values + 31) / 32; }
constexpr int kListPitch = kDistillMaxK + 4;   // floats of a row's list in the workspace

// Waves a SIMD that the registers are kept to: the latencies of a row's steps, one after the
// other, are covered by other rows.  A workgroup of 512 threads takes two of them.  (64 float32
// values a thread, 2048 x 16000, T = 2: 62.8 us with three waves, 72.5 with four, which spill; 64 as bf16,
// 4096 x 16000: 80.5 and 76.6; two exponentials of 40 float32 values, 4096 x 10000, T = 3: 85.4 and 98.3.
// These and row_plan's figures: inputs that change from call to call.)
template <typename T>
constexpr int distill_waves(int values, bool both, int tpr) {
    if (both) return values <= 16 ? 5 : values < 40 || (values == 40 && tpr > 256) ? 4 : tpr > 256 || values > 48 ? 2 : 3;
    return values < 64 || (values == 64 && (tpr > 256 || sizeof(T) == 2)) ? 4 : 3;
}

// WHOLE: a row to TPR threads, in their registers, so that z is read once.  PIECE_SUMS: a
// workgroup takes a piece of a row and leaves its largest value and its sums; PIECE_GRAD: the
// loss, and the gradient of its piece, from all pieces' sums.
// The listed classes and the label are taken out of the row (set to -inf) and have their
// parts of the sums, and their gradients, from the list, which the row's first wave
// works on: its teacher's side while the row is on its way, its student's side between
// the sums and the gradient.  The exponentials stay in registers from the sums to the
// gradient.
// 4096 x 20000 bf16, 32 listed (328 MB, 64 us at a large copy's rate): 88.5 us with T = 1, 91.4 with
// T = 2 and T = 4, 118.6 with T = 3, where both exponentials of a value are kept (eight waves to a
// row).  A compute unit holds three rows, each of which loads, sums and writes in turn: half of the
// time its vector units wait.
// 1024 x 1000 float32 8.1 us, 128 x 10 6.2: the latency of a row's steps, not its bytes (1.6, 0.002).
template <typename T, int TPR, int NC, int MODE, int EXPS, bool ST>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256, distill_waves<T>(NC * 16 / (int)sizeof(T), EXPS == TWO_EXPS, TPR)) void
distill_k(DistillArgs p) {
    constexpr bool BOTH = EXPS != ONE_EXP;
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int TB = TPR > 256 ? TPR : 256, RB = TB / TPR;
    constexpr int LW = TPR < 64 ? TPR : 64;      // lanes that work on the list
    __shared__ float slots[4 * (TB / 64)];
    extern __shared__ float lds[];
    int turn = 0, none = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    const bool lead = t < LW;
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
    // (BOTH not set: one temperature serves both, the other's terms have no weight or T = 1)
    const float iT = 1.f / temp, e1 = kLog2e, eT = !BOTH && !useT ? kLog2e : kLog2e * iT;
    const T* z = (const T*)p.z + r * p.ldz;

    // the list; entry k is the label
    float* at = lds + rl * distill_lds(p.lds_k, TPR * NC * V);
    int* cls = (int*)at;
    float *pr = at + (k + 1), *zc = at + 2 * (k + 1), *out = at + 4 * (k + 1);
    int* again = (int*)(at + 3 * (k + 1));
    uint32_t* mask = (uint32_t*)(out + 4);
    float rest = -INFINITY;
    if (lead) {
        for (int e = t; e <= k; e += LW) {
            int c = e < k ? (useT ? index[r * k + e] : -1) : (use1 ? labels[r] : -1);
            if ((unsigned)c >= (unsigned)p.C) c = -1;
            cls[e] = c;
            pr[e] = e < k && c >= 0 ? values[r * k + e] * iT : -INFINITY;
        }
        if (tail) rest = rests[r];
    }
    RowChunks<T, TPR, NC> x;
    if (MODE != PIECE_GRAD || p.dz) x.load(z, c0, c1, t, r >= p.exact);
    for (int e = t; e < (TPR * NC * V + 31) / 32; e += TPR) mask[e] = 0u;
    row_sync<TPR>();
    float tm = rest, ts = 0.f;
    bool twice = false;               // a class is listed twice
    if (lead) {
        bool bad = rest != rest;      // (a maximum drops a NaN)
        float lm = -INFINITY;         // the largest listed logit
        auto entry = [&](int e) {
            const int c = cls[e];
            // (dz may be z: the pieces' workgroups keep z at the listed classes for each other)
            float* kept = p.ws + 4 * p.rows * p.pieces + r * kListPitch;
            float v = 0.f;
            if (c >= 0) v = MODE == PIECE_GRAD ? kept[e] : ld1(z, c);
            zc[e] = v;
            if (MODE != PIECE_SUMS && c >= 0 && e < k) lm = fmaxf(lm, v);
            if (MODE == PIECE_SUMS && c >= c0 && c < c1) kept[e] = v;
            // whether the class is listed before (all of a row's entries are one wave's, the label
            // comes last)
            int seen = 0;
            if (c >= c0 && c < c1) {
                const uint32_t bit = 1u << ((c - c0) & 31);
                seen = (atomicOr(&mask[(c - c0) >> 5], bit) & bit) != 0;
            }
            if (MODE == PIECE_GRAD) {
                seen = 0;
#pragma unroll 4
                for (int o = 0; o < e; ++o) seen |= cls[o] == c;
            }
            again[e] = seen;
            twice |= seen && e < k;
            tm = fmaxf(tm, pr[e]);
            bad |= pr[e] != pr[e];
        };
        for (int e = t; e < k; e += LW) entry(e);
        if (t == k % LW) entry(k);
        // the teacher's probabilities
        tm = row_max<LW>(tm, slots, none);
        if (MODE != PIECE_SUMS) {
            lm = row_max<LW>(lm, slots, none);
            if (t == 0) out[3] = lm;  // (it waits there for the row's sums: registers)
        }
        for (int e = t; e < k; e += LW) ts += cls[e] >= 0 && tm > -INFINITY ? pow2((pr[e] - tm) * kLog2e) : 0.f;
        ts = row_sum<LW>(bad ? NAN : ts, slots, none) + (rest > -INFINITY ? pow2((rest - tm) * kLog2e) : 0.f);
    }
    // (a list without an entry, or of -inf alone, says nothing)
    const bool some = useT && !(tm == -INFINITY && ts == ts);
    row_sync<TPR>();

    // the row, then its exponentials: a of z / T (of z where only that is wanted), b of z
    float a[NC][V], b[EXPS == TWO_EXPS ? NC : 1][V];
    auto power = [&](float v) {         // exp(z) from exp(z / T)
        v *= v;
        return EXPS == FOURTH ? v * v : v;
    };
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        x.get(c, c0, c1, t, a[c]);
        const int i = (c * TPR + t) * V;
        const uint32_t gone = mask[i >> 5] >> (i & 31) & ((1u << V) - 1u);
        if (gone)
#pragma unroll
            for (int j = 0; j < V; ++j) a[c][j] = (gone >> j) & 1u ? -INFINITY : a[c][j];
    }
    // m: the largest of the classes that are not listed, and their sums of exp(z - m) and
    // exp((z - m) / T).  Relative to the row's largest value they would vanish where a listed class lies far
    // above them, and with them the rest's answer, which is a ratio of them.
    float m = -INFINITY, s1 = 0.f, so = 0.f;
    const f4* all = (const f4*)p.ws + r * p.pieces;
    if (MODE == PIECE_GRAD) {
        for (int e = t; e < p.pieces; e += TPR) m = fmaxf(m, all[e][0]);
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) m = fmaxf(m, a[c][j]);
    }
    if (MODE != PIECE_SUMS && lead && t == k % LW && cls[k] >= 0 && !again[k]) m = fmaxf(m, zc[k]);
    m = row_max<TPR>(m, slots, turn);
    // (nothing but -inf: sums of 0)
    const float base = m == -INFINITY ? 0.f : m;
    if (MODE != PIECE_GRAD || p.dz) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = a[c][j] - base;
                a[c][j] = pow2(d * eT);
                if constexpr (EXPS == TWO_EXPS) b[c][j] = pow2(d * e1);
                if (MODE == PIECE_GRAD) continue;
                so += a[c][j];
                if constexpr (EXPS == TWO_EXPS) s1 += b[c][j];
                else if constexpr (BOTH) s1 += power(a[c][j]);
            }
    }
    if (MODE == PIECE_GRAD)
        for (int e = t; e < p.pieces; e += TPR) {
            const f4 s = all[e];
            if (BOTH) s1 += s[1] * pow2((s[0] - base) * e1);
            so += s[2] * pow2((s[0] - base) * eT);
        }
    if (BOTH) row_sum2<TPR>(s1, so, slots, turn);
    else so = row_sum<TPR>(so, slots, turn);
    if (MODE == PIECE_SUMS) {
        if (t == 0) ((f4*)p.ws)[r * p.pieces + piece] = f4{m, s1, so, 0.f};
        return;
    }

    // the student's side of the list
    const int y = cls[k];
    const float a1 = use1 ? 1.f - alpha : 0.f, aT = some ? alpha * temp : 0.f;
    const float g1 = y >= 0 && use1 ? p.scale * w * a1 : 0.f, gT = p.scale * w * aT;
    const bool live = w != 0.f && (g1 != 0.f || gT != 0.f);   // (a row without a loss has no gradient, whatever it holds)
    float sT = 0.f, kT = 0.f;
    if (lead) {
        const float most = fmaxf(m, out[3]);     // of all classes
        // what the listed classes add: once each, the label's to the first sum (and to the
        // other classes' of the second, if it is not listed).  Sums over all classes are relative to most.
        float l1 = 0.f, lT = 0.f, ly = 0.f;
        for (int e = t; e <= k; e += LW) {
            if (cls[e] < 0 || again[e]) continue;
            const float d = zc[e] - most;
            if (BOTH) l1 += pow2(d * e1);
            if (e < k) lT += pow2(d * eT);
            else ly = pow2((zc[e] - base) * eT);
        }
        row_sum2<LW>(lT, ly, slots, none);
        const float away = m - most, far1 = pow2(away * e1), farT = pow2(away * eT);   // (NaN for a row of -inf)
        if (BOTH) s1 = s1 * far1 + row_sum<LW>(l1, slots, none);
        so += ly;
        sT = so * farT + lT;
        if (!BOTH) s1 = sT;
        const float lt = logf(ts), lq = logf(sT);
        float soft = 0.f, sp = 0.f;
        for (int e = t; e < k; e += LW) {
            if (cls[e] < 0 || !some) {
                pr[e] = 0.f;
                continue;
            }
            const float v = pr[e] - tm, pe = pow2(v * kLog2e) / ts, u = (zc[e] - most) * iT - lq, d = v - lt - u;
            pr[e] = pe;
            sp += pe;
            // both sides' probabilities add up to 1 (the student's with what it gives the classes
            // that are not listed): p log(p / q) - p + q in place of p log(p / q) keeps the sum
            // exact where p is near q
            if (pe > 0.f)
                soft += again[e] ? pe * d - pe : d > -1.f ? pe * (d + expm1f(-d)) : pe * d - pe + pow2(u * kLog2e);
            else if (pe != pe) soft = pe;
            else if (!again[e]) soft += pow2(u * kLog2e);
        }
        row_sum2<LW>(soft, sp, slots, none);
        float others = farT / sT;     // what gT times exp((z - m) / T) of a class that is not listed has
        const float q = so * farT / sT;
        if (!tail) {
            soft += q;
        } else {
            const float pe = some && rest > -INFINITY ? pow2((rest - tm) * kLog2e) / ts : 0.f;
            if (some) {
                const float d = (rest - tm) - lt - (logf(so) + away * iT - lq);
                if (pe > 0.f) soft += d > -1.f ? pe * (d + expm1f(-d)) : pe * d - pe + q;
                else soft += q;
            }
            // q - p of the rest is p - q of the list, which is the smaller and so the more
            // exact of the two where the rest is large
            others = so != 0.f ? (pe > 0.5f ? sp - lT / sT : q - pe) / so : 0.f;
        }
        kT = gT != 0.f ? gT * others : 0.f;
        if (t == 0) {
            if (ok && piece == 0) {
                float l = 0.f;
                if (y >= 0 && use1) l += a1 * (logf(s1) - (zc[k] - most));
                if (some) l += aT * temp * soft;
                p.loss[r] = w != 0.f ? w * l : 0.f;
            }
            out[0] = g1 != 0.f ? g1 / s1 * far1 : 0.f;
            out[1] = kT;
            out[2] = live ? 1.f : 0.f;
        }
    }
    if (!p.dz) return;
    row_sync<TPR>();
    T* dz = (T*)p.dz + r * p.lddz;
    const float k1 = out[0];
    kT = out[1];
    if (out[2] == 0.f)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                a[c][j] = 0.f;
                if constexpr (EXPS == TWO_EXPS) b[c][j] = 0.f;
            }
    // (dz may be z: what the list needs of z was read above, before a barrier)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int ch = c0 + (c * TPR + t) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (EXPS == TWO_EXPS) a[c][j] = __builtin_fmaf(kT, a[c][j], k1 * b[c][j]);
            else if constexpr (EXPS == ONE_EXP) a[c][j] *= kT + k1;
            else a[c][j] = __builtin_fmaf(kT, a[c][j], k1 * power(a[c][j]));
        }
        if (ok) st_chunk<ST>(dz + ch, c1 - ch, a[c]);
    }
    row_sync<TPR>();
    if (!lead) return;
#pragma unroll
    for (int d = 1; d < LW; d *= 2) twice |= __shfl_xor((int)twice, d) != 0;
    if (!ok || !live) return;
    const float most = fmaxf(m, out[3]);
    for (int e = t; e <= k; e += LW) {
        const int c = cls[e];
        if (c < c0 || c >= c1 || again[e]) continue;
        float pe = e < k ? pr[e] : 0.f;
        if (twice) {
            pe = 0.f;
            for (int o = 0; o < k; ++o) pe += cls[o] == c ? pr[o] : 0.f;
        }
        const float d = zc[e] - most;
        float g = g1 != 0.f ? g1 * (pow2(d * e1) / s1 - (c == y ? 1.f : 0.f)) : 0.f;
        if (gT != 0.f) g += e < k || !tail ? gT * (pow2(d * eT) / sT - pe) : kT * pow2((zc[e] - base) * eT);
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

// LDS of a row
template <int TPR>
struct TopSpace {
    u64 cand[kCandidates<TPR>];
    u64 border;
    int count;
    __device__ __forceinline__ void add(u64 key) {
        const int i = atomicAdd(&count, 1);
        if (i < kCandidates<TPR>) cand[i] = key;
    }
};
// The k largest of the m candidates, each placed by counting the larger ones: emit(i, key)
// takes the i-th.  Returns the k-th, 0 where there are fewer.
template <int TPR, class Emit>
__device__ __forceinline__ u64 rank_candidates(int k, int t, int m, TopSpace<TPR>& s, Emit emit) {
    if (t == 0) s.border = 0;
    row_sync<TPR>();
    for (int i = t; i < m; i += TPR) {
        const u64 key = s.cand[i];
        int larger = 0;
#pragma unroll 4
        for (int o = 0; o < m; ++o) larger += s.cand[o] > key;
        if (larger < k) emit(larger, key);
        if (larger == k - 1) s.border = key;
    }
    row_sync<TPR>();
    return s.border;
}

// The same of the keys that TPR threads hold, whatever they are; each(f) calls f(key) for
// those of a thread.  The k-th largest of the threads' own maxima is a bound that at least
// k keys reach, k exactly where all values are equal.  Keys laid out against the threads can
// leave too many; then the k largest are taken one by one.
template <int TPR, class Each, class Emit>
__device__ __forceinline__ u64 top_keys(int k, int t, TopSpace<TPR>& s, u64* slots, Each each, Emit emit) {
    constexpr int H = TPR < 256 ? TPR : 256;     // threads whose maxima are compared
    u64 best = 0;
    each([&](u64 key) { best = key > best ? key : best; });
    u64 lead = best;
    for (int d = H; d < TPR; d *= 2) {           // (TPR / H neighbours' maxima as one)
        const u64 o = shfl_xor64(lead, d / H);
        lead = o > lead ? o : lead;
    }
    row_sync<TPR>();
    if (t == 0) s.count = 0, s.border = 0;
    if (t % (TPR / H) == 0) s.cand[t / (TPR / H)] = lead;
    row_sync<TPR>();
    if (t < H) {
        const u64 mine = s.cand[t];
        int larger = 0;
        for (int o = 0; o < H; ++o) larger += s.cand[o] > mine;
        if (larger == k - 1 && mine) s.border = mine;     // (keys differ: one thread, or none)
    }
    row_sync<TPR>();
    const u64 bound = s.border;
    row_sync<TPR>();
    if (best >= bound)
        each([&](u64 key) {
            if (key >= bound && key) s.add(key);
        });
    row_sync<TPR>();
    const int m = s.count;
    if (m <= kCandidates<TPR>) return rank_candidates<TPR>(k, t, m, s, emit);
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

// Waves a SIMD that the registers are kept to (2048 x 16000 float32, 32 values a thread, five waves
// are two workgroups of 512 threads, six are three: 38.5 and 31.8 us).
template <typename T>
constexpr int top_waves(int values) { return values <= (sizeof(T) == 2 ? 40 : 32) ? 6 : values <= 40 ? 5 : 4; }

// Rows of a few candidates are finished by their first wave: the others are gone by then.
constexpr int kFew = 256;

// WHOLE: a row to TPR threads.  PIECE_SUMS: a workgroup takes a piece of a row and leaves
// the piece's k largest keys, the largest of the others and their sum.
//
// The row is cut into G groups of neighbouring threads' values.  The k-th largest of the
// groups' maxima is a bound that at least k values reach, and few more: about
// G ln(G / (G - k)) of random ones.  Those go to LDS, and the values under the bound are
// summed, relative to it; then the first wave places the candidates.  Where too many reach
// the bound (equal values, or values laid out against the threads) top_keys takes over, and
// where the values under it add up to less than 1, so that the bound may lie far above them,
// they are summed again relative to their largest.
// 4096 x 20000 bf16, k = 32 (164 MB, 32 us at a large copy's rate): 50.9 us, of which the vector
// instructions (about 17 a value, an exponential among them) are issued for 89%; k = 128: 95.0, whose
// candidates, about 177, the first wave alone places, in passes over all of them.  128 x 1000 float32 6.3
// us, and 8 x 131072 in pieces 12.2 + 6.6 for the merge: latency of 4 to 8 dependent steps.
template <typename T, int TPR, int NC, int MODE, int G>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256, top_waves<T>(NC * 16 / (int)sizeof(T))) void top_logits_k(TopArgs p) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int TB = TPR > 256 ? TPR : 256, RB = TB / TPR;
    constexpr int LW = TPR < 64 ? TPR : 64;
    __shared__ TopSpace<TPR> spaces[RB];
    __shared__ u64 slots[TB / 64];
    __shared__ __attribute__((aligned(16))) float maxima[RB][G];
    __shared__ float fslots[2 * (TB / 64)];
    int turn = 0, none = 0;
    const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
    TopSpace<TPR>& space = spaces[rl];
    long r = MODE == WHOLE ? (long)blockIdx.x * RB + rl : blockIdx.x / p.pieces;
    const bool ok = r < p.rows;
    if (!ok) r = p.rows - 1;
    const int piece = MODE == WHOLE ? 0 : (int)(blockIdx.x - r * p.pieces);
    const int c0 = piece * p.piece, c1 = min(p.C, c0 + p.piece);
    RowChunks<T, TPR, NC> x;
    x.load((const T*)p.z + r * p.ldz, c0, c1, t, r >= p.exact);
    float top[NC], best = -INFINITY;      // of the chunks, of the thread; NaN is the largest
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float v[V];
        x.get(c, c0, c1, t, v);
        top[c] = v[0];
#pragma unroll
        for (int j = 1; j < V; ++j) top[c] = max_nan(top[c], v[j]);
        best = max_nan(best, top[c]);
    }
    best = best != best ? INFINITY : best;
#pragma unroll
    for (int d = 1; d < TPR / G; d *= 2) best = fmaxf(best, __shfl_xor(best, d));
    if (t % (TPR / G) == 0) maxima[rl][t / (TPR / G)] = best;
    if (t == 0) space.count = 0;
    row_sync<TPR>();
    float bound;
    {
        // (a group's threads share the other groups)
        constexpr int S = TPR / G, N = G / S;
        const float* others = &maxima[rl][t % S * N];
        int larger = 0;
#pragma unroll 4
        for (int o = 0; o < N; o += 4) {
            const f4 v = *(const f4*)(others + o);
            larger += (v[0] > best) + (v[1] > best) + (v[2] > best) + (v[3] > best);
        }
#pragma unroll
        for (int d = 1; d < S; d *= 2) larger += __shfl_xor(larger, d);
        bound = -row_max<TPR>(larger < p.k ? -best : -INFINITY, fslots, turn);
    }
    // z / T - base / T, in powers of two, as one fma: shift is the rounded base / T, and the
    // sum is corrected by what the rounding left out
    const float eT = kLog2e / p.temp;
    const float base0 = rest_base(bound), shift = base0 * eT;
    float s = 0.f;
    x.again();
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float v[V];
        x.get(c, c0, c1, t, v);
        if (!(top[c] < bound)) {
            const int ch = c0 + (c * TPR + t) * V;
            uint32_t over = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool under = v[j] < bound;
                over |= under ? 0u : 1u << j;
                v[j] = under ? v[j] : -INFINITY;
            }
            if (c1 - ch < V) over &= c1 > ch ? (1u << (c1 - ch)) - 1u : 0u;
            for (; over; over &= over - 1) {
                const int j = __builtin_ctz(over);
                space.add(rank_key(x.one(c, j), ch + j));
            }
        }
        if (p.rest)
#pragma unroll
            for (int j = 0; j < V; ++j) s += pow2(__builtin_fmaf(v[j], eT, -shift));
    }
    s = row_sum<TPR>(s, fslots, turn);     // (its barrier is the candidates' too)
    s *= pow2(-__builtin_fmaf(base0, eT, -shift));
    row_sync<LW>();
    const int n = space.count;
    u64* keys = MODE == WHOLE ? nullptr : (u64*)p.ws + (r * p.pieces + piece) * p.k;
    auto emit = [&](int i, u64 key) {
        if (!ok) return;
        if (MODE == WHOLE) {
            p.values[r * p.k + i] = key_value(key);
            p.index[r * p.k + i] = (int)~(uint32_t)key;
        } else {
            keys[i] = key;
        }
    };
    auto give = [&](float m, float base, float sum) {     // (the others' largest value, their sum relative to base)
        if (t || !ok) return;
        if (MODE == WHOLE) p.rest[r] = base / p.temp + logf(sum);
        else ((f4*)((u64*)p.ws + (p.rows * p.pieces * p.k + 1) / 2 * 2))[r * p.pieces + piece] = f4{m, base, sum, 0.f};
    };
    if (n <= kFew && ((s >= 1.f && s < INFINITY && fabsf(bound) < INFINITY) || !p.rest)) {
        if (t >= LW) return;
        if (MODE == PIECE_SUMS)
            for (int i = n + t; i < p.k; i += LW) keys[i] = 0;
        // the candidates that are not among the k are others too: relative to the largest
        // of them, at least the bound
        float lead = -INFINITY;
        int place[kFew / LW];
#pragma unroll
        for (int q = 0; q < kFew / LW; ++q) {
            const int i = q * LW + t;
            place[q] = 0;
            if (q * LW >= n) continue;
            const u64 key = space.cand[min(i, n - 1)];
            int larger = 0;
#pragma unroll 4
            for (int o = 0; o < n; ++o) larger += space.cand[o] > key;
            place[q] = larger;
            if (i >= n) continue;
            if (larger < p.k) emit(larger, key);
            else lead = fmaxf(lead, key_value(key));
        }
        if (!p.rest) return;
        lead = row_max<LW>(lead, fslots, none);
        const float base = lead > bound ? rest_base(lead) : base0;
        float more = 0.f;
#pragma unroll
        for (int q = 0; q < kFew / LW; ++q) {
            const int i = q * LW + t;
            if (i < n && place[q] >= p.k) more += pow2((key_value(space.cand[i]) - base) * eT);
        }
        more = row_sum<LW>(more, fslots, none);
        give(fmaxf(lead, bound), base, s * pow2((base0 - base) * eT) + more);
        return;
    }
    // (rows that come here are few: they are read again, for registers that the others have)
    const T* z = (const T*)p.z + r * p.ldz;
    auto each = [&](auto f) {
#pragma unroll 1
        for (int c = 0; c < NC; ++c) {
            const int ch = c0 + (c * TPR + t) * V;
            if (ch >= c1) break;
            float v[V];
            chunk_values<T>(ld_chunk(z + ch, c1 - ch, r >= p.exact), v);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (ch + j < c1) f(rank_key(v[j], ch + j));
        }
    };
    if (MODE == PIECE_SUMS)
        for (int i = c1 - c0 + t; i < p.k; i += TPR) keys[i] = 0;
    const u64 border = n <= kCandidates<TPR> ? rank_candidates<TPR>(p.k, t, n, space, emit)
                                             : top_keys<TPR>(p.k, t, space, slots, each, emit);
    if (!p.rest) return;
    float m = -INFINITY;
    s = 0.f;
    each([&](u64 key) { m = key < border ? fmaxf(m, key_value(key)) : m; });
    m = row_max<TPR>(m, fslots, turn);
    const float base = rest_base(m);
    each([&](u64 key) { s += key < border ? pow2((key_value(key) - base) * eT) : 0.f; });
    give(m, base, row_sum<TPR>(s, fslots, turn));
}

// A row's answer from its pieces' lists, which are in descending order.  With j = 2 k / P
// (P pieces) at least k keys reach the ceil(k / j)-th largest of the pieces' j-th keys.  (8 rows of
// 32 pieces, k = 64: 6.6 us, barriers.)
constexpr int kMergeThreads = 1024, kMergeKeys = 4;
__global__ __launch_bounds__(kMergeThreads) void top_merge_k(TopArgs p) {
    constexpr int TPR = kMergeThreads;
    __shared__ TopSpace<TPR> space;
    __shared__ u64 slots[TPR / 64];
    __shared__ float fslots[2 * TPR / 64];
    int turn = 0;
    const int t = threadIdx.x;
    const long r = blockIdx.x;
    const u64* keys = (const u64*)p.ws + r * p.pieces * p.k;
    const f4* part = (const f4*)((const u64*)p.ws + (p.rows * p.pieces * p.k + 1) / 2 * 2) + r * p.pieces;
    const int n = p.pieces * p.k;
    const int jth = min(p.k, (2 * p.k + p.pieces - 1) / p.pieces), nth = (p.k + jth - 1) / jth;
    u64 v[kMergeKeys];
#pragma unroll
    for (int u = 0; u < kMergeKeys; ++u) v[u] = u * TPR + t < n ? keys[u * TPR + t] : 0;
    f4 mine = t < p.pieces ? part[t] : f4{-INFINITY, 0.f, 0.f, 0.f};
    u64 bound = 0;
    const bool few = p.pieces <= 64;
    if (few && t < p.pieces) {
        bound = keys[(long)t * p.k + jth - 1];
        space.cand[t] = bound;
    }
    if (t == 0) space.count = 0, space.border = 0;
    __syncthreads();
    if (few && t < p.pieces) {
        int larger = 0;
        for (int o = 0; o < p.pieces; ++o) larger += space.cand[o] > bound;
        if (larger == nth - 1) space.border = bound;     // (equal ones are 0: no bound)
    }
    __syncthreads();
    bound = space.border;
    __syncthreads();
    auto each = [&](auto f) {
#pragma unroll
        for (int u = 0; u < kMergeKeys; ++u)
            if (v[u]) f(v[u]);
        for (int i = kMergeKeys * TPR + t; i < n; i += TPR)
            if (keys[i]) f(keys[i]);
    };
    each([&](u64 key) {
        if (key >= bound) space.add(key);
    });
    __syncthreads();
    auto emit = [&](int i, u64 key) {
        p.values[r * p.k + i] = key_value(key);
        p.index[r * p.k + i] = (int)~(uint32_t)key;
    };
    const int m0 = space.count;
    const u64 border = m0 <= kCandidates<TPR> ? rank_candidates<TPR>(p.k, t, m0, space, emit)
                                              : top_keys<TPR>(p.k, t, space, slots, each, emit);
    if (!p.rest) return;
    const float eT = kLog2e / p.temp;
    float m = mine[0], s = 0.f;
    each([&](u64 key) { m = key < border ? fmaxf(m, key_value(key)) : m; });
    for (int i = t + TPR; i < p.pieces; i += TPR) m = fmaxf(m, part[i][0]);
    m = row_max<TPR>(m, fslots, turn);
    const float base = rest_base(m);
    each([&](u64 key) { s += key < border ? pow2((key_value(key) - base) * eT) : 0.f; });
    for (int i = t; i < p.pieces; i += TPR) {
        if (i >= TPR) mine = part[i];
        s += mine[2] != 0.f ? mine[2] * pow2((mine[1] - base) * eT) : 0.f;
    }
    s = row_sum<TPR>(s, fslots, turn);
    if (t == 0) p.rest[r] = base / p.temp + logf(s);
}

// ---- plans -------------------------------------------------------------------

// Threads of a row and chunks of a thread.  Rows that the registers of 512 threads do not
// hold are cut into pieces.  Where there are many rows, four waves to a row and more values a
// thread: more rows of a compute unit at once, whose steps cover each other (distillation of 4096 x 20000
// bf16, T = 2: 93.3 us, 101.1 with eight waves; 1024 x 16000 float32: 35.9 and 34.3).
// wide: values that a thread may keep there.  Top logits: 48 (4096 x 10000 bf16 32.0 us, 37.9 with
// eight; 16000: 41.8 and 40.8); distillation: 80, with two exponentials kept 48.
struct RowPlan {
    int tpr, nc;
    int pieces, piece;    // piece: classes
};
constexpr int kThreadValues = 64, kWideRows = 2048, kTopWide = 48, kDistillWide = 80, kTwoWide = 48;
// whether a row of TPR threads with `values` each is one of row_plan's with `wide`
constexpr bool planned(int tpr, int values, int wide) { return tpr != 256 || values <= wide; }
RowPlan row_plan(int V, long rows, int C, int k, int wide) {
    const int chunks = (C + V - 1) / V;
    // (up to 128 classes; 16384 x 100 float32, distillation, one buffer again and again: 20 us with a wave
    // to a row, 8.6 with 16 lanes)
    if (C <= 128 && k < 16) return {16, chunks <= 16 ? 1 : 2, 1, C};
    if (k <= 32)
        for (int nc : {1, 2, 4})
            if (chunks <= 64 * nc) return {64, nc, 1, C};
    for (int nc : {1, 2, 4})
        if (chunks <= 256 * nc) return {256, nc, 1, C};
    if (rows >= kWideRows)
        for (int nc : {6, 8, 10, 12, 16})
            if (nc * V <= wide && chunks <= 256 * nc) return {256, nc, 1, C};
    for (int nc : {4, 5, 6, 8, 12, 16})
        if (nc * V <= kThreadValues && chunks <= 512 * nc) return {512, nc, 1, C};
    // 256 workgroups with two chunks a thread at least, or as few as hold the row
    const long want = std::min<long>((256 + rows - 1) / std::max(rows, 1L), chunks / 512);
    const int pieces = (int)std::max<long>(want, (chunks + 256 * 8 - 1) / (256 * 8));
    const int per = (chunks + pieces - 1) / pieces;
    return {256, per <= 512 ? 2 : per <= 1024 ? 4 : 8, (chunks + per - 1) / per, per * V};
}

long exact_row(int dt, long rows, int C, long ld) {
    return rows - (dt == DT_BF16 ? tail_rows<bf16>(rows, C, ld) : tail_rows<float>(rows, C, ld));
}

int distill_exps(const DistillArgs& p) {
    if (p.step) return TWO_EXPS;
    if (!p.labels || p.alpha <= 0.f || p.alpha >= 1.f || p.temp == 1.f) return ONE_EXP;
    return p.temp == 2.f ? SQUARE : p.temp == 4.f ? FOURTH : TWO_EXPS;
}

// (hipErrorInvalidValue: a shape that row_plan does not make, and that has no kernel)
template <typename T, int TPR, int NC, int MODE>
hipError_t row_launch(const TopArgs& p, long wgs, hipStream_t st) {
    const dim3 grid((unsigned)wgs), block(TPR > 256 ? TPR : 256);
    constexpr int values = NC * 16 / (int)sizeof(T);
    if constexpr (TPR <= 64) launch((top_logits_k<T, TPR, NC, MODE, TPR>), grid, block, 0, st, p);
    else if constexpr (MODE != WHOLE || planned(TPR, values, kTopWide)) {
        if (p.k > 32) launch((top_logits_k<T, TPR, NC, MODE, 256>), grid, block, 0, st, p);
        else if constexpr (TPR != 256 || NC > 1) launch((top_logits_k<T, TPR, NC, MODE, 64>), grid, block, 0, st, p);
        else return hipErrorInvalidValue;   // (a wave's)
    } else return hipErrorInvalidValue;
    return hipGetLastError();
}
template <typename T, int TPR, int NC, int MODE>
hipError_t row_launch(const DistillArgs& p, long wgs, hipStream_t st) {
    if constexpr (TPR == 256 && NC == 1) return hipErrorInvalidValue;   // (a wave's)
    else {
        const dim3 grid((unsigned)wgs), block(TPR > 256 ? TPR : 256);
        constexpr int V = 16 / (int)sizeof(T), RB = TPR > 256 ? 1 : 256 / TPR;
        const unsigned lds = sizeof(float) * RB * distill_lds(p.lds_k, TPR * NC * V);
        const bool stream = MODE != PIECE_SUMS && p.dz && p.rows * p.C * (long)sizeof(T) >= kStreamBytes;
        const int exps = distill_exps(p);
        auto go = [&](auto exps) {
            constexpr int E = decltype(exps)::value;
            if (stream) launch((distill_k<T, TPR, NC, MODE, E, MODE != PIECE_SUMS>), grid, block, lds, st, p);
            else launch((distill_k<T, TPR, NC, MODE, E, false>), grid, block, lds, st, p);
        };
        if (exps == TWO_EXPS) {
            if constexpr (MODE != WHOLE || planned(TPR, NC * V, kTwoWide)) go(std::integral_constant<int, TWO_EXPS>());
            else return hipErrorInvalidValue;
        } else if (exps == SQUARE) go(std::integral_constant<int, SQUARE>());
        else if (exps == FOURTH) go(std::integral_constant<int, FOURTH>());
        else go(std::integral_constant<int, ONE_EXP>());
        return hipGetLastError();
    }
}

template <typename T, typename P>
hipError_t whole_rows(const P& p, RowPlan s, hipStream_t st) {
    const int rb = s.tpr < 256 ? 256 / s.tpr : 1;
    const long wgs = (p.rows + rb - 1) / rb;
    switch (s.tpr * 32 + s.nc) {
    case 16 * 32 + 1: return row_launch<T, 16, 1, WHOLE>(p, wgs, st);
    case 16 * 32 + 2:
        if constexpr (sizeof(T) == 4) return row_launch<T, 16, 2, WHOLE>(p, wgs, st);
        else return hipErrorInvalidValue;   // (128 bf16 classes are 16 chunks)
    case 64 * 32 + 1: return row_launch<T, 64, 1, WHOLE>(p, wgs, st);
    case 64 * 32 + 2: return row_launch<T, 64, 2, WHOLE>(p, wgs, st);
    case 64 * 32 + 4: return row_launch<T, 64, 4, WHOLE>(p, wgs, st);
    case 256 * 32 + 1: return row_launch<T, 256, 1, WHOLE>(p, wgs, st);
    case 256 * 32 + 2: return row_launch<T, 256, 2, WHOLE>(p, wgs, st);
    case 256 * 32 + 4: return row_launch<T, 256, 4, WHOLE>(p, wgs, st);
    case 256 * 32 + 6: return row_launch<T, 256, 6, WHOLE>(p, wgs, st);
    case 256 * 32 + 8: return row_launch<T, 256, 8, WHOLE>(p, wgs, st);
    case 256 * 32 + 10: return row_launch<T, 256, 10, WHOLE>(p, wgs, st);
    case 256 * 32 + 12:
        if constexpr (sizeof(T) == 4) return row_launch<T, 256, 12, WHOLE>(p, wgs, st);
        else return hipErrorInvalidValue;   // (row_plan: 80 values a thread)
    case 256 * 32 + 16:
        if constexpr (sizeof(T) == 4) return row_launch<T, 256, 16, WHOLE>(p, wgs, st);
        else return hipErrorInvalidValue;
    case 512 * 32 + 4: return row_launch<T, 512, 4, WHOLE>(p, wgs, st);
    case 512 * 32 + 5: return row_launch<T, 512, 5, WHOLE>(p, wgs, st);
    case 512 * 32 + 6: return row_launch<T, 512, 6, WHOLE>(p, wgs, st);
    case 512 * 32 + 8: return row_launch<T, 512, 8, WHOLE>(p, wgs, st);
    case 512 * 32 + 12:
        if constexpr (sizeof(T) == 4) return row_launch<T, 512, 12, WHOLE>(p, wgs, st);
        else return hipErrorInvalidValue;   // (64 values a thread)
    case 512 * 32 + 16:
        if constexpr (sizeof(T) == 4) return row_launch<T, 512, 16, WHOLE>(p, wgs, st);
        else return hipErrorInvalidValue;
    default: return hipErrorInvalidValue;
    }
}
template <typename T, int MODE, typename P>
hipError_t piece_rows(const P& p, int nc, long wgs, hipStream_t st) {
    return nc == 2   ? row_launch<T, 256, 2, MODE>(p, wgs, st)
           : nc == 4 ? row_launch<T, 256, 4, MODE>(p, wgs, st)
                     : row_launch<T, 256, 8, MODE>(p, wgs, st);
}

template <typename T>
hipError_t top_rows(TopArgs p, RowPlan s, hipStream_t st) {
    if (s.pieces == 1) return whole_rows<T>(p, s, st);
    hipError_t e = piece_rows<T, PIECE_SUMS>(p, s.nc, p.rows * p.pieces, st);
    if (e != hipSuccess) return e;
    launch(top_merge_k, dim3((unsigned)p.rows), dim3(kMergeThreads), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t distill_rows(DistillArgs p, RowPlan s, hipStream_t st) {
    if (s.pieces == 1) return whole_rows<T>(p, s, st);
    p.grid_pieces = s.pieces;
    hipError_t e = piece_rows<T, PIECE_SUMS>(p, s.nc, p.rows * s.pieces, st);
    if (e != hipSuccess) return e;
    p.grid_pieces = p.dz ? s.pieces : 1;
    return piece_rows<T, PIECE_GRAD>(p, s.nc, p.rows * p.grid_pieces, st);
}

}  // namespace

static long most_pieces(long rows, int C, int k) {
    return std::max(row_plan(4, rows, C, k, kTopWide).pieces, row_plan(8, rows, C, k, kTopWide).pieces);
}
static long row_threads(long rows, int C, int k, int wide) {
    long most = 0;
    for (int V : {4, 8}) {
        const RowPlan s = row_plan(V, rows, C, k, wide);
        const int rb = s.tpr < 256 ? 256 / s.tpr : 1;
        most = std::max(most, s.pieces > 1 ? rows * std::max(256 * s.pieces, kMergeThreads) : (rows + rb - 1) / rb * rb * s.tpr);
    }
    return most;
}
long top_logits_threads(long rows, int C, int k) { return row_threads(rows, C, k, kTopWide); }
long distill_threads(long rows, int C) { return std::max(row_threads(rows, C, 1, kDistillWide), row_threads(rows, C, 1, kTwoWide)); }
long top_logits_ws(long rows, int C, int k) {
    const long pieces = most_pieces(rows, C, k);
    return pieces > 1 ? (rows * pieces * (2L * k) + 3) / 4 * 4 + rows * pieces * 4 : 0;
}
long distill_ws(long rows, int C) {
    const long pieces = most_pieces(rows, C, 1);
    return pieces > 1 ? rows * (4 * pieces + kListPitch) : 0;
}

hipError_t launch_top_logits(int dt, TopArgs p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    const RowPlan s = row_plan(dt == DT_BF16 ? 8 : 4, p.rows, p.C, p.k, kTopWide);
    p.exact = exact_row(dt, p.rows, p.C, p.ldz);
    p.pieces = s.pieces;
    p.piece = s.piece;
    return dt == DT_BF16 ? top_rows<bf16>(p, s, st) : top_rows<float>(p, s, st);
}

hipError_t launch_distill(int dt, DistillArgs p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    const RowPlan s = row_plan(dt == DT_BF16 ? 8 : 4, p.rows, p.C, 1, distill_exps(p) == TWO_EXPS ? kTwoWide : kDistillWide);
    p.exact = exact_row(dt, p.rows, p.C, p.ldz);
    p.pieces = s.pieces;
    p.piece = s.piece;
    p.lds_k = p.step ? kDistillMaxK : p.k;
    return dt == DT_BF16 ? distill_rows<bf16>(p, s, st) : distill_rows<float>(p, s, st);
}

}  // namespace lpp
