// Adjusted logits: what a sampler does to a row of logits before it draws, and log-probabilities under the distribution
// that it really drew from.  With h_v = id v occurs in the row's history (the prompt of its group and the tokens of
// its response ahead of it) and c_v = how often among the latter, an element goes through
//   a = z_v + bias_v,   b = h_v ? (a > 0 ? a / rho : a rho) : a,   d = b - frequency c_v - presence [c_v > 0],
//   z'_v = mask bit v ? d / T : -inf.
//  adjust        z' of one row per sequence
//  logprob fwd   logp = z'_y - L, L = ln sum_v e^(z'_v), at every response row of a pack; z' is never stored
//  logprob bwd   dz_v = g (1[v = y] - e^(z'_v - L)) dz'_v / dz_v, the slope being (h_v ? (a > 0 ? 1 / rho : rho) : 1) / T, 0 where masked
//
// The history reaches a row as counters in LDS, 16 bits per id: bit 15 "in the prompt", below it the occurrences in the
// response (they stop at 32767).  A workgroup takes a slice of the vocabulary, so that its counters fit, and a run of rows; the
// counters are filled once, and from row to row only the tokens between them are added.  Integer atomics: the order does not matter.
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <algorithm>
#include <type_traits>

namespace sp {
namespace {

constexpr int AT = 512;                    // threads of a workgroup
constexpr int AWAVES = AT / 64;
constexpr int FEW_WAVES = 2;
constexpr int SLICE_MAX = 32768;           // ids of a slice at most: 64 KB of counters, two workgroups to a CU (half of it: forward 165 -> 180 us)
constexpr float A_LOWEST = -3.402823466e38f;

// eight consecutive elements, at any alignment of their own type
template <typename T> struct Pack8;
template <> struct Pack8<__bf16> {
    typedef __bf16 vec __attribute__((ext_vector_type(8), aligned(2)));
    vec x;
    template <bool PAST> __device__ __forceinline__ void load(const __bf16* p) {
        if constexpr (PAST) x = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p));
        else x = *reinterpret_cast<const vec*>(p);
    }
    template <bool PAST> __device__ __forceinline__ void store(__bf16* p) const {
        if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<vec*>(p));
        else *reinterpret_cast<vec*>(p) = x;
    }
};
template <> struct Pack8<float> {
    typedef float half __attribute__((ext_vector_type(4), aligned(4)));
    typedef float vec __attribute__((ext_vector_type(8)));
    vec x;
    template <bool PAST> __device__ __forceinline__ void load(const float* p) {
        const half* const q = reinterpret_cast<const half*>(p);
        half a, b;
        if constexpr (PAST) { a = __builtin_nontemporal_load(q); b = __builtin_nontemporal_load(q + 1); }
        else { a = q[0]; b = q[1]; }
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[e + 4] = b[e]; }
    }
    template <bool PAST> __device__ __forceinline__ void store(float* p) const {
        half* const q = reinterpret_cast<half*>(p);
        half a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) { a[e] = x[e]; b[e] = x[e + 4]; }
        if constexpr (PAST) { __builtin_nontemporal_store(a, q); __builtin_nontemporal_store(b, q + 1); }
        else { q[0] = a; q[1] = b; }
    }
};

// A slice [v0, v0 + n) of the vocabulary and the counters of its ids (two to a word)
struct Slice { int v0, n; unsigned* counts; };

__device__ __forceinline__ Slice slice_of(int index, int len, int vocab, unsigned* lds) {
    const int v0 = index * len;
    return Slice{v0, min(len, vocab - v0), lds};
}

template <int THREADS>
__device__ __forceinline__ void clear_counts(const Slice& s) {
    for (int i = threadIdx.x; i < (s.n + 7) / 8; i += THREADS) reinterpret_cast<i32x4*>(s.counts)[i] = i32x4{0, 0, 0, 0};
}

// Adds `count` tokens of the prompt, or of the response; those outside the slice (or the vocabulary) are passed over.  Four in flight per thread.
__device__ __forceinline__ void count_one(const Slice& s, unsigned k, bool may_saturate) {
    const int sh = 16 * (k & 1);
    unsigned* const w = &s.counts[k >> 1];
    if (!may_saturate) { atomicAdd(w, 1u << sh); return; }
    unsigned have = *w;
    while (((have >> sh) & 0x7fffu) != 0x7fffu) {
        const unsigned seen = atomicCAS(w, have, have + (1u << sh));
        if (seen == have) break;
        have = seen;
    }
}
template <int THREADS, typename F>
__device__ __forceinline__ void for_tokens(const Slice& s, const int* tokens, int count, F f) {
    for (int i = threadIdx.x; i < count; i += 4 * THREADS) {
        unsigned k[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) k[u] = i + u * THREADS < count ? (unsigned)tokens[i + u * THREADS] - (unsigned)s.v0 : 0xffffffffu;
#pragma unroll
        for (int u = 0; u < 4; ++u) if (k[u] < (unsigned)s.n) f(k[u]);
    }
}
template <int THREADS>
__device__ __forceinline__ void add_prompt(const Slice& s, const int* tokens, int count) {
    for_tokens<THREADS>(s, tokens, count, [&](unsigned k) { atomicOr(&s.counts[k >> 1], 0x8000u << (16 * (k & 1))); });
}
template <int THREADS>
__device__ __forceinline__ void add_generated(const Slice& s, const int* tokens, int count, bool may_saturate) {
    if (may_saturate) for_tokens<THREADS>(s, tokens, count, [&](unsigned k) { count_one(s, k, true); });
    else for_tokens<THREADS>(s, tokens, count, [&](unsigned k) { count_one(s, k, false); });
}

// Eight elements of a row after the bias: penalties and mask, ahead of the division by the temperature; slope (SLOPE): their
// derivative with respect to the raw elements, but for the temperature and the mask, multiplied in.  An element costs some twelve instructions if it
// is in the history of any of the wave's rows of eight, else two: few are.
template <bool SLOPE, bool HIST>
__device__ __forceinline__ void adjust8(float (&a)[8], float (&slope)[8], const AdjustRules& r, i32x4 counts, bool masked, unsigned bits) {
    if constexpr (HIST) {
        if (__builtin_amdgcn_ballot_w64(((counts[0] | counts[1]) | (counts[2] | counts[3])) != 0) != 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned c = e & 1 ? (unsigned)counts[e >> 1] >> 16 : (unsigned)counts[e >> 1] & 0xffffu;
                if (__builtin_amdgcn_ballot_w64(c != 0) != 0) {
                    const float f = c ? (a[e] > 0.f ? r.inv_repetition : r.repetition) : 1.f;
                    const float n = (float)(c & 0x7fffu);
                    a[e] = __builtin_fmaf(a[e], f, -__builtin_fmaf(n, r.frequency, n > 0.f ? r.presence : 0.f));
                    if constexpr (SLOPE) slope[e] *= f;
                }
            }
        }
    }
    if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned keep = (unsigned)__builtin_amdgcn_sbfe((int)bits, e, 1);
            a[e] = __uint_as_float((__float_as_uint(a[e]) & keep) | (0xff800000u & ~keep));
        }
    }
}

// Visits the slice of one row in vectors of eight, UNROLL of them in flight per thread, at the slice's end too (with the last ones one by one, five
// slices of 30392 ids took 182 us forward and 272 back, now 166 and 260): f(values, counts, mask bits, index
// of the first element within the slice, how many of them there are).  PAST: the row is read past the caches.
template <typename T, int THREADS, bool HIST, bool PAST, int UNROLL, typename F>
__device__ __forceinline__ void for_vectors(const T* row, const uint8_t* mask, const AdjustRules& r, const Slice& s, F f) {
    const int vecs = s.n / 8;
    const T* const z = row + s.v0;
    const float* const bias = r.bias ? r.bias + s.v0 : nullptr;
    const uint8_t* const bits = mask ? mask + s.v0 / 8 : nullptr;
    auto several = [&](int i, auto whole) __attribute__((always_inline)) {
        constexpr bool WHOLE = decltype(whole)::value;              // else the last ones again behind the slice's end, and not visited
        Pack8<T> x[UNROLL];
        Pack8<float> b[UNROLL];
        unsigned m[UNROLL];
        i32x4 c[UNROLL];
        auto at = [&](int u) __attribute__((always_inline)) { return WHOLE ? i + u * THREADS : min(i + u * THREADS, vecs - 1); };
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) x[u].template load<PAST>(z + 8 * at(u));
        if (bits)
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) m[u] = bits[at(u)];
        if (bias)
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) b[u].template load<false>(bias + 8 * at(u));
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            c[u] = i32x4{0, 0, 0, 0};
            if constexpr (HIST) c[u] = reinterpret_cast<const i32x4*>(s.counts)[at(u)];
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (!WHOLE && i + u * THREADS >= vecs) continue;
            float a[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = (float)x[u].x[e];
            if (bias)
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] += b[u].x[e];
            f(a, c[u], bits ? m[u] : 0xffu, 8 * (i + u * THREADS), 8);
        }
    };
    int i = threadIdx.x;
    for (; i + (UNROLL - 1) * THREADS < vecs; i += UNROLL * THREADS) several(i, std::true_type{});
    if (i < vecs) several(i, std::false_type{});
    if ((s.n & 7) && (int)threadIdx.x == vecs % THREADS) {          // the vocabulary's last, incomplete vector
        float a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = 8 * vecs + e < s.n ? (float)z[8 * vecs + e] + (bias ? bias[8 * vecs + e] : 0.f) : -INFINITY;
        i32x4 c{0, 0, 0, 0};
        if constexpr (HIST) c = reinterpret_cast<const i32x4*>(s.counts)[vecs];
        f(a, c, bits ? bits[vecs] : 0xffu, 8 * vecs, s.n & 7);
    }
}

template <bool PAST, typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8], int n) {
    if (n == 8) {
        Pack8<T> y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y.x[e] = (T)x[e];
        y.template store<PAST>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (e < n) p[e] = (T)x[e];
    }
}

struct AdjustArgs {
    const void* logits; void* out; int64_t stride, out_stride;
    const uint8_t* mask; int64_t mask_stride;            // bytes
    const int* prompt_tokens; const int* prompt_lens; int64_t prompt_stride;
    const int* resp_tokens; const int* resp_lens; int64_t resp_stride;
    AdjustRules rules;
    int first, n_groups, vocab, slice_len;               // first: sequence of the launch's first row
};

// One workgroup per (sequence, slice of at most ADJUST_VECS vectors to a thread), so that a slice's elements are all asked for ahead of the
// history, whose lookups wait for each other.  Two vectors: as every slice reads the whole history, longer slices serve long ones, shorter slices
// few rows.  152k ids in bf16 (us; one vector / two / four): 32 rows with 0.8k tokens 7.1 / 6.6 / 7.7, with 17k 16.0 / 12.0 / 12.7, 256 rows with
// 1.5k 35.9 / 28.8 (5.4 TB/s) / 29.9.  Bound: bytes, with few rows the latency of a launch and four lookups.  words[g] = first sequence of the launch's group g, one past the last behind them, then the
// number of the first group.
constexpr int ADJUST_VECS = 2;
template <typename T, bool HIST>
__global__ __launch_bounds__(AT) void adjust_kernel(SeqArg starts, AdjustArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned lds[];
    const int seq = a.first + blockIdx.y;
    const Slice s = slice_of(blockIdx.x, a.slice_len, a.vocab, lds);
    const int vecs = s.n / 8, loose = s.n & 7;
    const T* const z = (const T*)a.logits + seq * a.stride + s.v0;
    T* const out = (T*)a.out + seq * a.out_stride + s.v0;
    const float* const bias = a.rules.bias ? a.rules.bias + s.v0 : nullptr;
    const uint8_t* const bits = a.mask ? a.mask + seq * a.mask_stride + s.v0 / 8 : nullptr;
    float x[ADJUST_VECS][8];
    unsigned m[ADJUST_VECS];
    bool there[ADJUST_VECS];
#pragma unroll
    for (int u = 0; u < ADJUST_VECS; ++u) {
        const int i = threadIdx.x + u * AT;
        there[u] = i < vecs || (i == vecs && loose);
        if (!there[u]) continue;
        if (i < vecs) {
            Pack8<T> y;
            y.template load<false>(z + 8 * i);
            Pack8<float> b;
            if (bias) b.template load<false>(bias + 8 * i); else b.x = (typename Pack8<float>::vec)(0.f);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = (float)y.x[e] + b.x[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = e < loose ? (float)z[8 * i + e] + (bias ? bias[8 * i + e] : 0.f) : 0.f;
        }
        m[u] = bits ? bits[i] : 0xffu;
    }
    if constexpr (HIST) {
        clear_counts<AT>(s);
        int np = 0, nr = 0;
        const int* prompt = nullptr;
        if (a.prompt_tokens) {
            const int* const w = words_of(starts);
            int lo = 0, hi = a.n_groups;
            while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (w[mid] <= seq) lo = mid; else hi = mid; }
            const int g = w[a.n_groups + 1] + lo;
            prompt = a.prompt_tokens + g * a.prompt_stride;
            np = max(0, (int)min((int64_t)a.prompt_lens[g], a.prompt_stride));
        }
        if (a.resp_tokens) nr = max(0, (int)min((int64_t)a.resp_lens[seq], a.resp_stride));
        __syncthreads();
        add_prompt<AT>(s, prompt, np);
        add_generated<AT>(s, a.resp_tokens + seq * a.resp_stride, nr, nr > 0x7fff);
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < ADJUST_VECS; ++u) {
        if (!there[u]) continue;
        const int i = threadIdx.x + u * AT;
        i32x4 c{0, 0, 0, 0};
        if constexpr (HIST) c = reinterpret_cast<const i32x4*>(s.counts)[i];
        float none[8];
        adjust8<false, HIST>(x[u], none, a.rules, c, bits != nullptr, m[u]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] *= a.rules.inv_temperature;
        store8<false>(out + 8 * i, x[u], i < vecs ? 8 : loose);
    }
}

struct LogprobArgs {
    const void* logits; const int* labels; const int* tokens;
    const uint8_t* mask; int64_t mask_stride;            // bytes
    float* logp; float* lse;                             // forward out; backward: lse in
    const float* g; void* dlogits;
    uint32_t* tag;                                       // forward: the workspace's tag block, cleared as by every call that writes there
    float* parts;                                        // forward: (max, sum) per row, slice and wave, then a label's z' per row
    AdjustRules rules;
    int vocab, slice_len, n_slices, run, own, zero_prompt;
};

// (m, s) stands for s e^(m / T): differences are taken ahead of their scaling, so that they are exact at any magnitude, and start
// from the lowest finite value, so that elements of -inf contribute 0.
__device__ __forceinline__ void scaled_merge(float& m, float& s, float m2, float s2, float c) {
    const float mn = fmaxf(m, m2);
    s = s * __builtin_amdgcn_exp2f((m - mn) * c) + s2 * __builtin_amdgcn_exp2f((m2 - mn) * c);
    m = mn;
}
// over the lanes of a wave
__device__ __forceinline__ void scaled_wave(float& m, float& s, float c) {
    const float mn = wave_max(m);
    s = wave_sum(s * __builtin_amdgcn_exp2f((m - mn) * c));
    m = mn;
}
__device__ __forceinline__ float log_of(float m, float s, float inv_t) { return m * inv_t + __logf(s); }
// A row's results from its (m, s) and the label's z' (-inf: no id of the vocabulary).  No id allowed: L = -inf, and the log-probability of any
// label is -inf.  Where L's own rounding is large (rows of, say, -1e9 throughout: 64 and more) z' - L may come out above 0, which it is not: cut there.
// A NaN in the row is in L and stays.
__device__ __forceinline__ void finish_row(float m, float s, float z, float inv_t, float* logp, float* lse) {
    const float L = log_of(m, s, inv_t);
    *lse = L;
    const float d = z - L;
    const int bits = (int)bits_of(d);
    *logp = bits_of(L) == 0xff800000u ? -INFINITY : bits > 0 && bits <= 0x7f800000 ? 0.f : d;
}

// One workgroup per (slice, run of rows of the pack), its counters as the first row needs them; from row to row each wave adds to those of its
// own vectors.  Bound, at 1470 response rows of 152k ids in bf16 with bias and mask: the forward (447 MB, 163 us, 2.7 TB/s; 483 MB with mask and bias) by vector
// instructions, 118 for eight elements of a wave's rows, eight of them exponentials and a third for the 2.6 ids of every 512 that the history holds;
// the backward (1.05 GB, 219 us, 4.8 TB/s) by memory.  Four vectors of a row in flight per thread: with two 176 and 226 us.
template <typename T, int WAVES, bool HIST, bool BWD, bool PAST>
__global__ __launch_bounds__(64 * WAVES) void adjusted_logprob_kernel(TabArg table, LogprobArgs a) {
    constexpr int THREADS = 64 * WAVES;
    __shared__ float row_parts[2][2 * WAVES + 1];
    extern __shared__ __attribute__((aligned(16))) unsigned lds[];
    const int* const tab = table_of(table);
    const Slice s = slice_of(blockIdx.x, a.slice_len, a.vocab, lds);
    const int T_total = tab[1], t0 = blockIdx.y * a.run, t1 = min(t0 + a.run, T_total);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const float c = a.rules.inv_temperature * LOG2E;
    if (!BWD && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) a.tag[threadIdx.x] = 0u;
    int seg_end = t0, counted = 0, place = 0;
    bool prompt = false, may_saturate = false;
    for (int t = t0; t < t1; ++t) {
        if (t == seg_end) {                              // another segment: its prompt, its history up to this row
            const GroupDesc gd = load_group(tab, find_group_of_token(tab, t));
            const int local = t - gd.tok_base;
            prompt = local < gd.Lp;
            if (prompt) {
                seg_end = gd.tok_base + gd.Lp;
            } else {
                seg_end = gd.tok_base + sp::seg_end(gd, local);
                counted = gd.tok_base + seg_start(gd, local);
                may_saturate = seg_end - counted > 0x7fff;
                if constexpr (HIST) {
                    __syncthreads();                     // every wave is through with the segment before
                    clear_counts<THREADS>(s);
                    __syncthreads();
                    add_prompt<THREADS>(s, a.tokens + gd.tok_base, gd.Lp);
                    add_generated<THREADS>(s, a.tokens + counted, t + a.own - counted, may_saturate);
                    counted = t + a.own;
                    __syncthreads();
                }
            }
        }
        if (prompt) {
            if (!BWD && a.zero_prompt && blockIdx.x == 0 && threadIdx.x == 0) { a.logp[t] = 0.f; a.lse[t] = 0.f; }
            if (BWD && a.zero_prompt) {
                T* const out = (T*)a.dlogits + (int64_t)t * a.vocab + s.v0;
                const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                for (int i = threadIdx.x; i < (s.n + 7) / 8; i += THREADS) store8<PAST>(out + 8 * i, zero, min(8, s.n - 8 * i));
            }
            continue;
        }
        if constexpr (HIST) {
            // The tokens since the row before, by the wave that reads their counters: no wave waits for another from row to row.
            for (; counted < t + a.own; ++counted) {
                const unsigned k = (unsigned)a.tokens[counted] - (unsigned)s.v0;
                if (k < (unsigned)s.n && (int)(k >> 3) % THREADS == (int)threadIdx.x) count_one(s, k, may_saturate);
            }
            __builtin_amdgcn_wave_barrier();
        }
        const T* const row = (const T*)a.logits + (int64_t)t * a.vocab;
        const uint8_t* const mask = a.mask ? a.mask + t * a.mask_stride : nullptr;
        const unsigned label = (unsigned)a.labels[t] - (unsigned)s.v0;          // within the slice, if below s.n
        const int label_at = label < (unsigned)s.n ? (int)(label & ~7u) : -1;
        if constexpr (BWD) {
            T* const out = (T*)a.dlogits + (int64_t)t * a.vocab + s.v0;
            // (an L that is no number, or +inf, is the slope of the whole row, so that it ends as NaN)
            const float L = a.lse[t];
            const unsigned of_L = bits_of(L);
            const bool none = of_L == 0xff800000u;
            const float Lf = none ? 0.f : L, gt = none ? 0.f : (of_L & 0x7f800000u) == 0x7f800000u ? L : -a.g[t] * a.rules.inv_temperature;
            for_vectors<T, THREADS, HIST, PAST, 4>(row, mask, a.rules, s, [&](float (&x)[8], i32x4 cnt, unsigned bits, int at, int n) __attribute__((always_inline)) {
                float slope[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) slope[e] = gt;
                adjust8<true, HIST>(x, slope, a.rules, cnt, false, bits);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(__builtin_fmaf(x[e], a.rules.inv_temperature, -Lf) * LOG2E), 0.f, 1.f);      // (see finish_row)
                if (at == label_at)
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (e == (int)(label & 7)) x[e] -= 1.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= slope[e];
                if (mask)                                // 0 in masked places whatever the row's g and logits are
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(__float_as_uint(x[e]) & (unsigned)__builtin_amdgcn_sbfe((int)bits, e, 1));
                store8<PAST>(out + at, x, n);
            });
        } else {
            float m = A_LOWEST, sum = 0.f, z_label = -INFINITY;
            for_vectors<T, THREADS, HIST, false, 4>(row, mask, a.rules, s, [&](float (&x)[8], i32x4 cnt, unsigned bits, int at, int n) __attribute__((always_inline)) {
                float none[8];
                adjust8<false, HIST>(x, none, a.rules, cnt, mask != nullptr, bits);
                // against the reference from earlier elements, which serves as long as the exponentials stay in range
                float part = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) part += __builtin_amdgcn_exp2f((x[e] - m) * c);
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(part <= 16384.f)) != 0, 0)) {
                    float mx = x[0];
#pragma unroll
                    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
                    const float mn = fmaxf(m, mx);
                    part = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) part += __builtin_amdgcn_exp2f((x[e] - mn) * c);
                    sum *= __builtin_amdgcn_exp2f((m - mn) * c);
                    m = mn;
                }
                sum += part;
                if (at == label_at)
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (e == (int)(label & 7)) z_label = x[e] * a.rules.inv_temperature;
            });
            scaled_wave(m, sum, c);
            if (a.n_slices == 1) {
                // The workgroup has all of the row: no join.  (Two places in turn, from response row to response row, whatever lies between them: who
                // writes the next but one has met the reader at the barrier of the next.)
                float* const mine = row_parts[place];
                place ^= 1;
                if (lane == 0) { mine[2 * wave] = m; mine[2 * wave + 1] = sum; }
                if ((int)threadIdx.x == (label_at < 0 ? 0 : (label_at >> 3) % THREADS)) mine[2 * WAVES] = z_label;
                __syncthreads();
                if (threadIdx.x == 0) {
#pragma unroll
                    for (int i = 1; i < WAVES; ++i) scaled_merge(m, sum, mine[2 * i], mine[2 * i + 1], c);
                    finish_row(m, sum, mine[2 * WAVES], a.rules.inv_temperature, a.logp + t, a.lse + t);
                }
                continue;
            }
            float* const labels_z = a.parts + (int64_t)T_total * a.n_slices * WAVES * 2;
            if (label_at >= 0 && (int)threadIdx.x == (label_at >> 3) % THREADS) labels_z[t] = z_label;
            if (lane == 0) {
                float* const p = a.parts + (((int64_t)t * a.n_slices + blockIdx.x) * WAVES + wave) * 2;
                p[0] = m;
                p[1] = sum;
            }
        }
    }
}

// One wave per row joins the row's slices.
__global__ __launch_bounds__(256) void logprob_join_kernel(TabArg table, const int* __restrict__ labels, const float* __restrict__ parts,
                                                           float* __restrict__ logp, float* __restrict__ lse, int per_row, int vocab, float inv_t) {
    const int* const tab = table_of(table);
    const int T_total = tab[1], t = blockIdx.x * 4 + (threadIdx.x >> 6), l = threadIdx.x & 63;
    if (t >= T_total) return;
    const GroupDesc gd = load_group(tab, find_group_of_token(tab, t));
    if (t - gd.tok_base < gd.Lp) return;
    const float c = inv_t * LOG2E;
    float m = A_LOWEST, s = 0.f;
    for (int i = l; i < per_row; i += 64) {
        const float* const p = parts + ((int64_t)t * per_row + i) * 2;
        scaled_merge(m, s, p[0], p[1], c);
    }
    scaled_wave(m, s, c);
    if (l == 0) {
        const int y = labels[t];
        finish_row(m, s, y >= 0 && y < vocab ? parts[(int64_t)T_total * per_row * 2 + t] : -INFINITY, inv_t, logp + t, lse + t);
    }
}

template <typename F> void with_kernel(bool f32, bool hist, F f) {
    auto typed = [&](auto elem) { if (hist) f(elem, std::true_type{}); else f(elem, std::false_type{}); };
    if (f32) typed(float{}); else typed(__bf16{});
}

bool uses_history(const AdjustRules& r) { return r.repetition != 1.f || r.presence != 0.f || r.frequency != 0.f; }

}  // namespace

int adjust_slices(int64_t vocab) { return (int)((vocab + SLICE_MAX - 1) / SLICE_MAX); }

size_t adjust_parts_bytes(int64_t total_tokens, int64_t vocab) {
    return (size_t)total_tokens * ((size_t)adjust_slices(vocab) * AWAVES * 8 + 4);
}

hipError_t launch_adjust_logits(const void* logits, int64_t stride, void* out, int64_t out_stride, int64_t vocab, const AdjustRules& rules,
                                const uint32_t* mask, int64_t mask_stride, int n_groups, const int32_t* Gs,
                                const int* prompt_tokens, int prompt_stride, const int* prompt_lens,
                                const int* resp_tokens, int resp_stride, const int* resp_lens, bool f32, hipStream_t s) {
    AdjustArgs a{};
    a.logits = logits; a.out = out; a.stride = stride; a.out_stride = out_stride;
    a.mask = (const uint8_t*)mask; a.mask_stride = mask_stride * 4;
    a.prompt_tokens = prompt_stride > 0 ? prompt_tokens : nullptr; a.prompt_lens = prompt_lens; a.prompt_stride = prompt_stride;
    a.resp_tokens = resp_stride > 0 ? resp_tokens : nullptr; a.resp_lens = resp_lens; a.resp_stride = resp_stride;
    a.rules = rules;
    a.vocab = (int)vocab;
    int64_t n_seqs = 0;
    for (int g = 0; g < n_groups; ++g) n_seqs += Gs ? Gs[g] : 1;
    // Slices as long as their threads can hold, or half of that where the chip is not full (2 rows of 32k ids: 4.1 us against 4.8).
    a.slice_len = 8 * AT * ADJUST_VECS;
    if (n_seqs * ((vocab + a.slice_len - 1) / a.slice_len) < 256) a.slice_len /= ADJUST_VECS;
    const int64_t slices = (vocab + a.slice_len - 1) / a.slice_len;
    const bool hist = uses_history(rules) && (a.prompt_tokens || a.resp_tokens);
    const size_t lds = hist ? (size_t)a.slice_len * 2 : 0;
    // the groups of a launch are a kernel argument, and its rows a grid's second dimension: larger calls are several launches
    constexpr int MAX_GROUPS = SEQ_WORDS - 2, MAX_ROWS = 32768;
    int seq = 0, g = 0, left = 0;                        // left: sequences of group g that the launches so far have not served
    while (true) {
        while (g < n_groups && left == 0) { left = Gs ? Gs[g] : 1; if (left == 0) ++g; }
        if (g >= n_groups) break;
        SeqArg starts{};
        const int g0 = g;
        int n = 0, rows = 0;
        while (g < n_groups && n < MAX_GROUPS && rows < MAX_ROWS) {
            starts.words[n++] = seq + rows;
            const int take = left < MAX_ROWS - rows ? left : MAX_ROWS - rows;
            rows += take;
            left -= take;
            if (left > 0) break;
            ++g;
            if (g < n_groups) left = Gs ? Gs[g] : 1;
        }
        starts.words[n] = seq + rows;
        starts.words[n + 1] = g0;
        a.first = seq; a.n_groups = n;
        with_kernel(f32, hist, [&](auto elem, auto with) {
            hipLaunchKernelGGL((adjust_kernel<decltype(elem), decltype(with)::value>), dim3((unsigned)slices, (unsigned)rows), dim3(AT), lds, s, starts, a);
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        seq += rows;
    }
    return hipSuccess;
}

hipError_t launch_adjusted_logprob(bool bwd, const void* logits, const int* labels, const int* tokens, const uint32_t* mask, int64_t mask_stride,
                                   float* logp, float* lse, const float* g, void* dlogits, const AdjustRules& rules, const TabArg& tab,
                                   int64_t total_tokens, int64_t vocab, bool own_token, bool zero_prompt, float* parts, uint32_t* tag, bool f32,
                                   hipStream_t s) {
    LogprobArgs a{};
    a.logits = logits; a.labels = labels; a.tokens = tokens; a.mask = (const uint8_t*)mask; a.mask_stride = mask_stride * 4;
    a.logp = logp; a.lse = lse; a.g = g; a.dlogits = dlogits; a.parts = parts; a.tag = tag; a.rules = rules;
    a.vocab = (int)vocab;
    a.n_slices = adjust_slices(vocab);
    a.slice_len = (int)std::min<int64_t>(SLICE_MAX, (vocab + 7) / 8 * 8);
    a.own = own_token; a.zero_prompt = zero_prompt;
    // A small vocabulary leaves eight waves little to do between a row's lookups: two, as long as a thread has no more than eight vectors (1145 rows
    // of 5003 ids in float32: forward 10.5 us, gradient 11.9; with four waves 9.8 and 14.5, with eight 14.4 and 16.5).
    const int waves = a.slice_len > 8 * 64 * FEW_WAVES * 8 ? AWAVES : FEW_WAVES;
    // Runs: a workgroup's history is read once for its rows, and 2048 workgroups fill the chip four times over (1470 rows of 152k ids: forward
    // and backward 381 us, with half as many workgroups 429, with twice as many 380).
    const int64_t run = total_tokens * a.n_slices / 2048;
    a.run = (int)(run < 1 ? 1 : run > 16 ? 16 : run);
    while ((total_tokens + a.run - 1) / a.run > 65535) a.run *= 2;
    const bool hist = uses_history(rules);
    const size_t lds = hist ? (size_t)a.slice_len * 2 : 0;
    const dim3 grid((unsigned)a.n_slices, (unsigned)((total_tokens + a.run - 1) / a.run));
    // As the ordinary gradient: one that the Infinity Cache (256 MB) cannot hold is stored past the caches, and then the logits are read past
    // them (603 MB: the backward 224 us against 234, and the forward of the next call 169 against 186).
    const int64_t row = vocab * (f32 ? 4 : 2);
    const bool past = total_tokens * row > (int64_t)256 << 20 && row >= 8192;
    with_kernel(f32, hist, [&](auto elem, auto with) {
        typedef decltype(elem) T;
        constexpr bool H = decltype(with)::value;
        auto of = [&](auto size) {
            constexpr int W = decltype(size)::value;
            if (!bwd) hipLaunchKernelGGL((adjusted_logprob_kernel<T, W, H, false, false>), grid, dim3(64 * W), lds, s, tab, a);
            else if (past) hipLaunchKernelGGL((adjusted_logprob_kernel<T, W, H, true, true>), grid, dim3(64 * W), lds, s, tab, a);
            else hipLaunchKernelGGL((adjusted_logprob_kernel<T, W, H, true, false>), grid, dim3(64 * W), lds, s, tab, a);
        };
        if (waves == AWAVES) of(std::integral_constant<int, AWAVES>{}); else of(std::integral_constant<int, FEW_WAVES>{});
    });
    if (!bwd && a.n_slices > 1)
        hipLaunchKernelGGL(logprob_join_kernel, dim3((unsigned)((total_tokens + 3) / 4)), dim3(256), 0, s, tab, labels, parts, logp, lse,
                           a.n_slices * waves, (int)vocab, rules.inv_temperature);
    return hipGetLastError();
}

}  // namespace sp
