// Appending keys and values to a paged cache, with the rotary embedding on the way (Section 4.3, modification 2, for tokens as
// they are produced: a sequence's token j stands at position base + j, base being 0 for a prompt and Lp for a response).
// Token i of the new tokens of sequence s becomes token j = lens[s] + i: its k and q are rotated as by the rotary pass over a pack
// (same frequencies, same reduction of the angle in double, same fp32 sine and cosine), k and v go to row j % page of the page
// tables[s][j / page], and q, and if asked for k, to contiguous outputs as well.
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <algorithm>
#include <cmath>
#include <type_traits>

namespace sp {
namespace {

template <typename T> struct CacheVec8;
template <> struct CacheVec8<__bf16> { typedef bf16x8 type; };
template <> struct CacheVec8<float> { typedef float type __attribute__((ext_vector_type(8))); };

struct AppendFreq { double theta[64]; };      // theta_i = base^(-2 i / d), i < d / 2 <= 64

struct AppendArgs {
    const void* q; const void* k; const void* v; void* q_out; void* k_out; void* k_cache; void* v_cache;
    int64_t q_stride, k_stride, v_stride;     // elements from token to token
    const int* tables; const int* lens; const int* pos_base; int* lens_out;
    int64_t width, capacity;                  // pages of a sequence's table, tokens that they hold (at most MAX_TOKENS)
    int64_t n_pages;
    int first_seq, n_seqs, one_each, Hq, Hkv, log_page;
    int64_t first_token, n_tokens;            // of the launch
};

// A workgroup takes 512 / D tokens: each of its 256 threads evaluates one angle, which they exchange through LDS, and D / 16 lanes
// hold eight pairs each of a head, as in the rotary pass.  The heads of a token are those of q, of k and of v in this order; their
// rows are loaded ahead of the lookups.  Bound: bytes.  16.1k tokens of 32 + 8 + 8 heads of 128 with k_out, 430 MB: 80 us, 5.4 TB/s (86 us with stores
// that go through the caches, 88 with loads that do); one token each for 32 sequences: 5.3 us, a launch and three lookups that wait for each other.
// starts.words[i] = first of the launch's new tokens of its sequence i, one past the last behind.
template <typename T, int D>
__global__ __launch_bounds__(256) void append_kernel(SeqArg starts, AppendFreq f, AppendArgs a) {
    typedef typename CacheVec8<T>::type V8;
    constexpr int HALF = D / 2, TOKENS = 256 / HALF, LANES = D / 16, UNROLL = 6;
    __shared__ float cs[TOKENS][HALF], sn[TOKENS][HALF];
    const int* const w = words_of(starts);
    {   // lengths behind the call
        const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (a.lens_out && n < a.n_seqs) {
            const int seq = a.first_seq + (int)n;
            const int64_t have = a.lens[seq], now = have + (a.one_each ? 1 : w[n + 1] - w[n]);
            a.lens_out[seq] = have < 0 ? (int)have : (int)max(have, min(now, a.capacity));
        }
    }
    const int i0 = 8 * ((int)threadIdx.x % LANES), hg = (int)threadIdx.x / LANES % 8, tb = (int)threadIdx.x / HALF;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + (HALF == 64 ? __builtin_amdgcn_readfirstlane(tb) : tb);      // within the launch
    const bool valid = t < a.n_tokens;
    const int64_t tok = a.first_token + t;
    const int H = a.Hq + 2 * a.Hkv;
    auto source = [&](int h) -> const T* {
        if (h < a.Hq) return (const T*)a.q + tok * a.q_stride + (int64_t)h * D + i0;
        if (h < a.Hq + a.Hkv) return (const T*)a.k + tok * a.k_stride + (int64_t)(h - a.Hq) * D + i0;
        return (const T*)a.v + tok * a.v_stride + (int64_t)(h - a.Hq - a.Hkv) * D + i0;
    };
    V8 lo[UNROLL], hi[UNROLL];
    auto load = [&](int h0) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int h = h0 + 8 * u;
            if (!valid || h >= H) continue;
            const T* const p = source(h);
            lo[u] = __builtin_nontemporal_load(reinterpret_cast<const V8*>(p));
            hi[u] = __builtin_nontemporal_load(reinterpret_cast<const V8*>(p + HALF));
        }
    };
    load(hg);
    bool active = false;
    int64_t slot = -1;         // element offset of kv head 0's row in the caches, -1: the token is not stored
    if (valid) {
        int seq;
        int64_t i = 0;
        if (a.one_each) {
            seq = (int)t;
        } else {
            int b = 0, e = a.n_seqs;
            while (e - b > 1) { const int mid = (b + e) >> 1; if (w[mid] <= t) b = mid; else e = mid; }
            seq = b;
            i = t - w[b];
        }
        seq += a.first_seq;
        const int64_t have = a.lens[seq], j = have + i;
        active = have >= 0;
        if (active) {
            if (j < a.capacity) {
                const int64_t page = a.tables[seq * a.width + (j >> a.log_page)];
                if (page >= 0 && page < a.n_pages)
                    slot = (((page * a.Hkv) << a.log_page) + (j & ((1 << a.log_page) - 1))) * D;
            }
            const int64_t pos = j + (a.pos_base ? a.pos_base[seq] : 0);
            const int p = (int)threadIdx.x % HALF;
            const double ang = (double)pos * f.theta[p];
            const double red = ang - 6.283185307179586476925 * rint(ang * 0.15915494309189533577);   // into [-pi, pi]
            float sv, cv;
            sincosf((float)red, &sv, &cv);
            cs[tb][p] = cv;
            sn[tb][p] = sv;
        }
    }
    __syncthreads();
    if (!active) return;
    float c[8], s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { c[e] = cs[tb][i0 + e]; s[e] = sn[tb][i0 + e]; }
    const int64_t head_rows = (int64_t)D << a.log_page;      // from kv head to kv head of a page
    for (int h0 = hg; h0 < H; h0 += 8 * UNROLL) {
        if (h0 != hg) load(h0);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int h = h0 + 8 * u;
            if (h >= H) continue;
            V8 ylo = lo[u], yhi = hi[u];
            const bool is_v = h >= a.Hq + a.Hkv;
            if (!is_v) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = (float)lo[u][e], y = (float)hi[u][e];
                    ylo[e] = (T)(x * c[e] - y * s[e]);
                    yhi[e] = (T)(x * s[e] + y * c[e]);
                }
            }
            auto put = [&](T* p) {
                __builtin_nontemporal_store(ylo, reinterpret_cast<V8*>(p));
                __builtin_nontemporal_store(yhi, reinterpret_cast<V8*>(p + HALF));
            };
            if (h < a.Hq) { put((T*)a.q_out + (tok * a.Hq + h) * D + i0); continue; }
            const int kvh = h - a.Hq - (is_v ? a.Hkv : 0);
            if (slot >= 0) put((T*)(is_v ? a.v_cache : a.k_cache) + slot + kvh * head_rows + i0);
            if (!is_v && a.k_out) put((T*)a.k_out + (tok * a.Hkv + kvh) * D + i0);
        }
    }
}

}  // namespace

hipError_t launch_append(const KvCache& cache, const void* q, int64_t q_stride, void* q_out, int Hq, const void* k, int64_t k_stride,
                         void* k_out, const void* v, int64_t v_stride, int n_seqs, const int32_t* new_lens, const int* tables, int width,
                         const int* lens, const int* pos_base, int* lens_out, double base, hipStream_t s) {
    AppendFreq f{};
    const int d = cache.head_dim;
    for (int i = 0; i < d / 2; ++i) f.theta[i] = pow(base, -2.0 * (double)i / (double)d);
    AppendArgs a{};
    a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.k_out = k_out; a.k_cache = cache.k; a.v_cache = cache.v;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.tables = tables; a.lens = lens; a.pos_base = pos_base; a.lens_out = lens_out;
    a.width = width; a.log_page = cache.log_page; a.capacity = std::min<int64_t>((int64_t)width << cache.log_page, MAX_TOKENS); a.n_pages = cache.n_pages;
    a.one_each = !new_lens; a.Hq = Hq; a.Hkv = cache.n_kv_heads;
    // a launch's token counts are a kernel argument: more sequences than it holds are several launches
    constexpr int MAX_SEQS = SEQ_WORDS - 1;
    int64_t tok = 0;
    for (int seq = 0; seq < n_seqs;) {
        SeqArg starts{};
        int n = 0;
        int64_t tokens = 0;
        if (new_lens) {
            for (; n < MAX_SEQS && seq + n < n_seqs; ++n) { starts.words[n] = (int32_t)tokens; tokens += new_lens[seq + n]; }
            starts.words[n] = (int32_t)tokens;
        } else {
            n = n_seqs;
            tokens = n_seqs;
        }
        a.first_seq = seq; a.n_seqs = n; a.first_token = tok; a.n_tokens = tokens;
        const int per = 512 / d;
        const int64_t grid = std::max<int64_t>((tokens + per - 1) / per, lens_out ? (n + 255) / 256 : 0);
        auto launch = [&](auto elem, auto dim) {
            hipLaunchKernelGGL((append_kernel<decltype(elem), decltype(dim)::value>), dim3((unsigned)grid), dim3(256), 0, s, starts, f, a);
        };
        auto with_d = [&](auto elem) {
            if (d == 64) launch(elem, std::integral_constant<int, 64>{}); else launch(elem, std::integral_constant<int, 128>{});
        };
        if (grid > 0) {
            if (cache.f32) with_d(float{}); else with_d(__bf16{});
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        seq += n;
        tok += tokens;
    }
    return hipSuccess;
}

}  // namespace sp
