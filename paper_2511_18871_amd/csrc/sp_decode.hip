// Attention of one new token per sequence over the paged cache: the shared-prompt attention of Section 4.3 in the form of a rollout
// step.  The G sequences of a group read the pages of their common prompt, and each the pages of its own response.
//   S_j = scale <q, k_j> over the keys [0, Lp) of the prompt and [0, len) of the response,
//   o = sum_j e^(S_j - m) v_j / l, l = sum_j e^(S_j - m), lse = m + ln l; without a key o = 0 and lse = -inf.
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <type_traits>

namespace sp {
namespace {

struct DecodeArgs {
    const void* q; void* o; float* lse;
    const void* k_cache; const void* v_cache;
    const int* prompt_tables; const int* prompt_lens; const int* resp_tables; const int* resp_lens;
    int64_t prompt_width, resp_width, n_pages;
    int n_groups, n_seqs, Hq, Hkv, log_page;
    float scale;
    uint32_t* tag;
};

// One wave per row and q head, a key per lane and 64 keys at a time.
template <typename T, int D>
__global__ __launch_bounds__(256) void decode_kernel(TabArg starts, DecodeArgs a) {
    __shared__ float qs[4][D], ps[4][64];
    __shared__ int64_t rows[4][64];
    const int* const w = table_of(starts);
    const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    if (item >= (int64_t)a.n_seqs * a.Hq) return;
    const int seq = (int)(item / a.Hq), h = (int)(item % a.Hq), kvh = h / (a.Hq / a.Hkv);
    int lo = 0, hi = a.n_groups;
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (w[mid] <= seq) lo = mid; else hi = mid; }
    const int64_t Lr = max((int64_t)0, min((int64_t)a.resp_lens[seq], a.resp_width << a.log_page));
    const int64_t Lp = a.resp_lens[seq] < 0 || !a.prompt_tables ? 0 : max((int64_t)0, min((int64_t)a.prompt_lens[lo], a.prompt_width << a.log_page));
    for (int i = l; i < D; i += 64) qs[wave][i] = (float)((const T*)a.q)[item * D + i] * a.scale;
    __builtin_amdgcn_wave_barrier();
    float m = -3.402823466e38f, sum = 0.f, acc[D / 64] = {};
    for (int64_t j0 = 0; j0 < Lp + Lr; j0 += 64) {
        const int64_t j = j0 + l;
        int64_t row = -1;
        if (j < Lp + Lr) {
            const int64_t at = j < Lp ? j : j - Lp;
            const int page = j < Lp ? a.prompt_tables[lo * a.prompt_width + (at >> a.log_page)] : a.resp_tables[seq * a.resp_width + (at >> a.log_page)];
            if (page >= 0 && page < a.n_pages) row = ((((int64_t)page * a.Hkv + kvh) << a.log_page) + (at & ((1 << a.log_page) - 1))) * D;
        }
        float S = -INFINITY;
        if (row >= 0) {
            S = 0.f;
            for (int i = 0; i < D; ++i) S += qs[wave][i] * (float)((const T*)a.k_cache)[row + i];
        }
        float mx = S;
        for (int o = 32; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        const float mn = fmaxf(m, mx), p = __expf(S - mn), alpha = __expf(m - mn);
        float ts = p;
        for (int o = 32; o >= 1; o >>= 1) ts += __shfl_xor(ts, o, 64);
        sum = sum * alpha + ts;
        m = mn;
        ps[wave][l] = p;
        rows[wave][l] = row;
        __builtin_amdgcn_wave_barrier();
        for (int e = 0; e < D / 64; ++e) acc[e] *= alpha;
        for (int n = 0; n < 64; ++n)
            if (rows[wave][n] >= 0)
                for (int e = 0; e < D / 64; ++e) acc[e] += ps[wave][n] * (float)((const T*)a.v_cache)[rows[wave][n] + l + 64 * e];
        __builtin_amdgcn_wave_barrier();
    }
    for (int e = 0; e < D / 64; ++e) ((T*)a.o)[item * D + l + 64 * e] = (T)(sum > 0.f ? acc[e] / sum : 0.f);
    if (l == 0) a.lse[(int64_t)h * a.n_seqs + seq] = sum > 0.f ? m + __logf(sum) : -INFINITY;
}

}  // namespace

size_t decode_partial_bytes(int, int, int, int, int) { return 0; }

hipError_t launch_decode(const KvCache& cache, const void* q, void* o, float* lse, int Hq, int n_groups, int n_seqs, const TabArg& starts,
                         const int* prompt_tables, int prompt_width, const int* prompt_lens, const int* resp_tables, int resp_width,
                         const int* resp_lens, float scale, uint32_t* tag, float* partials, hipStream_t s) {
    DecodeArgs a{};
    a.q = q; a.o = o; a.lse = lse; a.k_cache = cache.k; a.v_cache = cache.v;
    a.prompt_tables = prompt_width > 0 ? prompt_tables : nullptr; a.prompt_lens = prompt_lens;
    a.resp_tables = resp_tables; a.resp_lens = resp_lens;
    a.prompt_width = prompt_width; a.resp_width = resp_width; a.n_pages = cache.n_pages;
    a.n_groups = n_groups; a.n_seqs = n_seqs; a.Hq = Hq; a.Hkv = cache.n_kv_heads; a.log_page = cache.log_page;
    a.scale = scale;
    a.tag = tag;
    const unsigned grid = (unsigned)(((int64_t)n_seqs * Hq + 3) / 4);
    auto launch = [&](auto elem, auto dim) {
        hipLaunchKernelGGL((decode_kernel<decltype(elem), decltype(dim)::value>), dim3(grid), dim3(256), 0, s, starts, a);
    };
    auto with_d = [&](auto elem) {
        if (cache.head_dim == 64) launch(elem, std::integral_constant<int, 64>{}); else launch(elem, std::integral_constant<int, 128>{});
    };
    if (cache.f32) with_d(float{}); else with_d(__bf16{});
    return hipGetLastError();
}

}  // namespace sp
