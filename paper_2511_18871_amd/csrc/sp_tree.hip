// Attention of drafted tokens that form trees, over the paged cache: several rows per sequence, each with the drafted tokens that it sees.
//   S_j = scale <q, k_j> over the prompt's keys, the sequence's own ahead of its drafted ones, and those drafted ones whose bit is set,
//   o = sum_j e^(S_j - m) v_j / l, l = sum_j e^(S_j - m), lse = m + ln l; without a key o = 0 and lse = -inf.
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <algorithm>

namespace sp {
namespace {

struct TreeArgs {
    const void* q; void* o; float* lse; const void* k_cache; const void* v_cache;
    const uint32_t* ancestors; int64_t mask_stride;
    const int* starts;                     // first token of each group, of each sequence; the number of tokens behind either
    const int* prompt_tables; const int* prompt_lens; const int* resp_tables; const int* resp_lens;
    int64_t prompt_width, resp_width, prompt_cap, resp_cap, n_pages;
    int n_groups, n_seqs, T, Hq, Hkv, rep, log_page;
    float c;
};

// One wave per token and q head: a lane scores one of 64 keys, then holds D / 64 elements of the output.
template <typename T, int D>
__global__ __launch_bounds__(64) void tree_kernel(TreeArgs a) {
    constexpr int E = D / 64;
    __shared__ float q[D], p[64];
    __shared__ int64_t at[64];
    const int l = threadIdx.x, tok = blockIdx.x, h = blockIdx.y, kvh = h / a.rep;
    auto find = [&](const int* w, int n) {
        int b = 0, e = n;
        while (e - b > 1) { const int mid = (b + e) >> 1; if (w[mid] <= tok) b = mid; else e = mid; }
        return b;
    };
    const int g = find(a.starts, a.n_groups);
    const int* const first = a.starts + a.n_groups + 1;
    const int s = find(first, a.n_seqs), node = tok - first[s], n = first[s + 1] - first[s];
    for (int e = l; e < D; e += 64) q[e] = (float)((const T*)a.q)[((int64_t)tok * a.Hq + h) * D + e];
    __syncthreads();
    float m = -3.4e38f / fmaxf(1.f, a.c), sum = 0.f, o[E];
    for (int i = 0; i < E; ++i) o[i] = 0.f;
    const int64_t own = a.resp_lens[s], base = own - n;
    const uint32_t* const row = a.ancestors ? a.ancestors + (int64_t)tok * a.mask_stride : nullptr;
    auto list = [&](const int* table, int64_t len, bool prompt) {
        for (int64_t j0 = 0; j0 < len; j0 += 64) {
            const int64_t j = j0 + l;
            int64_t k = -1;
            if (j < len) {
                const int64_t page = table[j >> a.log_page], i = j - base;
                const bool seen = prompt || i < 0 || (row ? row[i >> 5] >> (i & 31) & 1 : i <= node);
                if (seen && page >= 0 && page < a.n_pages) k = (((page * a.Hkv + kvh) << a.log_page) + (j & ((1 << a.log_page) - 1))) * D;
            }
            float x = -INFINITY;
            if (k >= 0) {
                x = 0.f;
                for (int e = 0; e < D; ++e) x += q[e] * (float)((const T*)a.k_cache)[k + e];
            }
            const float mn = fmaxf(m, wave_max(x)), alpha = __builtin_amdgcn_exp2f((m - mn) * a.c);
            const float w = k >= 0 ? __builtin_amdgcn_exp2f((x - mn) * a.c) : 0.f;
            m = mn;
            sum = sum * alpha + wave_sum(w);
            p[l] = w;
            at[l] = k;
            __syncthreads();
            for (int i = 0; i < E; ++i) o[i] *= alpha;
            for (int u = 0; u < 64; ++u)
                if (at[u] >= 0 && bits_of(p[u]) != 0)
                    for (int i = 0; i < E; ++i) o[i] += p[u] * (float)((const T*)a.v_cache)[at[u] + 64 * i + l];
            __syncthreads();
        }
    };
    if (own >= 0) {
        if (a.prompt_width) list(a.prompt_tables + g * a.prompt_width, min((int64_t)a.prompt_lens[g], a.prompt_cap), true);
        list(a.resp_tables + s * a.resp_width, min(own, a.resp_cap), false);
    }
    const bool none = bits_of(sum) == 0;
    for (int i = 0; i < E; ++i) ((T*)a.o)[((int64_t)tok * a.Hq + h) * D + 64 * i + l] = (T)(none ? 0.f : o[i] / sum);
    if (l == 0) a.lse[(int64_t)h * a.T + tok] = none ? -INFINITY : m * (a.c * LN2) + __logf(sum);
}

}  // namespace

hipError_t launch_tree(const KvCache& cache, const void* q, void* o, float* lse, int Hq, int n_groups, int n_seqs, int total, const int* starts,
                       const uint32_t* ancestors, int64_t mask_stride, const int* prompt_tables, int prompt_width, const int* prompt_lens,
                       const int* resp_tables, int resp_width, const int* resp_lens, float scale, hipStream_t s) {
    TreeArgs a{};
    a.q = q; a.o = o; a.lse = lse; a.k_cache = cache.k; a.v_cache = cache.v; a.ancestors = ancestors; a.mask_stride = mask_stride; a.starts = starts;
    a.prompt_tables = prompt_tables; a.prompt_lens = prompt_lens; a.resp_tables = resp_tables; a.resp_lens = resp_lens;
    a.prompt_width = prompt_width; a.resp_width = resp_width; a.n_pages = cache.n_pages;
    a.prompt_cap = std::min<int64_t>((int64_t)prompt_width << cache.log_page, MAX_TOKENS);
    a.resp_cap = std::min<int64_t>((int64_t)resp_width << cache.log_page, MAX_TOKENS);
    a.n_groups = n_groups; a.n_seqs = n_seqs; a.T = total; a.Hq = Hq; a.Hkv = cache.n_kv_heads; a.rep = Hq / cache.n_kv_heads; a.log_page = cache.log_page;
    a.c = scale * LOG2E;
    const dim3 grid((unsigned)total, (unsigned)Hq);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(64), 0, s, a); };
    if (cache.f32) { if (cache.head_dim == 64) launch(tree_kernel<float, 64>); else launch(tree_kernel<float, 128>); }
    else { if (cache.head_dim == 64) launch(tree_kernel<__bf16, 64>); else launch(tree_kernel<__bf16, 128>); }
    return hipGetLastError();
}

}  // namespace sp
