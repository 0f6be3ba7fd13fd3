// Attention of drafted tokens that form trees, over the paged cache: several rows per sequence, each with the drafted tokens that it sees.
//   S_j = scale <q, k_j> over the prompt's keys, the sequence's own ahead of its drafted ones, and those drafted ones whose bit is set,
//   o = sum_j e^(S_j - m) v_j / l, l = sum_j e^(S_j - m), lse = m + ln l; without a key o = 0 and lse = -inf.
//
// The kernels are those of one new token per sequence (sp_decode.hpp) with more rows to a list: a prompt is seen by the drafted tokens of all its
// sequences, a response by those of its own.  Only units of keys that hold drafted tokens look at the mask.
//
// Bound: the keys and values, read once for a list's rows as long as these are few; the matrix instructions from some hundred rows on; for a few
// sequences latency.  Measured (heads of 128, bf16, us of the kernel + of the join, medians of traced launches):
//   chunks of 192 to 256 tokens behind 4k to 8k, 32/8 heads     156 + 14   101 GFLOP, 650 TFLOP/s; matrix units are busy for 28 % of its cycles at 2.4 GHz, in the 16k prompt for 29
//   a prompt of 16k tokens, 32 answers, trees of 8, 40/8        124 + 10   87 GFLOP, 700 TFLOP/s
//   64 prompts of 64 to 192 tokens, 16 answers each, 3 to 5 drafted tokens, 28/4   177 + 39   0.84 GB read, 4.8 TB/s; half the rows are finished by one worker
//   a prompt of 1k tokens, 8 answers, trees of 16, 28/4         20 + 5     latency: plan, pages, first keys, code that comes from memory once
//   one sequence of 1k tokens, a tree of 8, 28/4                11 + 6     the same
#include "sp_decode.hpp"
#include <algorithm>
#include <type_traits>

namespace sp {
namespace {

constexpr int FEW_UNITS = 8192, SHORT_LIST = 512;      // below: which lists waves take by themselves

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t desc_bytes(int64_t lists) { return up256(((size_t)lists + 1) * sizeof(i32x4)); }

// Rows of slots at most, whatever the sequences' counts.  A worker leaves a slot per segment and one more for each worker that shares it.  A shared
// list of r rows takes at most r + 15 for its segments of a kv head; a solo one has blocks of 16 rows or more.
struct SlotRows { int64_t shared, prompts, responses; };
SlotRows slot_rows(int64_t n_groups, int64_t n_seqs, int64_t total, int64_t Hq, int64_t Hkv, bool f32) {
    const int64_t all = total * (Hq / Hkv), widest = std::min<int64_t>(WIDE_ROWS, (all + 15) / 16 * 16), solo = std::min<int64_t>(f32 ? SOLO_ROWS : TREE_SOLO_ROWS, all);
    const int64_t more = all / SOLO_ROWS;      // blocks of solo lists beyond the first
    SlotRows s;
    s.shared = !f32 && all > TREE_SOLO_ROWS ? PLAN_WGS * widest + Hkv * (2 * all + 16 * std::min(n_groups + n_seqs, 2 * all / (TREE_SOLO_ROWS + 1) + 1)) : 0;
    s.prompts = (4 * PLAN_WGS + Hkv * (n_groups + more)) * solo;
    s.responses = (4 * PLAN_WGS + Hkv * (n_groups + n_seqs + 2 * more)) * solo;
    return s;
}

}  // namespace

size_t tree_partial_bytes(int n_groups, int n_seqs, int64_t total, int Hq, int Hkv, int d, bool f32) {
    const SlotRows s = slot_rows(n_groups, n_seqs, total, Hq, Hkv, f32);
    const size_t rows = (size_t)(s.shared + s.prompts + s.responses);
    return desc_bytes((int64_t)n_groups + n_seqs) + up256(rows * 16) + up256(rows * d * 4);
}

size_t tree_table_bytes(int n_groups, int n_seqs) { return up256(((size_t)n_groups + n_seqs + 2) * 4); }

// units of 32 keys by 32 rows that the tables have room for
double tree_units(int n_groups, int n_seqs, int Hq, int Hkv, int64_t prompt_tokens, int64_t resp_tokens, const int32_t* starts) {
    const double rep = Hq / Hkv;
    double units = 0;
    for (int g = 0; g < n_groups; ++g) units += ((double)prompt_tokens / 32 + 1) * ((starts[g + 1] - starts[g]) * rep / SOLO_ROWS + 1);
    const int32_t* const first = starts + n_groups + 1;
    for (int s = 0; s < n_seqs; ++s) units += ((double)resp_tokens / 32 + 1) * ((first[s + 1] - first[s]) * rep / SOLO_ROWS + 1);
    return units * Hkv;
}

hipError_t launch_tree(const KvCache& cache, const void* q, void* o, float* lse, int Hq, int n_groups, int n_seqs, const int32_t* Gs, int total, const int32_t* starts, int* dev_starts,
                       const uint32_t* ancestors, int64_t mask_stride, const int* prompt_tables, int prompt_width, const int* prompt_lens,
                       const int* resp_tables, int resp_width, const int* resp_lens, float scale, uint32_t* tag, void* partials, hipStream_t s) {
    DecodeArgs a{};
    a.q = q; a.o = o; a.lse = lse; a.k_cache = (const char*)cache.k; a.v_cache = (const char*)cache.v;
    a.prompt_tables = prompt_tables; a.prompt_lens = prompt_lens; a.resp_tables = resp_tables; a.resp_lens = resp_lens;
    a.prompt_width = prompt_width; a.resp_width = resp_width; a.n_pages = (int)cache.n_pages;
    a.n_groups = n_groups; a.n_seqs = n_seqs; a.n_tok = total; a.Hq = Hq; a.Hkv = cache.n_kv_heads; a.rep = Hq / cache.n_kv_heads; a.log_page = cache.log_page;
    a.ancestors = ancestors; a.mask_stride = mask_stride;
    a.c = scale * LOG2E;
    a.m_none = -3.4e38f / fmaxf(1.f, a.c);
    a.tag = tag;
    const SlotRows slots = slot_rows(n_groups, n_seqs, total, Hq, a.Hkv, cache.f32);
    a.desc = (i32x4*)partials;
    a.stats = (float*)((char*)partials + desc_bytes((int64_t)n_groups + n_seqs));
    a.sums = a.stats + up256((size_t)(slots.shared + slots.prompts + slots.responses) * 16) / 4;
    a.prompt_base = slots.shared;
    a.resp_base = slots.shared + slots.prompts;
    // Groups and sequences of one count need no table of where they start
    const int32_t* const first = starts + n_groups + 1;
    a.members = starts[1] - starts[0];
    a.each = first[1] - first[0];
    for (int g = 1; g < n_groups; ++g) if (starts[g + 1] - starts[g] != a.members) a.members = 0;
    for (int i = 1; i < n_seqs; ++i) if (first[i + 1] - first[i] != a.each) a.each = 0;
    if (a.each == 0) a.members = 0;
    a.group_size = make_div(std::max(1, a.members));
    a.seq_size = make_div(std::max(1, a.each));
    TreeArg table;
    table.dev = nullptr;
    const int n_words = n_groups + n_seqs + 2;
    if (!a.members && n_words <= TREE_WORDS && total <= 0xffff) {
        for (int i = 0; i < n_words; ++i) table.words[i] = (uint16_t)starts[i];
    } else if (!a.members) {
        table.dev = dev_starts;
        const hipError_t e = launch_prepare(starts, n_words, dev_starts, tag, ReserveTag{}, TAG_CLEAR, false, n_groups, total, 0, 0, Schedule{}, KEYS_AS_PACKED, s);
        if (e != hipSuccess) return e;
    }
    bool groups_alike = true;              // of as many sequences
    for (int g = 1; Gs && g < n_groups; ++g) groups_alike = groups_alike && Gs[g] == Gs[0];
    a.group_seqs = make_div(std::max(1, Gs ? Gs[0] : 1));
    // Prompts ahead of their sequences' own keys, in one list: a row then leaves one set of sums, or none, in place of two, and a prompt is read for each of its
    // sequences, from the caches.  Where that is little, or up to eight times what the sums are (64 prompts of 64 to 192 tokens with 16 answers each, 28/4 heads: 242 ->
    // 216 us; 32 chains of 150 tokens behind prompts of 700, 32/8: 199 -> 146; 22 prompts of 400 with 18 answers, heads of 64, at the limit: 138 -> 141; a prompt of 16k
    // tokens with 32 answers 118 -> 254, hence not there).
    const double again = (double)(n_seqs - n_groups) * ((double)prompt_width * (1 << a.log_page)) * a.Hkv * 2 * cache.head_dim * 2;
    const double sums = (double)total * Hq * (4 * cache.head_dim + 16) * 2;
    a.joined = prompt_width > 0 && !cache.f32 && groups_alike && (again <= 32e6 || again <= 8 * sums);
    const int n_lists = n_groups + n_seqs;
    // (prompts, then responses)
    auto rows_of = [&](int i) { const int k = i < n_groups ? i : i + 1; return (int64_t)a.rep * (starts[k + 1] - starts[k]); };
    // Which lists are shared.  A segment of many rows costs a workgroup three units beside its own, and code that comes from memory once: not where all lists are
    // few units of 32 keys by 32 rows (one sequence of 1k tokens with 8 drafted ones, 28/4 heads: 17.2 -> 15.8 us), nor those whose tables hold few keys (64 prompts
    // of 64 to 192 tokens with 16 answers each: 245 -> 241 us; chunks of 150 tokens behind 700: 223 us without, 195 with, hence no more than that).
    constexpr int NEVER = 0x7fffffff;
    auto tokens_of = [&](int i) { return ((double)(i < n_groups ? prompt_width : resp_width) + (a.joined ? prompt_width : 0)) * (1 << a.log_page); };
    auto units_of = [&](int from) {        // of 32 keys by 32 rows that the tables of lists `from` ... have room for
        double units = 0;
        for (int i = from; i < n_lists; ++i) units += (tokens_of(i) / 32 + 1) * ((double)rows_of(i) / SOLO_ROWS + 1) * a.Hkv;
        return units;
    };
    a.joined = a.joined && units_of(n_groups) <= 2e9;
    const bool prompts = prompt_width > 0 && !a.joined;      // as lists of their own
    a.direct = !prompts && !cache.f32;
    const double units = units_of(prompts ? 0 : n_groups);
    const bool few = units <= FEW_UNITS;
    a.wide_prompts = cache.f32 || few || tokens_of(0) < SHORT_LIST ? NEVER : TREE_SOLO_ROWS;
    a.wide_resps = cache.f32 || few || tokens_of(n_groups) < SHORT_LIST ? NEVER : TREE_SOLO_ROWS;
    double units_shared = 0, units_solo = 0, units_256 = 0, weighted = 0;
    int solo_most = 0;                     // rows of the largest solo list
    for (int i = prompts ? 0 : n_groups; i < n_lists; ++i) {
        const int64_t rows = rows_of(i);
        if (rows > (i < n_groups ? a.wide_prompts : a.wide_resps)) {
            const double keys = tokens_of(i) / 64 + 1, more = (double)((rows + 127) / 128) * keys * a.Hkv;
            a.shared_rows = std::max(a.shared_rows, (int)std::min<int64_t>(WIDE_ROWS, (rows + 15) / 16 * 16));
            units_shared += more;
            units_256 += (double)((rows + 255) / 256) * keys * a.Hkv;
            weighted += more * keys;
        } else {
            solo_most = std::max(solo_most, (int)std::min<int64_t>(rows, TREE_SOLO_ROWS + 1));
            units_solo += (double)((rows + SOLO_ROWS - 1) / SOLO_ROWS) * (tokens_of(i) / 32 + 1) * a.Hkv;
        }
    }
    // tiles of 16 rows of a solo wave: as many as the largest such list has; of lists in several blocks three (241 us for those prompts, with two 262), or
    // two where units are few
    const int ns = cache.f32 ? 2 : solo_most > TREE_SOLO_ROWS ? (few ? 2 : 3) : std::max(1, (solo_most + 15) / 16);
    a.solo_rows = make_div(16 * ns);
    for (int i = prompts ? 0 : n_groups; i < n_lists; ++i) {
        if (rows_of(i) > (i < n_groups ? a.wide_prompts : a.wide_resps)) continue;
        int& solo = i < n_groups ? a.prompt_rows : a.resp_rows;
        solo = std::max(solo, (int)std::min<int64_t>(rows_of(i), 16 * ns));
    }
    // Workgroups of eight waves, where that leaves few of 256 rows empty and segments are long: they read keys and values half as often, but there is one to
    // a CU.  (4 chunks of 192 to 256 tokens behind 4k to 8k, 32/8 heads: 160 -> 150 us; a prompt of 1k tokens with 8 trees of 16, runs of two units: 27.5 us either way; 22
    // groups of short prompts 130 -> 177.)
    const bool eight = a.shared_rows && 2 * units_256 <= 1.2 * units_shared && weighted >= 32 * units_shared;
    const int nw = eight ? 8 : 4;
    a.shared_rows = std::min(a.shared_rows, 32 * nw);
    const unsigned grid = (unsigned)std::min<double>(4 * PLAN_WGS / nw, units_shared + units_solo / nw + 1);
    a.shared_cost = 2.f;                   // (64 short prompts with 16 answers each, all prompts shared: 1: 303 us, 2 and 4: 245; long answers beside a long prompt 104, 98, 108)
    a.kv_heads = make_div(a.Hkv);
    a.q_heads = make_div(Hq);
    a.heads_each = make_div(a.rep);
    a.block_rows = make_div(32 * nw);
    a.prompt_cap = (int)std::min<int64_t>((int64_t)prompt_width << a.log_page, MAX_TOKENS);
    a.resp_cap = (int)std::min<int64_t>((int64_t)resp_width << a.log_page, MAX_TOKENS);
    auto launch = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        auto with_lists = [&](auto many) {
            constexpr bool MANY = decltype(many)::value;
            auto with = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * (eight ? 8 : 4)), 0, s, table, a); };
            auto with_solo = [&](auto ns) {
                constexpr int NS = decltype(ns)::value;
                if (units_shared == 0) with(decode_kernel<D, 0, NS, MANY, true>);
                else if (eight) with(decode_kernel<D, 1, NS, MANY, true, 8>);
                else with(decode_kernel<D, 1, NS, MANY, true>);
            };
            if (cache.f32) with(decode_f32_kernel<D, MANY, true>);
            else if (ns == 1) with_solo(std::integral_constant<int, 1>{});
            else if (ns == 2) with_solo(std::integral_constant<int, 2>{});
            else with_solo(std::integral_constant<int, 3>{});
        };
        if (n_lists > 64) with_lists(std::true_type{}); else with_lists(std::false_type{});
        auto join = [&](auto dense) {
            const int64_t each = decltype(dense)::value ? 1024 / D : 4;
            const unsigned joins = (unsigned)(((int64_t)total * Hq + each - 1) / each);
            if (cache.f32) hipLaunchKernelGGL((decode_join_kernel<float, D, decltype(dense)::value, true>), dim3(joins), dim3(256), 0, s, table, a);
            else hipLaunchKernelGGL((decode_join_kernel<__bf16, D, decltype(dense)::value, true>), dim3(joins), dim3(256), 0, s, table, a);
        };
        if ((int64_t)total * Hq > 8192) join(std::true_type{}); else join(std::false_type{});
    };
    if (cache.head_dim == 64) launch(std::integral_constant<int, 64>{}); else launch(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace sp
