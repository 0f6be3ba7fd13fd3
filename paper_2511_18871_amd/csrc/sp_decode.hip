// Host side of the attention of one new token per sequence: what is launched for which lists (kernels: sp_decode.hpp).
#include "sp_decode.hpp"
#include <algorithm>
#include <type_traits>

namespace sp {
namespace {

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t desc_bytes(int n_groups, int n_seqs) { return up256(((size_t)n_groups + n_seqs + 1) * sizeof(i32x4)); }

// Rows of slots at most, whatever the groups' sizes: a slot per worker and one per segment of each kind.  Shared: a list of r rows has at
// most r / (64 nc) + 1 blocks of 64 nc <= 192 rows.
struct SlotRows { int64_t shared, prompts, responses; };
SlotRows slot_rows(int64_t n_groups, int64_t n_seqs, int64_t Hq, int64_t Hkv) {
    const int64_t rep = Hq / Hkv, all = n_seqs * rep, widest = std::min<int64_t>(64 * MAX_NC, (std::max(all, rep) + 63) / 64 * 64);
    const int64_t prompt_blocks = n_groups + all / SOLO_ROWS, resp_blocks = n_seqs * ((rep + SOLO_ROWS - 1) / SOLO_ROWS);
    SlotRows s;
    s.shared = all > SOLO_ROWS ? PLAN_WGS * widest + Hkv * (all + std::min(n_groups, all / (SOLO_ROWS + 1) + 1) * widest) : 0;
    if (rep > SOLO_ROWS) s.shared += Hkv * (all + n_seqs * widest);
    s.prompts = (4 * PLAN_WGS + Hkv * prompt_blocks) * std::min<int64_t>(SOLO_ROWS, all);
    s.responses = (4 * PLAN_WGS + Hkv * (prompt_blocks + resp_blocks)) * std::min<int64_t>(SOLO_ROWS, rep);
    return s;
}

}  // namespace

size_t decode_partial_bytes(int n_groups, int n_seqs, int Hq, int Hkv, int d) {
    const SlotRows s = slot_rows(n_groups, n_seqs, Hq, Hkv);
    const size_t rows = (size_t)(s.shared + s.prompts + s.responses);
    return desc_bytes(n_groups, n_seqs) + up256(rows * 8) + up256(rows * d * 4);
}

// units of all segments that the tables have room for
double decode_units(int n_groups, int n_seqs, int Hq, int Hkv, int64_t prompt_tokens, int64_t resp_tokens, const int32_t* Gs) {
    const double rep = Hq / Hkv;
    double units = 0;
    for (int g = 0; g < n_groups; ++g) units += ((double)prompt_tokens / 32 + 1) * ((Gs ? Gs[g] : 1) * rep / SOLO_ROWS + 1);
    return (units + ((double)resp_tokens / 32 + 1) * n_seqs * (rep / SOLO_ROWS + 1)) * Hkv;
}

hipError_t launch_decode(const KvCache& cache, const void* q, void* o, float* lse, int Hq, int n_groups, int n_seqs, const int32_t* Gs, const SeqArg& starts,
                         const int* prompt_tables, int prompt_width, const int* prompt_lens, const int* resp_tables, int resp_width,
                         const int* resp_lens, float scale, uint32_t* tag, void* partials, hipStream_t s) {
    DecodeArgs a{};
    a.q = q; a.o = o; a.lse = lse; a.k_cache = (const char*)cache.k; a.v_cache = (const char*)cache.v;
    a.prompt_tables = prompt_tables; a.prompt_lens = prompt_lens; a.resp_tables = resp_tables; a.resp_lens = resp_lens;
    a.prompt_width = prompt_width; a.resp_width = resp_width; a.n_pages = (int)cache.n_pages;
    a.n_groups = n_groups; a.n_seqs = n_seqs; a.Hq = Hq; a.Hkv = cache.n_kv_heads; a.rep = Hq / cache.n_kv_heads; a.log_page = cache.log_page;
    a.c = scale * LOG2E;
    a.m_none = -3.4e38f / fmaxf(1.f, a.c);
    a.tag = tag;
    const SlotRows slots = slot_rows(n_groups, n_seqs, Hq, a.Hkv);
    a.desc = (i32x4*)partials;
    a.stats = (float*)((char*)partials + desc_bytes(n_groups, n_seqs));
    a.sums = a.stats + up256((size_t)(slots.shared + slots.prompts + slots.responses) * 8) / 4;
    a.prompt_base = slots.shared;
    a.resp_base = slots.shared + slots.prompts;
    // Row tiles per wave if the rows of a shared list are dealt to as few workgroups as can hold them, as every workgroup reads the keys.  No
    // more than that: they are all computed (8 sequences of 7 heads to a kv head: 8.2 us with one, 10.7 with three).
    const bool prompts = prompt_width > 0;
    auto rows_of = [&](int g) { return (int64_t)a.rep * (Gs ? Gs[g] : 1); };
    a.nc = 1;
    auto widen = [&](int64_t rows) {
        if (rows <= SOLO_ROWS || cache.f32) return;
        const int64_t tiles = (rows + 15) / 16, blocks = (tiles + 4 * MAX_NC - 1) / (4 * MAX_NC), per = (tiles + blocks - 1) / blocks;
        a.nc = std::max(a.nc, (int)((per + 3) / 4));
    };
    for (int g = 0; prompts && g < n_groups; ++g) widen(rows_of(g));
    widen(a.rep);
    // rows of a slot, and workgroups: as many as units that the tables have room for, or as the units are dealt to
    double units_shared = 0, units_solo = 0;
    auto count = [&](int64_t rows, int64_t lists, double tokens, int& solo_rows) {
        if (rows > SOLO_ROWS && !cache.f32) {
            const int64_t tiles = (rows + 15) / 16, blocks = (rows + 64 * a.nc - 1) / (64 * a.nc);
            a.shared_rows = std::max(a.shared_rows, (int)(16 * ((tiles + blocks - 1) / blocks)));
            units_shared += (double)lists * blocks * (tokens / 64 + 1) * a.Hkv;
        } else {
            solo_rows = std::max(solo_rows, (int)std::min<int64_t>(rows, SOLO_ROWS));
            units_solo += (double)lists * ((rows + SOLO_ROWS - 1) / SOLO_ROWS) * (tokens / 32 + 1) * a.Hkv;
        }
    };
    for (int g = 0; prompts && g < n_groups; ++g) count(rows_of(g), 1, (double)prompt_width * (1 << a.log_page), a.prompt_rows);
    count(a.rep, n_seqs, (double)resp_width * (1 << a.log_page), a.resp_rows);
    const unsigned grid = (unsigned)std::min<double>(PLAN_WGS, units_shared + units_solo / 4 + 1);
    a.shared_cost = a.nc == 1 ? 3.f : a.nc == 2 ? 4.f : 5.5f;        // from their instructions; the 16k prompt takes 47 to 49 us with anything from 0.8 to 9
    a.kv_heads = make_div(a.Hkv);
    a.q_heads = make_div(Hq);
    a.heads_each = make_div(a.rep);
    a.block_rows = make_div(64 * a.nc);
    a.prompt_cap = (int)std::min<int64_t>((int64_t)prompt_width << a.log_page, MAX_TOKENS);
    a.resp_cap = (int)std::min<int64_t>((int64_t)resp_width << a.log_page, MAX_TOKENS);
    a.members = Gs ? Gs[0] : 1;
    for (int g = 1; Gs && g < n_groups; ++g) if (Gs[g] != Gs[0]) a.members = 0;
    a.group_size = make_div(std::max(1, a.members));
    auto launch = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        auto with_lists = [&](auto many) {
            constexpr bool MANY = decltype(many)::value;
            auto with = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, starts, a); };
            auto with_solo = [&](auto ns) {
                constexpr int NS = decltype(ns)::value;
                if (units_shared == 0) with(decode_kernel<D, 0, NS, MANY>);
                else if (a.nc == 1) with(decode_kernel<D, 1, NS, MANY>);
                else if (a.nc == 2) with(decode_kernel<D, 2, NS, MANY>);
                else with(decode_kernel<D, 3, NS, MANY>);
            };
            // one row tile per wave where 16 rows are the most (one sequence 5.7 us, with two tiles 6.5)
            if (cache.f32) with(decode_f32_kernel<D, MANY>);
            else if (std::max(a.prompt_rows, a.resp_rows) <= 16) with_solo(std::integral_constant<int, 1>{});
            else with_solo(std::integral_constant<int, 2>{});
        };
        if (n_groups + n_seqs > 64) with_lists(std::true_type{}); else with_lists(std::false_type{});
        auto join = [&](auto dense) {
            const int64_t each = decltype(dense)::value ? 1024 / D : 4;
            const unsigned joins = (unsigned)(((int64_t)n_seqs * Hq + each - 1) / each);
            if (cache.f32) hipLaunchKernelGGL((decode_join_kernel<float, D, decltype(dense)::value>), dim3(joins), dim3(256), 0, s, starts, a);
            else hipLaunchKernelGGL((decode_join_kernel<__bf16, D, decltype(dense)::value>), dim3(joins), dim3(256), 0, s, starts, a);
        };
        // More items than the chip holds waves (8192): most then have a few rows only.  (28.7k items of two or three: 13 us against 19; 1280 items
        // of 40: 12 against 9.)
        if ((int64_t)n_seqs * Hq > 8192) join(std::true_type{}); else join(std::false_type{});
    };
    if (cache.head_dim == 64) launch(std::integral_constant<int, 64>{}); else launch(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace sp
