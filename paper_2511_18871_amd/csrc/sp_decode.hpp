// Attention of one new token per sequence over the paged cache: the shared-prompt attention of Section 4.3 in the form of a rollout
// step.  The G sequences of a group read the pages of their common prompt, and each the pages of its own response.
//   S_j = scale <q, k_j> over the keys [0, Lp) of the prompt and [0, len) of the response,
//   o = sum_j e^(S_j - m) v_j / l, l = sum_j e^(S_j - m), lse = m + ln l; without a key o = 0 and lse = -inf.
//
// Bound: the keys and values, each read once.  (A prompt seen by more than 192 rows in bf16, 32 in float32, is read once for each block of as many: by
// workgroups that run side by side, so that memory is left alone, but the caches and the instructions are not.)  A LIST is what is walked together: the prompt of a group, seen by its G rep rows of
// each kv head (rep = n_q_heads / n_kv_heads; row r is q head r % rep of the group's sequence r / rep), or the response of a
// sequence, seen by its rep rows.  The units of keys of all lists lie one behind the other (list by list, in it block of rows by
// block, kv head by kv head: a SEGMENT each), and every worker takes an equal run of them, across segments: no worker waits for a
// longer one.  Where a worker leaves a segment it leaves unnormalised sums (m, l, sum p v) of its rows in the workspace; the join kernel adds up
// those of a row.  Lengths are on the device, so the dealing happens there, by every workgroup for itself.
//
// Products on matrix instructions of 16 x 16: S^T = K Q^T (keys x rows) leaves a lane with scores of one row, four keys in turn, and
// these are, rounded, the operand of O^T += V^T P^T as they stand, if the keys of V are taken in the same order.
//   a list of at most 32 rows   the worker is a wave: units of 32 keys through 16 KB of LDS of its own, no barriers
//   more rows                   the worker is a workgroup: its four waves share units of 64 keys and have up to 16 NC rows each
//
// Measured (heads of 128, bf16, us of the kernel + of the join; bytes are those of the keys and values):
//   32 answers of 8k to 15k tokens to 8 prompts, 32/8 heads   263 + 5     1.53 GB, 5.8 TB/s
//   64 prompts of 64 to 192 tokens, 16 answers each, 28/4     131 + 11    0.55 GB, 4.2 TB/s; the plan of 1088 lists takes 8 of it
//   a prompt of 16k tokens, 32 answers, 40/8                  38 + 9      91 MB; 36 MB of sums, written and read, take nearly as long
//   a prompt of 1k tokens, 8 answers, 28/4                    8 + 5       latency: launch, plan, pages, keys, sums one after the other
//   one sequence of 1k tokens, 28/4                           6 + 6       the same
// Whole calls: a prompt of 4k tokens, 32 answers, 28/4, 24 us (19 MB) and in float32, in seven blocks, 53 us (39 MB); in float32 8 sequences of 7k to 8k
// tokens, 32/8, 115 us (497 MB, 4.3 TB/s).
#pragma once
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <algorithm>
#include <type_traits>

namespace sp {
namespace {

#define SP_INLINE __attribute__((always_inline))      // lambdas: what they refer to has to stay in registers

constexpr int SOLO_ROWS = 32;              // rows of a segment that a wave takes by itself
// Drafted tokens
constexpr int WIDE_ROWS = 256;             // rows that a workgroup takes at most: 32 to a wave
constexpr int TREE_SOLO_ROWS = 48;         // rows of a list that a wave takes by itself where other lists are shared (bf16)
// Units that a worker takes at least, where few segments are dealt to many: it leaves 64 KB of sums or more, and pays its plan and first loads, whatever the run (a prompt
// of 1k tokens with 8 trees of 16: 28.0 us at 2, 24.9 at 3, 25.4 at 4, 26.7 at 6)
constexpr unsigned LEAST_RUN = 3;
constexpr int WIDE_PAD = 3;                // units that a segment of many rows costs beside its own: first loads, last product, sums
constexpr int MAX_NC = 3;                  // row tiles of 16 of a wave that shares its keys: 192 rows to a workgroup
constexpr int PLAN_WGS = 512;              // workgroups that the units are dealt to: two to a CU (one: 131 -> 164 us for the 64 prompts above)

typedef float f32x2 __attribute__((ext_vector_type(2)));

struct DecodeArgs {
    const void* q; void* o; float* lse;
    const char* k_cache; const char* v_cache;
    const int* prompt_tables; const int* prompt_lens; const int* resp_tables; const int* resp_lens;
    int64_t prompt_width, resp_width;
    int prompt_cap, resp_cap;              // tokens that a table holds (at most MAX_TOKENS)
    int members;                           // sequences of each group, 0: of several sizes
    int n_pages, n_groups, n_seqs, Hq, Hkv, rep, log_page;
    // Drafted tokens (kernels with TREE): rows belong to tokens in place of sequences
    int n_tok, each;                       // tokens; of each sequence, 0: of several counts
    Div seq_size;                          // of `each`
    const uint32_t* ancestors;             // a row per token, NULL: a chain
    int64_t mask_stride;
    Div solo_rows;                         // rows of a block of a solo list
    int wide_prompts, wide_resps;          // prompts, responses with more rows than this are shared
    // joined: a sequence's list is its prompt and behind it its own keys, and prompts are no lists; groups are of `group_seqs` sequences.  direct: a row
    // whose keys one worker has seen goes to o and lse at once
    bool joined, direct;
    Div group_seqs;
    int nc;                                // row tiles per wave of a shared segment
    float shared_cost;                     // of a shared unit, against a solo one
    Div group_size, block_rows;            // of `members`, of the rows of a shared segment (64 nc)
    Div kv_heads, q_heads, heads_each;     // of Hkv, Hq, rep
    float c, m_none;                       // softmax_scale * log2(e); reference point of a row that has not seen a key
    uint32_t* tag;
    i32x4* desc;                           // [0]: units of a worker, shared and solo; [1 + i], of list i: room ahead of it among its kind, units
                                           // of a segment, blocks ahead of it among its kind, room of a segment (-1: takes no part)
    // Slots of sums.  Worker w's sums of segment s (both counted within their kind) lie in slot w + s: either grows by one at a time.
    int shared_rows, prompt_rows, resp_rows;                 // rows of a slot of shared lists, and of solo prompts and responses
    int64_t prompt_base, resp_base;                          // first row of the solo prompts' slots, of the responses'
    float* stats;                          // per row of a slot: m, l
    float* sums;                           // per row: sum p v
};

__device__ const i32x4 zero_granule = {0, 0, 0, 0};      // what keys that are not there read

// ---- the plan --------------------------------------------------------------------------------------------

// inclusive sums over the lanes of a wave
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_add(int x) {
    return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int scan64(int x) {
    x = dpp_add<0x111, 0xf>(x); x = dpp_add<0x112, 0xf>(x); x = dpp_add<0x114, 0xf>(x); x = dpp_add<0x118, 0xf>(x);      // within 16 lanes
    x = dpp_add<0x142, 0xa>(x); return dpp_add<0x143, 0xc>(x);                                                      // across them
}
struct ListShape {                        // units of keys of a segment, `ahead` of them of the prompt (TREE); blocks of rows
    int rows, len, units, blocks, ahead; bool shared;
    // what a list adds to `ord`: its blocks, a shared list of drafted tokens its row tiles of 16
    template <bool TREE> __device__ __forceinline__ int places() const {
        if constexpr (TREE) { if (shared) return (rows + 15) >> 4; }
        return blocks;
    }
};
template <int NW> struct PlanShare { int sums[NW][5]; int list[NW], at[NW], ord[NW], rows[NW], len[NW], room[NW], ahead[NW]; };      // of the waves of a workgroup; where their runs start

// First tokens of the groups, the number of tokens, first tokens of the sequences, and that number again: in 16 bits among the kernel's arguments, or in
// the workspace.  (A table that is stored by a launch of its own costs 5 us for each 896 words.)
constexpr int TREE_WORDS = 1600;
struct TreeArg { const int* dev; uint16_t words[TREE_WORDS]; };
struct TreeStarts {
    const int* dev;
    const uint16_t* arg;
    __device__ __forceinline__ int operator[](int i) const { return dev ? dev[i] : arg[i]; }
};
__device__ __forceinline__ TreeStarts words_of(const TreeArg& t) {
    const uint64_t at = (uint64_t)(uintptr_t)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(TreeArg, words);
    return TreeStarts{t.dev, (const uint16_t*)(const __attribute__((address_space(4))) uint16_t*)at};
}
template <bool TREE> using StartsArg = std::conditional_t<TREE, TreeArg, SeqArg>;
template <bool TREE> using Starts = std::conditional_t<TREE, TreeStarts, const int*>;

// KIND 0: all lists are solo, 1: shared ones too.  TREE: a sequence has several rows per q head, one for each of its drafted tokens; `members` are
// the tokens of a group.
template <bool TREE> using ListIs = std::conditional_t<TREE, i32x4, i32x2>;      // rows, length; TREE: tokens of the prompt ahead of it
template <int KIND, bool TREE = false>
struct Lists {
    Starts<TREE> starts;                     // first sequence (token) of each group, where groups are of several sizes
    const DecodeArgs& a;
    // token counts of a list's rows and where they start (TREE)
    __device__ __forceinline__ int tokens(int i) const {
        const bool prompt = i < a.n_groups;
        if (a.members) return prompt ? a.members : a.each;
        const int k = prompt ? i : i + 1;
        return starts[k + 1] - starts[k];
    }
    __device__ __forceinline__ ListIs<TREE> read(int i) const {      // length -1: takes no part
        const bool prompt = i < a.n_groups;
        const int prompt_cap = a.prompt_cap, resp_cap = a.resp_cap;
        const int* const prompt_lens = a.prompt_lens;
        const int* const resp_lens = a.resp_lens - a.n_groups;
        const int n = prompt && !prompt_cap ? 0 : (prompt ? prompt_lens : resp_lens)[i];
        int members = 1;
        if constexpr (TREE) {
            if (a.joined && prompt) return i32x4{0, 0, 0, 0};
            members = tokens(i);
            const int len = min(max(n, -1), prompt ? prompt_cap : resp_cap);
            int ahead = 0;
            if (a.joined && len >= 0) {
                unsigned rest;
                ahead = min(max(prompt_lens[divmod((unsigned)(i - a.n_groups), a.group_seqs, rest)], 0), prompt_cap);
            }
            return i32x4{a.rep * members, len, ahead, 0};
        } else if (prompt) members = a.members ? a.members : starts[i + 1] - starts[i];
        if constexpr (!TREE) return i32x2{a.rep * members, min(max(n, -1), prompt ? prompt_cap : resp_cap)};
    }
    __device__ __forceinline__ ListShape shape(ListIs<TREE> x, int i) const {
        ListShape s;
        s.rows = x[0];
        s.len = x[1];
        s.shared = KIND && s.rows > (!TREE ? SOLO_ROWS : i < a.n_groups ? a.wide_prompts : a.wide_resps);
        auto units = [&](int n) { return n > 0 ? (int)(((unsigned)n + (s.shared ? 63u : 31u)) >> (s.shared ? 6 : 5)) : 0; };
        s.units = s.rows > 0 ? units(s.len) : 0;
        s.ahead = 0;
        if constexpr (TREE) { if (s.rows > 0) s.ahead = units(x[2]); s.units += s.ahead; }
        unsigned rest;
        if constexpr (TREE) s.blocks = s.rows <= 0 ? 0 : (int)divmod((unsigned)(s.rows - 1), s.shared ? a.block_rows : a.solo_rows, rest) + 1;
        else s.blocks = s.shared ? (int)divmod((unsigned)(s.rows - 1), a.block_rows, rest) + 1 : (s.rows + SOLO_ROWS - 1) / SOLO_ROWS;
        return s;
    }
    __device__ __forceinline__ int first_seq(int i) const {      // TREE: its first token
        if constexpr (TREE) return a.members ? (i >= a.n_groups ? (i - a.n_groups) * a.each : i * a.members) : starts[i >= a.n_groups ? i + 1 : i];
        else return i >= a.n_groups ? i - a.n_groups : a.members ? i * a.members : starts[i];
    }
};

// ceil(total / places), total < 2^31, places > 0: a float quotient that is low by 2^-20 at most, what it leaves divided in the same way, and
// what that leaves, which is below two places
__device__ __forceinline__ unsigned per_place(unsigned total, unsigned places) {
    const float inv = __builtin_amdgcn_rcpf((float)places) * 0.999999f;
    unsigned c = (unsigned)((float)total * inv);
    c += (unsigned)((float)(total - c * places) * inv);
    c += c * places < total;
    c += c * places < total;
    return max(c, 1u);
}
// floor(x / d), x < 2^31: a float quotient that is low by 2^-20 at most, what it leaves divided in the same way, and that is short by one at most
__device__ __forceinline__ unsigned quotient(unsigned x, unsigned d) {
    const float inv = __builtin_amdgcn_rcpf((float)d) * 0.999999f;
    unsigned q = (unsigned)((float)x * inv);
    q += (unsigned)((float)(x - q * d) * inv);
    return q + (x - q * d >= d);
}
// units of room that a segment has among those of its kind
template <bool TREE> __device__ __forceinline__ int room_of(int units, unsigned run, bool aligned) {
    return units <= 0 ? units : aligned ? (int)(per_place(units, run) * run) : TREE ? units + WIDE_PAD : units;
}

// What a worker does: `left` units from unit `at` of a list on (counted over the list's segments).
template <bool TREE> struct Work { bool shared; int worker, list, at, ord, left, room, pad; ListIs<TREE> list_is; };      // pad: units of a segment's room that are none

// The runs of either kind, from the units and segments of all lists.  Places are dealt by cost: a segment costs, for its rows and its sums, what one and a half of its
// units (shared) or one (solo) cost, and a shared unit what shared_cost solo ones do.  A worker that passes from one segment to another takes
// longer; where shared segments are long against the run, each is dealt to workers of its own, in room that is a multiple of the run (`aligned`: 37.8 us
// for the prompt of 16k tokens, 41.4 without).
struct Runs { unsigned shared_run, solo_run, used; bool aligned; };      // used: workgroups of shared segments
template <int KIND, bool TREE, int WGS>
__device__ __forceinline__ void shared_runs(const DecodeArgs& a, unsigned solo, unsigned solo_segs, unsigned shared, unsigned segs, Runs& r) {
    r = Runs{1, 1, 0, false};
    if constexpr (KIND) {
        if (shared == 0) return;
        const float cost = a.shared_cost * ((float)shared + (TREE ? (float)WIDE_PAD : 1.5f) * (float)segs);
        int wgs = (int)(WGS * (cost * __builtin_amdgcn_rcpf(cost + (float)solo + (float)solo_segs)));
        wgs = max(1, min(wgs, solo ? WGS - 1 : WGS));
        r.aligned = 4 * segs <= (unsigned)wgs;
        r.shared_run = r.aligned ? per_place(shared, wgs - segs) : per_place(shared + (TREE ? WIDE_PAD * segs : 0), wgs);
        if (TREE && r.aligned) r.shared_run = max(r.shared_run, LEAST_RUN);
    }
}

// Which run of the shared units a workgroup takes.  Drafted tokens: consecutive runs go to one XCD (workgroups are dealt round-robin over the 8), and
// the segments of a kv head lie one behind the other, so that the workgroups that read a head's keys for different rows find them in one L2.
template <bool TREE> __device__ __forceinline__ unsigned shared_worker(unsigned used) {
    if constexpr (!TREE) return blockIdx.x;
    const unsigned x = blockIdx.x & 7, each = used >> 3, more = used & 7;
    return x * each + min(x, more) + (blockIdx.x >> 3);
}

// Every workgroup makes the whole plan.  Written for few instructions: what a workgroup runs once comes from memory, 64 bytes at a time, and
// takes a cycle a byte.
// Up to 64 lists: a wave by itself, a list to a lane (one sequence of 1k tokens 5.7 us, by the workgroup 7.0; a group of 8 8.2 and 11.0).
template <int NW, int KIND, bool TREE>
__device__ __forceinline__ Work<TREE> find_work_in_lanes(const Lists<KIND, TREE>& ls, int wave, int lane) {
    constexpr int WGS = 4 * PLAN_WGS / NW;
    const DecodeArgs& a = ls.a;
    const int n = a.n_groups + a.n_seqs;
    const bool there = lane < n;
    ListIs<TREE> mine{};
    if (there) mine = ls.read(lane);
    const ListShape s = ls.shape(mine, lane);
    auto last = [](int x) SP_INLINE { return (unsigned)__builtin_amdgcn_readlane(x, 63); };
    const int solo_units = s.shared ? 0 : s.units * s.blocks, solo_blocks = s.shared ? 0 : s.blocks;
    const int to_solo = scan64(solo_units), ord_solo = scan64(solo_blocks);
    const unsigned solo = last(to_solo) * a.Hkv;
    int room = s.units, units = solo_units, to = to_solo, ord = ord_solo - solo_blocks;
    unsigned shared_room = 0;
    Runs runs{1, 1, 0, false};
    if constexpr (KIND) {
        const int shared_units = s.shared ? s.units * s.blocks : 0, shared_blocks = s.shared ? s.template places<TREE>() : 0;
        const int ord_shared = scan64(shared_blocks), segments = TREE ? scan64(s.shared ? s.blocks : 0) : ord_shared;
        shared_runs<KIND, TREE, WGS>(a, solo, last(ord_solo) * a.Hkv, last(scan64(shared_units)) * a.Hkv, last(segments) * a.Hkv, runs);
        if (s.shared) { room = room_of<TREE>(s.units, runs.shared_run, runs.aligned); units = room * s.blocks; ord = ord_shared - shared_blocks; }
        const int to_shared = scan64(s.shared ? units : 0);
        if (s.shared) to = to_shared;
        shared_room = last(to_shared) * a.Hkv;
        if (shared_room) runs.used = per_place(shared_room, runs.shared_run);
    }
    if (solo) runs.solo_run = per_place(solo, NW * (WGS - runs.used));
    if (blockIdx.x == 0 && wave == 0) {          // what the join needs to know
        if (there) a.desc[1 + lane] = i32x4{to - units, s.units, ord, s.len < 0 ? -1 : room};
        if (lane == 0) a.desc[0] = i32x4{(int)runs.shared_run, (int)runs.solo_run, 0, 0};
    }
    Work<TREE> work;
    work.shared = blockIdx.x < runs.used;
    work.worker = work.shared ? (int)shared_worker<TREE>(runs.used) : (int)(blockIdx.x - runs.used) * NW + wave;
    const unsigned run = work.shared ? runs.shared_run : runs.solo_run, all = work.shared ? shared_room : solo, pos = (unsigned)work.worker * run;
    // (through a lane read: without it the compiler left the comparison out and took the difference, wrapped, as it was)
    work.left = pos < all ? __builtin_amdgcn_readfirstlane((int)min(run, all - pos)) : 0;
    const unsigned from = (unsigned)(to - units) * a.Hkv, end = (unsigned)to * a.Hkv;
    const int src = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(s.shared == work.shared && pos >= from && pos < end)) - 1;
    auto of = [&](int x) SP_INLINE { return __builtin_amdgcn_readlane(x, src & 63); };
    work.list = src & 63;
    work.at = (int)(pos - (unsigned)of((int)from));
    work.ord = of(ord);
    work.room = of(room);
    work.pad = TREE && work.shared && !runs.aligned ? WIDE_PAD : 0;
    if constexpr (TREE) work.list_is = i32x4{of(mine[0]), of(mine[1]), of(mine[2]), 0};
    else work.list_is = i32x2{of(mine[0]), of(mine[1])};
    return work;
}

// More lists: a thread adds up the units of its share of them (they lie in LDS meanwhile, if there are no more than n_held), the workgroup their sums.
template <int NW, int KIND, bool TREE>
__device__ __forceinline__ Work<TREE> find_work(const Lists<KIND, TREE>& ls, ListIs<TREE>* held, int n_held, PlanShare<NW>& share, int wave, int lane) {
    constexpr int SUMS = KIND ? TREE ? 5 : 4 : 2;       // solo units and blocks, shared units and blocks (TREE: and places)
    constexpr int WGS = 4 * PLAN_WGS / NW, ALL = 64 * NW;
    const DecodeArgs& a = ls.a;
    const int n = a.n_groups + a.n_seqs, per = (n + 64 * NW - 1) / (64 * NW), i0 = min(n, (int)threadIdx.x * per), i1 = min(n, i0 + per);
    const bool in_lds = n <= n_held;
    if (in_lds) {
        for (int i = threadIdx.x; i < n; i += ALL * 4) {      // four reads in flight
            ListIs<TREE> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) if (i + ALL * u < n) x[u] = ls.read(i + ALL * u);
#pragma unroll
            for (int u = 0; u < 4; ++u) if (i + ALL * u < n) held[i + ALL * u] = x[u];
        }
        __syncthreads();
    }
    auto list_of = [&](int i) SP_INLINE { return in_lds ? held[i] : ls.read(i); };
    int own[SUMS] = {}, to[SUMS];
    unsigned all[SUMS];
    auto add = [&](int (&sum)[SUMS], const ListShape& s, int room) SP_INLINE {
        sum[0] += s.shared ? 0 : room * s.blocks;
        sum[1] += s.shared ? 0 : s.blocks;
        if constexpr (KIND) {
            sum[2] += s.shared ? room * s.blocks : 0;
            sum[3] += s.shared ? s.blocks : 0;
            if constexpr (TREE) sum[SUMS - 1] += s.shared ? s.template places<TREE>() : 0;
        }
    };
    constexpr int SHARED = KIND ? 2 : 0, SEGS = KIND ? 3 : 1;      // places in `sums`
    auto over_waves = [&](int k) SP_INLINE {       // to[k], inclusive, and all[k] from own[k]
        to[k] = scan64(own[k]);
        __syncthreads();
        if (lane == 63) share.sums[wave][k] = to[k];
        __syncthreads();
        unsigned sum = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) { const int x = share.sums[w][k]; to[k] += w < wave ? x : 0; sum += x; }
        all[k] = sum * a.Hkv;
    };
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        const ListShape s = ls.shape(list_of(i), i);
        add(own, s, s.units);
    }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) over_waves(k);
    Runs runs{1, 1, 0, false};
    if constexpr (KIND) {
        shared_runs<KIND, TREE, WGS>(a, all[0], all[1], all[SHARED], all[SEGS], runs);
        if (runs.aligned || TREE) {
            own[SHARED] = 0;
#pragma unroll 1
            for (int i = i0; i < i1; ++i) {
                const ListShape s = ls.shape(list_of(i), i);
                own[SHARED] += s.shared ? room_of<TREE>(s.units, runs.shared_run, runs.aligned) * s.blocks : 0;
            }
            over_waves(SHARED);
        }
        if (all[SHARED]) runs.used = per_place(all[SHARED], runs.shared_run);
    }
    if (all[0]) runs.solo_run = per_place(all[0], NW * (WGS - runs.used));
    // this workgroup's runs start at `first` and multiples of the run behind it
    Work<TREE> work;
    const bool shared = work.shared = blockIdx.x < runs.used;
    const unsigned run = shared ? runs.shared_run : runs.solo_run, many = shared ? 1 : NW, first = (shared ? shared_worker<TREE>(runs.used) : NW * (blockIdx.x - runs.used)) * run;
    const bool tells = blockIdx.x == 0;          // the first workgroup writes down what the join needs to know
    const int mine = KIND && shared ? SHARED : 0;
    const unsigned through = (unsigned)(mine ? to[SHARED] : to[0]) * a.Hkv, ahead = through - (unsigned)(mine ? own[SHARED] : own[0]) * a.Hkv;
    if (tells || (ahead < first + many * run && through > first)) {
        int at[SUMS];
#pragma unroll
        for (int k = 0; k < SUMS; ++k) at[k] = to[k] - own[k];
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            const ListIs<TREE> x = list_of(i);
            const ListShape s = ls.shape(x, i);
            const int units = s.shared ? at[SHARED] : at[0], blocks = s.shared ? at[SUMS - 1] : at[1], room = s.shared ? room_of<TREE>(s.units, runs.shared_run, runs.aligned) : s.units;
            const unsigned from = (unsigned)units * a.Hkv, end = from + (unsigned)(room * s.blocks) * a.Hkv;
            if (s.shared == shared)
#pragma unroll 1
                for (unsigned k = 0; k < many; ++k) {
                    const unsigned pos = first + k * run;
                    if (pos >= from && pos < end) {
                        share.list[k] = i; share.at[k] = (int)(pos - from); share.ord[k] = blocks;
                        share.rows[k] = x[0]; share.len[k] = x[1]; share.room[k] = room;
                        if constexpr (TREE) share.ahead[k] = x[2];
                    }
                }
            if (tells) a.desc[1 + i] = i32x4{units, s.units, blocks, s.len < 0 ? -1 : room};
            add(at, s, room);
        }
        if (tells && threadIdx.x == 0) a.desc[0] = i32x4{(int)runs.shared_run, (int)runs.solo_run, 0, 0};
    }
    __syncthreads();
    auto scalar = [](int x) SP_INLINE { return __builtin_amdgcn_readfirstlane(x); };      // the same in every lane, which the compiler does not see
    const int slot = shared ? 0 : wave;
    const unsigned pos = first + slot * run, end = mine ? all[SHARED] : all[0];
    work.left = pos < end ? scalar((int)min(run, end - pos)) : 0;
    work.worker = scalar(shared ? (int)shared_worker<TREE>(runs.used) : (int)(blockIdx.x - runs.used) * NW + wave);
    work.list = scalar(share.list[slot]);
    work.at = scalar(share.at[slot]);
    work.ord = scalar(share.ord[slot]);
    work.room = scalar(share.room[slot]);
    work.pad = TREE && shared && !runs.aligned ? WIDE_PAD : 0;
    if constexpr (TREE) work.list_is = i32x4{share.rows[slot], share.len[slot], share.ahead[slot], 0};
    else work.list_is = i32x2{share.rows[slot], share.len[slot]};
    return work;
}

// A place among the units: of list `list` segment `seg` (block * n_kv_heads + kv head; drafted tokens: kv head * blocks + block), unit `t`
template <int KIND, bool TREE = false>
struct Cursor {
    const Lists<KIND, TREE>& ls;
    const bool shared;
    int list, seg, t, units, segs, rows, len, blocks, ord, places;
    int ahead, ahead_len;                  // units and tokens of the prompt that are the first of the list (TREE)
    __device__ __forceinline__ Cursor(const Lists<KIND, TREE>& l, Work<TREE>& w) : ls(l), shared(w.shared), list(w.list), ord(w.ord) {
        load(w.list_is);
        const float inv = __builtin_amdgcn_rcpf((float)w.room);        // a quotient, what it leaves divided again, and a step to either side
        seg = (int)((float)w.at * inv);
        seg += (int)((float)(w.at - seg * w.room) * inv);
        seg = __builtin_amdgcn_readfirstlane(seg);
        seg -= seg * w.room > w.at;
        seg += (unsigned)(seg + 1) * w.room <= (unsigned)w.at;
        t = w.at - seg * w.room;
        if (TREE && w.pad) {
            if (t >= units) {                                      // behind the segment's last unit
                w.left -= w.room - t;
                t = units - 1;
                if (w.left > 0) next();
            }
        } else if (w.room > units) w.left = min(w.left, units - t);        // a run of the segment's own, the last one shorter
    }
    __device__ __forceinline__ bool load(ListIs<TREE> x) {
        const ListShape s = ls.shape(x, list);
        auto scalar = [](int x) SP_INLINE { return __builtin_amdgcn_readfirstlane(x); };
        rows = scalar(s.rows); len = scalar(s.len); units = scalar(s.units); blocks = scalar(s.blocks);
        if constexpr (TREE) { ahead = scalar(s.ahead); ahead_len = scalar(x[2]); }
        places = TREE ? scalar(s.template places<TREE>()) : blocks;
        segs = blocks * ls.a.Hkv;
        return s.shared == shared;
    }
    __device__ __forceinline__ int kv_head() const {      // TREE
        return blocks > 1 ? __builtin_amdgcn_readfirstlane((int)((unsigned)seg / (unsigned)blocks)) : seg;
    }
    // the next unit; there is one
    __device__ __forceinline__ void next() {
        if (++t < units) return;
        t = 0;
        if (++seg < segs) return;
        seg = 0;
        ord += places;
        do {
            ++list;
            if (load(ls.read(list))) { if (units > 0) return; ord += places; }
        } while (list < ls.a.n_groups + ls.a.n_seqs - 1);
    }
};

// Rows of a segment: where they come from, and the slot that they go to
struct SegmentRows {
    int seq0, rep, row0, rows, Hq, kvh, block;          // rows row0 ... row0 + rows - 1 of the list
    int64_t base;                                // of row0 among the rows of sums
    Div heads_each;
    template <int KIND, bool TREE> __device__ __forceinline__ SegmentRows(const Cursor<KIND, TREE>& c, const DecodeArgs& a, int worker) {
        if constexpr (TREE) {
            kvh = c.kv_head();
            block = c.seg - kvh * c.blocks;
        } else {
            unsigned k;
            block = c.blocks > 1 ? (int)divmod((unsigned)c.seg, a.kv_heads, k) : 0;
            kvh = c.blocks > 1 ? (int)k : c.seg;
        }
        const int per = !c.shared ? (TREE ? (int)a.solo_rows.d : SOLO_ROWS) : TREE ? (int)a.block_rows.d : 16 * (((((c.rows + 15) >> 4)) + c.blocks - 1) / c.blocks);
        row0 = block * per;
        rows = min(per, c.rows - row0);
        seq0 = c.ls.first_seq(c.list);
        rep = a.rep; Hq = a.Hq; heads_each = a.heads_each;
        if constexpr (TREE && KIND) {
            if (c.shared) {      // (the segment's own rows lie behind those of the segments ahead of it, not each in room for the largest)
                base = (int64_t)worker * a.shared_rows + ((int64_t)c.ord * a.Hkv + kvh * c.places + block * (per >> 4)) * 16;
                return;
            }
        }
        const int64_t slot = (int64_t)worker + (int64_t)c.ord * a.Hkv + c.seg;
        base = c.shared ? slot * a.shared_rows : c.list < a.n_groups ? a.prompt_base + slot * a.prompt_rows : a.resp_base + slot * a.resp_rows;
    }
    __device__ __forceinline__ int64_t q_row(int r) const {        // row of q and o
        unsigned hr;
        const int member = (int)divmod((unsigned)(row0 + r), heads_each, hr);
        return (int64_t)(seq0 + member) * Hq + kvh * rep + (int)hr;
    }
};

// ---- rows of a wave ---------------------------------------------------------------------------------------

// LDS tiles: a row per key, its granules of 16 bytes permuted so that neither 16 rows of one granule (K) nor four rows of a block
// of 16 columns (V, read transposed) meet in a bank
template <int D> __device__ __forceinline__ int kv_swz(int r) {
    if constexpr (D == 128) return swz(r);
    else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
template <int D> __device__ __forceinline__ int kv_off(int row, int granule) { return row * (2 * D) + ((granule ^ kv_swz<D>(row)) << 4); }

template <int D, int NC>
struct Rows {
    static_assert(NC <= 4, "one element of m and l per tile");
    f32x4 o[NC][D / 16];       // lane: row l % 16 of tile c, elements 16 dt + 4 (l / 16) + i
    f32x4 m, l;                // (vectors: arrays of these ended up in LDS)
    bf16x8 q[NC][D / 32];
    __device__ __forceinline__ void clear(float m_none) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            m[c] = m_none; l[c] = 0.f;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) o[c][dt] = f32x4{0, 0, 0, 0};
        }
    }
};

__device__ __forceinline__ unsigned lds_address(const char* p) {
    return __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)p);
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() {
    if constexpr (N == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if constexpr (N == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
}

// (All NC row tiles that a wave has room for are computed, also where it has fewer: branches between them kept the reads from LDS from
// running ahead of the products, and branches around them cost registers.)
// Scores of 32 keys at LDS address `k`, keys not in `bits` masked: s[c][kt][i] is key 16 kt + 4 (l / 16) + i of row l % 16 of tile c
// (an operand's granule is its first one's with a constant xored in, which leaves the address of the first in a register only)
template <int D, int NC>
__device__ __forceinline__ void scores(const Rows<D, NC>& r, unsigned k, unsigned bits, int l, f32x4 (&s)[NC][2]) {
    const unsigned at = k + kv_off<D>(l & 15, l >> 4);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        bf16x8 a[D / 32];
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) a[ks] = lds_at_row8((at ^ (ks << 6)) + kt * (32 * D));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            s[c][kt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) s[c][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[ks], r.q[c][ks], s[c][kt], 0, 0, 0);
        }
    }
    if (bits != 0xffffffffu) {
        const unsigned mine = bits >> (4 * (l >> 4));
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[c][kt][i] = mine >> (16 * kt + i) & 1 ? s[c][kt][i] : -INFINITY;
    }
}

// Weights of 32 keys from their scores, in two parts of bf16 as the second product needs them: a weight's upper 16 bits, which is not above
// it, and what that leaves, rounded.  Both go through the matrix instructions, and 2^-15 of the weight is lost at most, so that o is off as with unrounded weights
// (32 answers to a prompt of 16k tokens: o off by 1.66e-3 of its 2-norm, the rounding of o itself, where weights rounded once left 1.92e-3; for 39 us instead of
// 37, while calls that wait for keys cost the same).  The second part has 2^-20 of the weight added, so that it is 0 only with
// the weight: it would turn an infinite value into NaN.
// They are taken against the reference m that the row has from earlier keys, any finite one serving as well, as long as they stay in
// range: only if a lane's eight sum to more than 2^14 (or to infinity, as they do for a row that has not seen a key) does the wave
// take the rows' maxima for new references, scale what it has and take the weights again.  A NaN among the scores stays in the row's sum, whichever way the
// compiler took the comparison, and a score of +inf becomes one, as it would in a softmax of the whole row.  (With the maximum of every 32 keys, 128 rows and short runs
// rescaled nearly every time: 110 instructions a tile instead of 30.)  Differences are taken ahead of their scaling, so that they are exact at any
// magnitude: of a scaled reference the rounding alone passes the exponential's range for scores above 2^30, and the chunks of a row differ in it.
template <int D, int NC>
__device__ __forceinline__ void weights(Rows<D, NC>& r, const f32x4 (&s)[NC][2], float c2, bf16x8 (&p)[NC][2]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float sum;
        auto take = [&](float m) SP_INLINE {
            sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = __builtin_amdgcn_exp2f((s[c][e >> 2][e & 3] - m) * c2);
                sum += x;
                const float high = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
                p[c][0][e] = __builtin_bit_cast(__bf16, (unsigned short)(__float_as_uint(x) >> 16));
                p[c][1][e] = (__bf16)__builtin_fmaf(x, 1.f + 0x1p-20f, -high);
            }
        };
        take(r.m[c]);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= 16384.f)) != 0, 0)) {
            float mx = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])), fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3])));
            mx = quad_max(mx);
            const float mn = fmaxf(r.m[c], mx), alpha = __builtin_amdgcn_exp2f((r.m[c] - mn) * c2);
            r.l[c] *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) r.o[c][dt][i] *= alpha;
            r.m[c] = mn;
            take(mn);
        }
        r.l[c] += sum;
    }
}

// Which of 32 keys a row of drafted token `node` sees, the first of them being drafted token j (negative: as many keys are ahead of the drafted ones,
// which all see).  `mask`: the token's row of `words` words, NULL: a chain.
__device__ __forceinline__ unsigned drafted_bits(const uint32_t* mask, int words, int node, int j) {
    if (!mask) return low_bits(node - j + 1);
    const int w = j >> 5, shift = j & 31;
    auto word = [&](int i) SP_INLINE { return i < 0 ? 0xffffffffu : i < words ? mask[i] : 0u; };
    return (unsigned)((((uint64_t)word(w + 1) << 32) | word(w)) >> shift);
}

// A list's drafted tokens: its keys from `base` on are tokens `first`, first + 1, ... of q (a prompt has none: base is beyond its keys)
struct Drafted {
    int base, first, words;
    template <int KIND> __device__ __forceinline__ void of(const Lists<KIND, true>& ls, int list) {
        const DecodeArgs& a = ls.a;
        base = 0x7fffffff;
        if (list < a.n_groups) return;
        const int n = __builtin_amdgcn_readfirstlane(ls.tokens(list));
        base = __builtin_amdgcn_readfirstlane(a.resp_lens[list - a.n_groups]) - n;      // (of the length that was given: the table may hold less)
        first = __builtin_amdgcn_readfirstlane(ls.first_seq(list));
        words = (n + 31) >> 5;
    }
    // of the 32 keys from `key` on, which row `row` of the segment sees (rows behind the last: those of the last)
    __device__ __forceinline__ unsigned bits(const DecodeArgs& a, const SegmentRows& seg, int row, int key) const {
        unsigned hr;
        const int node = (int)divmod((unsigned)(seg.row0 + min(row, seg.rows - 1)), seg.heads_each, hr);
        return drafted_bits(a.ancestors ? a.ancestors + (int64_t)(first + node) * a.mask_stride : nullptr, words, node, key - base);
    }
};

// Scores of 32 keys from `key` on that rows do not see, in units that hold drafted tokens
template <int D, int NC>
__device__ __forceinline__ void hide(const DecodeArgs& a, const SegmentRows& seg, const Drafted& drafted, int row0, int key, int l, f32x4 (&s)[NC][2]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const unsigned mine = drafted.bits(a, seg, row0 + 16 * c + (l & 15), key) >> (4 * (l >> 4));
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[c][kt][i] = mine >> (16 * kt + i) & 1 ? s[c][kt][i] : -INFINITY;
    }
}

// A weight of 0 does not leave out an infinite or NaN value in a product.  Where rows see some of the keys only, such elements are therefore taken out
// of the values, and the row's statistics say so: the join then adds them to the rows that see their keys.
__device__ __forceinline__ i32x4 only_finite(i32x4 w, bool& found) {      // bf16
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool low = (w[i] & 0x7f80) == 0x7f80, high = (w[i] & 0x7f800000) == 0x7f800000;
        found |= low || high;
        w[i] &= (low ? (int)0xffff0000 : -1) & (high ? 0xffff : -1);
    }
    return w;
}
// of `granules` of 16 bytes at LDS address `at`, 64 lanes (or more: `step`) in turn; true if any was found (by this lane)
__device__ __forceinline__ bool clean(unsigned at, int first, int granules, int step) {
    bool any = false;
    for (int g = first; g < granules; g += step) {
        auto* const p = (__attribute__((address_space(3))) i32x4*)(uintptr_t)(at + 16u * g);
        bool found = false;
        const i32x4 w = only_finite(*p, found);
        if (found) *p = w;
        any |= found;
    }
    return any;
}

// O^T += V^T P^T over 32 keys at LDS address `v`
template <int D, int NC>
__device__ __forceinline__ void add_values(Rows<D, NC>& r, unsigned v, const bf16x8 (&p)[NC][2], int l) {
    const unsigned at = v + kv_off<D>(4 * (l >> 4) + ((l & 15) >> 2), (l & 3) >> 1) + ((l & 1) << 3);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
        s16x4 half[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
            half[kt] = lds_at_tr4((at ^ (dt << 5)) + kt * (32 * D));
        const bf16x8 a = cat4(half[0], half[1]);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int part = 1; part >= 0; --part) r.o[c][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[c][part], r.o[c][dt], 0, 0, 0);
        }
    }
}

// Pages of a list's keys, `count` of its table: a lane holds one of 64 page numbers, from page `first` on; `bad`: some of them are none of the cache's
// (what the table holds behind the list's last page is padding and does not matter)
struct Pages {
    const int* table; int count, n_pages, first, held, lane; bool bad;
    __device__ __forceinline__ int at(int page) {
        need(page);
        return __builtin_amdgcn_readlane(held, page - first);
    }
    __device__ __forceinline__ void need(int page) { if ((unsigned)(page - first) >= 64u) load(page); }
    __device__ __forceinline__ void load(int page) {
        first = page;
        const bool used = page + lane < count;
        held = used ? table[page + lane] : -1;
        bad = __builtin_amdgcn_ballot_w64(used && (unsigned)held >= (unsigned)n_pages) != 0;
    }
};

__device__ __forceinline__ int pages_of(int len, int log_page) { return (int)(((unsigned)len + (1u << log_page) - 1) >> log_page); }

__device__ __forceinline__ uint64_t uniform64(uint64_t x) {
    return ((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)x);
}

// Copies of keys and values into LDS, 16 keys at a time (which lie in one page)
template <int D>
struct Copier {
    static constexpr int ROW = 2 * D, PER_ROW = ROW / 16, ROWS = 64 / PER_ROW, COPIES = 16 / ROWS;      // copies of 16 keys
    unsigned voff[COPIES];
    int row0;
    uint64_t zero;
    __device__ __forceinline__ Copier(int l) {
        row0 = l / PER_ROW;
#pragma unroll
        for (int u = 0; u < COPIES; ++u) {
            const int row = u * ROWS + row0;
            voff[u] = row * ROW + (((l % PER_ROW) ^ kv_swz<D>(row)) << 4);
        }
        zero = (uint64_t)(uintptr_t)&zero_granule;
    }
    // `valid` of the 16 rows at `src` (negative or zero: none) to LDS address `dst`; rows that are not there read as zero, whatever memory holds
    __device__ __forceinline__ void rows16(uint64_t src, int valid, unsigned dst) const {
        src = uniform64(src);
        dst = __builtin_amdgcn_readfirstlane(dst);
        valid = __builtin_amdgcn_readfirstlane(valid);
        if (valid >= 16) {
#pragma unroll
            for (int u = 0; u < COPIES; ++u) async_copy16_sm(src, voff[u], dst + 1024u * u);
        } else {
#pragma unroll
            for (int u = 0; u < COPIES; ++u) {
                const uint64_t at = u * ROWS + row0 < valid ? src + voff[u] : zero;
                asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(at), "s"(dst + 1024u * u) : "memory");
            }
        }
    }
};

template <int D, int NC>
__device__ __forceinline__ void load_rows(Rows<D, NC>& r, const __bf16* q, const SegmentRows& pr, int row0, int tiles, int l) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int row = row0 + 16 * c + (l & 15);
        const bool there = c < tiles && row < pr.rows;
        const __bf16* const p = q + pr.q_row(there ? row : 0) * D + 8 * (l >> 4);
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) r.q[c][ks] = *reinterpret_cast<const bf16x8*>(p + 32 * ks);
    }
}

// Statistics of a row of a slot: m and l; TREE: also l of the weights as the second product took them, and whether values were left out of it
template <bool TREE> __device__ __forceinline__ void put_stats(const DecodeArgs& a, int64_t row, float m, float l, float l_product, bool left_out) {
    if constexpr (TREE) *reinterpret_cast<f32x4*>(a.stats + row * 4) = f32x4{m, l, l_product, left_out ? 1.f : 0.f};
    else *reinterpret_cast<f32x2*>(a.stats + row * 2) = f32x2{m, l};
}

template <bool TREE, int D, int NC>
__device__ __forceinline__ void store_rows(const Rows<D, NC>& r, const DecodeArgs& a, const SegmentRows& pr, int row0, int tiles, int l, bool left_out = false) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int row = row0 + 16 * c + (l & 15);
        const float lt = quad_sum(r.l[c]);
        if (c >= tiles || row >= pr.rows) continue;
        float* const out = a.sums + (pr.base + row) * D + 4 * (l >> 4);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(out + 16 * dt) = r.o[c][dt];
        if (l < 16) put_stats<TREE>(a, pr.base + row, r.m[c], lt, lt, left_out);
    }
}

// Rows whose keys this worker has all seen (TREE): o and lse, and a mark for the join
constexpr float DONE = 2.f;
template <int D, int NC>
__device__ __forceinline__ void finish_rows(const Rows<D, NC>& r, const DecodeArgs& a, const SegmentRows& pr, int tiles, int l) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int row = 16 * c + (l & 15);
        const float lt = quad_sum(r.l[c]);
        if (c >= tiles || row >= pr.rows) continue;
        const bool none = bits_of(lt) == 0;
        const float inv = 1.f / lt;
        unsigned hr;
        const int tok = pr.seq0 + (int)divmod((unsigned)(pr.row0 + row), pr.heads_each, hr), h = pr.kvh * pr.rep + (int)hr;
        __bf16* const out = (__bf16*)a.o + ((int64_t)tok * pr.Hq + h) * D + 4 * (l >> 4);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            bf16x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (__bf16)(none ? 0.f : r.o[c][dt][i] * inv);
            *reinterpret_cast<bf16x4*>(out + 16 * dt) = y;
        }
        if (l < 16) {
            a.lse[(int64_t)h * a.n_tok + tok] = none ? -INFINITY : r.m[c] * (a.c * LN2) + __logf(lt);
            *reinterpret_cast<f32x4*>(a.stats + (pr.base + row) * 4) = f32x4{0.f, 0.f, 0.f, DONE};
        }
    }
}

// NC: row tiles of a wave in a shared segment, 0: no list is shared.  NS: in a solo one.  NW: waves of a workgroup; eight (TREE) for lists of many rows.
template <int D, int NC, int NS, bool MANY, bool TREE = false, int NW = 4>
__global__ __launch_bounds__(64 * NW, 2) void decode_kernel(StartsArg<TREE> starts, DecodeArgs a) {
    constexpr int KEYS16 = 32 * D, KIND = NC > 0;       // bytes of 16 keys
    __shared__ __attribute__((aligned(1024))) char lds[4 * NW * KEYS16];
    __shared__ PlanShare<NW> share;
    // Wide segments of drafted tokens: values were left out of the products; some pages are none of the cache's; pages of 16 keys each
    __shared__ int left_out, bad_pages, place[TREE && KIND ? 256 : 1];
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63;
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    const Lists<KIND, TREE> ls{words_of(starts), a};
    Work<TREE> work;
    if constexpr (MANY) {
        work = find_work<NW>(ls, reinterpret_cast<ListIs<TREE>*>(lds), (int)(sizeof(lds) / sizeof(ListIs<TREE>)), share, w, l);
        __syncthreads();                             // the lists' place is free
    } else {
        work = find_work_in_lanes<NW>(ls, w, l);
    }
    if (work.left == 0) return;
    Cursor<KIND, TREE> at(ls, work);
    if (TREE && work.left <= 0) return;
    auto kv_head = [&]() SP_INLINE {
        if constexpr (TREE) return at.kv_head();
        unsigned k = (unsigned)at.seg;
        if (KIND && at.blocks > 1) divmod((unsigned)at.seg, a.kv_heads, k);
        return (int)k;
    };
    int kvh = kv_head();
    Pages pages;
    pages.lane = l;
    pages.n_pages = a.n_pages;
    Drafted drafted;
    // The part of the list that the unit lies in: its length and first unit (TREE: the prompt's or the sequence's own)
    int part_len = 0, part_unit = 0;
    auto prompt_of = [&]() SP_INLINE {             // table of the prompt ahead of the list's keys
        unsigned rest;
        return a.prompt_tables + (int64_t)divmod((unsigned)(at.list - a.n_groups), a.group_seqs, rest) * a.prompt_width;
    };
    auto table_of_list = [&]() SP_INLINE {
        const bool prompt = at.list < a.n_groups;
        pages.table = prompt ? a.prompt_tables + at.list * a.prompt_width : a.resp_tables + (at.list - a.n_groups) * a.resp_width;
        if constexpr (TREE) {
            drafted.of(ls, at.list);
            const bool ahead = at.t < at.ahead;
            if (ahead) pages.table = prompt_of();
            part_len = ahead ? at.ahead_len : at.len;
            part_unit = ahead ? 0 : at.ahead;
            pages.count = pages_of(part_len, a.log_page);
        } else {
            pages.count = pages_of(at.len, a.log_page);
        }
    };
    auto length = [&]() SP_INLINE { return TREE ? part_len : at.len; };
    auto unit = [&]() SP_INLINE { return TREE ? at.t - part_unit : at.t; };
    auto next = [&]() SP_INLINE {
        const int list = at.list;
        at.next();
        if (at.list != list || (TREE && at.ahead > 0 && (at.t == 0 || at.t == at.ahead))) { table_of_list(); if (!TREE || !work.shared) pages.load(0); }
        if (at.t == 0) kvh = kv_head();
    };
    table_of_list();
    const Copier<D> copy(l);
    const uint64_t kc = uniform64((uint64_t)(uintptr_t)a.k_cache), vc = uniform64((uint64_t)(uintptr_t)a.v_cache);
    // byte offset of a key's row in either cache, for a page of the cache
    auto offset = [&](int key, int page) SP_INLINE {
        return ((((uint64_t)(unsigned)page * a.Hkv + kvh) << a.log_page) + (key & ((1 << a.log_page) - 1))) * (2 * D);
    };
    // the same of 16 keys, and how many of them there are
    auto locate = [&](int key, uint64_t& off, int& valid) SP_INLINE {
        valid = min(16, length() - key);
        off = 0;
        if (valid <= 0) return;
        const int page = __builtin_amdgcn_readfirstlane(pages.at(key >> a.log_page));
        if ((unsigned)page >= (unsigned)a.n_pages) { valid = 0; return; }
        off = offset(key, page);
    };
    // whether all of `count` keys are there (the pages held include the last one's; if any of those held is none, it is looked at in turn)
    auto whole = [&](int key, int count) SP_INLINE {
        if (key + count > length()) return false;
        pages.need(key >> a.log_page);
        pages.need((key + count - 1) >> a.log_page);
        return !pages.bad && (unsigned)((key >> a.log_page) - pages.first) < 64u;
    };
    const __bf16* const q = (const __bf16*)a.q;
    const unsigned buf = lds_address(lds);

    if (!KIND || !work.shared) {
        // One wave: K and V of a unit in turn.  The next K is copied while the weights and the second product run, the next V under the
        // next scores, also from segment to segment.
        Rows<D, NS> r;
        const unsigned kb = buf + w * 4 * KEYS16, vb = kb + 2 * KEYS16;
        uint64_t off[2];
        int valid[2];
        auto fetch = [&]() SP_INLINE {
            const int key = 32 * unit();
            if (whole(key, 32)) {
                valid[0] = valid[1] = 16;
                off[0] = offset(key, __builtin_amdgcn_readfirstlane(pages.at(key >> a.log_page)));
                off[1] = a.log_page > 4 ? off[0] + KEYS16 : offset(key + 16, __builtin_amdgcn_readfirstlane(pages.at((key + 16) >> a.log_page)));
            } else {
                locate(key, off[0], valid[0]);
                locate(key + 16, off[1], valid[1]);
            }
        };
        auto issue = [&](uint64_t cache, unsigned dst) SP_INLINE {
            copy.rows16(cache + off[0], valid[0], dst);
            copy.rows16(cache + off[1], valid[1], dst + KEYS16);
        };
        constexpr int N = 2 * Copier<D>::COPIES;
        pages.load(32 * unit() >> a.log_page);
        fetch();
        issue(kc, kb);
        issue(vc, vb);
        while (true) {
            SegmentRows seg(at, a, work.worker);
            const int tiles = (seg.rows + 15) >> 4;
            load_rows(r, q, seg, 0, tiles, l);
            r.clear(a.m_none);
            bool more = true, same = true, left_out = false;
            const bool from_first = at.t == 0;
            bool to_last = false;
            while (same) {
                const unsigned bits = low_bits(valid[0]) | low_bits(valid[1]) << 16;
                f32x4 s[NS][2];
                bf16x8 pw[NS][2];
                wait_copies<N>();
                scores(r, kb, bits, l, s);
                bool some = false;             // whether rows see some of the unit's keys only
                if constexpr (TREE) {
                    some = at.t >= at.ahead && 32 * (int64_t)unit() + 32 > drafted.base;
                    if (some) hide<D>(a, seg, drafted, 0, 32 * unit(), l, s);
                }
                wait_lds();
                more = --work.left > 0;
                same = more && at.t + 1 < at.units;
                if constexpr (TREE) to_last = at.t + 1 == at.units;
                if (more) { next(); fetch(); issue(kc, kb); }
                weights(r, s, a.c, pw);
                if (more) wait_copies<N>(); else wait_copies<0>();
                if (TREE && some) {
                    left_out |= __builtin_amdgcn_ballot_w64(clean(vb, l, 2 * KEYS16 / 16, 64)) != 0;
                    wait_lds();
                }
                add_values(r, vb, pw, l);
                wait_lds();
                if (more) issue(vc, vb);
            }
            if (TREE && a.direct && from_first && to_last && !left_out) finish_rows(r, a, seg, tiles, l);
            else store_rows<TREE>(r, a, seg, 0, tiles, l, left_out);
            if (!more) return;
        }
    } else if constexpr (TREE) {
        // Many drafted tokens: four or eight waves of 32 rows, products on matrix instructions of 32 x 32, software-pipelined as in the forward over a pack: while
        // step j's matrix instructions form O^T += V(j-1)^T P(j-1)^T and S(j+1) = K(j+1) Q^T, its vector ones turn S(j) into P(j), a score to a
        // matrix instruction (two, heads of 64).  Four waves: two buffers of 64 keys each of K and of V, a barrier per step; V(j) and K(j+2) are copied under step
        // j, and two workgroups share a CU.  A weight is rounded once, to bf16, and o divided by the sum of the rounded ones, which takes what their errors have in
        // common out of it (o off by 1.76e-3 of its 2-norm against 1.66e-3 with weights in two parts, whose second product would be of twice the instructions); lse
        // has the sum of the others.  An element is off by 2^-8 of sum p |v| and of |o| for the weights, at most, and by 2^-8 of |o| for its own rounding.
        // Heads of 128: 256 registers to a wave, and 88 to 104 bytes of scratch, written where a segment starts and read there, where pages are looked
        // up, values cleaned or drafted tokens masked, and behind the last step; steps without drafted tokens do not touch it.
        // Eight waves: four buffers each, two steps to a barrier; a copy serves twice the rows and has twice the time.
        constexpr int TILE = 4 * KEYS16, KS = D / 16, MF = 2 * KS, DB = D / 32, PER = 32 / (2 * MF), RD = 3, NB = NW == 8 ? 4 : 2;
        const int c32 = l & 31, hh = l >> 5, j16 = l & 15;
        unsigned row_at[KS], tr_at[DB][2];         // operands within the first buffers
#pragma unroll
        for (int i = 0; i < KS; ++i) { row_at[i] = buf + kv_off<D>(c32, 2 * i + hh); asm volatile("" : "+v"(row_at[i])); }
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int col4 = 32 * db + 16 * ((l >> 4) & 1) + 4 * (j16 & 3);
                tr_at[db][half] = buf + NB * TILE + kv_off<D>(4 * hh + (j16 >> 2) + 8 * half, col4 >> 3) + ((col4 & 4) << 1);
                asm volatile("" : "+v"(tr_at[db][half]));
            }
        auto ldK = [&](int b, int i) SP_INLINE { return lds_at_row8(row_at[i >> 1] + TILE * b + 2 * KEYS16 * (i & 1)); };
        auto ldV = [&](int b, int i) SP_INLINE {
            const int off = TILE * b + KEYS16 * (i / DB);
            return cat4(lds_at_tr4(tr_at[i % DB][0] + off), lds_at_tr4(tr_at[i % DB][1] + off));
        };
        auto operand = [&](const unsigned (&p)[16], int i) SP_INLINE {      // of product i of O^T: keys 16 (i / DB) ...
            typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
            const int k = 4 * (i / DB);
            return __builtin_bit_cast(bf16x8, u32x4{p[k], p[k + 1], p[k + 2], p[k + 3]});
        };
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        auto pack2 = [&](float x, float y) SP_INLINE { return __builtin_bit_cast(unsigned, bf16x2{(__bf16)x, (__bf16)y}); };
        auto sum2 = [&](unsigned p, float acc) SP_INLINE {
            return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, p), bf16x2{(__bf16)1.f, (__bf16)1.f}, acc, false);
        };
        const float cs = a.c;
        const f32x16 zero16 = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        while (true) {
            const SegmentRows seg(at, a, work.worker);
            const int total = min(work.left, at.units - at.t), tile0 = at.t;
            const int* const own_table = a.resp_tables + (at.list - a.n_groups) * a.resp_width;
            const int* const table = at.list < a.n_groups ? a.prompt_tables + at.list * a.prompt_width : own_table;
            const int* const table_ahead = at.ahead ? prompt_of() : nullptr;
            // tile j is of the prompt ahead or not; its first key there, and the keys from it on
            auto is_ahead = [&](int j) SP_INLINE { return tile0 + j < at.ahead; };
            auto key_of = [&](int j) SP_INLINE { return 64 * (tile0 + j - (is_ahead(j) ? 0 : at.ahead)); };
            auto keys_from = [&](int j) SP_INLINE { return (is_ahead(j) ? at.ahead_len : at.len) - key_of(j); };
            const bool active = 32 * w < seg.rows;
            // Pages of every 16 keys of up to 64 tiles, -1: none, filled in by all threads ahead of their use
            auto fill = [&](int j, int tiles) SP_INLINE {
                if ((int)threadIdx.x >= 4 * tiles) return;
                const int jt = j + ((int)threadIdx.x >> 2), in_tile = 16 * ((int)threadIdx.x & 3);
                int page = -1;
                if (tile0 + jt < at.units && in_tile < keys_from(jt)) {
                    page = (is_ahead(jt) ? table_ahead : table)[(unsigned)(key_of(jt) + in_tile) >> a.log_page];
                    if ((unsigned)page >= (unsigned)a.n_pages) { page = -1; bad_pages = 1; }
                }
                place[(4 * j + threadIdx.x) & 255] = page;
            };
            struct Tile { uint64_t off; int valid; };      // this wave's 16 keys of a tile
            auto fetch = [&](int j) SP_INLINE {
                const int page = __builtin_amdgcn_readfirstlane(place[(4 * j + (w & 3)) & 255]), in_tile = 16 * (w & 3);
                return Tile{offset(key_of(j) + in_tile, max(page, 0)), page < 0 ? 0 : min(16, keys_from(j) - in_tile)};
            };
            auto copy_k = [&](int j, int b) SP_INLINE {         // K(j) into buffer b; of eight waves, the first four
                if (j >= total || (NW == 8 && w >= 4)) return;
                const Tile t = fetch(j);
                copy.rows16(kc + t.off, t.valid, buf + (unsigned)b * TILE + (w & 3) * KEYS16);
            };
            auto copy_v = [&](int j, int b) SP_INLINE {
                if (j >= total || (NW == 8 && w < 4)) return;
                const Tile t = fetch(j);
                copy.rows16(vc + t.off, t.valid, buf + (unsigned)(NB + b) * TILE + (w & 3) * KEYS16);
            };
            auto tail = [&](int j) SP_INLINE { return !is_ahead(j) && key_of(j) + (int64_t)64 > drafted.base; };      // holds drafted tokens
            bool bad = false;
            auto mask = [&](int j, f32x16 (&S)[2]) SP_INLINE {
                const bool some = tail(j);
                const int n = keys_from(j);
                if (!some && !bad && n >= 64) return;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    unsigned bits = low_bits(n - 32 * kb);
                    if (bad) bits &= (place[(4 * j + 2 * kb) & 255] < 0 ? 0xffff0000u : ~0u) & (place[(4 * j + 2 * kb + 1) & 255] < 0 ? 0xffffu : ~0u);
                    if (some) bits &= drafted.bits(a, seg, 32 * w + c32, key_of(j) + 32 * kb);
                    mask16(S[kb], bits >> (4 * hh));
                }
            };
            // takes infinite and NaN values out of those of V(j) ... V(j + n - 1), in buffers from b on, that hold drafted tokens; every wave its share.  (Not out of the
            // others, whose keys all rows see: the join would not add them.)
            auto clean_tiles = [&](int j, int n, int b) SP_INLINE {
                if (j + n <= 0 || !tail(j + n - 1)) return;        // tiles behind the first one with drafted tokens hold some as well
#pragma unroll
                for (int i = 0; i < n; ++i)
                    if (tail(j + i) && clean(buf + (unsigned)(NB + ((b + i) & (NB - 1))) * TILE, threadIdx.x, TILE / 16, 64 * NW)) left_out = 1;
                wait_lds();
                __syncthreads();
            };
            __syncthreads();                           // the last segment's reads from LDS are done
            if (threadIdx.x == 0) left_out = bad_pages = 0;
            bf16x8 qreg[KS];
            {
                const __bf16* const p = q + seg.q_row(min(32 * w + c32, seg.rows - 1)) * D + 8 * hh;
#pragma unroll
                for (int i = 0; i < KS; ++i) qreg[i] = *reinterpret_cast<const bf16x8*>(p + 16 * i);
            }
            // V(-1), which P = 0 is multiplied with: LDS may hold what reads as NaN
            for (int i = threadIdx.x; i < TILE / 16; i += 64 * NW) *(__attribute__((address_space(3))) i32x4*)(uintptr_t)(buf + (2 * NB - 1) * TILE + 16 * i) = i32x4{0, 0, 0, 0};
            wait_lds();
            __syncthreads();
            fill(0, 64);
            wait_lds();
            __syncthreads();
            bad = bad_pages;
            copy_k(0, 0);
            copy_k(1, 1);
            if constexpr (NB == 4) { copy_k(2, 2); copy_v(0, 0); }
            f32x16 o[DB], sA[2], sB[2];
            unsigned pA[16], pB[16];
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] = zero16;
#pragma unroll
            for (int i = 0; i < 16; ++i) { pA[i] = 0u; pB[i] = 0u; }
            float m = a.m_none, lsum = 0.f, lprod = 0.f;
            wait_copies<0>();
            wait_lds();
            __syncthreads();
            if (active) {
#pragma unroll
                for (int i = 0; i < MF; ++i) sA[i & 1] = mfma32(ldK(0, i), qreg[i >> 1], i < 2 ? zero16 : sA[i & 1]);
                mask(0, sA);
                float mx = sA[0][0];
#pragma unroll
                for (int e = 1; e < 32; ++e) mx = fmaxf(mx, sA[e >> 4][e & 15]);
                m = fmaxf(m, pair_max(mx));
            }
            // A row's weights are 2^(S c - R).  R is m c as rounded, where that is small, so that one operation makes the exponent; else m c itself, and
            // differences are taken ahead of their scaling, in the branch below, which then every step takes.  d = R - m c.
            constexpr float LARGE = 4194304.f;
            auto beyond = [&](float x) SP_INLINE { return !(fabsf(x * cs) <= LARGE); };
            auto offset_of = [&](float x) SP_INLINE { return beyond(x) ? 0.f : __builtin_fmaf(-x, cs, x * cs); };
            auto step = [&](int j, auto par, f32x16 (&S)[2], f32x16 (&Snext)[2], const unsigned (&p)[16], unsigned (&pnew)[16]) SP_INLINE {
                constexpr int R = decltype(par)::value;
                mask(j, S);
                __builtin_amdgcn_sched_barrier(0);
                const float mc = m * cs;
                float tsum = 0.f, tprod = 0.f, pe[32];
                auto valu = [&](int e) SP_INLINE {
                    pe[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[e >> 4][e & 15], cs, -mc));
                    asm volatile("" : "+v"(pe[e]));
                    if (e >= 1) { tsum += pe[e - 1]; asm volatile("" : "+v"(tsum)); }
                    if (e >= 2 && (e & 1) == 0) { pnew[(e - 2) >> 1] = pack2(pe[e - 2], pe[e - 1]); asm volatile("" : "+v"(pnew[(e - 2) >> 1])); }
                    if (e >= 3 && (e & 1) == 1) { tprod = sum2(pnew[(e - 3) >> 1], tprod); asm volatile("" : "+v"(tprod)); }
                };
                auto operand_at = [&](int i) SP_INLINE { return i < MF ? ldV((R + NB - 1) % NB, i) : ldK((R + 1) % NB, i - MF); };
                bf16x8 ring[RD];
#pragma unroll
                for (int i = 0; i < RD - 1; ++i) ring[i] = operand_at(i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 2 * MF; ++i) {
                    if (i + RD - 1 < 2 * MF) ring[(i + RD - 1) % RD] = operand_at(i + RD - 1);
                    if (i < MF) o[i % DB] = mfma32(ring[i % RD], operand(p, i), o[i % DB]);
                    else Snext[i & 1] = mfma32(ring[i % RD], qreg[(i - MF) >> 1], i < MF + 2 ? zero16 : Snext[i & 1]);
#pragma unroll
                    for (int e = 0; e < PER; ++e) valu(PER * i + e);
                    __builtin_amdgcn_sched_barrier(0);
                }
                tsum += pe[31];
                pnew[15] = pack2(pe[30], pe[31]);
                tprod = sum2(pnew[15], tprod);
                if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(tsum <= 16384.f) || beyond(m)) != 0, 0)) {
                    float mx = S[0][0];
#pragma unroll
                    for (int e = 1; e < 32; ++e) mx = fmaxf(mx, S[e >> 4][e & 15]);
                    const float mn = fmaxf(m, pair_max(mx)), d = offset_of(mn);
                    const float alpha = __builtin_amdgcn_exp2f(__builtin_fmaf(m - mn, cs, offset_of(m) - d));
                    lsum *= alpha;
                    lprod *= alpha;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
                    m = mn;
                    tsum = tprod = 0.f;
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[k >> 3][(2 * k) & 15] - mn, cs, -d));
                        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[k >> 3][((2 * k) & 15) + 1] - mn, cs, -d));
                        tsum += p0 + p1;
                        pnew[k] = pack2(p0, p1);
                        tprod = sum2(pnew[k], tprod);
                    }
                }
                lsum += tsum;
                lprod += tprod;
            };
            int vlast = NB - 1;        // buffer of the last V
            // step j, and whether it was the last one; P of an odd count of steps is in the other registers
            auto even = [&](int j, auto r) SP_INLINE {
                if (active) step(j, r, sA, sB, pA, pB);
                if (j + 1 < total) return false;
#pragma unroll
                for (int i = 0; i < 16; ++i) pA[i] = pB[i];
                vlast = decltype(r)::value;
                return true;
            };
            auto odd = [&](int j, auto r) SP_INLINE {
                if (active) step(j, r, sB, sA, pB, pA);
                vlast = decltype(r)::value;
                return j + 1 >= total;
            };
            auto arrived = [&](int j) SP_INLINE {        // what was copied under the last steps; then the next pages, far ahead of their use
                wait_copies<0>();
                __syncthreads();
                if ((j & 31) == 0 && j > 0 && j + 32 < total) fill(j + 32, 32);
                if ((j & 31) == 4) bad = bad_pages;
            };
            constexpr std::integral_constant<int, 0> b0{};
            constexpr std::integral_constant<int, 1> b1{};
            if constexpr (NB == 4) {
                constexpr std::integral_constant<int, 2> b2{};
                constexpr std::integral_constant<int, 3> b3{};
                for (int j = 0;; j += 4) {
                    arrived(j);
                    clean_tiles(j - 1, 2, 3);
                    copy_v(j + 1, 1); copy_v(j + 2, 2); copy_k(j + 3, 3); copy_k(j + 4, 0);
                    if (even(j, b0) || odd(j + 1, b1)) break;
                    arrived(j + 2);
                    clean_tiles(j + 1, 2, 1);
                    copy_v(j + 3, 3); copy_v(j + 4, 0); copy_k(j + 5, 1); copy_k(j + 6, 2);
                    if (even(j + 2, b2) || odd(j + 3, b3)) break;
                }
            } else {
                for (int j = 0;; j += 2) {
                    arrived(j);
                    clean_tiles(j - 1, 1, 1);
                    copy_v(j, 0); copy_k(j + 2, 0);
                    if (even(j, b0)) break;
                    arrived(j + 1);
                    clean_tiles(j, 1, 0);
                    copy_v(j + 1, 1); copy_k(j + 3, 1);
                    if (odd(j + 1, b1)) break;
                }
            }
            wait_copies<0>();
            __syncthreads();
            clean_tiles(total - 1, 1, vlast);
            if (active) {
#pragma unroll
                for (int i = 0; i < MF; ++i) {
                    const unsigned off = TILE * vlast + KEYS16 * (i / DB);
                    const bf16x8 x = cat4(lds_at_tr4(tr_at[i % DB][0] + off), lds_at_tr4(tr_at[i % DB][1] + off));
                    o[i % DB] = mfma32(x, operand(pA, i), o[i % DB]);
                }
                // from R to m c
                const float f = __builtin_amdgcn_exp2f(offset_of(m)), lt = pair_sum(lsum) * f, lp = pair_sum(lprod) * f;
                const int row = 32 * w + c32;
                if (row < seg.rows && a.direct && tile0 == 0 && total == at.units && !left_out) {
                    const bool none = bits_of(lt) == 0;
                    const float inv = f / lp;
                    unsigned hr;
                    const int tok = seg.seq0 + (int)divmod((unsigned)(seg.row0 + row), seg.heads_each, hr), h = seg.kvh * seg.rep + (int)hr;
                    __bf16* const out = (__bf16*)a.o + ((int64_t)tok * seg.Hq + h) * D + 4 * hh;
#pragma unroll
                    for (int n = 0; n < 4 * DB; ++n) {
                        bf16x4 y;
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = (__bf16)(none ? 0.f : o[n >> 2][4 * (n & 3) + i] * inv);
                        *reinterpret_cast<bf16x4*>(out + 32 * (n >> 2) + 8 * (n & 3)) = y;
                    }
                    if (hh == 0) {
                        a.lse[(int64_t)h * a.n_tok + tok] = none ? -INFINITY : m * (a.c * LN2) + __logf(lt);
                        *reinterpret_cast<f32x4*>(a.stats + (seg.base + row) * 4) = f32x4{0.f, 0.f, 0.f, DONE};
                    }
                } else if (row < seg.rows) {
                    float* const out = a.sums + (seg.base + row) * D + 4 * hh;
#pragma unroll
                    for (int n = 0; n < 4 * DB; ++n) {
                        const f32x16& x = o[n >> 2];
                        const int r = 4 * (n & 3);
                        *reinterpret_cast<f32x4*>(out + 32 * (n >> 2) + 8 * (n & 3)) = f32x4{x[r] * f, x[r + 1] * f, x[r + 2] * f, x[r + 3] * f};
                    }
                    if (hh == 0) put_stats<true>(a, seg.base + row, m, lt, lp, left_out);
                }
            }
            work.left -= total;
            if (at.t + total >= at.units) work.left -= work.pad;
            if (work.left <= 0) return;
            at.t += total - 1;
            next();
        }
    } else if constexpr (KIND) {
        // Four waves: a unit of K and V in one half of LDS while the next is copied into the other, a wave copying 16 keys of each,
        // also from segment to segment.
        Rows<D, NC> r;
        unsigned half = 0;
        unsigned lo = 0, hi = 0;               // which of the next unit's keys there are
        auto issue = [&](unsigned dst) SP_INLINE {
            uint64_t mine = 0;
            int valid = 16;
            lo = hi = 0xffffffffu;
            const int key = 64 * at.t;
            if (whole(key, 64)) {
                mine = offset(key + 16 * w, __builtin_amdgcn_readfirstlane(pages.at((key + 16 * w) >> a.log_page)));
            } else {
                lo = hi = 0;
#pragma unroll 1
                for (int h = 0; h < 4; ++h) {
                    uint64_t off;
                    int v;
                    locate(key + 16 * h, off, v);
                    if (h == w) { mine = off; valid = v; }
                    (h < 2 ? lo : hi) |= low_bits(v) << (16 * (h & 1));
                }
            }
            copy.rows16(kc + mine, valid, dst + w * KEYS16);
            copy.rows16(vc + mine, valid, dst + (4 + w) * KEYS16);
        };
        pages.load(64 * at.t >> a.log_page);
        issue(buf);
        while (true) {
            SegmentRows seg(at, a, work.worker);
            const int n = (seg.rows + 15) >> 4, t0 = w * n >> 2, tiles = ((w + 1) * n >> 2) - t0;
            load_rows(r, q, seg, 16 * t0, tiles, l);
            r.clear(a.m_none);
            bool more = true, same = true;
            while (same) {
                const unsigned here[2] = {lo, hi};
                wait_copies<0>();
                __syncthreads();
                const unsigned kb = buf + half * 8 * KEYS16, vb = kb + 4 * KEYS16;
                half ^= 1;
                more = --work.left > 0;
                same = more && at.t + 1 < at.units;
                if (more) { next(); issue(buf + half * 8 * KEYS16); }
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    f32x4 s[NC][2];
                    bf16x8 pw[NC][2];
                    scores(r, kb + 2 * h * KEYS16, h ? here[1] : here[0], l, s);
                    weights(r, s, a.c, pw);
                    add_values(r, vb + 2 * h * KEYS16, pw, l);
                }
            }
            store_rows<TREE>(r, a, seg, 16 * t0, tiles, l);
            if (!more) return;
        }
    }
}

// ---- float32: all workers are waves, K and V are read straight into the operands' registers ------------------------------

// Products on float32 matrix instructions of 16 x 16 x 4.  S^T: lane group j = l / 16 contracts elements [j D / 4, (j + 1) D / 4) of its key, so
// that it reads them in pieces of 16 bytes.  O^T += V^T P^T: step i contracts keys 4 j + i, whose weight is score i of the lane, and row m of
// tile (h, e) is element 64 h + 4 m + e, so that V is read in pieces of 16 bytes as well.
template <int D, bool MANY, bool TREE = false>
__global__ __launch_bounds__(256, 2) void decode_f32_kernel(StartsArg<TREE> starts, DecodeArgs a) {
    __shared__ ListIs<TREE> lists[4096];
    __shared__ PlanShare<4> share;
    constexpr int NC = SOLO_ROWS / 16, HALVES = D / 64;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, m16 = l & 15, j = l >> 4;
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    const Lists<0, TREE> ls{words_of(starts), a};
    Work<TREE> work;
    if constexpr (MANY) work = find_work<4>(ls, lists, 4096, share, w, l); else work = find_work_in_lanes<4>(ls, w, l);
    if (work.left == 0) return;
    Cursor<0, TREE> at(ls, work);
    Pages pages;
    pages.lane = l;
    pages.n_pages = a.n_pages;
    while (true) {
        SegmentRows seg(at, a, work.worker);
        const bool prompt = at.list < a.n_groups;
        pages.table = prompt ? a.prompt_tables + at.list * a.prompt_width : a.resp_tables + (at.list - a.n_groups) * a.resp_width;
        pages.count = pages_of(at.len, a.log_page);
        const int run = min(work.left, at.units - at.t), key0 = 32 * at.t, key1 = (int)min((unsigned)at.len, 32u * (unsigned)(at.t + run));
        pages.load(key0 >> a.log_page);
        Drafted drafted;
        if constexpr (TREE) drafted.of(ls, at.list);
        const int tiles = (seg.rows + 15) >> 4;
        float q[NC][D / 4];
        f32x4 o[NC][HALVES][4];
        float m[NC], sum[NC];
        bool left_out = false;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int row = 16 * c + m16;
            const float* const src = (const float*)a.q + seg.q_row(row < seg.rows ? row : 0) * D + j * (D / 4);
#pragma unroll
            for (int e = 0; e < D / 4; e += 4) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(src + e);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[c][e + i] = x[i];
            }
            m[c] = a.m_none; sum[c] = 0.f;
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[c][h][e] = f32x4{0, 0, 0, 0};
        }
        for (int key = key0; key < key1; key += 16) {
            const int valid = min(16, key1 - key), page = __builtin_amdgcn_readfirstlane(pages.at(key >> a.log_page));
            if (page < 0 || page >= a.n_pages) continue;
            const int64_t row = ((((int64_t)page * a.Hkv + seg.kvh) << a.log_page) + (key & ((1 << a.log_page) - 1)));
            // keys behind the last one read the first one's row; their scores are masked, and their values taken for zero
            const float* const kp = (const float*)a.k_cache + (row + (m16 < valid ? m16 : 0)) * D + j * (D / 4);
            f32x4 k[D / 16], v[4][HALVES];
#pragma unroll
            for (int e = 0; e < D / 16; ++e) k[e] = *reinterpret_cast<const f32x4*>(kp + 4 * e);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float* const vp = (const float*)a.v_cache + (row + (4 * j + i < valid ? 4 * j + i : 0)) * D + 4 * m16;
#pragma unroll
                for (int h = 0; h < HALVES; ++h) v[i][h] = *reinterpret_cast<const f32x4*>(vp + 64 * h);
                if (valid < 16 && 4 * j + i >= valid)
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) v[i][h] = f32x4{0, 0, 0, 0};
            }
            bool some = false;
            if constexpr (TREE) {
                some = key + (int64_t)16 > drafted.base;
                if (some) {
                    bool found = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const unsigned x = bits_of(v[i][h][e]);
                                const bool bad = (x & 0x7f800000u) == 0x7f800000u;
                                v[i][h][e] = __uint_as_float(bad ? 0u : x);
                                found |= bad;
                            }
                    left_out |= __builtin_amdgcn_ballot_w64(found) != 0;
                }
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (c > 0 && c >= tiles) continue;
                f32x4 s = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < D / 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e >> 2][e & 3], q[c][e], s, 0, 0, 0);
                if (valid < 16)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[i] = 4 * j + i < valid ? s[i] : -INFINITY;
                if (TREE && some) {
                    const unsigned mine = drafted.bits(a, seg, 16 * c + m16, key) >> (4 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[i] = mine >> i & 1 ? s[i] : -INFINITY;
                }
                const float mn = fmaxf(m[c], quad_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])))), alpha = __builtin_amdgcn_exp2f((m[c] - mn) * a.c);
                m[c] = mn;
                float part = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) { s[i] = __builtin_amdgcn_exp2f((s[i] - mn) * a.c); part += s[i]; }
                sum[c] = sum[c] * alpha + part;
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[c][h][e][i] *= alpha;
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[c][h][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i][h][e], s[i], o[c][h][e], 0, 0, 0);
                    }
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int row = 16 * c + m16;
            const float lt = quad_sum(sum[c]);
            if (row >= seg.rows) continue;
            float* const out = a.sums + (seg.base + row) * D + 16 * j;
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(out + 64 * h + 4 * i) = f32x4{o[c][h][0][i], o[c][h][1][i], o[c][h][2][i], o[c][h][3][i]};
            if (j == 0) put_stats<TREE>(a, seg.base + row, m[c], lt, lt, left_out);
        }
        work.left -= run;
        if (work.left == 0) return;
        at.t += run - 1;
        at.next();
    }
}

// ---- the join ------------------------------------------------------------------------------------------------

// One wave per sequence and q head: o = sum_c e^(m_c - M) O_c / sum_c e^(m_c - M) l_c over the chunks of the prompt and of the response.
// Bound: the latency of two loads that wait for each other (where the sums are; the sums and their statistics) and of fetching code that
// runs once.  Hence even lanes find the prompt's chunks and odd ones the response's with the same instructions, the lanes that hold a row (D / 4)
// load its statistics too and keep a maximum of their own, and these meet at the end.  DENSE: such lanes do all of an item, and a
// wave takes 256 / D of them.
// Drafted tokens: 115k rows of 64 short prompts' answers 39 us, 76 MB, bound by vector instructions (45 with integer divisions and four chunks at a time; four rows one after
// the other to the same lanes, which share the search, 2 us less there and 1 more for chunks behind long responses).
template <typename T, int D, bool DENSE, bool TREE = false>
__global__ __launch_bounds__(256) void decode_join_kernel(StartsArg<TREE> starts, DecodeArgs a) {
    constexpr int LANES = D / 4, EACH = DENSE ? LANES : 64, AT_ONCE = EACH / LANES, DEPTH = TREE && DENSE ? 2 : 4;
    const Starts<TREE> w = words_of(starts);
    const int l = threadIdx.x & (EACH - 1), mine = l / LANES, e0 = 4 * (l % LANES);
    const int64_t item = DENSE ? (int64_t)blockIdx.x * (256 / EACH) + threadIdx.x / EACH
                               : (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n_rows = TREE ? a.n_tok : a.n_seqs;
    if (item >= (int64_t)n_rows * a.Hq) return;
    unsigned in_seq, hr;
    const int tok = (int)divmod((unsigned)item, a.q_heads, in_seq), h = (int)in_seq;      // token, or sequence
    const int kvh = (int)divmod((unsigned)h, a.heads_each, hr);
    int g = 0, first, members = a.members, seq = tok, node = 0, own = 1;      // `own` rows of the sequence per q head, this one's number
    if (members) {
        unsigned rest;
        g = (int)divmod((unsigned)tok, a.group_size, rest);
        first = tok - (int)rest;
        if constexpr (TREE) { seq = (int)divmod((unsigned)tok, a.seq_size, rest); node = (int)rest; own = a.each; }
    } else {
        if constexpr (TREE) {
            // the last of the groups, and of the sequences, that starts at the token or ahead of it: as many candidates at a time as the row has lanes
            auto of_row = [](bool b) {
                const uint64_t all = __builtin_amdgcn_ballot_w64(b);
                const unsigned half = half_of_lane(all);
                return EACH == 64 ? __popcll(all) : __popc(EACH == 32 ? half : half >> (threadIdx.x & 31 & ~(EACH - 1)) & ((1u << (EACH & 31)) - 1));
            };
            int ge = a.n_groups, sb = a.n_groups + 1, se = sb + a.n_seqs;
            while (__builtin_amdgcn_ballot_w64(ge - g > 1 || se - sb > 1)) {
                const int gs = (ge - g + EACH - 1) / EACH, ss = (se - sb + EACH - 1) / EACH, gi = g + l * gs, si = sb + l * ss;
                const int gw = w[min(gi, ge - 1)], sw = w[min(si, se - 1)];
                g += (of_row(gi < ge && gw <= tok) - 1) * gs;
                sb += (of_row(si < se && sw <= tok) - 1) * ss;
                ge = min(ge, g + gs);
                se = min(se, sb + ss);
            }
            seq = sb - a.n_groups - 1;
            node = tok - w[sb];
            own = w[sb + 1] - w[sb];
        } else {
            int hi = a.n_groups;
            while (hi - g > 1) { const int mid = (g + hi) >> 1; if (w[mid] <= tok) g = mid; else hi = mid; }
        }
        first = w[g];
        members = w[g + 1] - first;
    }
    // The side's chunks: consecutive slots, those of the workers that had units of this row's segment, from the first one's on.  Rows of slots
    // are below 2^32: a workspace of so many has more than 1 TB.
    const bool resp = l & 1;
    const i32x4 run = a.desc[0], d = a.desc[1 + (resp ? a.n_groups + seq : g)];
    const int rows = resp ? own * a.rep : members * a.rep, row = resp ? node * a.rep + (int)hr : (tok - first) * a.rep + (int)hr;
    const bool shared = sizeof(T) == 2 && rows > (!TREE ? SOLO_ROWS : resp ? a.wide_resps : a.wide_prompts);
    int per = TREE ? (int)a.solo_rows.d : SOLO_ROWS;
    if (sizeof(T) == 2) {
        unsigned rest;
        const int blocks = (int)divmod((unsigned)(rows - 1), a.block_rows, rest) + 1;
        if (shared) per = TREE ? (int)a.block_rows.d : 16 * ((((rows + 15) >> 4) + blocks - 1) / blocks);
    }
    int block, segment;
    if constexpr (TREE) {
        Div by = a.solo_rows;
        if (shared) by = a.block_rows;
        unsigned rest;
        block = (int)divmod((unsigned)row, by, rest);
        segment = kvh * ((int)divmod((unsigned)(rows - 1), by, rest) + 1) + block;
    } else {
        block = rows > per ? row / per : 0;
        segment = block * a.Hkv + kvh;
    }
    const unsigned each = shared ? run[0] : run[1], from = (unsigned)d[0] * a.Hkv + (unsigned)segment * d[3];
    const unsigned worker0 = TREE ? quotient(from, each) : from / each, worker1 = TREE ? quotient(from + d[1] - 1, each) : (from + d[1] - 1) / each;
    const unsigned stride = shared ? a.shared_rows : resp ? a.resp_rows : a.prompt_rows;
    unsigned at = (unsigned)(shared ? 0 : resp ? a.resp_base : a.prompt_base) + (worker0 + (unsigned)d[2] * a.Hkv + segment) * stride + row - block * per;
    if (TREE && shared)
        at = worker0 * stride + ((unsigned)d[2] * a.Hkv + kvh * ((rows + 15) >> 4) + block * (per >> 4)) * 16 + row - block * per;
    const int count = d[1] > 0 ? (int)(worker1 - worker0) + 1 : 0;
    auto prompts = [](unsigned x) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x00, 0xf, 0xf, true); };     // of the even lanes
    auto resps = [](unsigned x) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x55, 0xf, 0xf, true); };       // of the odd ones
    const bool part = (int)resps(d[3]) >= 0;
    const int n_p = part ? (int)prompts(count) : 0, n = part ? n_p + (int)resps(count) : 0;
    const unsigned at_p = prompts(at), at_r = resps(at), stride_p = prompts(stride), stride_r = resps(stride);
    typedef std::conditional_t<TREE, f32x4, f32x2> Stats;
    if constexpr (TREE) {
        if (a.direct && n == 1 && a.stats[(uint64_t)(n_p ? at_p : at_r) * 4 + 3] == DONE) return;
    }
    float M = a.m_none, L = 0.f, LP = 0.f;             // LP: of the weights that the products took (TREE)
    bool left_out = false;
    f32x4 acc = {0, 0, 0, 0};
    for (int i = 0; i < n; i += DEPTH * AT_ONCE) {
        Stats st[DEPTH];
        f32x4 x[DEPTH];
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            const int k = min(i + u * AT_ONCE + mine, n - 1);              // behind the last: again, and not counted
            const unsigned at_k = k < n_p ? at_p + k * stride_p : at_r + (k - n_p) * stride_r;
            st[u] = *reinterpret_cast<const Stats*>(a.stats + (uint64_t)at_k * (sizeof(Stats) / 4));
            x[u] = *reinterpret_cast<const f32x4*>(a.sums + (uint64_t)at_k * D + e0);
        }
        float mn = M;
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) mn = fmaxf(mn, st[u][0]);
        const float alpha = __builtin_amdgcn_exp2f((M - mn) * a.c);
        M = mn;
        L *= alpha;
        if constexpr (TREE) LP *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= alpha;
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            if (i + u * AT_ONCE + mine >= n) continue;                     // (not with a weight of 0: sums may be infinite)
            const float wt = __builtin_amdgcn_exp2f((st[u][0] - mn) * a.c);
            L += wt * st[u][1];
            if constexpr (TREE) { LP += wt * st[u][2]; left_out |= bits_of(st[u][3]) != 0; }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += wt * x[u][e];
        }
    }
#pragma unroll
    for (int o = EACH / 2; o >= LANES; o >>= 1) {
        const float m2 = __shfl_xor(M, o, 64), mn = fmaxf(M, m2), wt = __builtin_amdgcn_exp2f((M - mn) * a.c), wt2 = __builtin_amdgcn_exp2f((m2 - mn) * a.c);
        M = mn;
        L = L * wt + __shfl_xor(L, o, 64) * wt2;
        if constexpr (TREE) { LP = LP * wt + __shfl_xor(LP, o, 64) * wt2; left_out |= (bool)__shfl_xor((int)left_out, o, 64); }
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = acc[e] * wt + __shfl_xor(acc[e], o, 64) * wt2;
    }
    // Without a key L is 0, and a NaN among the scores is in L
    const bool none = bits_of(L) == 0;
    const float inv = 1.f / (TREE ? LP : L);
    if constexpr (TREE) {
        // Infinite and NaN values that the products left out: those of the keys that the row sees, from the first unit with drafted ones on
        if (left_out) {
            const int len = min(a.resp_lens[seq], a.resp_cap), base = a.resp_lens[seq] - own, words = (own + 31) >> 5;
            const uint32_t* const mask = a.ancestors ? a.ancestors + (int64_t)tok * a.mask_stride : nullptr;
            for (int key = max(base & ~63, 0); key < len; ++key) {
                const int page = a.resp_tables[seq * a.resp_width + (key >> a.log_page)];
                if ((unsigned)page >= (unsigned)a.n_pages || !(drafted_bits(mask, words, node, key - base) & 1)) continue;
                const T* const v = (const T*)a.v_cache + (((((int64_t)page * a.Hkv + kvh) << a.log_page) + (key & ((1 << a.log_page) - 1))) * D + e0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = (float)v[e];
                    if ((bits_of(x) & 0x7f800000u) == 0x7f800000u) acc[e] += x;
                }
            }
        }
    }
    if (mine == 0) {
        typedef T out4 __attribute__((ext_vector_type(4)));
        out4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (T)(none ? 0.f : acc[e] * inv);
        *reinterpret_cast<out4*>((T*)a.o + item * D + e0) = y;
    }
    if (l == 0) a.lse[(int64_t)h * n_rows + tok] = none ? -INFINITY : M * (a.c * LN2) + __logf(L);
}

}  // namespace
}  // namespace sp
