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
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <algorithm>
#include <type_traits>

namespace sp {
namespace {

#define SP_INLINE __attribute__((always_inline))      // lambdas: what they refer to has to stay in registers

constexpr int SOLO_ROWS = 32;              // rows of a segment that a wave takes by itself
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
struct ListShape { int rows, len, units, blocks; bool shared; };      // units of keys of a segment; blocks of rows
struct PlanShare { int sums[4][4]; int list[4], at[4], ord[4], rows[4], len[4], room[4]; };      // of the waves of a workgroup; where their runs start

// KIND 0: all lists are solo, 1: shared ones too
template <int KIND>
struct Lists {
    const int* starts;                       // first sequence of each group, where groups are of several sizes
    const DecodeArgs& a;
    __device__ __forceinline__ i32x2 read(int i) const {      // rows and length, -1: takes no part
        const bool prompt = i < a.n_groups;
        const int prompt_cap = a.prompt_cap, resp_cap = a.resp_cap;
        const int* const prompt_lens = a.prompt_lens;
        const int* const resp_lens = a.resp_lens - a.n_groups;
        const int n = prompt && !prompt_cap ? 0 : (prompt ? prompt_lens : resp_lens)[i];
        int members = 1;
        if (prompt) members = a.members ? a.members : starts[i + 1] - starts[i];
        return i32x2{a.rep * members, min(max(n, -1), prompt ? prompt_cap : resp_cap)};
    }
    __device__ __forceinline__ ListShape shape(i32x2 x) const {
        ListShape s;
        s.rows = x[0];
        s.len = x[1];
        s.shared = KIND && s.rows > SOLO_ROWS;
        s.units = s.rows > 0 && s.len > 0 ? (int)(((unsigned)s.len + (s.shared ? 63u : 31u)) >> (s.shared ? 6 : 5)) : 0;
        unsigned rest;
        s.blocks = s.shared ? (int)divmod((unsigned)(s.rows - 1), a.block_rows, rest) + 1 : (s.rows + SOLO_ROWS - 1) / SOLO_ROWS;
        return s;
    }
    __device__ __forceinline__ int first_seq(int i) const { return i >= a.n_groups ? i - a.n_groups : a.members ? i * a.members : starts[i]; }
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
// units of room that a segment has among those of its kind
__device__ __forceinline__ int room_of(int units, unsigned run, bool aligned) { return aligned && units > 0 ? (int)(per_place(units, run) * run) : units; }

// What a worker does: `left` units from unit `at` of a list on (counted over the list's segments).
struct Work { bool shared; int worker, list, at, ord, left, room; i32x2 list_is; };

// The runs of either kind, from the units and segments of all lists.  Places are dealt by cost: a segment costs, for its rows and its sums, what one and a half of its
// units (shared) or one (solo) cost, and a shared unit what shared_cost solo ones do.  A worker that passes from one segment to another takes
// longer; where shared segments are long against the run, each is dealt to workers of its own, in room that is a multiple of the run (`aligned`: 37.8 us
// for the prompt of 16k tokens, 41.4 without).
struct Runs { unsigned shared_run, solo_run, used; bool aligned; };      // used: workgroups of shared segments
template <int KIND>
__device__ __forceinline__ void shared_runs(const DecodeArgs& a, unsigned solo, unsigned solo_segs, unsigned shared, unsigned segs, Runs& r) {
    r = Runs{1, 1, 0, false};
    if constexpr (KIND) {
        if (shared == 0) return;
        const float cost = a.shared_cost * ((float)shared + 1.5f * (float)segs);
        int wgs = (int)(PLAN_WGS * (cost * __builtin_amdgcn_rcpf(cost + (float)solo + (float)solo_segs)));
        wgs = max(1, min(wgs, solo ? PLAN_WGS - 1 : PLAN_WGS));
        r.aligned = 4 * segs <= (unsigned)wgs;
        r.shared_run = per_place(shared, r.aligned ? wgs - segs : wgs);
    }
}

// Every workgroup makes the whole plan.  Written for few instructions: what a workgroup runs once comes from memory, 64 bytes at a time, and
// takes a cycle a byte.
// Up to 64 lists: a wave by itself, a list to a lane (one sequence of 1k tokens 5.7 us, by the workgroup 7.0; a group of 8 8.2 and 11.0).
template <int KIND>
__device__ __forceinline__ Work find_work_in_lanes(const Lists<KIND>& ls, int wave, int lane) {
    const DecodeArgs& a = ls.a;
    const int n = a.n_groups + a.n_seqs;
    const bool there = lane < n;
    i32x2 mine{0, 0};
    if (there) mine = ls.read(lane);
    const ListShape s = ls.shape(mine);
    auto last = [](int x) SP_INLINE { return (unsigned)__builtin_amdgcn_readlane(x, 63); };
    const int solo_units = s.shared ? 0 : s.units * s.blocks, solo_blocks = s.shared ? 0 : s.blocks;
    const int to_solo = scan64(solo_units), ord_solo = scan64(solo_blocks);
    const unsigned solo = last(to_solo) * a.Hkv;
    int room = s.units, units = solo_units, to = to_solo, ord = ord_solo - solo_blocks;
    unsigned shared_room = 0;
    Runs runs{1, 1, 0, false};
    if constexpr (KIND) {
        const int shared_units = s.shared ? s.units * s.blocks : 0, shared_blocks = s.shared ? s.blocks : 0;
        const int ord_shared = scan64(shared_blocks);
        shared_runs<KIND>(a, solo, last(ord_solo) * a.Hkv, last(scan64(shared_units)) * a.Hkv, last(ord_shared) * a.Hkv, runs);
        if (s.shared) { room = room_of(s.units, runs.shared_run, runs.aligned); units = room * s.blocks; ord = ord_shared - shared_blocks; }
        const int to_shared = scan64(s.shared ? units : 0);
        if (s.shared) to = to_shared;
        shared_room = last(to_shared) * a.Hkv;
        if (shared_room) runs.used = per_place(shared_room, runs.shared_run);
    }
    if (solo) runs.solo_run = per_place(solo, 4 * (PLAN_WGS - runs.used));
    if (blockIdx.x == 0 && wave == 0) {          // what the join needs to know
        if (there) a.desc[1 + lane] = i32x4{to - units, s.units, ord, s.len < 0 ? -1 : room};
        if (lane == 0) a.desc[0] = i32x4{(int)runs.shared_run, (int)runs.solo_run, 0, 0};
    }
    Work work;
    work.shared = blockIdx.x < runs.used;
    work.worker = work.shared ? (int)blockIdx.x : (int)(blockIdx.x - runs.used) * 4 + wave;
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
    work.list_is = i32x2{of(mine[0]), of(mine[1])};
    return work;
}

// More lists: a thread adds up the units of its share of them (they lie in LDS meanwhile, if there are no more than n_held), the workgroup their sums.
template <int KIND>
__device__ __forceinline__ Work find_work(const Lists<KIND>& ls, i32x2* held, int n_held, PlanShare& share, int wave, int lane) {
    constexpr int SUMS = KIND ? 4 : 2;       // solo units and blocks, shared units and blocks
    const DecodeArgs& a = ls.a;
    const int n = a.n_groups + a.n_seqs, per = (n + 255) >> 8, i0 = min(n, (int)threadIdx.x * per), i1 = min(n, i0 + per);
    const bool in_lds = n <= n_held;
    if (in_lds) {
        for (int i = threadIdx.x; i < n; i += 256 * 4) {      // four reads in flight
            i32x2 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) if (i + 256 * u < n) x[u] = ls.read(i + 256 * u);
#pragma unroll
            for (int u = 0; u < 4; ++u) if (i + 256 * u < n) held[i + 256 * u] = x[u];
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
        }
    };
    auto over_waves = [&](int k) SP_INLINE {       // to[k], inclusive, and all[k] from own[k]
        to[k] = scan64(own[k]);
        __syncthreads();
        if (lane == 63) share.sums[wave][k] = to[k];
        __syncthreads();
        unsigned sum = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) { const int x = share.sums[w][k]; to[k] += w < wave ? x : 0; sum += x; }
        all[k] = sum * a.Hkv;
    };
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
        const ListShape s = ls.shape(list_of(i));
        add(own, s, s.units);
    }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) over_waves(k);
    Runs runs{1, 1, 0, false};
    if constexpr (KIND) {
        shared_runs<KIND>(a, all[0], all[1], all[SUMS - 2], all[SUMS - 1], runs);
        if (runs.aligned) {
            own[SUMS - 2] = 0;
#pragma unroll 1
            for (int i = i0; i < i1; ++i) {
                const ListShape s = ls.shape(list_of(i));
                own[SUMS - 2] += s.shared ? room_of(s.units, runs.shared_run, true) * s.blocks : 0;
            }
            over_waves(SUMS - 2);
        }
        if (all[SUMS - 2]) runs.used = per_place(all[SUMS - 2], runs.shared_run);
    }
    if (all[0]) runs.solo_run = per_place(all[0], 4 * (PLAN_WGS - runs.used));
    // this workgroup's runs start at `first` and multiples of the run behind it
    Work work;
    const bool shared = work.shared = blockIdx.x < runs.used;
    const unsigned run = shared ? runs.shared_run : runs.solo_run, many = shared ? 1 : 4, first = (shared ? blockIdx.x : 4 * (blockIdx.x - runs.used)) * run;
    const bool tells = blockIdx.x == 0;          // the first workgroup writes down what the join needs to know
    const int mine = KIND && shared ? SUMS - 2 : 0;
    const unsigned through = (unsigned)(mine ? to[SUMS - 2] : to[0]) * a.Hkv, ahead = through - (unsigned)(mine ? own[SUMS - 2] : own[0]) * a.Hkv;
    if (tells || (ahead < first + many * run && through > first)) {
        int at[SUMS];
#pragma unroll
        for (int k = 0; k < SUMS; ++k) at[k] = to[k] - own[k];
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            const i32x2 x = list_of(i);
            const ListShape s = ls.shape(x);
            const int units = s.shared ? at[SUMS - 2] : at[0], blocks = s.shared ? at[SUMS - 1] : at[1], room = room_of(s.units, runs.shared_run, s.shared && runs.aligned);
            const unsigned from = (unsigned)units * a.Hkv, end = from + (unsigned)(room * s.blocks) * a.Hkv;
            if (s.shared == shared)
#pragma unroll 1
                for (unsigned k = 0; k < many; ++k) {
                    const unsigned pos = first + k * run;
                    if (pos >= from && pos < end) {
                        share.list[k] = i; share.at[k] = (int)(pos - from); share.ord[k] = blocks;
                        share.rows[k] = x[0]; share.len[k] = x[1]; share.room[k] = room;
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
    const unsigned pos = first + slot * run, end = mine ? all[SUMS - 2] : all[0];
    work.left = pos < end ? scalar((int)min(run, end - pos)) : 0;
    work.worker = scalar(shared ? (int)blockIdx.x : (int)(blockIdx.x - runs.used) * 4 + wave);
    work.list = scalar(share.list[slot]);
    work.at = scalar(share.at[slot]);
    work.ord = scalar(share.ord[slot]);
    work.room = scalar(share.room[slot]);
    work.list_is = i32x2{share.rows[slot], share.len[slot]};
    return work;
}

// A place among the units: of list `list` segment `seg` (block * n_kv_heads + kv head), unit `t`
template <int KIND>
struct Cursor {
    const Lists<KIND>& ls;
    const bool shared;
    int list, seg, t, units, segs, rows, len, blocks, ord;
    __device__ __forceinline__ Cursor(const Lists<KIND>& l, Work& w) : ls(l), shared(w.shared), list(w.list), ord(w.ord) {
        load(w.list_is);
        const float inv = __builtin_amdgcn_rcpf((float)w.room);        // a quotient, what it leaves divided again, and a step to either side
        seg = (int)((float)w.at * inv);
        seg += (int)((float)(w.at - seg * w.room) * inv);
        seg = __builtin_amdgcn_readfirstlane(seg);
        seg -= seg * w.room > w.at;
        seg += (unsigned)(seg + 1) * w.room <= (unsigned)w.at;
        t = w.at - seg * w.room;
        if (w.room > units) w.left = min(w.left, units - t);        // a run of the segment's own, the last one shorter
    }
    __device__ __forceinline__ bool load(i32x2 x) {
        const ListShape s = ls.shape(x);
        auto scalar = [](int x) SP_INLINE { return __builtin_amdgcn_readfirstlane(x); };
        rows = scalar(s.rows); len = scalar(s.len); units = scalar(s.units); blocks = scalar(s.blocks);
        segs = blocks * ls.a.Hkv;
        return s.shared == shared;
    }
    // the next unit; there is one
    __device__ __forceinline__ void next() {
        if (++t < units) return;
        t = 0;
        if (++seg < segs) return;
        seg = 0;
        ord += blocks;
        do {
            ++list;
            if (load(ls.read(list))) { if (units > 0) return; ord += blocks; }
        } while (list < ls.a.n_groups + ls.a.n_seqs - 1);
    }
};

// Rows of a segment: where they come from, and the slot that they go to
struct SegmentRows {
    int seq0, rep, row0, rows, Hq, kvh, block;          // rows row0 ... row0 + rows - 1 of the list
    int64_t base;                                // of row0 among the rows of sums
    Div heads_each;
    template <int KIND> __device__ __forceinline__ SegmentRows(const Cursor<KIND>& c, const DecodeArgs& a, int worker) {
        unsigned k;
        block = c.blocks > 1 ? (int)divmod((unsigned)c.seg, a.kv_heads, k) : 0;
        kvh = c.blocks > 1 ? (int)k : c.seg;
        const int per = c.shared ? 16 * (((((c.rows + 15) >> 4)) + c.blocks - 1) / c.blocks) : SOLO_ROWS;
        row0 = block * per;
        rows = min(per, c.rows - row0);
        seq0 = c.ls.first_seq(c.list);
        rep = a.rep; Hq = a.Hq; heads_each = a.heads_each;
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

template <int D, int NC>
__device__ __forceinline__ void store_rows(const Rows<D, NC>& r, const DecodeArgs& a, const SegmentRows& pr, int row0, int tiles, int l) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int row = row0 + 16 * c + (l & 15);
        const float lt = quad_sum(r.l[c]);
        if (c >= tiles || row >= pr.rows) continue;
        float* const out = a.sums + (pr.base + row) * D + 4 * (l >> 4);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(out + 16 * dt) = r.o[c][dt];
        if (l < 16) *reinterpret_cast<f32x2*>(a.stats + (pr.base + row) * 2) = f32x2{r.m[c], lt};
    }
}

// NC: row tiles of a wave in a shared segment, 0: no list is shared.  NS: in a solo one.
template <int D, int NC, int NS, bool MANY>
__global__ __launch_bounds__(256, 2) void decode_kernel(SeqArg starts, DecodeArgs a) {
    constexpr int KEYS16 = 32 * D, KIND = NC > 0;       // bytes of 16 keys
    __shared__ __attribute__((aligned(1024))) char lds[16 * KEYS16];
    __shared__ PlanShare share;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63;
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    const Lists<KIND> ls{words_of(starts), a};
    Work work;
    if constexpr (MANY) {
        work = find_work<KIND>(ls, reinterpret_cast<i32x2*>(lds), (int)sizeof(lds) / 8, share, w, l);
        __syncthreads();                             // the lists' place is free
    } else {
        work = find_work_in_lanes<KIND>(ls, w, l);
    }
    if (work.left == 0) return;
    Cursor<KIND> at(ls, work);
    auto kv_head = [&]() SP_INLINE {
        unsigned k = (unsigned)at.seg;
        if (KIND && at.blocks > 1) divmod((unsigned)at.seg, a.kv_heads, k);
        return (int)k;
    };
    int kvh = kv_head();
    Pages pages;
    pages.lane = l;
    pages.n_pages = a.n_pages;
    auto table_of_list = [&]() SP_INLINE {
        const bool prompt = at.list < a.n_groups;
        pages.table = prompt ? a.prompt_tables + at.list * a.prompt_width : a.resp_tables + (at.list - a.n_groups) * a.resp_width;
        pages.count = pages_of(at.len, a.log_page);
    };
    auto next = [&]() SP_INLINE {
        const int list = at.list;
        at.next();
        if (at.list != list) { table_of_list(); pages.load(0); }
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
        valid = min(16, at.len - key);
        off = 0;
        if (valid <= 0) return;
        const int page = __builtin_amdgcn_readfirstlane(pages.at(key >> a.log_page));
        if ((unsigned)page >= (unsigned)a.n_pages) { valid = 0; return; }
        off = offset(key, page);
    };
    // whether all of `count` keys are there (the pages held include the last one's; if any of those held is none, it is looked at in turn)
    auto whole = [&](int key, int count) SP_INLINE {
        if (key + count > at.len) return false;
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
            const int key = 32 * at.t;
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
        pages.load(32 * at.t >> a.log_page);
        fetch();
        issue(kc, kb);
        issue(vc, vb);
        while (true) {
            SegmentRows seg(at, a, work.worker);
            const int tiles = (seg.rows + 15) >> 4;
            load_rows(r, q, seg, 0, tiles, l);
            r.clear(a.m_none);
            bool more = true, same = true;
            while (same) {
                const unsigned bits = low_bits(valid[0]) | low_bits(valid[1]) << 16;
                f32x4 s[NS][2];
                bf16x8 pw[NS][2];
                wait_copies<N>();
                scores(r, kb, bits, l, s);
                wait_lds();
                more = --work.left > 0;
                same = more && at.t + 1 < at.units;
                if (more) { next(); fetch(); issue(kc, kb); }
                weights(r, s, a.c, pw);
                if (more) wait_copies<N>(); else wait_copies<0>();
                add_values(r, vb, pw, l);
                wait_lds();
                if (more) issue(vc, vb);
            }
            store_rows(r, a, seg, 0, tiles, l);
            if (!more) return;
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
            store_rows(r, a, seg, 16 * t0, tiles, l);
            if (!more) return;
        }
    }
}

// ---- float32: all workers are waves, K and V are read straight into the operands' registers ------------------------------

// Products on float32 matrix instructions of 16 x 16 x 4.  S^T: lane group j = l / 16 contracts elements [j D / 4, (j + 1) D / 4) of its key, so
// that it reads them in pieces of 16 bytes.  O^T += V^T P^T: step i contracts keys 4 j + i, whose weight is score i of the lane, and row m of
// tile (h, e) is element 64 h + 4 m + e, so that V is read in pieces of 16 bytes as well.
template <int D, bool MANY>
__global__ __launch_bounds__(256, 2) void decode_f32_kernel(SeqArg starts, DecodeArgs a) {
    __shared__ i32x2 lists[4096];
    __shared__ PlanShare share;
    constexpr int NC = SOLO_ROWS / 16, HALVES = D / 64;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, m16 = l & 15, j = l >> 4;
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    const Lists<0> ls{words_of(starts), a};
    Work work;
    if constexpr (MANY) work = find_work<0>(ls, lists, 4096, share, w, l); else work = find_work_in_lanes<0>(ls, w, l);
    if (work.left == 0) return;
    Cursor<0> at(ls, work);
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
        const int tiles = (seg.rows + 15) >> 4;
        float q[NC][D / 4];
        f32x4 o[NC][HALVES][4];
        float m[NC], sum[NC];
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
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (c > 0 && c >= tiles) continue;
                f32x4 s = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < D / 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e >> 2][e & 3], q[c][e], s, 0, 0, 0);
                if (valid < 16)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[i] = 4 * j + i < valid ? s[i] : -INFINITY;
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
            if (j == 0) *reinterpret_cast<f32x2*>(a.stats + (seg.base + row) * 2) = f32x2{m[c], lt};
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
template <typename T, int D, bool DENSE>
__global__ __launch_bounds__(256) void decode_join_kernel(SeqArg starts, DecodeArgs a) {
    constexpr int LANES = D / 4, EACH = DENSE ? LANES : 64, AT_ONCE = EACH / LANES, DEPTH = 4;
    const int* const w = words_of(starts);
    const int l = threadIdx.x & (EACH - 1), mine = l / LANES, e0 = 4 * (l % LANES);
    const int64_t item = DENSE ? (int64_t)blockIdx.x * (256 / EACH) + threadIdx.x / EACH
                               : (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (item >= (int64_t)a.n_seqs * a.Hq) return;
    unsigned in_seq, hr;
    const int seq = (int)divmod((unsigned)item, a.q_heads, in_seq), h = (int)in_seq;
    const int kvh = (int)divmod((unsigned)h, a.heads_each, hr);
    int g = 0, first, members = a.members;
    if (members) {
        unsigned rest;
        g = (int)divmod((unsigned)seq, a.group_size, rest);
        first = seq - (int)rest;
    } else {
        int hi = a.n_groups;
        while (hi - g > 1) { const int mid = (g + hi) >> 1; if (w[mid] <= seq) g = mid; else hi = mid; }
        first = w[g];
        members = w[g + 1] - first;
    }
    // The side's chunks: consecutive slots, those of the workers that had units of this row's segment, from the first one's on.  Rows of slots
    // are below 2^32: a workspace of so many has more than 1 TB.
    const bool resp = l & 1;
    const i32x4 run = a.desc[0], d = a.desc[1 + (resp ? a.n_groups + seq : g)];
    const int rows = resp ? a.rep : members * a.rep, row = resp ? (int)hr : (seq - first) * a.rep + (int)hr;
    const bool shared = sizeof(T) == 2 && rows > SOLO_ROWS;
    int per = SOLO_ROWS;
    if (sizeof(T) == 2) {
        unsigned rest;
        const int blocks = (int)divmod((unsigned)(rows - 1), a.block_rows, rest) + 1;
        if (shared) per = 16 * ((((rows + 15) >> 4) + blocks - 1) / blocks);
    }
    const int block = rows > per ? row / per : 0, segment = block * a.Hkv + kvh;
    const unsigned each = shared ? run[0] : run[1], from = (unsigned)d[0] * a.Hkv + (unsigned)segment * d[3];
    const unsigned worker0 = from / each, worker1 = (from + d[1] - 1) / each;
    const unsigned stride = shared ? a.shared_rows : resp ? a.resp_rows : a.prompt_rows;
    const unsigned at = (unsigned)(shared ? 0 : resp ? a.resp_base : a.prompt_base) + (worker0 + (unsigned)d[2] * a.Hkv + segment) * stride + row - block * per;
    const int count = d[1] > 0 ? (int)(worker1 - worker0) + 1 : 0;
    auto prompts = [](unsigned x) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x00, 0xf, 0xf, true); };     // of the even lanes
    auto resps = [](unsigned x) { return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x55, 0xf, 0xf, true); };       // of the odd ones
    const bool part = (int)resps(d[3]) >= 0;
    const int n_p = part ? (int)prompts(count) : 0, n = part ? n_p + (int)resps(count) : 0;
    const unsigned at_p = prompts(at), at_r = resps(at), stride_p = prompts(stride), stride_r = resps(stride);
    float M = a.m_none, L = 0.f;
    f32x4 acc = {0, 0, 0, 0};
    for (int i = 0; i < n; i += DEPTH * AT_ONCE) {
        f32x2 st[DEPTH];
        f32x4 x[DEPTH];
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            const int k = min(i + u * AT_ONCE + mine, n - 1);              // behind the last: again, and not counted
            const unsigned at_k = k < n_p ? at_p + k * stride_p : at_r + (k - n_p) * stride_r;
            st[u] = *reinterpret_cast<const f32x2*>(a.stats + (uint64_t)at_k * 2);
            x[u] = *reinterpret_cast<const f32x4*>(a.sums + (uint64_t)at_k * D + e0);
        }
        float mn = M;
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) mn = fmaxf(mn, st[u][0]);
        const float alpha = __builtin_amdgcn_exp2f((M - mn) * a.c);
        M = mn;
        L *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= alpha;
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            if (i + u * AT_ONCE + mine >= n) continue;                     // (not with a weight of 0: sums may be infinite)
            const float wt = __builtin_amdgcn_exp2f((st[u][0] - mn) * a.c);
            L += wt * st[u][1];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += wt * x[u][e];
        }
    }
#pragma unroll
    for (int o = EACH / 2; o >= LANES; o >>= 1) {
        const float m2 = __shfl_xor(M, o, 64), mn = fmaxf(M, m2), wt = __builtin_amdgcn_exp2f((M - mn) * a.c), wt2 = __builtin_amdgcn_exp2f((m2 - mn) * a.c);
        M = mn;
        L = L * wt + __shfl_xor(L, o, 64) * wt2;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = acc[e] * wt + __shfl_xor(acc[e], o, 64) * wt2;
    }
    // Without a key L is 0, and a NaN among the scores is in L
    const bool none = bits_of(L) == 0;
    const float inv = 1.f / L;
    if (mine == 0) {
        typedef T out4 __attribute__((ext_vector_type(4)));
        out4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (T)(none ? 0.f : acc[e] * inv);
        *reinterpret_cast<out4*>((T*)a.o + item * D + e0) = y;
    }
    if (l == 0) a.lse[(int64_t)h * a.n_seqs + seq] = none ? -INFINITY : M * (a.c * LN2) + __logf(L);
}

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
