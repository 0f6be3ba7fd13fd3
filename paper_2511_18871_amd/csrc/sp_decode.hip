// Attention of one new token per sequence over the paged cache: the shared-prompt attention of Section 4.3 in the form of a rollout
// step.  The G sequences of a group read the pages of their common prompt, and each the pages of its own response.
//   S_j = scale <q, k_j> over the keys [0, Lp) of the prompt and [0, len) of the response,
//   o = sum_j e^(S_j - m) v_j / l, l = sum_j e^(S_j - m), lse = m + ln l; without a key o = 0 and lse = -inf.
//
// Bound: the keys and values, each read once.  A LIST is what is walked together: the prompt of a group, seen by its G rep rows of
// each kv head (rep = n_q_heads / n_kv_heads; row r is q head r % rep of the group's sequence r / rep), or the response of a
// sequence, seen by its rep rows.  Lists are cut into chunks of keys; a chunk leaves unnormalised sums (m, l, sum p v) of its rows in the
// workspace, and the join kernel adds up those of a row.  Lengths are on the device, so the cutting happens there: every workgroup
// adds up the tiles of all lists, derives the chunk that fills the chip, and finds its own piece (Plan).
//
// Products on matrix instructions of 16 x 16: S^T = K Q^T (keys x rows) leaves a lane with scores of one row, four keys in turn, and
// these are, rounded, the operand of O^T += V^T P^T as they stand, if the keys of V are taken in the same order.
//   a list of at most 32 rows   a wave takes a piece by itself: 32 keys at a time through 16 KB of LDS of its own, no barriers
//   more rows                   the four waves of a workgroup share 64 keys at a time and have up to 16 NC rows each
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <algorithm>
#include <type_traits>

namespace sp {
namespace {

constexpr int SOLO_ROWS = 32;              // rows of a list that a wave takes by itself
constexpr int MAX_NC = 3;                  // row tiles of 16 of a wave that shares its keys: 192 rows to a workgroup
constexpr int PLAN_WGS = 512;              // workgroups that the pieces are made for: two to a CU
constexpr int PLAN_SOLO = 4 * PLAN_WGS;    // pieces of single waves, at most, that the chunk is made for

struct DecodeArgs {
    const void* q; void* o; float* lse;
    const char* k_cache; const char* v_cache;
    const int* prompt_tables; const int* prompt_lens; const int* resp_tables; const int* resp_lens;
    int64_t prompt_width, resp_width;
    int prompt_cap, resp_cap;              // tokens that a table holds (at most 2^31 - 1)
    int members;                           // sequences of each group, 0: of several sizes
    Div group_size, block_rows;            // of `members`, of the rows of a shared piece
    int n_pages, n_groups, n_seqs, Hq, Hkv, rep, log_page;
    int nc, tile_shift;                    // row tiles per wave of a shared piece; see find_piece()
    Div kv_heads, q_heads, heads_each;     // of Hkv, Hq, rep
    float c, m_none;                       // softmax_scale * log2(e); reference point of a row that has not seen a key
    uint32_t* tag;
    int2* desc;                            // per list: first row of its sums, chunks (-1: a sequence that takes no part)
    float* stats;                          // per row of sums: m, l, l of the rounded weights, 0
    float* sums;                           // per row: sum p v
};

__device__ const i32x4 zero_granule = {0, 0, 0, 0};      // what keys that are not there read

// ---- the plan --------------------------------------------------------------------------------------------

// over the lanes of a wave: inclusive sums, and the maximum or the sum in every lane
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp_add(int x) {
    return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int scan64(int x) {
    x = dpp_add<0x111, 0xf>(x); x = dpp_add<0x112, 0xf>(x); x = dpp_add<0x114, 0xf>(x); x = dpp_add<0x118, 0xf>(x);      // within 16 lanes
    x = dpp_add<0x142, 0xa>(x); return dpp_add<0x143, 0xc>(x);                                                      // across them
}
template <int CTRL> __device__ __forceinline__ float rotated16(float x) {
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, false));
}
// the four lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quad_max(float x) {
    x = pair_max(x);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
    x = pair_sum(x);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, rotated16<0x128>(x)); x = fmaxf(x, rotated16<0x124>(x)); x = fmaxf(x, rotated16<0x122>(x)); x = fmaxf(x, rotated16<0x121>(x));
    return quad_max(x);
}
__device__ __forceinline__ float wave_sum(float x) {
    x += rotated16<0x128>(x); x += rotated16<0x124>(x); x += rotated16<0x122>(x); x += rotated16<0x121>(x);
    return quad_sum(x);
}

struct ListShape { int rows, len, tiles, blocks; bool shared; };      // tiles of 32 keys; blocks of rows that a piece holds
struct Piece { int list, chunk, kvh, block, base, chunk_tiles, rows, len, blocks; bool shared; };
struct PlanShare { int sums[4][3]; int left[4], list[4], base[4]; };     // of the waves of a workgroup; their pieces

struct Lists {
    const int* starts;                       // first sequence of each group, where groups are of several sizes
    const i32x2* held;                       // rows and length of each list in LDS, or nullptr
    const DecodeArgs& a;
    __device__ __forceinline__ i32x2 read(int i) const {
        const bool prompt = i < a.n_groups;
        const int prompt_cap = a.prompt_cap, resp_cap = a.resp_cap;
        const int* const prompt_lens = a.prompt_lens;
        const int* const resp_lens = a.resp_lens - a.n_groups;
        const int n = prompt && !prompt_cap ? 0 : (prompt ? prompt_lens : resp_lens)[i];
        int members = 1;
        if (prompt) members = a.members ? a.members : starts[i + 1] - starts[i];
        return i32x2{a.rep * members, min(max(n, -1), prompt ? prompt_cap : resp_cap)};
    }
    template <bool F32> __device__ __forceinline__ ListShape shape(i32x2 x) const {
        ListShape s;
        s.rows = x[0];
        s.len = x[1];
        s.tiles = s.rows > 0 && s.len > 0 ? (int)(((unsigned)s.len + 31u) >> 5) : 0;
        s.shared = !F32 && s.rows > SOLO_ROWS;
        unsigned rest;
        s.blocks = s.shared ? (int)divmod((unsigned)(s.rows - 1), a.block_rows, rest) + 1 : (s.rows + SOLO_ROWS - 1) / SOLO_ROWS;
        return s;
    }
    template <bool F32> __device__ __forceinline__ ListShape shape(int i) const { return shape<F32>(held ? held[i] : read(i)); }
};

// A chunk and its reciprocal.  Whole numbers: the least chunk of `unit` tiles with chunk * places >= total.  (The quotients are below the
// number of places, a few thousand, so that a float is off by one at most.)
struct Chunk {
    int tiles; float inv;
    __device__ __forceinline__ Chunk(int64_t total, int places, int unit) {
        const int step = places * unit;
        int c = (int)fminf((float)total * __builtin_amdgcn_rcpf((float)step), 1e8f);
        c += (int64_t)c * step < total;
        c += (int64_t)c * step < total;
        tiles = max(c, 1) * unit;
        inv = __builtin_amdgcn_rcpf((float)tiles);
    }
    __device__ __forceinline__ int of(int n) const {       // chunks of n tiles
        int c = (int)((float)n * inv);
        c -= c > 0 && (int64_t)c * tiles >= n;
        c += (int64_t)c * tiles < n;
        return c + ((int64_t)c * tiles < n);
    }
};

// The piece of this wave (of a shared list: of the workgroup).  Every workgroup makes the whole plan: its threads add up the tiles of
// all lists, leaving them in LDS (n_held of them fit).  Pieces of shared lists come first, one per workgroup, then those of
// single waves, four per workgroup.  The chunk of either kind follows from the tiles (row blocks counted) per place, the places being
// dealt by tiles, so there are no more pieces than places and one per list, block and kv head.
// (tile_shift: tiles are added up in units that keep their sum within 31 bits, rounded up.)
// Written for few instructions: what a workgroup runs once comes from memory, 64 bytes at a time.
template <bool F32>
__device__ __forceinline__ bool find_piece(const TabArg& starts, const DecodeArgs& a, i32x2* held, int n_held, PlanShare& share, int wave, int lane, Piece& p) {
    const int n = a.n_groups + a.n_seqs;
    const Lists ls{table_of(starts), n <= n_held ? held : nullptr, a};
    int shared_tiles = 0, solo_tiles = 0;
    for (int i = threadIdx.x; i < n; i += 256) {
        const i32x2 x = ls.read(i);
        if (ls.held) held[i] = x;
        const ListShape s = ls.shape<F32>(x);
        const int t = ((s.tiles + (1 << a.tile_shift) - 1) >> a.tile_shift) * s.blocks;
        shared_tiles += s.shared ? t : 0;
        solo_tiles += s.shared ? 0 : t;
    }
    auto over_waves = [&](int k, int& before, int& all) {      // of a sum that each wave has left in share.sums[.][k]
        const int s0 = share.sums[0][k], s1 = share.sums[1][k], s2 = share.sums[2][k], s3 = share.sums[3][k];
        before = (wave > 0 ? s0 : 0) + (wave > 1 ? s1 : 0) + (wave > 2 ? s2 : 0);
        all = s0 + s1 + s2 + s3;
    };
    shared_tiles = scan64(shared_tiles);
    solo_tiles = scan64(solo_tiles);
    if (lane == 63) { share.sums[wave][0] = shared_tiles; share.sums[wave][1] = solo_tiles; }
    __syncthreads();
    int before, sum_shared, sum_solo;
    over_waves(0, before, sum_shared);
    over_waves(1, before, sum_solo);
    const int64_t t_shared = ((int64_t)sum_shared << a.tile_shift) * a.Hkv, t_solo = ((int64_t)sum_solo << a.tile_shift) * a.Hkv;
    int shared_wgs = t_shared > 0 ? max(1, (int)(PLAN_WGS * ((float)t_shared * __builtin_amdgcn_rcpf((float)(t_shared + t_solo))))) : 0;
    if (t_solo > 0) shared_wgs = min(shared_wgs, PLAN_WGS - 1);
    const Chunk chunk_shared(t_shared, max(1, min(shared_wgs, PLAN_WGS)), 2), chunk_solo(t_solo, 4 * max(1, PLAN_WGS - shared_wgs), 1);      // shared: whole stages of 64 keys
    auto pick = [&](bool shared) {
        Chunk c = chunk_solo;
        if (shared) { c.tiles = chunk_shared.tiles; c.inv = chunk_shared.inv; }
        return c;
    };
    const int per = (n + 255) >> 8, i0 = min(n, (int)threadIdx.x * per), i1 = min(n, i0 + per);
    int n_shared = 0, n_solo = 0, rows = 0;
    for (int i = i0; i < i1; ++i) {
        const ListShape s = ls.shape<F32>(i);
        const int chunks = pick(s.shared).of(s.tiles), count = chunks * s.blocks * a.Hkv;
        n_shared += s.shared ? count : 0;
        n_solo += s.shared ? 0 : count;
        rows += chunks * a.Hkv * s.rows;
    }
    int to_shared = scan64(n_shared), to_solo = scan64(n_solo), to_rows = scan64(rows);
    __syncthreads();
    if (lane == 63) { share.sums[wave][0] = to_shared; share.sums[wave][1] = to_solo; share.sums[wave][2] = to_rows; }
    __syncthreads();
    int all_shared, all_solo, all_rows;
    over_waves(0, before, all_shared); to_shared += before;
    over_waves(1, before, all_solo); to_solo += before;
    over_waves(2, before, all_rows); to_rows += before;
    const bool shared = (int)blockIdx.x < all_shared;
    const int first = shared ? (int)blockIdx.x : ((int)blockIdx.x - all_shared) * 4, many = shared ? 1 : 4;      // this workgroup's pieces
    const int to = shared ? to_shared : to_solo, from = to - (shared ? n_shared : n_solo);
    const bool tells = blockIdx.x == 0;          // the first workgroup writes down what the join needs to know of each list
    if (tells || (from < first + many && to > first)) {
        int at = from, base = to_rows - rows;
        for (int i = i0; i < i1; ++i) {
            const ListShape s = ls.shape<F32>(i);
            const int chunks = pick(s.shared).of(s.tiles), count = s.shared == shared ? chunks * s.blocks * a.Hkv : 0;
            for (int k = max(at, first); k < min(at + count, first + many); ++k) {
                share.list[k - first] = i; share.left[k - first] = k - at; share.base[k - first] = base;
            }
            if (tells) a.desc[i] = int2{base, i >= a.n_groups && s.len < 0 ? -1 : chunks};
            at += count;
            base += chunks * a.Hkv * s.rows;
        }
    }
    __syncthreads();
    if (!shared && first + wave >= all_solo) return false;
    const int slot = shared ? 0 : wave;
    auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };      // the same in every lane, which the compiler does not see
    p.list = scalar(share.list[slot]);
    p.base = scalar(share.base[slot]);
    const ListShape s = ls.shape<F32>(p.list);
    p.rows = scalar(s.rows); p.len = scalar(s.len); p.blocks = scalar(s.blocks);
    p.shared = shared;
    p.chunk_tiles = scalar(shared ? chunk_shared.tiles : chunk_solo.tiles);
    unsigned rest;
    int left = (int)divmod((unsigned)scalar(share.left[slot]), a.kv_heads, rest);
    p.kvh = (int)rest;
    p.block = 0;
    if (p.blocks > 1) { p.block = left % p.blocks; left /= p.blocks; }
    p.chunk = left;
    return true;
}

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
    f32x4 o[NC][D / 16];       // lane: row l % 16 of tile c, elements 16 dt + 4 (l / 16) + i
    float m[NC], l[NC], lr[NC];
    bf16x8 q[NC][D / 32];
    __device__ __forceinline__ void clear(float m_none) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            m[c] = m_none; l[c] = 0.f; lr[c] = 0.f;
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

// Scores of 32 keys at LDS address `k`, keys not in `bits` masked: s[c][kt][i] is key 16 kt + 4 (l / 16) + i of row l % 16 of tile c
// (an operand's granule is its first one's with a constant xored in, which leaves the address of the first in a register only)
template <int D, int NC>
__device__ __forceinline__ void scores(const Rows<D, NC>& r, unsigned k, unsigned bits, int tiles, int l, f32x4 (&s)[NC][2]) {
    const unsigned at = k + kv_off<D>(l & 15, l >> 4);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
        bf16x8 a[D / 32];
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) a[ks] = lds_at_row8((at ^ (ks << 6)) + kt * (32 * D));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (c > 0 && c >= tiles) continue;
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

// Weights of 32 keys from their scores, rounded to bf16 as the second product needs them: the rounding of a weight, 2^-9 at most
// of it, is like that of o itself, and the sum that divides o is of the rounded ones (lr).
template <int D, int NC>
__device__ __forceinline__ void weights(Rows<D, NC>& r, const f32x4 (&s)[NC][2], float c2, int tiles, bf16x8 (&p)[NC]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c > 0 && c >= tiles) continue;
        float mx = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])), fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3])));
        mx = quad_max(mx);
        if (__builtin_amdgcn_ballot_w64(mx > r.m[c]) != 0) {
            const float mn = fmaxf(r.m[c], mx), alpha = __builtin_amdgcn_exp2f((r.m[c] - mn) * c2);
            r.l[c] *= alpha; r.lr[c] *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) r.o[c][dt][i] *= alpha;
            r.m[c] = mn;
        }
        const float mc = r.m[c] * c2;
        float sum = 0.f, rounded = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][e >> 2][e & 3], c2, -mc));
            sum += x;
            p[c][e] = (__bf16)x;
        }
        const bf16x8 one = {(__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f, (__bf16)1.f};
        rounded = dot8(p[c], one, 0.f);
        r.l[c] += sum;
        r.lr[c] += rounded;
    }
}

// O^T += V^T P^T over 32 keys at LDS address `v`
template <int D, int NC>
__device__ __forceinline__ void add_values(Rows<D, NC>& r, unsigned v, const bf16x8 (&p)[NC], int tiles, int l) {
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
            if (c > 0 && c >= tiles) continue;
            r.o[c][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[c], r.o[c][dt], 0, 0, 0);
        }
    }
}

// Pages of a list's keys: a lane holds one of 64 page numbers, from page `first` on
struct Pages {
    const int* table; int width, first, held, lane;
    __device__ __forceinline__ int at(int page) {
        if (page - first >= 64) load(page);
        return __builtin_amdgcn_readlane(held, page - first);
    }
    __device__ __forceinline__ void load(int page) {
        first = page;
        held = page + lane < width ? table[page + lane] : -1;
    }
};

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

// Where the rows of a piece come from and go to
struct PieceRows {
    int seq0, rep, rows, Hq, kvh;
    int64_t base;                       // of row 0 among the rows of sums
    Div heads_each;
    __device__ __forceinline__ int64_t q_row(int r) const {        // row of q and o
        unsigned hr;
        const int member = (int)divmod((unsigned)r, heads_each, hr);
        return (int64_t)(seq0 + member) * Hq + kvh * rep + (int)hr;
    }
};

template <int D, int NC>
__device__ __forceinline__ void load_rows(Rows<D, NC>& r, const __bf16* q, const PieceRows& pr, int row0, int tiles, int l) {
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
__device__ __forceinline__ void store_rows(const Rows<D, NC>& r, const DecodeArgs& a, const PieceRows& pr, int row0, int tiles, int l) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int row = row0 + 16 * c + (l & 15);
        const float lt = quad_sum(r.l[c]), lrt = quad_sum(r.lr[c]);
        if (c >= tiles || row >= pr.rows) continue;
        float* const out = a.sums + (pr.base + row) * D + 4 * (l >> 4);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(out + 16 * dt) = r.o[c][dt];
        if (l < 16) *reinterpret_cast<f32x4*>(a.stats + (pr.base + row) * 4) = f32x4{r.m[c], lt, lrt, 0.f};
    }
}

template <int D, int NC>
__global__ __launch_bounds__(256, 2) void decode_kernel(TabArg starts, DecodeArgs a) {
    constexpr int KEYS16 = 32 * D;               // bytes of 16 keys
    __shared__ __attribute__((aligned(1024))) char lds[16 * KEYS16];
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63;
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    __shared__ PlanShare share;
    Piece p;
    const bool has = find_piece<false>(starts, a, reinterpret_cast<i32x2*>(lds), (int)sizeof(lds) / 8, share, w, l, p);
    __syncthreads();                             // the lists' place is free
    if (!has) return;
    const bool prompt = p.list < a.n_groups;
    const int own = p.list - a.n_groups;
    const int key0 = p.chunk * p.chunk_tiles * 32, key1 = (int)min((unsigned)p.len, (unsigned)key0 + 32u * p.chunk_tiles);
    PieceRows pr{prompt ? (a.members ? p.list * a.members : table_of(starts)[p.list]) : own, a.rep, p.rows, a.Hq, p.kvh, p.base + ((int64_t)p.chunk * a.Hkv + p.kvh) * p.rows, a.heads_each};
    Pages pages{prompt ? a.prompt_tables + p.list * a.prompt_width : a.resp_tables + own * a.resp_width, (int)(prompt ? a.prompt_width : a.resp_width), 0, 0, l};
    pages.load(key0 >> a.log_page);
    const Copier<D> copy(l);
    const uint64_t kc = uniform64((uint64_t)(uintptr_t)a.k_cache), vc = uniform64((uint64_t)(uintptr_t)a.v_cache);
    // byte offset of 16 keys in either cache and how many of them there are
    auto locate = [&](int key, uint64_t& at, int& valid) {
        valid = min(16, key1 - key);
        at = 0;
        if (valid <= 0) return;
        const int page = __builtin_amdgcn_readfirstlane(pages.at(key >> a.log_page));
        if (page < 0 || page >= a.n_pages) { valid = 0; return; }
        at = ((((uint64_t)(unsigned)page * a.Hkv + p.kvh) << a.log_page) + (key & ((1 << a.log_page) - 1))) * (2 * D);
    };
    const __bf16* const q = (const __bf16*)a.q;
    const unsigned buf = lds_address(lds);

    if (!p.shared) {
        // one wave: K and V of 32 keys in turn, the next K copied while the weights and the second product run, the next V under the next scores
        Rows<D, 2> r;
        const int row0 = p.block * SOLO_ROWS, tiles = min(2, (p.rows - row0 + 15) >> 4);
        load_rows(r, q, pr, row0, tiles, l);
        r.clear(a.m_none);
        const unsigned kb = buf + w * 4 * KEYS16, vb = kb + 2 * KEYS16;
        uint64_t at[2];
        int valid[2];
        auto fetch = [&](int key) { locate(key, at[0], valid[0]); locate(key + 16, at[1], valid[1]); };
        auto issue = [&](uint64_t cache, unsigned dst) {
            copy.rows16(cache + at[0], valid[0], dst);
            copy.rows16(cache + at[1], valid[1], dst + KEYS16);
        };
        constexpr int N = 2 * Copier<D>::COPIES;
        fetch(key0);
        issue(kc, kb);
        issue(vc, vb);
        for (int key = key0; key < key1; key += 32) {
            const unsigned bits = low_bits(valid[0]) | low_bits(valid[1]) << 16;
            const bool more = key + 32 < key1;
            f32x4 s[2][2];
            bf16x8 pw[2];
            wait_copies<N>();
            scores(r, kb, bits, tiles, l, s);
            wait_lds();
            if (more) { fetch(key + 32); issue(kc, kb); }
            weights(r, s, a.c, tiles, pw);
            if (more) wait_copies<N>(); else wait_copies<0>();
            add_values(r, vb, pw, tiles, l);
            wait_lds();
            if (more) issue(vc, vb);
        }
        store_rows(r, a, pr, row0, tiles, l);
    } else {
        // four waves: 64 keys of K and V in one half of LDS while the next 64 are copied into the other, a wave copying 16 keys of each
        Rows<D, NC> r;
        const int all = (p.rows + 15) >> 4, per = (all + p.blocks - 1) / p.blocks, first = p.block * per, n = min(per, all - first);
        const int t0 = first + (w * n >> 2), tiles = ((w + 1) * n >> 2) - (w * n >> 2), row0 = 16 * t0;
        load_rows(r, q, pr, row0, tiles, l);
        r.clear(a.m_none);
        uint64_t at;
        int valid[4];
        auto issue = [&](int key, unsigned dst) {
            uint64_t mine = 0;
            int v_mine = 0;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                locate(key + 16 * h, at, valid[h]);
                if (h == w) { mine = at; v_mine = valid[h]; }
            }
            copy.rows16(kc + mine, v_mine, dst + w * KEYS16);
            copy.rows16(vc + mine, v_mine, dst + (4 + w) * KEYS16);
        };
        unsigned half = 0;
        issue(key0, buf);
        for (int key = key0; key < key1; key += 64) {
            const unsigned lo = low_bits(valid[0]) | low_bits(valid[1]) << 16, hi = low_bits(valid[2]) | low_bits(valid[3]) << 16;
            wait_copies<0>();
            __syncthreads();
            const unsigned kb = buf + half * 8 * KEYS16, vb = kb + 4 * KEYS16;
            half ^= 1;
            if (key + 64 < key1) issue(key + 64, buf + half * 8 * KEYS16);
            if (tiles > 0) {
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    f32x4 s[NC][2];
                    bf16x8 pw[NC];
                    scores(r, kb + 2 * h * KEYS16, h ? hi : lo, tiles, l, s);
                    weights(r, s, a.c, tiles, pw);
                    add_values(r, vb + 2 * h * KEYS16, pw, tiles, l);
                }
            }
        }
        store_rows(r, a, pr, row0, tiles, l);
    }
}

// ---- float32: the same pieces, all of single waves, K and V read straight into the operands' registers ------------------------------

// Products on float32 matrix instructions of 16 x 16 x 4.  S^T: lane group j = l / 16 contracts elements [j D / 4, (j + 1) D / 4) of its key, so
// that it reads them in pieces of 16 bytes.  O^T += V^T P^T: step i contracts keys 4 j + i, whose weight is score i of the lane, and row m of
// tile (h, e) is element 64 h + 4 m + e, so that V is read in pieces of 16 bytes as well.
template <int D>
__global__ __launch_bounds__(256, 2) void decode_f32_kernel(TabArg starts, DecodeArgs a) {
    __shared__ i32x2 lists[4096];
    __shared__ PlanShare share;
    constexpr int NC = SOLO_ROWS / 16, HALVES = D / 64;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = threadIdx.x & 63, m16 = l & 15, j = l >> 4;
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    Piece p;
    if (!find_piece<true>(starts, a, lists, 4096, share, w, l, p)) return;
    const bool prompt = p.list < a.n_groups;
    const int own = p.list - a.n_groups;
    const int key0 = p.chunk * p.chunk_tiles * 32, key1 = (int)min((unsigned)p.len, (unsigned)key0 + 32u * p.chunk_tiles);
    PieceRows pr{prompt ? (a.members ? p.list * a.members : table_of(starts)[p.list]) : own, a.rep, p.rows, a.Hq, p.kvh, p.base + ((int64_t)p.chunk * a.Hkv + p.kvh) * p.rows, a.heads_each};
    Pages pages{prompt ? a.prompt_tables + p.list * a.prompt_width : a.resp_tables + own * a.resp_width, (int)(prompt ? a.prompt_width : a.resp_width), 0, 0, l};
    pages.load(key0 >> a.log_page);
    const int row0 = p.block * SOLO_ROWS, tiles = min(NC, (p.rows - row0 + 15) >> 4);
    float q[NC][D / 4];
    f32x4 o[NC][HALVES][4];
    float m[NC], sum[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int row = row0 + 16 * c + m16;
        const float* const src = (const float*)a.q + pr.q_row(c < tiles && row < pr.rows ? row : 0) * D + j * (D / 4);
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
        int valid = min(16, key1 - key);
        const int page = pages.at(key >> a.log_page);
        if (page < 0 || page >= a.n_pages) continue;
        const int64_t row = ((((int64_t)page * a.Hkv + p.kvh) << a.log_page) + (key & ((1 << a.log_page) - 1)));
        // keys behind the last one read the first one's row and are masked
        const float* const kp = (const float*)a.k_cache + (row + (m16 < valid ? m16 : 0)) * D + j * (D / 4);
        f32x4 k[D / 16], v[4][HALVES];
#pragma unroll
        for (int e = 0; e < D / 16; ++e) k[e] = *reinterpret_cast<const f32x4*>(kp + 4 * e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* const vp = (const float*)a.v_cache + (row + (4 * j + i < valid ? 4 * j + i : 0)) * D + 4 * m16;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) v[i][h] = *reinterpret_cast<const f32x4*>(vp + 64 * h);
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
        const int row = row0 + 16 * c + m16;
        const float lt = quad_sum(sum[c]);
        if (c >= tiles || row >= pr.rows) continue;
        float* const out = a.sums + (pr.base + row) * D + 16 * j;
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(out + 64 * h + 4 * i) = f32x4{o[c][h][0][i], o[c][h][1][i], o[c][h][2][i], o[c][h][3][i]};
        if (j == 0) *reinterpret_cast<f32x4*>(a.stats + (pr.base + row) * 4) = f32x4{m[c], lt, lt, 0.f};
    }
}

// ---- the join ------------------------------------------------------------------------------------------------

// One wave per sequence and q head: o = sum_c e^(m_c - M) O_c / sum_c e^(m_c - M) l_c over the chunks of the prompt and of the response.
// Bound: the latency of three loads that wait for each other (where the sums are, the statistics, the sums); the first sums are
// therefore asked for with the statistics.  D / 4 lanes hold a row, so that a wave has 4 x 256 / D rows in flight.
template <typename T, int D>
__global__ __launch_bounds__(256) void decode_join_kernel(TabArg starts, DecodeArgs a) {
    constexpr int LANES = D / 4, AT_ONCE = 64 / LANES, DEPTH = 4;
    const int* const w = table_of(starts);
    const int l = threadIdx.x & 63, mine = l / LANES, e0 = 4 * (l % LANES);
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (item >= (int64_t)a.n_seqs * a.Hq) return;
    unsigned in_seq;
    const int seq = (int)divmod((unsigned)item, a.q_heads, in_seq), h = (int)in_seq;
    unsigned hr;
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
    int2 dp = a.desc[g];
    const int2 dr = a.desc[a.n_groups + seq];
    if (dr.y < 0) dp.y = 0;
    const int prompt_rows = members * a.rep;
    const int64_t base_p = dp.x + (int64_t)kvh * prompt_rows + (seq - first) * a.rep + hr, base_r = dr.x + (int64_t)kvh * a.rep + hr;
    const int n = dp.y + max(dr.y, 0);
    auto row_of = [&](int i) { return i < dp.y ? base_p + (int64_t)i * (a.Hkv * prompt_rows) : base_r + (int64_t)(i - dp.y) * (a.Hkv * a.rep); };
    float M = a.m_none, L = 0.f, LR = 0.f;
    f32x4 acc = {0, 0, 0, 0};
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int count = min(64, n - i0);
        f32x4 st = {a.m_none, 0.f, 0.f, 0.f}, x[DEPTH];
        if (l < count) st = *reinterpret_cast<const f32x4*>(a.stats + row_of(i0 + l) * 4);
        auto fetch = [&](int i) {
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                const int k = i + u * AT_ONCE + mine;
                x[u] = f32x4{0, 0, 0, 0};
                if (k < count) x[u] = *reinterpret_cast<const f32x4*>(a.sums + row_of(i0 + k) * D + e0);
            }
        };
        fetch(0);
        const float mn = fmaxf(M, wave_max(st[0])), alpha = __builtin_amdgcn_exp2f((M - mn) * a.c), wt = __builtin_amdgcn_exp2f((st[0] - mn) * a.c);
        M = mn;
        L = L * alpha + wt * st[1];            // lanes hold their chunks' shares of the sums
        LR = LR * alpha + wt * st[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= alpha;
        for (int i = 0; i < count; i += DEPTH * AT_ONCE) {
            if (i > 0) fetch(i);
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                const float f = __shfl(wt, (i + u * AT_ONCE + mine) & 63, 64);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += f * x[u][e];
            }
        }
    }
    L = wave_sum(L);
    LR = wave_sum(LR);
#pragma unroll
    for (int o = 32; o >= LANES; o >>= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
    const float inv = L > 0.f ? 1.f / LR : 0.f;
    if (mine == 0) {
        typedef T out4 __attribute__((ext_vector_type(4)));
        out4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (T)(L > 0.f ? acc[e] * inv : 0.f);
        *reinterpret_cast<out4*>((T*)a.o + item * D + e0) = y;
    }
    if (l == 0) a.lse[(int64_t)h * a.n_seqs + seq] = L > 0.f ? M * (a.c * LN2) + __logf(L) : -INFINITY;
}

int64_t most_rows(int n_seqs, int Hq, int rep) {       // rows of sums: a chunk more than the plan's places per list
    const int64_t in_group = (int64_t)n_seqs * rep;
    return PLAN_WGS * std::min<int64_t>(64 * MAX_NC, in_group) + PLAN_SOLO * std::min<int64_t>(SOLO_ROWS, in_group) + 2 * (int64_t)n_seqs * Hq;
}
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t desc_bytes(int n_groups, int n_seqs) { return up256(((size_t)n_groups + n_seqs) * sizeof(int2)); }

}  // namespace

size_t decode_partial_bytes(int n_groups, int n_seqs, int Hq, int Hkv, int d) {
    const size_t rows = (size_t)most_rows(n_seqs, Hq, Hq / Hkv);
    return desc_bytes(n_groups, n_seqs) + up256(rows * 16) + up256(rows * d * 4);
}

hipError_t launch_decode(const KvCache& cache, const void* q, void* o, float* lse, int Hq, int n_groups, int n_seqs, const int32_t* Gs, const TabArg& starts,
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
    a.desc = (int2*)partials;
    a.stats = (float*)((char*)partials + desc_bytes(n_groups, n_seqs));
    a.sums = a.stats + up256((size_t)most_rows(n_seqs, Hq, a.rep) * 16) / 4;
    int64_t shared = 0, solo = 0;
    int widest = 0;
    auto rows_of = [&](int g) { return (int64_t)a.rep * (Gs ? Gs[g] : 1); };
    auto per_wave = [](int64_t rows) {      // row tiles per wave if the rows are dealt to as few workgroups as can hold them
        const int64_t tiles = (rows + 15) / 16, blocks = (tiles + 4 * MAX_NC - 1) / (4 * MAX_NC), per = (tiles + blocks - 1) / blocks;
        return (int)((per + 3) / 4);
    };
    const bool prompts = prompt_width > 0;
    for (int g = 0; g < n_groups; ++g)
        if (prompts && rows_of(g) > SOLO_ROWS && !cache.f32) widest = std::max(widest, per_wave(rows_of(g)));
    if (a.rep > SOLO_ROWS && !cache.f32) widest = std::max(widest, per_wave(a.rep));
    a.nc = std::max(1, widest);
    a.kv_heads = make_div(a.Hkv);
    a.q_heads = make_div(Hq);
    a.heads_each = make_div(a.rep);
    a.block_rows = make_div(64 * a.nc);
    a.prompt_cap = (int)std::min<int64_t>((int64_t)prompt_width << a.log_page, 0x7fffffff);
    a.resp_cap = (int)std::min<int64_t>((int64_t)resp_width << a.log_page, 0x7fffffff);
    a.members = Gs ? Gs[0] : 1;
    for (int g = 1; Gs && g < n_groups; ++g) if (Gs[g] != Gs[0]) a.members = 0;
    a.group_size = make_div(std::max(1, a.members));
    {   // tiles at most
        const double most = ((double)n_groups * prompt_width + (double)n_seqs * resp_width) * (1 << a.log_page) / 32 *
                            ((double)n_seqs * a.rep / SOLO_ROWS + 1) + n_groups + n_seqs;
        while (most / (double)((int64_t)1 << a.tile_shift) + n_groups + n_seqs > 2e9) ++a.tile_shift;
    }
    // the plan's places and one piece per list, block and kv head, or a piece per tile (stage of two) that the tables have room for
    int64_t tiles_shared = 0, tiles_solo = 0;
    auto count = [&](int64_t rows, int64_t lists, int64_t width) {
        const int64_t tiles = (((width << a.log_page) + 31) >> 5) < ((int64_t)1 << 26) ? ((width << a.log_page) + 31) >> 5 : (int64_t)1 << 26;
        const bool sh = rows > SOLO_ROWS && !cache.f32;
        const int64_t blocks = lists * (sh ? (rows + 64 * a.nc - 1) / (64 * a.nc) : (rows + SOLO_ROWS - 1) / SOLO_ROWS);
        (sh ? shared : solo) += blocks;
        (sh ? tiles_shared : tiles_solo) += blocks * (sh ? (tiles + 1) / 2 : tiles);
    };
    if (prompts) for (int g = 0; g < n_groups; ++g) count(rows_of(g), 1, prompt_width);
    count(a.rep, n_seqs, resp_width);
    int64_t grid = PLAN_WGS + shared * a.Hkv + (solo * a.Hkv + 3) / 4 + 1;
    grid = std::max<int64_t>(1, std::min(grid, tiles_shared * a.Hkv + (tiles_solo * a.Hkv + 3) / 4));
    auto launch = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        if (cache.f32) hipLaunchKernelGGL((decode_f32_kernel<D>), dim3((unsigned)grid), dim3(256), 0, s, starts, a);
        else if (a.nc == 1) hipLaunchKernelGGL((decode_kernel<D, 1>), dim3((unsigned)grid), dim3(256), 0, s, starts, a);
        else if (a.nc == 2) hipLaunchKernelGGL((decode_kernel<D, 2>), dim3((unsigned)grid), dim3(256), 0, s, starts, a);
        else hipLaunchKernelGGL((decode_kernel<D, 3>), dim3((unsigned)grid), dim3(256), 0, s, starts, a);
        const unsigned joins = (unsigned)(((int64_t)n_seqs * Hq + 3) / 4);
        if (cache.f32) hipLaunchKernelGGL((decode_join_kernel<float, D>), dim3(joins), dim3(256), 0, s, starts, a);
        else hipLaunchKernelGGL((decode_join_kernel<__bf16, D>), dim3(joins), dim3(256), 0, s, starts, a);
    };
    if (cache.head_dim == 64) launch(std::integral_constant<int, 64>{}); else launch(std::integral_constant<int, 128>{});
    return hipGetLastError();
}

}  // namespace sp
