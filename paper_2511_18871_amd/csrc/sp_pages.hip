// Pages of the paged cache when sequences branch: keeping the accepted ones of drafted tokens, forking sequences, and fitting tables of
// pages to their sequences' lengths.  A page is free while no table holds it (its count in `refs` is 0); free pages are given out
// in ascending order, to requests in the order of their sequences and places, so that results do not depend on how the work is dealt.
#include "sp_common.hpp"
#include "sp_launch.hpp"
#include <algorithm>

namespace sp {
namespace {

constexpr int CHUNK = 4096;        // pages whose free ones are counted together: 64 words of 64 bits
typedef unsigned long long u64;

// inclusive sums over the lanes of a wave
__device__ __forceinline__ int scan_lanes(int x) {
    const int l = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(x, o, 64); x += l >= o ? y : 0; }
    return x;
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }
__device__ __forceinline__ u64 ballot(bool b) { return __builtin_amdgcn_ballot_w64(b); }
// (no shifts of 64 bits by a lane's own amount: half_of_lane())
__device__ __forceinline__ int lanes_below(u64 set) { return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(set >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)set, 0u)); }
__device__ __forceinline__ bool has_lane(u64 set) { return half_of_lane(set) >> (threadIdx.x & 31) & 1; }

// ---- keep ----------------------------------------------------------------------------------------------------

struct KeepArgs {
    char* k; char* v;
    int64_t layer_bytes;                   // from layer to layer
    const int* tables; const int* lens; const int* kept; const int* n_kept; int* lens_out;
    int64_t width, capacity, n_pages, kept_width;
    int items, per_wave, Hkv, log_page;    // items: layers * 2 * Hkv of a sequence
    Div heads;
};

// Token lens + kept[i] of a sequence becomes its token lens + i.  A wave looks 64 entries of the list up at a time, a lane each, and moves their rows of `per_wave`
// (layer, K or V, head) in turn, 64 AHEAD lanes of 16 bytes on their way.  It reads a batch of rows ahead of writing any, and kept ascends, so that
// kept[j] >= j > i for j > i: no row that is still to be read is written over.
// Bound: bytes, and for small calls four loads that wait for each other: 3.5 us for 8 paths in 2 layers; 128 paths in 16 layers 45 us for 193 MB, 4.3 TB/s.
constexpr int KEEP_AHEAD = 4;
template <int ROW>        // bytes of a row
__global__ __launch_bounds__(256) void keep_kernel(KeepArgs a) {
    constexpr int LANES = ROW / 16, ROWS = 64 / LANES;
    __shared__ int64_t moves[4][64][2];    // bytes from the head's place in page 0: from, to
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), seq = blockIdx.x;
    const int item0 = ((int)blockIdx.y * 4 + w) * a.per_wave;
    if (item0 >= a.items) return;
    const int64_t have = a.lens[seq];
    const int* const kept = a.kept + seq * a.kept_width;
    const int* const table = a.tables + seq * a.width;
    const int most = have < 0 ? 0 : (int)min((int64_t)max(a.n_kept[seq], 0), a.kept_width);
    auto row_of = [&](int64_t j) -> int64_t {
        const int64_t page = table[j >> a.log_page];
        return page < 0 || page >= a.n_pages ? -1 : (((page * a.Hkv) << a.log_page) + (j & ((1 << a.log_page) - 1))) * ROW;
    };
    int n = 0;                             // of the list up to its first entry that does not ascend or that the table has no room for
    for (bool more = true; more && n < most;) {
        const int i = n + l, x = i < most ? kept[i] : -1, before = i > 0 && i < most ? kept[i - 1] : -1;
        const u64 bad = ~ballot(x > before && have + x < a.capacity);
        const int run = bad ? __ffsll(bad) - 1 : 64;
        n += run;
        more = run == 64;
        const bool moves_row = l < run && x != i;
        const int64_t from = moves_row ? row_of(have + x) : -1, to = moves_row ? row_of(have + i) : -1;
        const bool both = from >= 0 && to >= 0;
        const u64 set = ballot(both);
        if (both) { moves[w][lanes_below(set)][0] = from; moves[w][lanes_below(set)][1] = to; }
        const int count = __popcll(set);
        __builtin_amdgcn_wave_barrier();
        for (int item = item0; item < min(item0 + a.per_wave, a.items); ++item) {
            unsigned head;
            const int lk = (int)divmod((unsigned)item, a.heads, head);
            char* const base = (lk & 1 ? a.v : a.k) + (lk >> 1) * a.layer_bytes + (((int64_t)head * ROW) << a.log_page) + (l % LANES) * 16;
            for (int r0 = l / LANES; r0 < count; r0 += ROWS * KEEP_AHEAD) {
                i32x4 x[KEEP_AHEAD];
#pragma unroll
                for (int u = 0; u < KEEP_AHEAD; ++u)
                    if (r0 + ROWS * u < count) x[u] = *reinterpret_cast<const i32x4*>(base + moves[w][r0 + ROWS * u][0]);
#pragma unroll
                for (int u = 0; u < KEEP_AHEAD; ++u)
                    if (r0 + ROWS * u < count) *reinterpret_cast<i32x4*>(base + moves[w][r0 + ROWS * u][1]) = x[u];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    if (item0 == 0 && l == 0) a.lens_out[seq] = (int)(have + n);
}

// ---- free pages ------------------------------------------------------------------------------------------------

struct Pool { int* refs; u64* free; int* counts; int64_t n_pages; int n_chunks; };      // free: a bit per page; counts: of each chunk

// which pages of chunk `c` are free, and how many (256 threads)
__device__ __forceinline__ void count_chunk(const Pool& p, int64_t c, int* sh) {
    const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
    int sum = 0, refs[CHUNK / 256];
#pragma unroll
    for (int i = 0; i < CHUNK / 256; ++i) {
        const int64_t page = c * CHUNK + i * 256 + threadIdx.x;
        refs[i] = page < p.n_pages ? p.refs[page] : 1;
    }
#pragma unroll
    for (int i = 0; i < CHUNK / 256; ++i) {
        const u64 set = ballot(refs[i] == 0);
        sum += __popcll(set);
        if (l == 0) p.free[c * 64 + i * 4 + w] = set;
    }
    if (l == 0) sh[w] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.counts[c] = sh[0] + sh[1] + sh[2] + sh[3];
}

// The free page that request first + l gets in lane l < n (-1: none is left).  Each lane holds one of a chunk's 64 words; a request finds its word among them by their ranks,
// then its bit by halves: 36 -> 30 us for the two calls of a step of 1024 sequences, against words that deal out their bits one by one.
// `mine`: the chunk's count, a lane each, among the first 64 chunks.
__device__ __forceinline__ int first_counts(const Pool& p) {
    const int l = threadIdx.x & 63;
    return l < p.n_chunks ? p.counts[l] : 0;
}
__device__ __forceinline__ int take_pages(const Pool& p, int mine, int64_t first, int n) {
    const int l = threadIdx.x & 63;
    const int64_t nth = first + l;
    int got = -1, given = 0;
    int64_t before = 0;                    // free pages ahead of the chunk
    for (int64_t c0 = 0; c0 < p.n_chunks && given < n; c0 += 64) {
        if (c0) mine = c0 + l < p.n_chunks ? p.counts[c0 + l] : 0;
        const int to = scan_lanes(mine);
        if (before + last_lane(to) > first + given) {
            u64 here = ballot(mine > 0 && before + to > first + given && before + to - mine < first + n);
            while (here) {
                const int k = __ffsll(here) - 1;
                here &= here - 1;
                const int64_t ahead = before + __builtin_amdgcn_readlane(to - mine, k);
                const int count = __builtin_amdgcn_readlane(mine, k);
                const u64 word = p.free[(c0 + k) * 64 + l];
                const int mask = __popcll(word), rank = scan_lanes(mask) - mask;
                const bool asks = l < n && nth >= ahead && nth < ahead + count;
                int r = asks ? (int)(nth - ahead) : 0, at = 0;
#pragma unroll
                for (int o = 32; o; o >>= 1) at += __shfl(rank, at + o, 64) <= r ? o : 0;      // the last word that starts at r or ahead of it
                r -= __shfl(rank, at, 64);
                const unsigned low_half = (unsigned)__shfl((int)word, at, 64), high_half = (unsigned)__shfl((int)(word >> 32), at, 64);
                const bool high = r >= __popc(low_half);
                r -= high ? __popc(low_half) : 0;
                unsigned bits = high ? high_half : low_half;
                int bit = high ? 32 : 0;
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    const int low = __popc(bits & ((1u << o) - 1));
                    if (r >= low) { r -= low; bits >>= o; bit += o; }
                }
                if (asks) got = (int)((c0 + k) * CHUNK + at * 64 + bit);
                given = (int)min((int64_t)n, ahead + count - first);
            }
        }
        before += last_lane(to);
    }
    return got;
}

// ---- fit -------------------------------------------------------------------------------------------------------

constexpr int FIT_AHEAD = 4;           // pieces of 64 places that a wave looks at together
struct FitArgs {
    Pool pool;
    int* tables; const int* lens; int* missing; int* wants; uint32_t* tag;
    int64_t width; int n_seqs, log_page;
};
__device__ __forceinline__ int64_t pages_needed(const FitArgs& a, int seq) {
    const int64_t n = a.lens[seq];
    return n < 0 ? -1 : min((n + (1 << a.log_page) - 1) >> a.log_page, a.width);
}

// One wave per sequence: what lies behind its last page goes back, and its empty places ahead are counted.
__global__ __launch_bounds__(256) void release_kernel(FitArgs a) {
    const int l = threadIdx.x & 63, seq = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (blockIdx.x == 0 && threadIdx.x < 64) a.tag[l] = 0u;
    if (seq >= a.n_seqs) return;
    const int64_t need = pages_needed(a, seq);
    int wants = 0;
    for (int64_t c0 = 0; need >= 0 && c0 < a.width; c0 += 64) {
        const int64_t c = c0 + l;
        const int page = c < a.width ? a.tables[seq * a.width + c] : -1;
        const bool held = page >= 0 && page < a.pool.n_pages;
        wants += __popcll(ballot(c < need && !held));
        if (c < a.width && c >= need && page != -1) {
            if (held) atomicSub(&a.pool.refs[page], 1);
            a.tables[seq * a.width + c] = -1;
        }
    }
    if (l == 0) a.wants[seq] = wants;
}

__global__ __launch_bounds__(256) void count_free_kernel(Pool p) {
    __shared__ int sh[4];
    count_chunk(p, blockIdx.x, sh);
}

// One wave per sequence: its empty places get pages.  The first workgroup says how many places of all got none.
__global__ __launch_bounds__(256) void assign_kernel(FitArgs a) {
    __shared__ int sh[4];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), seq0 = (int)blockIdx.x * 4, seq = seq0 + w;
    auto over_workgroup = [&](int x) {
        x = last_lane(scan_lanes(x));
        __syncthreads();
        if (l == 0) sh[w] = x;
        __syncthreads();
        return sh[0] + sh[1] + sh[2] + sh[3];
    };
    if (blockIdx.x == 0 && a.missing) {
        int all = 0, free = 0;
        for (int s = threadIdx.x; s < a.n_seqs; s += 256) all += a.wants[s];
        for (int c = threadIdx.x; c < a.pool.n_chunks; c += 256) free += a.pool.counts[c];
        all = over_workgroup(all);
        free = over_workgroup(free);
        if (threadIdx.x == 0) a.missing[0] = max(0, all - free);
    }
    // places are looked at FIT_AHEAD * 64 at a time, the first of them while the sums are on their way
    int left = seq < a.n_seqs ? a.wants[seq] : 0;
    const int counts = first_counts(a.pool);
    const int64_t need = left > 0 ? pages_needed(a, seq) : 0;
    int* const table = a.tables + seq * a.width;
    int page[FIT_AHEAD];
    auto look_up = [&](int64_t c0) {
#pragma unroll
        for (int u = 0; u < FIT_AHEAD; ++u) page[u] = c0 + 64 * u + l < need ? table[c0 + 64 * u + l] : 0;
    };
    look_up(0);
    int ahead = 0;
    for (int s = threadIdx.x; s < seq0; s += 256) ahead += a.wants[s];
    ahead = over_workgroup(ahead);
    for (int s = seq0; s < min(seq, a.n_seqs); ++s) ahead += a.wants[s];
    for (int64_t c0 = 0; left > 0 && c0 < need; c0 += 64 * FIT_AHEAD) {
        if (c0) look_up(c0);
#pragma unroll
        for (int u = 0; u < FIT_AHEAD; ++u) {
            const bool empty = c0 + 64 * u + l < need && (page[u] < 0 || page[u] >= a.pool.n_pages);
            const u64 set = ballot(empty);
            const int n = __popcll(set);
            if (n == 0) continue;
            const int got = __shfl(take_pages(a.pool, counts, ahead, n), lanes_below(set) & 63, 64);
            if (empty) {
                table[c0 + 64 * u + l] = got;
                if (got >= 0) a.pool.refs[got] = 1;
            }
            ahead += n;
            left -= n;
        }
    }
}

// The same in one launch, for what one workgroup sees at a time: FIT_PLACES places of all tables in FIT_ITEMS pieces of 64, and 64 pages to a thread.  The places that
// want a page are listed in LDS, in order; a lane keeps a bit per page of its own, and a wave deals out the free ones among 64 at a time.
// Bound: the launch, three loads that wait for each other, and code that runs once.
constexpr int FIT_PLACES = 16384, FIT_ITEMS = 2048, FIT_PAGES = 65536;
__global__ __launch_bounds__(1024) void fit_small_kernel(FitArgs a, Div pieces) {      // pieces: of 64 places of a table
    __shared__ int places[FIT_PLACES];
    __shared__ u64 sets[FIT_ITEMS];        // of a piece's places, those that want a page
    __shared__ int first[FIT_ITEMS], sums[16];
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid < 64) a.tag[l] = 0u;
    const int items = a.n_seqs * (int)pieces.d, width = (int)a.width;
    auto place_of = [&](int item, int& seq) {
        unsigned piece;
        seq = (int)divmod((unsigned)item, pieces, piece);
        return (int)piece * 64 + l;
    };
    // what lies behind a sequence's last page goes back
    for (int i0 = w; i0 < items; i0 += 16 * FIT_AHEAD) {
        int page[FIT_AHEAD], seq[FIT_AHEAD], c[FIT_AHEAD], len[FIT_AHEAD];
#pragma unroll
        for (int u = 0; u < FIT_AHEAD; ++u) {
            c[u] = place_of(min(i0 + 16 * u, items - 1), seq[u]);
            page[u] = c[u] < width ? a.tables[seq[u] * width + c[u]] : -1;
            len[u] = a.lens[seq[u]];
        }
#pragma unroll
        for (int u = 0; u < FIT_AHEAD; ++u) {
            if (i0 + 16 * u >= items) break;
            const int need = len[u] < 0 ? 0 : (int)min(((int64_t)len[u] + (1 << a.log_page) - 1) >> a.log_page, (int64_t)width);
            const bool held = page[u] >= 0 && page[u] < a.pool.n_pages;
            const u64 set = ballot(c[u] < need && !held);
            if (l == 0) sets[i0 + 16 * u] = set;
            if (len[u] >= 0 && c[u] >= need && page[u] != -1) {
                if (held) atomicSub(&a.pool.refs[page[u]], 1);
                a.tables[seq[u] * width + c[u]] = -1;
            }
        }
    }
    __threadfence();                       // the counts that fell are read below
    __syncthreads();
    auto over_waves = [&](int x, int& all) {       // the sum over earlier threads and over all
        const int to = scan_lanes(x);
        __syncthreads();
        if (l == 63) sums[w] = to;
        __syncthreads();
        int ahead = to - x;
        all = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) { ahead += i < w ? sums[i] : 0; all += sums[i]; }
        return ahead;
    };
    int total;
    {
        const int n0 = 2 * tid < items ? __popcll(sets[2 * tid]) : 0, n1 = 2 * tid + 1 < items ? __popcll(sets[2 * tid + 1]) : 0;
        const int at = over_waves(n0 + n1, total);
        first[2 * tid] = at;
        first[2 * tid + 1] = at + n0;
    }
    if (total == 0) {
        if (tid == 0 && a.missing) a.missing[0] = 0;
        return;
    }
    // free pages: lane l of a wave looks at pages page0 + 64 j
    const int n_pages = (int)a.pool.n_pages, turns = (n_pages + 1023) >> 10, page0 = w * 64 * turns + l;
    u64 mask = 0;
    int found = 0;                         // of the wave
    for (int j0 = 0; j0 < turns; j0 += 8) {
        int refs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) refs[j] = j0 + j < turns && page0 + 64 * (j0 + j) < n_pages ? a.pool.refs[page0 + 64 * (j0 + j)] : 1;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            mask |= (u64)(refs[j] == 0) << ((j0 + j) & 63);
            found += __popcll(ballot(refs[j] == 0));
        }
    }
    __syncthreads();
    for (int item = w; item < items; item += 16) {
        const u64 set = sets[item];
        int seq;
        const int c = place_of(item, seq);
        if (has_lane(set)) places[first[item] + lanes_below(set)] = seq * width + c;
    }
    int all, nth = over_waves(l == 0 ? found : 0, all);       // (its barriers stand behind the list as well)
    nth = __builtin_amdgcn_readfirstlane(nth);
    if (tid == 0 && a.missing) a.missing[0] = max(0, total - all);
    for (int j = 0; j < turns && nth < total; ++j) {
        const bool free = mask >> j & 1;
        const u64 set = ballot(free);
        const int k = nth + lanes_below(set);
        if (free && k < total) {
            a.tables[places[k]] = page0 + 64 * j;
            a.pool.refs[page0 + 64 * j] = 1;
        }
        nth += __popcll(set);
    }
    // places that no page was left for
    for (int i = all + tid; i < total; i += 1024) a.tables[places[i]] = -1;
}

// ---- fork ------------------------------------------------------------------------------------------------------

struct ForkArgs {
    Pool pool;
    char* k; char* v;
    int64_t layer_bytes, row_bytes;
    const int* parents; const int* src_tables; const int* src_lens;
    int* tables; int* lens_out; int* order; uint32_t* tag;
    int64_t src_width, width, capacity;    // capacity: tokens that both tables hold
    int n_seqs, n_src, Hkv, log_page;
    bool mark_orphans;                     // lens_out of sequences without a parent becomes -1
};
struct Child { int parent; int64_t len, whole; int rest; bool takes; int last; };      // takes: a page for the `rest` tokens of page `last`
__device__ __forceinline__ Child child_of(const ForkArgs& a, int seq) {
    Child c{-1, 0, 0, 0, false, -1};
    const int parent = a.parents[seq];
    if (parent < 0 || parent >= a.n_src) return c;
    c.parent = parent;
    c.len = min((int64_t)a.src_lens[parent], a.capacity);
    if (c.len < 0) return c;
    c.whole = c.len >> a.log_page;
    c.rest = (int)(c.len & ((1 << a.log_page) - 1));
    if (c.rest) c.last = a.src_tables[parent * a.src_width + c.whole];
    c.takes = c.rest && c.last >= 0 && c.last < a.pool.n_pages;
    return c;
}

// Counts free pages; one workgroup more numbers the children that need one.
__global__ __launch_bounds__(256) void fork_count_kernel(ForkArgs a) {
    __shared__ int sh[4];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    if ((int)blockIdx.x < a.pool.n_chunks) { count_chunk(a.pool, blockIdx.x, sh); return; }
    if (threadIdx.x < 64) a.tag[l] = 0u;
    int before = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 256) {
        const int s = s0 + threadIdx.x;
        const bool takes = s < a.n_seqs && child_of(a, s).takes;
        const u64 set = ballot(takes);
        __syncthreads();
        if (l == 0) sh[w] = __popcll(set);
        __syncthreads();
        int at = before + lanes_below(set);
        for (int i = 0; i < 4; ++i) { at += i < w ? sh[i] : 0; before += sh[i]; }
        if (s < a.n_seqs) a.order[s] = at;
    }
}

// A workgroup takes K or V of a layer of a child, and copies the tokens of its last page; the first of a child writes its table.
__global__ __launch_bounds__(256) void fork_kernel(ForkArgs a) {
    __shared__ int page_of_child;
    const int seq = blockIdx.x, layer = blockIdx.y >> 1;
    const Child c = child_of(a, seq);
    const bool tells = blockIdx.y == 0;
    if (c.parent < 0) {
        if (a.mark_orphans && tells && threadIdx.x == 0) a.lens_out[seq] = -1;
        return;
    }
    if (!tells && !c.takes) return;
    int to = -1;
    if (c.takes) {
        if (threadIdx.x < 64) {
            const int got = take_pages(a.pool, first_counts(a.pool), a.order[seq], 1);
            if (threadIdx.x == 0) page_of_child = got;
        }
        __syncthreads();
        to = __builtin_amdgcn_readfirstlane(page_of_child);
    }
    const bool none = c.takes && to < 0;
    if (tells) {
        if (threadIdx.x == 0) a.lens_out[seq] = none ? -1 : (int)c.len;
        for (int64_t i = threadIdx.x; i < a.width; i += 256) {
            int page = -1;
            if (!none && c.len >= 0 && i < c.whole) {
                page = a.src_tables[c.parent * a.src_width + i];
                if (page >= 0 && page < a.pool.n_pages) atomicAdd(&a.pool.refs[page], 1);
            } else if (!none && c.rest && i == c.whole) {
                page = c.takes ? to : c.last;
                if (c.takes) a.pool.refs[to] = 1;
            }
            a.tables[seq * a.width + i] = page;
        }
    }
    if (to < 0) return;
    char* const base = (blockIdx.y & 1 ? a.v : a.k) + layer * a.layer_bytes;
    const int64_t page_bytes = a.row_bytes << a.log_page, granules = c.rest * a.row_bytes / 16;
    for (int h = 0; h < a.Hkv; ++h) {
        const i32x4* const src = reinterpret_cast<const i32x4*>(base + ((int64_t)c.last * a.Hkv + h) * page_bytes);
        i32x4* const dst = reinterpret_cast<i32x4*>(base + ((int64_t)to * a.Hkv + h) * page_bytes);
        for (int64_t i = threadIdx.x; i < granules; i += 256) dst[i] = src[i];
    }
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
int64_t chunks_of(int64_t n_pages) { return (n_pages + CHUNK - 1) / CHUNK; }

// behind the tag: a word per sequence, bits of the free pages, counts
Pool make_pool(int* refs, int64_t n_pages, int n_seqs, void* room) {
    char* const at = (char*)room + up256((size_t)n_seqs * 4);
    const int64_t chunks = chunks_of(n_pages);
    return Pool{refs, (u64*)at, (int*)(at + (size_t)chunks * 512), n_pages, (int)chunks};
}

}  // namespace

size_t pages_room_bytes(int64_t n_pages, int n_seqs) { return up256((size_t)n_seqs * 4) + (size_t)chunks_of(n_pages) * 516; }

hipError_t launch_keep(const KvCache& cache, int n_layers, int64_t layer_stride, int n_seqs, const int* tables, int width, const int* lens,
                       const int* kept, int kept_width, const int* n_kept, int* lens_out, hipStream_t s) {
    const int elem = cache.f32 ? 4 : 2, row = cache.head_dim * elem;
    KeepArgs a{};
    a.k = (char*)cache.k; a.v = (char*)cache.v; a.layer_bytes = layer_stride * elem;
    a.tables = tables; a.lens = lens; a.kept = kept; a.n_kept = n_kept; a.lens_out = lens_out;
    a.width = width; a.capacity = std::min<int64_t>((int64_t)width << cache.log_page, MAX_TOKENS); a.n_pages = cache.n_pages; a.kept_width = kept_width;
    a.items = n_layers * 2 * cache.n_kv_heads; a.Hkv = cache.n_kv_heads; a.log_page = cache.log_page;
    a.heads = make_div(cache.n_kv_heads);
    // as many items to a wave as leave the chip twice its waves (16384)
    a.per_wave = (int)std::max<int64_t>(1, std::min<int64_t>(8, (int64_t)n_seqs * a.items / 16384));
    const dim3 grid((unsigned)n_seqs, (unsigned)((a.items + 4 * a.per_wave - 1) / (4 * a.per_wave)));
    if (row == 128) hipLaunchKernelGGL(keep_kernel<128>, grid, dim3(256), 0, s, a);
    else if (row == 256) hipLaunchKernelGGL(keep_kernel<256>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(keep_kernel<512>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_fit(int* refs, int64_t n_pages, int log_page, int n_seqs, int* tables, int width, const int* lens, int* missing, uint32_t* tag,
                      void* room, hipStream_t s) {
    FitArgs a{};
    a.pool = make_pool(refs, n_pages, n_seqs, room);
    a.tables = tables; a.lens = lens; a.missing = missing; a.wants = (int*)room; a.tag = tag;
    a.width = width; a.n_seqs = n_seqs; a.log_page = log_page;
    const int64_t pieces = ((int64_t)width + 63) / 64;
    if (n_seqs * pieces <= FIT_ITEMS && (int64_t)n_seqs * width <= FIT_PLACES && n_pages <= FIT_PAGES) {
        hipLaunchKernelGGL(fit_small_kernel, dim3(1), dim3(1024), 0, s, a, make_div((int)pieces));
        return hipGetLastError();
    }
    const dim3 waves((unsigned)((n_seqs + 3) / 4));
    hipLaunchKernelGGL(release_kernel, waves, dim3(256), 0, s, a);
    hipLaunchKernelGGL(count_free_kernel, dim3((unsigned)a.pool.n_chunks), dim3(256), 0, s, a.pool);
    hipLaunchKernelGGL(assign_kernel, waves, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_fork(const KvCache& cache, int n_layers, int64_t layer_stride, int* refs, int n_seqs, const int* parents, int n_src, const int* src_tables,
                       int src_width, const int* src_lens, int* tables, int width, int* lens_out, bool mark_orphans, uint32_t* tag, void* room, hipStream_t s) {
    const int elem = cache.f32 ? 4 : 2;
    ForkArgs a{};
    a.pool = make_pool(refs, cache.n_pages, n_seqs, room);
    a.k = (char*)cache.k; a.v = (char*)cache.v; a.layer_bytes = layer_stride * elem; a.row_bytes = (int64_t)cache.head_dim * elem;
    a.parents = parents; a.src_tables = src_tables; a.src_lens = src_lens; a.tables = tables; a.lens_out = lens_out; a.order = (int*)room; a.tag = tag;
    a.src_width = src_width; a.width = width; a.capacity = std::min<int64_t>((int64_t)std::min(src_width, width) << cache.log_page, MAX_TOKENS);
    a.n_seqs = n_seqs; a.n_src = n_src; a.Hkv = cache.n_kv_heads; a.log_page = cache.log_page;
    a.mark_orphans = mark_orphans;
    hipLaunchKernelGGL(fork_count_kernel, dim3((unsigned)a.pool.n_chunks + 1), dim3(256), 0, s, a);
    hipLaunchKernelGGL(fork_kernel, dim3((unsigned)n_seqs, (unsigned)(2 * n_layers)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sp
