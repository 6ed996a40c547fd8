// Keeping a paged key-value cache (gfx950, wave64): writing new tokens,
// copying, reserving, forking, freeing and compacting pages (Sec. 2.2: the
// engine manages sequences in a paged KV cache).
//
// All of it is data movement.  The bytes of tokens and pages go through
// 16-byte loads and stores, several in flight per lane; the caches of all
// layers are served by one launch, whose arguments carry their addresses.
//
// Free pages.  The n-th lowest free page is found from a bit per page and a
// count per block of 2048 pages: survey_kernel writes both, one launch ahead,
// and every wave that hands out pages then finds its own by rank (select),
// without an atomic and without waiting for another workgroup.  So the
// outcome does not depend on the order that workgroups run in.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "wq_cache.h"
#include "wq_device.h"
#include "wq_host.h"
#include "wq_internal.h"

namespace wq {
namespace cache {
namespace {

using dev::gbl;
using dev::u32x4;
using namespace host;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBlockPages = 2048;              // pages of one count: 32 bits for each lane of a wave
constexpr int kBlockWords = kBlockPages / 32;  // 64
constexpr int kGroupSeqs = 16;                 // sequences of one survey workgroup
constexpr int kGroupForks = kThreads;
constexpr int kUnroll = 4;
constexpr int kSegment = kThreads * kUnroll * 16;  // bytes a workgroup copies at once

struct Arrays {
    uint16_t* p[WQ_CACHE_MAX_ARRAYS];
};

// ------------------------------------------------------------- wave tools

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }

__device__ __forceinline__ int inclusive_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1, 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2, 3
    return v;
}
__device__ __forceinline__ int wave_sum(int v) { return __builtin_amdgcn_readlane(inclusive_scan(v), 63); }
__device__ __forceinline__ int count_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
__device__ __forceinline__ int from_lane(int v, int lane) { return __builtin_amdgcn_ds_bpermute(lane * 4, v); }

// Sum of a[0 .. n) over a wave; the lanes take turns.  Their first values can be
// asked for ahead.
__device__ __forceinline__ int first_of(const int32_t* a, int n) { return lane_id() < n ? a[lane_id()] : 0; }
__device__ __forceinline__ int sum_of(const int32_t* a, int n, int first) {
    int v = first;
    for (int i = lane_id() + 64; i < n; i += 64) v += a[i];
    return wave_sum(v);
}
__device__ __forceinline__ int sum_of(const int32_t* a, int n) { return sum_of(a, n, first_of(a, n)); }
// The same of up to 2^16 values of 0 .. 2^28, whose sum may pass 32 bits.
__device__ __forceinline__ int64_t long_sum_of(const int32_t* a, int n) {
    int64_t v = first_of(a, n);
    for (int i = lane_id() + 64; i < n; i += 64) v += a[i];
    return ((int64_t)wave_sum((int)(v >> 24)) << 24) + wave_sum((int)(v & 0xFFFFFF));
}

// ------------------------------------------------------------- free pages

struct Pool {
    const uint32_t* bits;    // bit p % 32 of word p / 32: page p is free
    const int32_t* counts;   // free pages of each block
    int blocks;
};

// Position of set bit k of w (k below its number of set bits).
__device__ __forceinline__ int nth_bit(uint32_t w, int k) {
    int at = 0;
#pragma unroll
    for (int half = 16; half >= 1; half >>= 1) {
        const int low = __popc((w >> at) & ((1u << half) - 1u));
        if (k >= low) {
            k -= low;
            at += half;
        }
    }
    return at;
}

// The free page of rank `rank` in every lane whose rank is not negative (and
// below the number of free pages).  All 64 lanes take part.
__device__ __forceinline__ int select(const Pool& pool, int rank) {
    const int lane = lane_id();
    int page = -1, base = 0;
    for (int b0 = 0; b0 < pool.blocks; b0 += 64) {
        const int cnt = b0 + lane < pool.blocks ? pool.counts[b0 + lane] : 0;
        const int inc = inclusive_scan(cnt);
        const int first = base + inc - cnt;
        const int total = base + __builtin_amdgcn_readlane(inc, 63);
        uint64_t pending = __builtin_amdgcn_ballot_w64(rank >= base && rank < total);
        while (pending) {
            const int want = __builtin_amdgcn_readlane(rank, __builtin_ctzll(pending));
            const int j = __builtin_ctzll(__builtin_amdgcn_ballot_w64(want >= first && want < first + cnt));
            const int start = __builtin_amdgcn_readlane(first, j), size = __builtin_amdgcn_readlane(cnt, j);
            const int word = (int)pool.bits[(int64_t)(b0 + j) * kBlockWords + lane];
            const int pc = __popc((uint32_t)word);
            const int before = start + inclusive_scan(pc) - pc;
            int lo = 0;
#pragma unroll
            for (int step = 32; step >= 1; step >>= 1)
                if (from_lane(before, lo + step) <= rank) lo += step;
            const uint32_t w = (uint32_t)from_lane(word, lo);
            const int k = rank - from_lane(before, lo);
            const bool mine = rank >= start && rank < start + size;
            if (mine) page = ((b0 + j) * kBlockWords + lo) * 32 + nth_bit(w, k);
            pending &= ~__builtin_amdgcn_ballot_w64(mine);
        }
        base = total;
        if (!__builtin_amdgcn_ballot_w64(rank >= total)) break;
    }
    return page;
}

// Free pages below page p (the same p in every lane).
__device__ __forceinline__ int free_below(const Pool& pool, int p) {
    const int block = p / kBlockPages;
    int n = sum_of(pool.counts, min(block, pool.blocks));
    if (block >= pool.blocks) return n;
    const int first = block * kBlockPages + lane_id() * 32;
    uint32_t w = pool.bits[(int64_t)block * kBlockWords + lane_id()];
    if (p < first + 32) w &= p <= first ? 0u : (1u << (p - first)) - 1u;
    return n + wave_sum(__popc(w));
}

struct Survey {
    const int32_t* refs;
    int32_t num_pages;
    uint32_t* bits;
    int32_t* counts;
    int32_t blocks;
    // Pages wanted: `need` of each sequence or fork, `group` of each workgroup's.
    int32_t* need;
    int32_t* group;
    int32_t items;
    const int32_t* table;
    int64_t max_pages;
    int32_t log2_page;
    // reserve
    const int32_t* old_lens;
    const int32_t* new_lens;
    // fork
    const int32_t* lens;
    const int32_t* src;
    const int32_t* dst;
    int32_t num_seqs;
    int32_t* length;  // [items] of each fork's source, -1: skipped
};

// Table entries [lo, hi) in which a growing sequence may lack pages.
__device__ __forceinline__ void grown(int old_len, int new_len, int log2_page, int64_t max_pages, int& lo, int& hi) {
    const int64_t page = int64_t(1) << log2_page;
    lo = (int)min<int64_t>(((int64_t)max(old_len, 0) + page - 1) >> log2_page, max_pages);
    hi = (int)min<int64_t>(((int64_t)max(new_len, 0) + page - 1) >> log2_page, max_pages);
}

// A fork's sequences and length; false where the pair is skipped.
__device__ __forceinline__ bool fork_of(const Survey& p, int i, int& s, int& d, int& len) {
    s = p.src[i];
    d = p.dst[i];
    if ((uint32_t)s >= (uint32_t)p.num_seqs || (uint32_t)d >= (uint32_t)p.num_seqs) return false;
    len = p.lens[s];
    return len >= 0 && len <= (p.max_pages << p.log2_page);
}

enum { kNothing, kReserve, kFork };

// Workgroups below `blocks` survey 2048 pages each; the others count the
// pages that their sequences (or forks) want.
template <int WHAT>
__global__ __launch_bounds__(kThreads) void survey_kernel(const Survey p) {
    __shared__ int sums[kWaves];
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    int mine = 0;
    if ((int)blockIdx.x < p.blocks) {
        const int first = blockIdx.x * kBlockPages + wave * (kBlockPages / kWaves);
        int refs[kBlockPages / kThreads];
#pragma unroll
        for (int i = 0; i < kBlockPages / kThreads; ++i) {
            const int page = first + i * 64 + lane;
            refs[i] = page < p.num_pages ? p.refs[page] : 1;
        }
#pragma unroll
        for (int i = 0; i < kBlockPages / kThreads; ++i) {
            const uint64_t free = __builtin_amdgcn_ballot_w64(refs[i] <= 0);
            mine += __popcll(free);
            if (lane < 2) p.bits[(first + i * 64) / 32 + lane] = (uint32_t)(free >> (32 * lane));
        }
        if (lane == 0) sums[wave] = mine;
        __syncthreads();
        if (threadIdx.x == 0) p.counts[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
        return;
    }
    const int g = blockIdx.x - p.blocks;
    if constexpr (WHAT == kReserve) {
        constexpr int kPer = kGroupSeqs / kWaves;
        const int s0 = g * kGroupSeqs + wave * kPer;
        int lo = 0, hi = 0;
        if (lane < kPer && s0 + lane < p.items) grown(p.old_lens[s0 + lane], p.new_lens[s0 + lane], p.log2_page, p.max_pages, lo, hi);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (s0 + i >= p.items) break;
            const int a = __builtin_amdgcn_readlane(lo, i), b = __builtin_amdgcn_readlane(hi, i);
            const int32_t* row = p.table + (int64_t)(s0 + i) * p.max_pages;
            int n = 0;
            for (int e = a + lane; e < b; e += 64) n += row[e] < 0;
            n = b > a ? wave_sum(n) : 0;
            if (lane == 0) p.need[s0 + i] = n;
            mine += n;
        }
        if (lane == 0) sums[wave] = mine;
        __syncthreads();
        if (threadIdx.x == 0) p.group[g] = sums[0] + sums[1] + sums[2] + sums[3];
    } else if constexpr (WHAT == kFork) {
        const int i = g * kGroupForks + threadIdx.x;
        bool need = false;
        int s, d, len, length = -1;
        if (i < p.items && fork_of(p, i, s, d, len)) {
            length = len;
            if (len & ((1 << p.log2_page) - 1)) {
                const int tail = p.table[(int64_t)s * p.max_pages + (len >> p.log2_page)];
                need = (uint32_t)tail < (uint32_t)p.num_pages;
            }
        }
        if (i < p.items) {
            p.need[i] = need;
            p.length[i] = length;
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(need);
        if (lane == 0) sums[wave] = __popcll(m);
        __syncthreads();
        if (threadIdx.x == 0) p.group[g] = sums[0] + sums[1] + sums[2] + sums[3];
    }
}

// ------------------------------------------------------------- reserve

struct Reserve {
    Survey s;
    int32_t* table;
    int32_t* refs;
    int32_t* shortfall;
    int32_t groups;
};

// One workgroup per sequence.
__global__ __launch_bounds__(kThreads) void reserve_kernel(const Reserve p) {
    __shared__ int wants[kWaves];
    const int s = blockIdx.x, g = s / kGroupSeqs, lane = lane_id(), wave = threadIdx.x >> 6;
    const Pool pool{p.s.bits, p.s.counts, p.s.blocks};
    const int need = p.s.need[s];
    if (need == 0 && s != 0) return;
    // (Tables may want more pages than 32 bits count: 2^16 rows of 2^24 entries.)
    const int64_t missing = long_sum_of(p.s.group, p.groups) - sum_of(pool.counts, pool.blocks);
    if (s == 0 && threadIdx.x == 0) *p.shortfall = (int32_t)min<int64_t>(max<int64_t>(missing, 0), INT32_MAX);
    if (missing > 0 || need == 0) return;
    int rank = sum_of(p.s.group, g) + sum_of(p.s.need + g * kGroupSeqs, s - g * kGroupSeqs);
    int lo, hi;
    grown(p.s.old_lens[s], p.s.new_lens[s], p.s.log2_page, p.s.max_pages, lo, hi);
    int32_t* row = p.table + (int64_t)s * p.s.max_pages;
    for (int e0 = lo; e0 < hi; e0 += kThreads) {
        const int e = e0 + (int)threadIdx.x;
        const bool want = e < hi && row[e] < 0;
        const uint64_t m = __builtin_amdgcn_ballot_w64(want);
        if (lane == 0) wants[wave] = __popcll(m);
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            before += w < wave ? wants[w] : 0;
            all += wants[w];
        }
        __syncthreads();
        if (m) {
            const int page = select(pool, want ? rank + before + count_below(m) : -1);
            if (want && page >= 0) {
                row[e] = page;
                p.refs[page] = 1;
            }
        }
        rank += all;
    }
}

// ---------------------------------------------------------------- free

struct Free {
    int32_t* table;
    int32_t* refs;
    const int32_t* lens;
    const int32_t* seqs;
    int64_t max_pages;
    int32_t num_seqs, num_pages, log2_page, window, sinks;
};

// One workgroup per listed sequence and kThreads of its entries.  The entry is
// taken with an exchange, so that a sequence listed twice gives each page up once.
__global__ __launch_bounds__(kThreads) void free_kernel(const Free p) {
    const int s = p.seqs[blockIdx.x];
    if ((uint32_t)s >= (uint32_t)p.num_seqs) return;
    const int64_t len = p.lens[s];
    for (int64_t e = (int64_t)blockIdx.y * kThreads + threadIdx.x; e < p.max_pages; e += (int64_t)gridDim.y * kThreads) {
        const int64_t first = e << p.log2_page, last = first + (int64_t(1) << p.log2_page) - 1;
        if (first < p.sinks || (p.window > 0 && last + p.window > len)) continue;
        int32_t* entry = p.table + (int64_t)s * p.max_pages + e;
        if (*entry < 0) continue;
        const int page = atomicExch(entry, -1);
        if ((uint32_t)page < (uint32_t)p.num_pages) atomicSub(p.refs + page, 1);
    }
}

// ---------------------------------------------------------------- copies

// Copies `chunks` pieces of 16 bytes, piece i from src + 8 at(i) to dst + 8 at(i).
template <typename AT>
__device__ __forceinline__ void copy_pieces(const uint16_t* src, uint16_t* dst, int begin, int chunks, AT at) {
    u32x4 v[kUnroll];
    int64_t off[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
        const int i = begin + j * kThreads + (int)threadIdx.x;
        if (i < chunks) {
            off[j] = at(i);
            v[j] = __builtin_nontemporal_load(gbl(reinterpret_cast<const u32x4*>(src) + off[j]));
        }
    }
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
        const int i = begin + j * kThreads + (int)threadIdx.x;
        if (i < chunks) __builtin_nontemporal_store(v[j], gbl(reinterpret_cast<u32x4*>(dst) + off[j]));
    }
}

struct Copy {
    const int32_t* src;
    const int32_t* dst;
    const int32_t* moves;  // their number on the device; NULL: `count`
    int32_t count, num_pages;
    int64_t page_bytes;
    int32_t segments;  // of one page
    // compact: the table's new numbers, by the workgroups with blockIdx.y == arrays
    const int32_t* table;
    int32_t* new_table;
    const int32_t* map;
    int64_t entries;
    int32_t arrays;
};

__global__ __launch_bounds__(kThreads) void copy_kernel(const Copy p, const Arrays arrays) {
    if ((int)blockIdx.y == p.arrays) {
        for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < p.entries; i += (int64_t)gridDim.x * kThreads) {
            const int e = p.table[i];
            p.new_table[i] = (uint32_t)e < (uint32_t)p.num_pages ? p.map[e] : e;
        }
        return;
    }
    uint16_t* cache = arrays.p[blockIdx.y];
    const int64_t items = (int64_t)(p.moves ? *p.moves : p.count) * p.segments;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int i = (int)(item / p.segments), segment = (int)(item % p.segments);
        const int a = p.src[i], b = p.dst[i];
        if ((uint32_t)a >= (uint32_t)p.num_pages || (uint32_t)b >= (uint32_t)p.num_pages) continue;
        const int64_t at = (int64_t)segment * kSegment;
        const int chunks = (int)(min<int64_t>(kSegment, p.page_bytes - at) / 16);
        copy_pieces(cache + ((int64_t)a * p.page_bytes + at) / 2, cache + ((int64_t)b * p.page_bytes + at) / 2, 0, chunks, [](int c) { return (int64_t)c; });
    }
}

// ----------------------------------------------------------------- fork

struct Fork {
    Survey s;
    int32_t* table;
    int32_t* refs;
    int32_t* lens;
    int32_t* shortfall;
    int32_t groups;
    int32_t kv_heads, head_dim, arrays;
};

// (A kernel, so that a captured call replays it.)
__global__ void zero_kernel(int32_t* word) {
    if (threadIdx.x == 0) *word = 0;
}

// Workgroups (i, y): fork i, caches y, y + gridDim.y, ...  Those with y = 0
// write the row as well.  Lengths are those that the survey found, so that all
// of a fork's workgroups go by the same one, also where a sequence is in both lists.
__global__ __launch_bounds__(kThreads) void fork_kernel(const Fork p, const Arrays arrays) {
    __shared__ int shared_page;
    const Pool pool{p.s.bits, p.s.counts, p.s.blocks};
    const int i = blockIdx.x, g = i / kGroupForks, lane = lane_id();
    // What waits for no other load comes first (36 forks, 32 caches: 19.8 -> 19.3 us).
    const int32_t* needs = p.s.need + g * kGroupForks;
    const int len = p.s.length[i], s = p.s.src[i], d = p.s.dst[i];
    const bool need = p.s.need[i] != 0;
    const int wanted = first_of(p.s.group, p.groups), there = first_of(pool.counts, pool.blocks);
    const int before = first_of(p.s.group, g), ahead = first_of(needs, i - g * kGroupForks);
    const int missing = sum_of(p.s.group, p.groups, wanted) - sum_of(pool.counts, pool.blocks, there);
    if (i == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.shortfall = max(missing, 0);
    if (missing > 0 || len < 0) return;
    const int page_size = 1 << p.s.log2_page, full = len >> p.s.log2_page, part = len & (page_size - 1);
    const int32_t* from = p.table + (int64_t)s * p.s.max_pages;
    const int tail = need ? from[full] : -1;
    int page = -1;
    if (need) {
        if (threadIdx.x < 64) {
            const int rank = sum_of(p.s.group, g, before) + sum_of(needs, i - g * kGroupForks, ahead);
            const int found = select(pool, lane == 0 ? rank : -1);
            if (lane == 0) shared_page = found;
        }
        __syncthreads();
        page = shared_page;
    }
    if (blockIdx.y == 0) {
        int32_t* to = p.table + (int64_t)d * p.s.max_pages;
        for (int64_t e = threadIdx.x; e < p.s.max_pages; e += kThreads) {
            int v = -1;
            if (e < full) {
                v = from[e];
                if ((uint32_t)v < (uint32_t)p.s.num_pages) atomicAdd(p.refs + v, 1);
            } else if (e == full && need) {
                v = page;
            }
            to[e] = v;
        }
        if (threadIdx.x == 0) {
            p.lens[d] = len;
            if (page >= 0) p.refs[page] = 1;
        }
    }
    if (page < 0) return;
    if ((uint32_t)tail >= (uint32_t)p.s.num_pages) return;
    const int per_token = p.head_dim / 8;
    const int run = part * per_token;  // pieces of one kv head, contiguous
    const int chunks = p.kv_heads * run;
    const int64_t page_pieces = (int64_t)p.kv_heads * page_size * per_token;
    for (int c = blockIdx.y; c < p.arrays; c += gridDim.y) {
        const uint16_t* src = arrays.p[c] + (int64_t)tail * page_pieces * 8;
        uint16_t* dst = arrays.p[c] + (int64_t)page * page_pieces * 8;
        for (int at = 0; at < chunks; at += kThreads * kUnroll)
            copy_pieces(src, dst, at, chunks, [&](int k) {
                const int head = k / run;
                return (int64_t)head * page_size * per_token + (k - head * run);
            });
    }
}

// --------------------------------------------------------------- compact

struct Compact {
    const int32_t* refs;
    int32_t* new_refs;
    int32_t* live;
    int32_t* map;
    int32_t* src;
    int32_t* dst;
    int32_t* moves;
    Pool pool;
    int32_t num_pages;
};

// One lane per page.
__global__ __launch_bounds__(kThreads) void number_kernel(const Compact p) {
    const int p0 = blockIdx.x * kThreads + (threadIdx.x & ~63), page = p0 + lane_id();
    const int live = p.num_pages - sum_of(p.pool.counts, p.pool.blocks);
    const int holes = free_below(p.pool, live);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *p.live = live;
        *p.moves = holes;
    }
    if (p0 >= p.num_pages) return;
    const bool in = page < p.num_pages;
    const bool free = in && (p.pool.bits[page / 32] >> (page % 32) & 1);
    const uint64_t free_mask = __builtin_amdgcn_ballot_w64(free);
    const bool moves = in && !free && page >= live;
    int to = page;
    if (__builtin_amdgcn_ballot_w64(moves)) {
        const int before = free_below(p.pool, p0) + count_below(free_mask);  // free pages below this one
        const int rank = page - live - (before - holes);                     // pages in use in [live, page)
        const int found = select(p.pool, moves ? rank : -1);
        if (moves && found >= 0) {
            to = found;
            p.src[rank] = page;
            p.dst[rank] = to;
        }
    }
    if (!in) return;
    p.map[page] = to;
    // Every count is written by the page that it comes from, and read by no other.
    if (!free) p.new_refs[to] = p.refs[page];
    if (page >= live) p.new_refs[page] = 0;
}

// ---------------------------------------------------------------- append

struct Append {
    const uint16_t* k;
    const uint16_t* v;
    uint16_t* k_cache;
    uint16_t* v_cache;
    const int32_t* table;
    const int32_t* lens;
    const int32_t* starts;
    int64_t k_stride, v_stride, max_pages;
    int32_t num_seqs, num_tokens, kv_heads, head_dim, log2_page, num_pages;
    int32_t tokens;  // of one workgroup, at most kAppendTokens
};

constexpr int kAppendTokens = 16;

// One workgroup writes the keys and values of `tokens` consecutive rows.  The
// slot of each row is found once, by one lane, and shared; each lane then
// moves the same 16-byte piece of every row.
__global__ __launch_bounds__(kThreads) void append_kernel(const Append p) {
    __shared__ int64_t slots[kAppendTokens];  // piece offset of the row's slot in head 0; -1: not written
    const int t0 = blockIdx.x * p.tokens, n = min(p.tokens, p.num_tokens - t0);
    const int per_token = p.head_dim / 8;
    const int pieces = p.kv_heads * per_token;
    const int64_t head_pieces = (int64_t)per_token << p.log2_page;
    if ((int)threadIdx.x < 64) {
        const int lane = lane_id(), t = t0 + min(lane, n - 1);
        int s = t, place_back = 1;  // the row is this many tokens from its sequence's end
        if (p.starts) {
            // The sequence of row t0: the last one that starts at or before it.
            int low = 0;
            for (int b = 0; b < p.num_seqs; b += 64) {
                const bool at = b + lane < p.num_seqs && p.starts[b + lane + 1] <= t0;
                const uint64_t m = __builtin_amdgcn_ballot_w64(at);
                low += __popcll(m);
                if (m != ~0ull) break;
            }
            s = min(low, p.num_seqs - 1);
            while (s + 1 < p.num_seqs && p.starts[s + 1] <= t) ++s;
            place_back = p.starts[s] <= t ? p.starts[s + 1] - t : 0;
        }
        const int64_t len = p.lens[s];
        const int64_t place = len - place_back;
        const int64_t entry = place >> p.log2_page;
        int64_t slot = -1;
        if (place_back > 0 && place >= 0 && entry < p.max_pages) {
            const int page = p.table[(int64_t)s * p.max_pages + entry];
            if ((uint32_t)page < (uint32_t)p.num_pages)
                slot = (int64_t)page * p.kv_heads * head_pieces + (place & ((1 << p.log2_page) - 1)) * per_token;
        }
        if (lane < n) slots[lane] = slot;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * pieces; i += kThreads) {
        const bool value = i >= pieces;
        const int c = value ? i - pieces : i;
        const int head = c / per_token;
        const int64_t off = head * head_pieces + (c - head * per_token);
        const u32x4* src = reinterpret_cast<const u32x4*>(value ? p.v : p.k) + c;
        u32x4* dst = reinterpret_cast<u32x4*>(value ? p.v_cache : p.k_cache) + off;
        const int64_t stride = (value ? p.v_stride : p.k_stride) / 8;
        for (int t = 0; t < n; t += kUnroll) {
            u32x4 w[kUnroll];
#pragma unroll
            for (int j = 0; j < kUnroll; ++j)
                if (t + j < n) w[j] = *gbl(src + (int64_t)(t0 + t + j) * stride);
#pragma unroll
            for (int j = 0; j < kUnroll; ++j)
                if (t + j < n && slots[t + j] >= 0) *gbl(dst + slots[t + j]) = w[j];
        }
    }
}

// ------------------------------------------------------------------ host

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }

// The workspace, in 16-byte steps: counts, bits, needs, lengths, group sums, then
// compact's map and moves (a move's count first).
struct Layout {
    int64_t blocks, counts, bits, need, length, group, map, moves, total;
};
Layout layout_of(int64_t num_pages, int64_t num_seqs) {
    Layout l{};
    l.blocks = ceil_div(num_pages, kBlockPages);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up16(bytes);
        return here;
    };
    l.counts = take(4 * l.blocks);
    l.bits = take(4 * l.blocks * kBlockWords);
    l.need = take(4 * num_seqs);
    l.length = take(4 * num_seqs);
    l.group = take(4 * ceil_div(num_seqs, kGroupSeqs));
    l.map = take(4 * num_pages);
    l.moves = take(16 + 8 * num_pages);
    l.total = at;
    return l;
}

wq_status check_pool(const char* fn, int64_t num_seqs, int64_t num_pages, int64_t max_pages) {
    WQ_TRY(in_range(fn, "num_seqs", num_seqs, 1, WQ_CACHE_MAX_SEQS));
    WQ_TRY(in_range(fn, "num_pages", num_pages, 1, WQ_CACHE_MAX_PAGES));
    return in_range(fn, "max_pages_per_seq", max_pages, 1, WQ_CACHE_MAX_PAGES);
}

wq_status check_page_size(const char* fn, int64_t page_size) {
    if (!is_pow2(page_size) || page_size > WQ_CACHE_MAX_PAGE_SIZE)
        return err(WQ_ERR_UNSUPPORTED, "%s: page_size must be a power of two in [1, %lld] (got %lld)", fn,
                   (long long)WQ_CACHE_MAX_PAGE_SIZE, (long long)page_size);
    return WQ_OK;
}

wq_status check_heads(const char* fn, int64_t kv_heads, int64_t head_dim) {
    WQ_TRY(in_range(fn, "num_kv_heads", kv_heads, 1, WQ_CACHE_MAX_KV_HEADS));
    if (head_dim < 8 || head_dim % 8 != 0 || head_dim > WQ_CACHE_MAX_HEAD_DIM)
        return err(WQ_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of 8 in [8, %lld] (got %lld)", fn,
                   (long long)WQ_CACHE_MAX_HEAD_DIM, (long long)head_dim);
    return WQ_OK;
}

wq_status check_arrays(const char* fn, void* const* caches, int64_t n, Arrays& out) {
    if (!caches) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(in_range(fn, "num_caches", n, 1, WQ_CACHE_MAX_ARRAYS));
    for (int64_t i = 0; i < n; ++i) {
        if (!caches[i]) return err(WQ_ERR_INVALID_ARG, "%s: caches[%lld] is null", fn, (long long)i);
        if (!aligned(caches[i], 16)) return err(WQ_ERR_MISALIGNED, "%s: caches[%lld] must be 16-byte aligned", fn, (long long)i);
        out.p[i] = static_cast<uint16_t*>(caches[i]);
    }
    return WQ_OK;
}

wq_status check_workspace(const char* fn, const void* workspace, size_t bytes, const Layout& l) {
    if (!workspace || bytes < (size_t)l.total)
        return err(WQ_ERR_INVALID_ARG, "%s: a workspace of %lld bytes is needed (got %zu)", fn, (long long)l.total, workspace ? bytes : (size_t)0);
    if (!aligned(workspace, 16)) return err(WQ_ERR_MISALIGNED, "%s: workspace must be 16-byte aligned", fn);
    return WQ_OK;
}

template <typename... P>
bool words_aligned(P... p) {
    return (aligned(p, 4) && ...);
}

// No two of the spans overlap.
template <int N>
bool disjoint(const Span (&s)[N]) {
    for (int i = 0; i < N; ++i)
        for (int j = i + 1; j < N; ++j)
            if (overlaps(s[i], s[j])) return false;
    return true;
}

template <typename T>
T* at(void* workspace, int64_t offset) {
    return reinterpret_cast<T*>(static_cast<char*>(workspace) + offset);
}

Survey survey_of(const int32_t* refs, int64_t num_pages, void* ws, const Layout& l) {
    Survey s{};
    s.refs = refs;
    s.num_pages = (int32_t)num_pages;
    s.bits = at<uint32_t>(ws, l.bits);
    s.counts = at<int32_t>(ws, l.counts);
    s.blocks = (int32_t)l.blocks;
    s.need = at<int32_t>(ws, l.need);
    s.length = at<int32_t>(ws, l.length);
    s.group = at<int32_t>(ws, l.group);
    return s;
}

// Workgroups of a copy over `arrays` caches: a few for every CU, the rest of
// the pages in a loop.
int64_t copy_blocks(int64_t items, int64_t arrays) { return std::max<int64_t>(1, std::min(items, ceil_div(4096, arrays))); }

}  // namespace
}  // namespace cache
}  // namespace wq

using namespace wq::cache;
using wq::host::err;
using wq::host::span;
using wq::host::Span;

extern "C" {

wq_status wq_cache_append(const uint16_t* k_new, const uint16_t* v_new, uint16_t* k_cache, uint16_t* v_cache,
                          const int32_t* block_table, const int32_t* seq_lens, const int32_t* q_starts,
                          int64_t num_seqs, int64_t num_tokens, int64_t num_kv_heads, int64_t head_dim,
                          int64_t k_stride, int64_t v_stride, int64_t page_size, int64_t num_pages,
                          int64_t max_pages_per_seq, void* stream) {
    static const char* fn = "wq_cache_append";
    if (!k_new || !v_new || !k_cache || !v_cache || !block_table || !seq_lens)
        return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(wq::host::in_range(fn, "num_seqs", num_seqs, 1, (int64_t)1 << 20));
    WQ_TRY(wq::host::in_range(fn, "num_tokens", num_tokens, 1, WQ_CACHE_MAX_TOKENS));
    WQ_TRY(check_heads(fn, num_kv_heads, head_dim));
    WQ_TRY(check_page_size(fn, page_size));
    WQ_TRY(wq::host::in_range(fn, "num_pages", num_pages, 1, INT32_MAX));
    WQ_TRY(wq::host::in_range(fn, "max_pages_per_seq", max_pages_per_seq, 1, INT32_MAX));
    if (!q_starts && num_tokens != num_seqs)
        return err(WQ_ERR_INVALID_ARG, "%s: without q_starts there is one new token per sequence (%lld tokens, %lld sequences)", fn,
                   (long long)num_tokens, (long long)num_seqs);
    const int64_t row = num_kv_heads * head_dim;
    for (const int64_t stride : {k_stride, v_stride})
        if (stride < row || stride % 8 != 0 || stride > ((int64_t)1 << 32))
            return err(WQ_ERR_INVALID_ARG, "%s: strides must be multiples of 8 of at least num_kv_heads * head_dim (got %lld)", fn, (long long)stride);
    if (!wq::host::aligned(k_new, 16) || !wq::host::aligned(v_new, 16) || !wq::host::aligned(k_cache, 16) || !wq::host::aligned(v_cache, 16))
        return err(WQ_ERR_MISALIGNED, "%s: k_new, v_new and the caches must be 16-byte aligned", fn);
    if (!words_aligned(block_table, seq_lens, q_starts)) return err(WQ_ERR_MISALIGNED, "%s: tables and lengths must be 4-byte aligned", fn);
    const uint64_t cache_bytes = (uint64_t)num_pages * row * page_size * 2;
    const Span k = span(k_cache, cache_bytes), v = span(v_cache, cache_bytes);
    if (overlaps(k, v)) return err(WQ_ERR_INVALID_ARG, "%s: the caches overlap", fn);
    const Span inputs[] = {span(k_new, ((uint64_t)(num_tokens - 1) * k_stride + row) * 2), span(v_new, ((uint64_t)(num_tokens - 1) * v_stride + row) * 2),
                           span(block_table, (uint64_t)num_seqs * max_pages_per_seq * 4), span(seq_lens, (uint64_t)num_seqs * 4),
                           span(q_starts, q_starts ? (uint64_t)(num_seqs + 1) * 4 : 0)};
    for (const Span& in : inputs)
        if (overlaps(k, in) || overlaps(v, in)) return err(WQ_ERR_INVALID_ARG, "%s: a cache overlaps an input", fn);

    Append p{};
    p.k = k_new;
    p.v = v_new;
    p.k_cache = k_cache;
    p.v_cache = v_cache;
    p.table = block_table;
    p.lens = seq_lens;
    p.starts = q_starts;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.max_pages = max_pages_per_seq;
    p.num_seqs = (int32_t)num_seqs;
    p.num_tokens = (int32_t)num_tokens;
    p.kv_heads = (int32_t)num_kv_heads;
    p.head_dim = (int32_t)head_dim;
    p.log2_page = wq::host::log2_of(page_size);
    p.num_pages = (int32_t)num_pages;
    // One row per workgroup until there are a few workgroups for every CU.
    p.tokens = (int32_t)std::min<int64_t>(kAppendTokens, std::max<int64_t>(1, num_tokens / 2048));
    (void)hipGetLastError();
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)ceil_div(num_tokens, p.tokens)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), p);
    return wq::host::hip_result(fn, hipGetLastError());
}

wq_status wq_cache_copy_pages(void* const* caches, int64_t num_caches, int64_t page_bytes, int64_t num_pages,
                              const int32_t* src, const int32_t* dst, int64_t count, void* stream) {
    static const char* fn = "wq_cache_copy_pages";
    Arrays arrays;
    WQ_TRY(check_arrays(fn, caches, num_caches, arrays));
    WQ_TRY(wq::host::in_range(fn, "num_pages", num_pages, 1, WQ_CACHE_MAX_PAGES));
    WQ_TRY(wq::host::in_range(fn, "count", count, 0, num_pages));
    if (page_bytes < 16 || page_bytes % 16 != 0 || page_bytes > ((int64_t)1 << 30))
        return err(WQ_ERR_INVALID_ARG, "%s: page_bytes must be a multiple of 16 in [16, 2^30] (got %lld)", fn, (long long)page_bytes);
    if (count == 0) return WQ_OK;
    if (!src || !dst) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    if (!words_aligned(src, dst)) return err(WQ_ERR_MISALIGNED, "%s: src and dst must be 4-byte aligned", fn);
    Copy p{};
    p.src = src;
    p.dst = dst;
    p.count = (int32_t)count;
    p.num_pages = (int32_t)num_pages;
    p.page_bytes = page_bytes;
    p.segments = (int32_t)ceil_div(page_bytes, kSegment);
    p.arrays = (int32_t)num_caches;
    (void)hipGetLastError();
    hipLaunchKernelGGL(copy_kernel, dim3((unsigned)copy_blocks(count * p.segments, num_caches), (unsigned)num_caches), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), p, arrays);
    return wq::host::hip_result(fn, hipGetLastError());
}

wq_status wq_page_workspace_size(int64_t num_pages, int64_t num_seqs, size_t* bytes) {
    static const char* fn = "wq_page_workspace_size";
    if (!bytes) return err(WQ_ERR_INVALID_ARG, "%s: null output pointer", fn);
    WQ_TRY(check_pool(fn, num_seqs, num_pages, 1));
    *bytes = (size_t)layout_of(num_pages, num_seqs).total;
    return WQ_OK;
}

wq_status wq_cache_reserve(int32_t* block_table, int32_t* refs, const int32_t* old_lens, const int32_t* new_lens,
                           int64_t num_seqs, int64_t page_size, int64_t num_pages, int64_t max_pages_per_seq,
                           int32_t* shortfall, void* workspace, size_t workspace_bytes, void* stream) {
    static const char* fn = "wq_cache_reserve";
    if (!block_table || !refs || !old_lens || !new_lens || !shortfall) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(check_pool(fn, num_seqs, num_pages, max_pages_per_seq));
    WQ_TRY(check_page_size(fn, page_size));
    if (!words_aligned(block_table, refs, old_lens, new_lens, shortfall)) return err(WQ_ERR_MISALIGNED, "%s: every array must be 4-byte aligned", fn);
    const Layout l = layout_of(num_pages, num_seqs);
    WQ_TRY(check_workspace(fn, workspace, workspace_bytes, l));
    const Span written[] = {span(block_table, (uint64_t)num_seqs * max_pages_per_seq * 4), span(refs, (uint64_t)num_pages * 4), span(shortfall, 4),
                            span(workspace, (uint64_t)l.total)};
    const Span read[] = {span(old_lens, (uint64_t)num_seqs * 4), span(new_lens, (uint64_t)num_seqs * 4)};
    bool apart = disjoint(written);
    for (const Span& w : written)
        for (const Span& r : read) apart = apart && !overlaps(w, r);
    if (!apart) return err(WQ_ERR_INVALID_ARG, "%s: arrays overlap", fn);

    Reserve p{};
    p.s = survey_of(refs, num_pages, workspace, l);
    p.s.items = (int32_t)num_seqs;
    p.s.table = block_table;
    p.s.max_pages = max_pages_per_seq;
    p.s.log2_page = wq::host::log2_of(page_size);
    p.s.old_lens = old_lens;
    p.s.new_lens = new_lens;
    p.table = block_table;
    p.refs = refs;
    p.shortfall = shortfall;
    p.groups = (int32_t)ceil_div(num_seqs, kGroupSeqs);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    hipLaunchKernelGGL((survey_kernel<kReserve>), dim3((unsigned)(l.blocks + p.groups)), dim3(kThreads), 0, st, p.s);
    hipLaunchKernelGGL(reserve_kernel, dim3((unsigned)num_seqs), dim3(kThreads), 0, st, p);
    return wq::host::hip_result(fn, hipGetLastError());
}

wq_status wq_cache_free(int32_t* block_table, int32_t* refs, const int32_t* seq_lens, const int32_t* seqs,
                        int64_t count, int64_t window, int64_t sinks, int64_t num_seqs, int64_t page_size,
                        int64_t num_pages, int64_t max_pages_per_seq, void* stream) {
    static const char* fn = "wq_cache_free";
    if (!block_table || !refs || !seq_lens) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(check_pool(fn, num_seqs, num_pages, max_pages_per_seq));
    WQ_TRY(check_page_size(fn, page_size));
    WQ_TRY(wq::host::in_range(fn, "count", count, 0, num_seqs));
    WQ_TRY(wq::host::in_range(fn, "window", window, 0, (int64_t)1 << 30));
    WQ_TRY(wq::host::in_range(fn, "sinks", sinks, 0, (int64_t)1 << 30));
    if (count == 0) return WQ_OK;
    if (!seqs) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    if (!words_aligned(block_table, refs, seq_lens, seqs)) return err(WQ_ERR_MISALIGNED, "%s: every array must be 4-byte aligned", fn);
    const Span table = span(block_table, (uint64_t)num_seqs * max_pages_per_seq * 4), counts = span(refs, (uint64_t)num_pages * 4);
    const Span lens = span(seq_lens, (uint64_t)num_seqs * 4), list = span(seqs, (uint64_t)count * 4);
    if (overlaps(table, counts) || overlaps(table, lens) || overlaps(table, list) || overlaps(counts, lens) || overlaps(counts, list))
        return err(WQ_ERR_INVALID_ARG, "%s: arrays overlap", fn);
    Free p{};
    p.table = block_table;
    p.refs = refs;
    p.lens = seq_lens;
    p.seqs = seqs;
    p.max_pages = max_pages_per_seq;
    p.num_seqs = (int32_t)num_seqs;
    p.num_pages = (int32_t)num_pages;
    p.log2_page = wq::host::log2_of(page_size);
    p.window = (int32_t)window;
    p.sinks = (int32_t)sinks;
    (void)hipGetLastError();
    hipLaunchKernelGGL(free_kernel, dim3((unsigned)count, (unsigned)std::min<int64_t>(64, ceil_div(max_pages_per_seq, kThreads))), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), p);
    return wq::host::hip_result(fn, hipGetLastError());
}

wq_status wq_cache_fork(void* const* caches, int64_t num_caches, int32_t* block_table, int32_t* refs,
                        int32_t* seq_lens, const int32_t* src, const int32_t* dst, int64_t count,
                        int64_t num_seqs, int64_t num_kv_heads, int64_t head_dim, int64_t page_size,
                        int64_t num_pages, int64_t max_pages_per_seq, int32_t* shortfall, void* workspace,
                        size_t workspace_bytes, void* stream) {
    static const char* fn = "wq_cache_fork";
    if (!block_table || !refs || !seq_lens || !shortfall) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    Arrays arrays;
    WQ_TRY(check_arrays(fn, caches, num_caches, arrays));
    WQ_TRY(check_pool(fn, num_seqs, num_pages, max_pages_per_seq));
    WQ_TRY(check_heads(fn, num_kv_heads, head_dim));
    WQ_TRY(check_page_size(fn, page_size));
    WQ_TRY(wq::host::in_range(fn, "count", count, 0, num_seqs));
    if (count > 0 && (!src || !dst)) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    if (!words_aligned(block_table, refs, seq_lens, src, dst, shortfall)) return err(WQ_ERR_MISALIGNED, "%s: every array must be 4-byte aligned", fn);
    const Layout l = layout_of(num_pages, num_seqs);
    WQ_TRY(check_workspace(fn, workspace, workspace_bytes, l));
    const Span written[] = {span(block_table, (uint64_t)num_seqs * max_pages_per_seq * 4), span(refs, (uint64_t)num_pages * 4),
                            span(seq_lens, (uint64_t)num_seqs * 4), span(shortfall, 4), span(workspace, (uint64_t)l.total)};
    bool apart = disjoint(written);
    for (const Span& w : written) {
        apart = apart && !overlaps(w, span(src, (uint64_t)count * 4)) && !overlaps(w, span(dst, (uint64_t)count * 4));
        for (int64_t i = 0; i < num_caches; ++i)
            apart = apart && !overlaps(w, span(caches[i], (uint64_t)num_pages * num_kv_heads * page_size * head_dim * 2));
    }
    if (!apart) return err(WQ_ERR_INVALID_ARG, "%s: arrays overlap", fn);

    Fork p{};
    p.s = survey_of(refs, num_pages, workspace, l);
    p.s.items = (int32_t)count;
    p.s.table = block_table;
    p.s.max_pages = max_pages_per_seq;
    p.s.log2_page = wq::host::log2_of(page_size);
    p.s.lens = seq_lens;
    p.s.src = src;
    p.s.dst = dst;
    p.s.num_seqs = (int32_t)num_seqs;
    p.table = block_table;
    p.refs = refs;
    p.lens = seq_lens;
    p.shortfall = shortfall;
    p.groups = (int32_t)ceil_div(count, kGroupForks);
    p.kv_heads = (int32_t)num_kv_heads;
    p.head_dim = (int32_t)head_dim;
    p.arrays = (int32_t)num_caches;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    if (count == 0) {
        hipLaunchKernelGGL(zero_kernel, dim3(1), dim3(64), 0, st, shortfall);
        return wq::host::hip_result(fn, hipGetLastError());
    }
    hipLaunchKernelGGL((survey_kernel<kFork>), dim3((unsigned)(l.blocks + p.groups)), dim3(kThreads), 0, st, p.s);
    const int64_t per_fork = std::max<int64_t>(1, std::min(num_caches, ceil_div(4096, count)));
    hipLaunchKernelGGL(fork_kernel, dim3((unsigned)count, (unsigned)per_fork), dim3(kThreads), 0, st, p, arrays);
    return wq::host::hip_result(fn, hipGetLastError());
}

wq_status wq_cache_compact(void* const* caches, int64_t num_caches, int64_t page_bytes, const int32_t* block_table,
                           const int32_t* refs, int32_t* new_table, int32_t* new_refs, int32_t* live,
                           int64_t num_seqs, int64_t num_pages, int64_t max_pages_per_seq, void* workspace,
                           size_t workspace_bytes, void* stream) {
    static const char* fn = "wq_cache_compact";
    if (!block_table || !refs || !new_table || !new_refs || !live) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    Arrays arrays;
    WQ_TRY(check_arrays(fn, caches, num_caches, arrays));
    WQ_TRY(check_pool(fn, num_seqs, num_pages, max_pages_per_seq));
    if (page_bytes < 16 || page_bytes % 16 != 0 || page_bytes > ((int64_t)1 << 30))
        return err(WQ_ERR_INVALID_ARG, "%s: page_bytes must be a multiple of 16 in [16, 2^30] (got %lld)", fn, (long long)page_bytes);
    if (!words_aligned(block_table, refs, new_table, new_refs, live)) return err(WQ_ERR_MISALIGNED, "%s: every array must be 4-byte aligned", fn);
    const Layout l = layout_of(num_pages, num_seqs);
    WQ_TRY(check_workspace(fn, workspace, workspace_bytes, l));
    const uint64_t table_bytes = (uint64_t)num_seqs * max_pages_per_seq * 4, refs_bytes = (uint64_t)num_pages * 4;
    const Span written[] = {span(new_table, table_bytes), span(new_refs, refs_bytes), span(live, 4), span(workspace, (uint64_t)l.total)};
    const Span read[] = {span(block_table, table_bytes), span(refs, refs_bytes)};
    bool apart = disjoint(written);
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 2; ++j)
            apart = apart && (!overlaps(written[i], read[j]) || (i == j && written[i].lo == read[j].lo));
        for (int64_t c = 0; c < num_caches; ++c) apart = apart && !overlaps(written[i], span(caches[c], (uint64_t)num_pages * page_bytes));
    }
    if (!apart) return err(WQ_ERR_INVALID_ARG, "%s: arrays overlap", fn);

    const Survey s = survey_of(refs, num_pages, workspace, l);
    Compact c{};
    c.refs = refs;
    c.new_refs = new_refs;
    c.live = live;
    c.map = at<int32_t>(workspace, l.map);
    c.moves = at<int32_t>(workspace, l.moves);
    c.src = c.moves + 4;
    c.dst = c.src + num_pages;
    c.pool = Pool{s.bits, s.counts, s.blocks};
    c.num_pages = (int32_t)num_pages;
    Copy p{};
    p.src = c.src;
    p.dst = c.dst;
    p.moves = c.moves;
    p.num_pages = (int32_t)num_pages;
    p.page_bytes = page_bytes;
    p.segments = (int32_t)ceil_div(page_bytes, kSegment);
    p.table = block_table;
    p.new_table = new_table;
    p.map = c.map;
    p.entries = num_seqs * max_pages_per_seq;
    p.arrays = (int32_t)num_caches;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    hipLaunchKernelGGL((survey_kernel<kNothing>), dim3((unsigned)l.blocks), dim3(kThreads), 0, st, s);
    hipLaunchKernelGGL(number_kernel, dim3((unsigned)ceil_div(num_pages, kThreads)), dim3(kThreads), 0, st, c);
    hipLaunchKernelGGL(copy_kernel, dim3((unsigned)copy_blocks(ceil_div(num_pages, 2) * p.segments, num_caches), (unsigned)num_caches + 1),
                       dim3(kThreads), 0, st, p, arrays);
    return wq::host::hip_result(fn, hipGetLastError());
}

}  // extern "C"
