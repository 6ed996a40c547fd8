// Causal attention with a sliding window and sinks over a paged KV cache
// (gfx950, wave64), for single tokens and for prompts: one pass over the
// visible keys and values with the running maximum and sum of the softmax.
//
// Rows.  A kv head serves G query heads, so the n new tokens of a sequence are
// n G rows (row r: token r / G, head r % G) against the same keys and values.
// Both kernels put rows on the columns of the matrix cores and compute
// S^T = K Q^T and O^T = V^T P^T.  A lane then holds scores of one row only: the
// softmax needs one exchange between lanes per tile, the factors that rescale O
// are a lane's own, and S^T leaves the matrix cores in the layout that the next
// product takes P^T in, with the tokens of a tile in another order, which V is
// read in as well.  P never leaves the registers.
//
//   few_kernel   sequences with up to 16 rows (decoding).  Bound by the bytes
//                of the cache: no LDS, keys and values go from memory to the
//                matrix cores' registers, 32 tokens per wave and step, and the
//                cache is split over workgroups by the sequences' lengths.
//   tile_kernel  all others.  Bound by the matrix cores: 128 rows per
//                workgroup, 64-token tiles through LDS.
//
// Where the cache is split, merge kernels join the parts.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "wq_device.h"
#include "wq_host.h"
#include "wq_internal.h"
#include "wq_window.h"

namespace wq {
namespace window {
namespace {

using dev::gbl;
using dev::u32x4;
using namespace host;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kFewRows = 16;    // rows of few_kernel
constexpr int kFewTokens = 32;  // tokens of one of its steps
constexpr int kTileRows = 128;  // rows of a workgroup of tile_kernel, 32 per wave
constexpr int kTileTokens = 64;
// Tiles of which some row of a workgroup does not see every token: where its
// rows' windows begin and end, (rows / 64 + 2) each, and where the sinks end.
constexpr int kEdges = 16;
constexpr float kRescale = 8.0f;  // see Softmax

template <typename T>
struct Type;
template <>
struct Type<_Float16> {
    typedef _Float16 Vec8 __attribute__((ext_vector_type(8)));
    static constexpr uint16_t kNaN = 0x7E00;
    static constexpr uint32_t kExponent = 0x7C00;
    static constexpr float kLift = 7.0f;     // see Softmax
    static constexpr float kFine = 2048.0f;  // see few_body
    static __device__ __forceinline__ float4v mfma16(Vec8 a, Vec8 b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float16v mfma32(Vec8 a, Vec8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Type<__bf16> {
    typedef __bf16 Vec8 __attribute__((ext_vector_type(8)));
    static constexpr uint16_t kNaN = 0x7FC0;
    static constexpr uint32_t kExponent = 0x7F80;
    static constexpr float kLift = 0.0f, kFine = 1.0f;  // it has the range of fp32
    static __device__ __forceinline__ float4v mfma16(Vec8 a, Vec8 b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float16v mfma32(Vec8 a, Vec8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

template <typename T>
__device__ __forceinline__ uint16_t bits_of(float x) {
    return __builtin_bit_cast(uint16_t, static_cast<T>(x));
}
template <typename T>
__device__ __forceinline__ float value_of(uint32_t bits) {
    return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(bits)));
}

// The word with those of its two 16-bit values cleared that are not finite.
template <typename T>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
    constexpr uint32_t e = Type<T>::kExponent;
    const uint32_t lo = (w & e) == e ? 0u : w & 0xFFFFu, hi = (w >> 16 & e) == e ? 0u : w & 0xFFFF0000u;
    return lo | hi;
}
// A value that is not finite as it is, 0 for the others.
template <typename T>
__device__ __forceinline__ float other_part(uint32_t bits) {
    return (bits & Type<T>::kExponent) == Type<T>::kExponent ? value_of<T>(bits) : 0.0f;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

struct Params {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* table;
    const int32_t* lens;
    const int32_t* starts;
    uint16_t* out;
    int64_t max_pages, q_stride, out_stride;
    int64_t page_stride;  // elements of a page
    int32_t num_seqs, num_tokens, max_query, num_pages, hq, hkv, group, log2_page, max_seq_len;
    int32_t window, sinks;
    float c;           // |scale| log2(e): scores in log2 units
    uint32_t q_and, q_xor;  // scale < 0 changes the signs of q, scale = 0 makes it zero (with c = 1)
    // few_kernel
    int32_t units;     // per kv head, at most
    int32_t round;     // units per kv head that run at once
    int32_t few_slots; // rows of a unit's partial results
    float* few_acc;    // [unit][kv head][few_slots][head_dim]
    float2* few_ml;    // [unit][kv head][few_slots]: (m, l)
    int2* few_units;   // [sequence][kv head]: first unit, units
    // tile_kernel
    int32_t splits;
    float* tile_acc;   // [token][q head][splits][head_dim]
    float2* tile_ml;
    int32_t few_rows;  // sequences of up to so many rows are few_kernel's, all others tile_kernel's
};

// ------------------------------------------------------------- sequences

struct Seq {
    int first, n, len;  // first row of q, new tokens, tokens
    bool bad;           // its outputs are NaN
    __device__ __forceinline__ bool few(const Params& p) const { return n * p.group <= p.few_rows; }
};

__device__ __forceinline__ Seq seq_of(const Params& p, int s) {
    Seq q;
    q.first = s;
    q.n = 1;
    if (p.starts) {
        q.first = p.starts[s];
        const int end = p.starts[s + 1];
        q.n = q.first < 0 || end > p.num_tokens || end < q.first ? 0 : end - q.first;
    }
    q.len = p.lens[s];
    q.bad = q.len > p.max_seq_len || q.len > (p.max_pages << p.log2_page) || q.n > q.len || q.n > p.max_query;
    return q;
}

// The tokens that new tokens at positions [lo, hi] see, in tiles of TOKENS:
// those of the sinks below `start`, then all from `start` on.
template <int TOKENS>
struct Tiles {
    int first;       // no token below it is in the window of the first
    int start;       // first, down to a multiple of TOKENS
    int sink_tiles, count;
    // A window of 0 holds no token: `first` is then the start of the tile after hi's, so
    // that no aligned group of tokens up to hi's reaches it.
    __device__ __forceinline__ Tiles(const Params& p, int lo, int hi) {
        first = p.window > 0 ? max(0, lo - p.window + 1) : (hi + TOKENS) & ~(TOKENS - 1);
        start = first & ~(TOKENS - 1);
        sink_tiles = (min(p.sinks, start) + TOKENS - 1) / TOKENS;
        count = p.window > 0 || p.sinks > 0 ? sink_tiles + (hi - start + TOKENS) / TOKENS : 0;
    }
    __device__ __forceinline__ int token(int tile) const { return tile < sink_tiles ? tile * TOKENS : start + (tile - sink_tiles) * TOKENS; }
};

__device__ __forceinline__ bool sees(const Params& p, int place, int t) { return t <= place && (t < p.sinks || t > place - p.window); }

// ------------------------------------------------------------ lane tools

__device__ __forceinline__ int inclusive_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1, 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2, 3
    return v;
}
__device__ __forceinline__ int wave_max(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }

// The values of lanes l and l ^ 32 (HALVES) or l and l ^ 16, lower lane first.
template <bool HALVES>
__device__ __forceinline__ void pair_values(float x, float& lo, float& hi) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    uint32_t e0, e1;
    if constexpr (HALVES) {
        auto p = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        e0 = p[0];
        e1 = p[1];
    } else {
        auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        e0 = p[0];
        e1 = p[1];
    }
    lo = __builtin_bit_cast(float, e0);
    hi = __builtin_bit_cast(float, e1);
}
template <bool HALVES>
__device__ __forceinline__ float pair_max(float x) {
    float a, b;
    pair_values<HALVES>(x, a, b);
    return fmaxf(a, b);
}
template <bool HALVES>
__device__ __forceinline__ float pair_sum(float x) {
    float a, b;
    pair_values<HALVES>(x, a, b);
    return a + b;
}

// Softmax.  m is the reference that a row's weights 2^(c s - c m + kLift) are formed
// against, l this lane's share of their sum.  m follows the row's largest score
// only when that passes it by more than kRescale in log2 units, so a wave
// rarely has to rescale its accumulators; weights then reach at most 2^(8 + kLift),
// and their sums are fp32.  The lift, which is the same in every part of a row and so
// leaves the quotient, puts binary16's weights at the top of its range (2^15 <
// 65504): below 2^-14 that type is off by up to 2^-25 however small the weight,
// 2^-32 of the row's largest with the lift, 2^-25 without.
template <typename T>
struct Softmax {
    float m = -INFINITY, l = 0.0f;
    // Given the row's largest new score: whether any row of the wave needs a new
    // reference, and if so the factor for this row (1 where it keeps its own, so
    // that no row's bits depend on the others).
    __device__ __forceinline__ bool advance(float mx, float c, float& factor) {
        const bool need = (mx - m) * c > kRescale;
        if (!__builtin_amdgcn_ballot_w64(need)) return false;
        factor = need ? exp2_((m - mx) * c) : 1.0f;
        m = need ? mx : m;
        l *= factor;
        return true;
    }
    // kLift - c m, or 0 while nothing is visible (every weight is then 2^-inf = 0).
    __device__ __forceinline__ float shift(float c) const { return m == -INFINITY ? 0.0f : fmaf(m, -c, Type<T>::kLift); }
};

// ------------------------------------------------------ few rows: the split
//
// The visible tokens of every few-row sequence are cut into steps of 32 tokens
// and the steps into units, each one workgroup's (per kv head).  The lengths
// are on the device, so every wave works the cut out for itself: T steps to a
// unit at most, and then which sequence unit u falls in.  The steps of a
// sequence are dealt evenly over its units.
//
// A launch lasts about r (T + kUnitCost) steps when the units fill r rounds of
// workgroups (two to a CU).  What counts is that the longest sequences come out
// even, so T is a whole fraction of the longest: for one round and for two, the
// smaller such T that fits, and then the better of both.  Up to 64 sequences, one to
// a lane; the plain T beyond.  Against the plain T alone, 24/8 heads of 128: 16 sequences
// of 4096 tokens 53.2 -> 49.4 us, 7 of 9000 52.3 -> 49.2, 20 of 5000 71.6 -> 70.5, but 33 of
// 4096 99.0 -> 100.5 and 48 of 4096 133 -> 146; ragged ones are the same (16 of 4000 to
// 20000: 119, 64 of up to 30000: 370).  kUnitCost from 0 to 8 changes 48 sequences of up to
// 30000 tokens (96 to 98 us) by less than runs differ.
constexpr int kUnitCost = 4;

struct Unit {
    int seq, steps, chunk, first, count;  // steps of the sequence; which of its `count` units, the first of them
};

__device__ __forceinline__ int few_steps(const Params& p, int s) {
    const Seq q = seq_of(p, s);
    if (q.n == 0 || !q.few(p)) return 0;
    if (q.bad) return 1;
    return max(1, Tiles<kFewTokens>(p, q.len - q.n, q.len - 1).count);
}

// ceil(a / b) for 0 <= a <= 2^22, 1 <= b: the estimate is off by one at most.
__device__ __forceinline__ int ceil_quotient(int a, int b) {
    const int n = a + b - 1;
    int q = (int)((float)n * __builtin_amdgcn_rcpf((float)b));
    const int r = n - q * b;
    return q + (r >= b ? 1 : r < 0 ? -1 : 0);
}

__device__ __forceinline__ bool unit_of(const Params& p, int u, Unit& out) {
    if (p.units == p.num_seqs) {
        out = Unit{u, few_steps(p, u), 0, u, 1};
        return out.steps > 0;
    }
    const int lane = threadIdx.x & 63;
    const int per = (p.num_seqs + 63) / 64;  // lane i has sequences [i per, (i + 1) per)
    const int s0 = min(lane * per, p.num_seqs), s1 = min(s0 + per, p.num_seqs);
    const int steps0 = s0 < s1 ? few_steps(p, s0) : 0;
    auto steps_of = [&](int s) { return s == s0 ? steps0 : few_steps(p, s); };
    int sum = 0, most = 0;
    for (int s = s0; s < s1; ++s) {
        sum += steps_of(s);
        most = max(most, steps_of(s));
    }
    const int total = last_lane(inclusive_scan(sum));
    // sum of ceil(steps / T) <= total / T + sequences, so this T always fits.
    int t = max(1, ceil_quotient(total, p.units - p.num_seqs));
    if (per == 1) {
        most = wave_max(most);
        int cost = 2 * (t + kUnitCost);
#pragma unroll
        for (int r = 1; r <= 2; ++r) {
            const int room = min(r * p.round, p.units);
            const int k0 = max(1, (int)((float)most * (float)room * __builtin_amdgcn_rcpf((float)max(total, 1))));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int tk = max(1, ceil_quotient(most, max(1, k0 - k)));
                const int need = last_lane(inclusive_scan(ceil_quotient(sum, tk)));
                if (need <= room && r * (tk + kUnitCost) < cost) {
                    cost = r * (tk + kUnitCost);
                    t = tk;
                }
            }
        }
    }
    int mine = 0;
    for (int s = s0; s < s1; ++s) mine += ceil_quotient(steps_of(s), t);
    int first = inclusive_scan(mine) - mine;
    const bool here = u >= first && u < first + mine;
    const uint64_t owner = __builtin_amdgcn_ballot_w64(here);
    if (owner == 0) return false;
    int s = s0, steps = steps0, n = ceil_quotient(steps0, t);
    if (here) {
        while (u >= first + n) {
            first += n;
            steps = few_steps(p, ++s);
            n = ceil_quotient(steps, t);
        }
    }
    const int from = __builtin_ctzll(owner);
    out.seq = __builtin_amdgcn_readlane(s, from);
    out.steps = __builtin_amdgcn_readlane(steps, from);
    out.first = __builtin_amdgcn_readlane(first, from);
    out.count = __builtin_amdgcn_readlane(n, from);
    out.chunk = u - out.first;
    return true;
}

// Output address of row r of a sequence.
__device__ __forceinline__ uint16_t* out_row(const Params& p, const Seq& q, int kvh, int r, int dim) {
    return p.out + (int64_t)(q.first + r / p.group) * p.out_stride + (int64_t)(kvh * p.group + r % p.group) * dim;
}

// o = acc / l; rows that see nothing are zero.
template <typename T>
__device__ __forceinline__ uint16_t finish(const Params& p, float acc, float l) {
    if (p.window == 0 && p.sinks == 0) return l != l ? Type<T>::kNaN : 0;
    return l != l ? Type<T>::kNaN : bits_of<T>(acc / l);
}

// One step's keys and values in registers.  Lane (i = lane % 16, g = lane / 16):
//   k[a][ks]  key of token 8 (i / 4) + 4 a + i % 4, dims 32 ks + 8 g .. + 7;
//   v[j]      value of token 8 g + j, dims VW i .. VW i + VW - 1.
// The matrix cores' row i of key tile a is then token 8 (i / 4) + 4 a + i % 4, so
// that they leave the scores of tokens 8 g + 4 a + r in lane group g: the
// tokens whose values it holds.
//
// Keys are fetched again as soon as the scores are formed and values as soon as
// they are weighted, so a wave always has between half a step and a whole one
// (16 KB at head_dim 128) in flight, in one set of registers.  Every path
// issues the same loads (past the last step, of one row again), so that the
// waits that the compiler counts stay exact; the table entries of a step are
// asked for before the loads of the one ahead of it, so that waiting for them
// waits for no key or value.
// WHOLE: pages of 8 tokens or more, so that 8 aligned tokens share one.
// WAVES: 4 where the cache is split, 8 where a workgroup takes a sequence whole
// (516 tokens of 64 dims, 2 kv heads: 8.9 -> 8.2 us; 64 sequences of up to 2004, 4
// kv heads: 28.3 -> 22.6 against the split).
template <int D, int WAVES>
struct FewShared {
    float acc[WAVES][kFewRows][D];
    float m[WAVES][kFewRows], l[WAVES][kFewRows];
    // Tokens that only some rows see and whose values are not all finite, once
    // for each lane that met one.  16 new tokens at most have 15 such tokens at
    // the end and 15 where their windows begin, in 16 lanes each.
    int others, other[512];
};

template <typename T, int D, bool WHOLE, int WAVES>
__device__ __forceinline__ void few_body(const Params& p, int block, FewShared<D, WAVES>& sh) {
    constexpr int kOthers = sizeof(sh.other) / sizeof(sh.other[0]);
    using Vec8 = typename Type<T>::Vec8;
    constexpr int kKs = D / 32, kVw = D / 16;
    typedef uint32_t VLoad __attribute__((ext_vector_type(kVw / 2)));
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = block % p.hkv, u = block / p.hkv;
    Unit un;
    if (!unit_of(p, u, un)) return;
    const Seq q = seq_of(p, un.seq);
    const int rows = q.n * p.group;
    // (The merge reads this only where the sequence has units.)
    if (p.units > p.num_seqs && un.chunk == 0 && tid == 0) p.few_units[un.seq * p.hkv + kvh] = make_int2(un.first, un.count);
    if (q.bad) {
        for (int64_t x = tid; x < (int64_t)rows * D; x += (WAVES * 64)) out_row(p, q, kvh, (int)(x / D), D)[x % D] = Type<T>::kNaN;
        return;
    }
    if (tid == 0) sh.others = 0;
    __syncthreads();
    const Tiles<kFewTokens> tiles(p, q.len - q.n, q.len - 1);
    const int begin = (int)((int64_t)tiles.count * un.chunk / un.count), end = (int)((int64_t)tiles.count * (un.chunk + 1) / un.count);
    const int place = q.len - q.n + min(i / p.group, q.n - 1);  // of the lane's row
    const int last = q.len - 1;

    Vec8 qf[kKs];
    {
        const int r = min(i, rows - 1);
        const uint16_t* src = p.q + (int64_t)(q.first + r / p.group) * p.q_stride + (int64_t)(kvh * p.group + r % p.group) * D + g * 8;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            u32x4 w = *gbl(reinterpret_cast<const u32x4*>(src + ks * 32));
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (w[e] & p.q_and) ^ p.q_xor;
            qf[ks] = __builtin_bit_cast(Vec8, w);
        }
    }

    const int32_t* trow = p.table + (int64_t)un.seq * p.max_pages;
    const int page_mask = (1 << p.log2_page) - 1;
    const uint16_t* kbase = p.k + ((int64_t)kvh << p.log2_page) * D + g * 8;
    const uint16_t* vbase = p.v + ((int64_t)kvh << p.log2_page) * D + i * kVw;
    int bad = 0;

    // Visible to some row.  Only pages of such tokens are looked up: a token that
    // is not stands for `safe`, which is, and is masked.
    auto used = [&](int t) { return t <= last && (t < p.sinks || t >= tiles.first); };
    const int safe = p.window > 0 ? last : 0;
    auto lookup = [&](int t) { return trow[t >> p.log2_page]; };
    auto checked = [&](int page) {
        bad |= (uint32_t)page >= (uint32_t)p.num_pages;
        return (uint32_t)page >= (uint32_t)p.num_pages ? 0 : page;
    };
    auto offset = [&](int page, int t) { return (int64_t)page * p.page_stride + (int64_t)((t & page_mask) * D); };
    // The token of a lane's keys in step t0 (t0 < 0: past the last step), and the
    // first of its values.  Of a group of 8 in one page, the first used token
    // stands for all.
    auto key_token = [&](int t0, int a) { return t0 + (i >> 2) * 8 + a * 4 + (i & 3); };
    auto page_token = [&](int t) { return t < p.sinks ? t : max(t, tiles.first); };
    struct Pages {
        int k[2], v[8];
    };
    auto or_safe = [&](int t0, int t) { return t0 >= 0 && used(t) ? t : safe; };
    auto pages_of = [&](int t0) {
        Pages pg;
        if constexpr (WHOLE) {
            const int kt = t0 + (i >> 2) * 8, vt = t0 + g * 8;
            pg.k[0] = lookup(or_safe(t0, min(page_token(kt), kt + 7)));
            pg.v[0] = lookup(or_safe(t0, min(page_token(vt), vt + 7)));
        } else {
            for (int a = 0; a < 2; ++a) pg.k[a] = lookup(or_safe(t0, key_token(t0, a)));
#pragma unroll
            for (int j = 0; j < 8; ++j) pg.v[j] = lookup(or_safe(t0, t0 + g * 8 + j));
        }
        return pg;
    };
    u32x4 k[2][kKs];
    VLoad v[8];
    auto load_keys = [&](int t0, const Pages& pg) {
        const int page = checked(pg.k[0]);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const int t = key_token(t0, a);
            // (A group's page is any of its tokens': whether this one is used does not matter.)
            const uint16_t* src = kbase + offset(WHOLE || a == 0 ? page : checked(pg.k[1]), t0 < 0 ? safe : WHOLE ? t : or_safe(t0, t));
#pragma unroll
            for (int ks = 0; ks < kKs; ++ks) k[a][ks] = *gbl(reinterpret_cast<const u32x4*>(src + ks * 32));
        }
    };
    auto load_values = [&](int t0, const Pages& pg) {
        if constexpr (WHOLE) {
            const uint16_t* src = vbase + offset(checked(pg.v[0]), t0 < 0 ? 0 : t0 + g * 8);
            const int step = t0 < 0 ? 0 : D;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __builtin_nontemporal_load(gbl(reinterpret_cast<const VLoad*>(src + j * step)));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                v[j] = __builtin_nontemporal_load(gbl(reinterpret_cast<const VLoad*>(vbase + offset(checked(pg.v[j]), or_safe(t0, t0 + g * 8 + j)))));
        }
    };

    Softmax<T> sm;
    // Sums of values times weights, and (times kFine) of values times what rounding took
    // from the weights.
    constexpr bool kApart = Type<T>::kFine != 1.0f;
    float4v o[kVw], fine[kApart ? kVw : 1];
#pragma unroll
    for (int m = 0; m < kVw; ++m) o[m] = fine[kApart ? m : 0] = float4v{0, 0, 0, 0};

    // Waves take steps in turn.
    const int lo = q.len - q.n;
    int step = begin + wave;
    if (step < end) {
        auto token_of = [&](int st) { return st < end ? tiles.token(st) : -1; };
        int t0 = tiles.token(step);
        Pages pg = pages_of(t0);
        load_keys(t0, pg);
        load_values(t0, pg);
        pg = pages_of(token_of(step + WAVES));
        for (;;) {
            const int t1 = token_of(step + WAVES);
            const Pages after = pages_of(token_of(step + 2 * WAVES));
            float4v st[2];
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                st[a] = float4v{0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < kKs; ++ks) st[a] = Type<T>::mfma16(__builtin_bit_cast(Vec8, k[a][ks]), qf[ks], st[a]);
            }
            load_keys(t1, pg);
            // Every row sees every token of the step, or some are masked.
            const bool all = t0 + kFewTokens - 1 <= lo && (t0 + kFewTokens - 1 < p.sinks || t0 > last - p.window);
            if (!all) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = t0 + g * 8 + j;
                    if (!sees(p, place, t)) st[j / 4][j % 4] = -INFINITY;
                    const bool any = used(t), every = t <= lo && (t < p.sinks || t > last - p.window);
                    bool clean = true;
#pragma unroll
                    for (int e = 0; e < kVw / 2; ++e) {
                        const uint32_t w = v[j][e], f = finite_part<T>(w);
                        clean = clean && (w == f || every);
                        v[j][e] = every ? w : any ? f : 0u;
                    }
                    if (any && !clean) sh.other[min(atomicAdd(&sh.others, 1), kOthers - 1)] = t;
                }
            }
            float mx = fmaxf(fmaxf(fmaxf(st[0][0], st[0][1]), fmaxf(st[0][2], st[0][3])), fmaxf(fmaxf(st[1][0], st[1][1]), fmaxf(st[1][2], st[1][3])));
            mx = pair_max<true>(pair_max<false>(mx));
            float f;
            if (sm.advance(mx, p.c, f)) {
#pragma unroll
                for (int m = 0; m < kVw; ++m) {
                    o[m] *= f;
                    if constexpr (kApart) fine[m] *= f;
                }
            }
            const float shift = sm.shift(p.c);
            // A weight is two values of the type, its rounding and what that leaves: memory
            // bounds this kernel, so the second product costs little (48 sequences 98.0 ->
            // 98.7 us), and the output's own rounding is then its largest error (fp16, 512
            // tokens: 3.1e-4 -> 2.0e-4 of the output's norm).  What rounding leaves of a weight
            // of 2^15 is at most 2^4 in binary16, and is multiplied by 2^11, so that it too
            // reaches down as far as the type allows (2^-36 in place of 2^-25); sums of their own
            // take 20 to 32 registers (head_dim 64: 16 sequences of up to 20000 tokens 59.8 -> 61.4
            // us, 200 of up to 2004 42.9 -> 43.3; head_dim 128 within 1%).
            Vec8 pf, rest;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = exp2_(fmaf(st[j / 4][j % 4], p.c, shift));
                sm.l += w;
                pf[j] = static_cast<T>(w);
                rest[j] = static_cast<T>((w - static_cast<float>(pf[j])) * Type<T>::kFine);
            }
            // V^T: the 8 tokens x kVw dims that a lane holds, turned 2 x 2 at a time.
            u32x4 vf[kVw];
            ushort2v top = {0, 0};
#pragma unroll
            for (int m = 0; m < kVw; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    vf[m][j] = __builtin_amdgcn_perm(v[2 * j + 1][m / 2], v[2 * j][m / 2], m & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int m = 0; m < kVw; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort2v, vf[m][j] & 0x7FFF7FFFu));
#pragma unroll
            for (int m = 0; m < kVw; ++m) o[m] = Type<T>::mfma16(__builtin_bit_cast(Vec8, vf[m]), pf, o[m]);
            // What is not finite takes part in the first product only: `rest` may be 0 or
            // below.
            if (__builtin_amdgcn_ballot_w64(max(top.x, top.y) >= Type<T>::kExponent)) {
#pragma unroll
                for (int m = 0; m < kVw; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) vf[m][j] = finite_part<T>(vf[m][j]);
            }
#pragma unroll
            for (int m = 0; m < kVw; ++m) {
                float4v& sum = kApart ? fine[m] : o[m];
                sum = Type<T>::mfma16(__builtin_bit_cast(Vec8, vf[m]), rest, sum);
            }
            load_values(t1, pg);
            if (t1 < 0) break;
            pg = after;
            t0 = t1;
            step += WAVES;
        }
    }

    // The waves' states are joined through LDS.  A wave that met a page outside
    // the cache leaves a NaN sum.
    if constexpr (kApart) {
#pragma unroll
        for (int m = 0; m < kVw; ++m) o[m] += fine[m] * (1.0f / Type<T>::kFine);
    }
    float l = pair_sum<true>(pair_sum<false>(sm.l));
    if (__builtin_amdgcn_ballot_w64(bad != 0)) l = NAN;
    if (g == 0) {
        sh.m[wave][i] = sm.m;
        sh.l[wave][i] = l;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int m = 0; m < kVw; m += 4)
            *reinterpret_cast<float4v*>(&sh.acc[wave][i][(g * 4 + r) * kVw + m]) = float4v{o[m][r], o[m + 1][r], o[m + 2][r], o[m + 3][r]};
    __syncthreads();
    for (int x = tid; x < rows * D; x += (WAVES * 64)) {
        const int r = x / D, d = x % D;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sh.m[w][r]);
        const float ms = m == -INFINITY ? 0.0f : m;
        float sum = 0.0f, acc = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = sh.m[w][r] == -INFINITY ? 0.0f : exp2_((sh.m[w][r] - ms) * p.c);
            sum += sh.l[w][r] == 0.0f ? 0.0f : sh.l[w][r] * f;
            acc += sh.m[w][r] == -INFINITY ? 0.0f : sh.acc[w][r][d] * f;
        }
        // What is not finite goes to the rows that see it, whatever its weight.
        for (int x2 = 0; x2 < min(sh.others, kOthers); ++x2) {
            const int t = sh.other[x2];
            if (sees(p, lo + r / p.group, t)) acc += other_part<T>(vbase[offset(checked(lookup(t)), t) - i * kVw + d]);
        }
        if (un.count == 1) {
            out_row(p, q, kvh, r, D)[d] = finish<T>(p, acc, sum);
        } else {
            const int64_t slot = ((int64_t)u * p.hkv + kvh) * p.few_slots + r;
            p.few_acc[slot * D + d] = acc;
            if (d == 0) p.few_ml[slot] = make_float2(m, sum);
        }
    }
}

template <typename T, int D, bool WHOLE, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 4 ? 2 : 1) void few_kernel(const Params p) {
    __shared__ __align__(16) FewShared<D, WAVES> sh;
    few_body<T, D, WHOLE, WAVES>(p, blockIdx.x, sh);
}

// Joins `count` parts of one row; part i at slot base + i step.  256 threads.
template <typename T, int D>
__device__ __forceinline__ void merge_row(const Params& p, const float* acc, const float2* ml, int64_t base, int64_t step, int count, uint16_t* dst) {
    constexpr int kCols = D / 4, kSlots = kThreads / kCols;
    __shared__ float sh_m[kSlots], sh_l[kSlots];
    __shared__ float4v sh_a[kSlots][kCols];
    const int slot = threadIdx.x / kCols, col = threadIdx.x % kCols;
    float m = -INFINITY, l = 0.0f;
    float4v a = {0, 0, 0, 0};
    constexpr int kBatch = 4;
    for (int c0 = slot; c0 < count; c0 += kSlots * kBatch) {
        float2 h[kBatch];
        float4v v[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int64_t at = base + min(c0 + j * kSlots, count - 1) * step;
            h[j] = ml[at];
            v[j] = *reinterpret_cast<const float4v*>(acc + at * D + col * 4);
        }
        float to = m;
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (c0 + j * kSlots < count) to = fmaxf(to, h[j].x);
        const float ms = to == -INFINITY ? 0.0f : to;
        const float f0 = m == -INFINITY ? 0.0f : exp2_((m - ms) * p.c);
        l *= f0;
        a *= f0;
        m = to;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (c0 + j * kSlots >= count) continue;
            if (h[j].y == 0.0f) continue;  // the part saw nothing
            const float f = h[j].x == -INFINITY ? 1.0f : exp2_((h[j].x - ms) * p.c);
            l = fmaf(h[j].y, f, l);
            a += v[j] * f;
        }
    }
    if (col == 0) {
        sh_m[slot] = m;
        sh_l[slot] = l;
    }
    sh_a[slot][col] = a;
    __syncthreads();
    if ((int)threadIdx.x < D) {
        const float* col_a = reinterpret_cast<const float*>(&sh_a[0][0]) + threadIdx.x;
        float top = -INFINITY;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) top = fmaxf(top, sh_m[s]);
        const float ms = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f, total = 0.0f;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) {
            if (sh_l[s] == 0.0f) continue;
            const float f = sh_m[s] == -INFINITY ? 1.0f : exp2_((sh_m[s] - ms) * p.c);
            sum = fmaf(sh_l[s], f, sum);
            total = fmaf(col_a[s * D], f, total);
        }
        dst[threadIdx.x] = finish<T>(p, total, sum);
    }
}

// One workgroup per (sequence, kv head, row).
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void few_merge_kernel(const Params p) {
    const int kvh = blockIdx.x % p.hkv, r = blockIdx.x / p.hkv % p.few_slots, s = blockIdx.x / p.hkv / p.few_slots;
    const int2 units = p.few_units[s * p.hkv + kvh];
    const Seq q = seq_of(p, s);
    if (q.bad || !q.few(p) || r >= q.n * p.group || units.y <= 1) return;
    merge_row<T, D>(p, p.few_acc, p.few_ml, ((int64_t)units.x * p.hkv + kvh) * p.few_slots + r, (int64_t)p.hkv * p.few_slots, units.y,
                    out_row(p, q, kvh, r, D));
}

// ----------------------------------------------------------- many rows

typedef __attribute__((address_space(3))) uint8_t lds_u8;

template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
    if constexpr (N > 0) {
        unrolled<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

template <typename V>
__device__ __forceinline__ V lds_read(uint32_t addr) {
    return *reinterpret_cast<__attribute__((address_space(3))) V*>((lds_u8*)(size_t)addr);
}
template <typename V>
__device__ __forceinline__ void lds_write(uint32_t addr, V v) {
    *reinterpret_cast<__attribute__((address_space(3))) V*>((lds_u8*)(size_t)addr) = v;
}
// Four 16-bit values of a 4 x 16 block of each 16-lane group, turned: lane 4 r +
// c reads values 4 c .. 4 c + 3 of row r, lane i gets value i of rows 0 .. 3.
__device__ __forceinline__ u32x2 lds_read_turned(uint32_t addr) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(lds_u8*)(size_t)addr));
}

// 16 bytes per lane from memory straight into LDS, lane after lane.  Written out
// because the compiler puts a wait for every load in flight before any LDS read
// that follows its own form; the waits are written out too.
__device__ __forceinline__ void dma16(const uint16_t* src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(lds) : "memory");
}
// The same from base + offset + IMM bytes to IMM bytes further on.
template <int IMM>
__device__ __forceinline__ void dma16_at(const uint16_t* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 offset:%3" ::"v"(offset), "s"(base), "s"(lds), "n"(IMM) : "memory");
}
// A barrier behind which every wave's loads are done.
__device__ __forceinline__ void dma_done_and_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Tiles in LDS: a token's D values are 16-byte pieces, piece c at place c ^ s(t).
// The places are chosen by permuting which piece each lane fetches.
//   keys    16 consecutive lanes read the same piece of 16 tokens: s spreads
//           them over all banks;
//   values  32 lanes read 64 bytes of each of 4 tokens: s moves each token's to
//           banks of its own.
template <int D>
__device__ __forceinline__ int key_place(int t) {
    return D == 128 ? t & 15 : t >> 1 & 7;
}
template <int D>
__device__ __forceinline__ int value_place(int t) {
    return D == 128 ? (t & 3) << 2 : (t >> 1 & 1) << 2;
}

struct RowTile {
    int s;
    Seq seq;
    int row0, rows;
};

// Row tile `tile`, the sequences in order; of a sequence the last tiles, which
// see most, come first.
__device__ __forceinline__ bool find_tile(const Params& p, int tile, RowTile& out) {
    const int lane = threadIdx.x & 63;
    int s = -1;
    for (int s0 = 0; s0 < p.num_seqs; s0 += 64) {
        int n = 0;
        if (s0 + lane < p.num_seqs) {
            const Seq q = seq_of(p, s0 + lane);
            // (An invalid one may have more rows than the launch has tiles for: one writes its NaN.)
            n = q.few(p) ? 0 : q.bad ? min(q.n, 1) : (q.n * p.group + kTileRows - 1) / kTileRows;
        }
        const int inc = inclusive_scan(n);
        const uint64_t owner = __builtin_amdgcn_ballot_w64(tile >= inc - n && tile < inc);
        if (owner) {
            const int j = __builtin_ctzll(owner);
            s = s0 + j;
            tile -= __builtin_amdgcn_readlane(inc - n, j);
            break;
        }
        tile -= last_lane(inc);
    }
    if (s < 0) return false;
    out.s = __builtin_amdgcn_readfirstlane(s);
    out.seq = seq_of(p, out.s);
    const int all_rows = out.seq.n * p.group;
    out.row0 = ((all_rows + kTileRows - 1) / kTileRows - 1 - tile) * kTileRows;
    out.rows = min(kTileRows, all_rows - out.row0);
    return true;
}

// A lane's outputs: of its row, dims 32 dt + 8 (r / 4) + 4 h + r % 4.
template <typename T, int D, int DT>
__device__ __forceinline__ void write_rows(const Params& p, uint16_t* dst, const float16v (&o)[DT], float l, int h) {
    const bool blind = p.window == 0 && p.sinks == 0;
    const float inv = 1.0f / l;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            uint16_t e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) e[r] = l != l ? Type<T>::kNaN : blind ? 0 : bits_of<T>(o[dt][r4 * 4 + r] * inv);
            const u32x2 w = {(uint32_t)e[0] | (uint32_t)e[1] << 16, (uint32_t)e[2] | (uint32_t)e[3] << 16};
            *gbl(reinterpret_cast<u32x2*>(dst + dt * 32 + r4 * 8 + h * 4)) = w;
        }
}

// Workgroups: kv heads fastest (each XCD then has its own, whose keys and
// values stay in its L2), then splits, then row tiles.
// WHOLE: pages of 16 tokens or more.
template <int D>
struct TileShared {
    uint8_t tiles[2][2][kTileTokens * D * 2];  // keys, values
    unsigned long long partly[kEdges];
    int edge[kEdges], bad;
};

template <typename T, int D, bool WHOLE>
__device__ __forceinline__ void tile_body(const Params& p, int block, TileShared<D>& sh) {
    using Vec8 = typename Type<T>::Vec8;
    constexpr int kKs = D / 16;                      // key pieces of 16 dims
    constexpr int kDt = D / 32;                      // output tiles of 32 dims
    constexpr int kPieces = D / 8;                   // 16-byte pieces of a token
    constexpr uint32_t kTileBytes = kTileTokens * D * 2;
    constexpr int kLoads = kTileBytes / 16 / kThreads;  // per lane and array
    constexpr int kTokensPerLoad = 64 / kPieces;        // of one wave

    const int tid = threadIdx.x, lane = tid & 63, i = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = block % p.hkv, split = block / p.hkv % p.splits;
    RowTile rt;
    if (!find_tile(p, block / p.hkv / p.splits, rt)) return;
    const Seq& q = rt.seq;
    const int s = rt.s, row0 = rt.row0, rows = rt.rows, all_rows = q.n * p.group;
    if (q.bad) {
        if (split == 0)
            for (int64_t x = tid; x < (int64_t)all_rows * D; x += kThreads) out_row(p, q, kvh, (int)(x / D), D)[x % D] = Type<T>::kNaN;
        return;
    }
    const int lo = q.len - q.n + row0 / p.group, hi = q.len - q.n + (row0 + rows - 1) / p.group;  // positions of the rows
    const Tiles<kTileTokens> tiles(p, lo, hi);
    const int begin = (int)((int64_t)tiles.count * split / p.splits), end = (int)((int64_t)tiles.count * (split + 1) / p.splits);

    const int row = row0 + wave * 32 + i;  // the lane's
    const bool row_ok = row < all_rows;
    // Positions of the wave's rows, of which there may be none.
    const bool idle = row0 + wave * 32 >= all_rows;
    const int wlo = q.len - q.n + min(row0 + wave * 32, all_rows - 1) / p.group, whi = q.len - q.n + min(row0 + wave * 32 + 31, all_rows - 1) / p.group;
    const int clamped = min(row, all_rows - 1);
    const int place = q.len - q.n + clamped / p.group;
    Vec8 qf[kKs];
    {
        const uint16_t* src = p.q + (int64_t)(q.first + clamped / p.group) * p.q_stride + (int64_t)(kvh * p.group + clamped % p.group) * D + h * 8;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
            u32x4 w = *gbl(reinterpret_cast<const u32x4*>(src + ks * 16));
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (w[e] & p.q_and) ^ p.q_xor;
            qf[ks] = __builtin_bit_cast(Vec8, w);
        }
    }

    const int32_t* trow = p.table + (int64_t)s * p.max_pages;
    const int page_mask = (1 << p.log2_page) - 1;
    const uint16_t* kbase = p.k + ((int64_t)kvh << p.log2_page) * D;
    const uint16_t* vbase = p.v + ((int64_t)kvh << p.log2_page) * D;
    const uint32_t lds0 = (uint32_t)(size_t)(lds_u8*)&sh.tiles[0][0][0];
    int bad = 0;

    auto used = [&](int t) { return t <= hi && (t < p.sinks || t >= tiles.first); };
    auto checked = [&](int page) {
        if ((uint32_t)page < (uint32_t)p.num_pages) return page;
        bad = 1;
        return 0;
    };
    // A wave fetches 16 tokens of a tile.  In pages of 16 or more they share one,
    // whose number is a scalar load: a lane's offsets from the first token are then
    // the same in every tile, and the addresses cost no vector instruction.
    const int piece = lane % kPieces, in = lane / kPieces;
    uint32_t key_off[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) key_off[j] = (uint32_t)(in * D + (piece ^ key_place<D>(j * kTokensPerLoad + in)) * 8) * 2;
    const uint32_t value_off = (uint32_t)(in * D + (piece ^ value_place<D>(in)) * 8) * 2;
    // A token that no row sees stands for `safe`, which one does, and is masked.
    // The page of the tile after the one that is fetched is asked for in advance.
    const int safe = p.window > 0 ? hi : 0;
    auto page_of = [&](int step) {
        const int t0 = tiles.token(step) + wave * 16;
        const int t = step < end && t0 <= hi && (t0 < p.sinks || t0 + 15 >= tiles.first) ? t0 : safe;
        return ((const __attribute__((address_space(4))) int32_t*)trow)[__builtin_amdgcn_readfirstlane(t >> p.log2_page)];
    };
    int page_ahead = WHOLE && begin < end ? page_of(begin) : 0;
    auto fetch = [&](int step, int buffer) {
        const int t0 = tiles.token(step) + wave * 16;
        const uint32_t kdst = lds0 + (buffer * 2) * kTileBytes + wave * (kTileBytes / kWaves);
        if constexpr (WHOLE) {
            const int page = __builtin_amdgcn_readfirstlane(checked(page_ahead));
            page_ahead = page_of(step + 1);
            const int64_t off = (int64_t)page * p.page_stride + (int64_t)((t0 & page_mask) * D);
            const uint16_t *ks = kbase + off, *vs = vbase + off;
            unrolled<kLoads>([&](auto j) {
                dma16_at<j * 1024>(ks, key_off[j], kdst);
                dma16_at<j * 1024>(vs, value_off, kdst + kTileBytes);
            });
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int t = t0 + j * kTokensPerLoad + in;
                const int page = checked(trow[(used(t) ? t : safe) >> p.log2_page]);
                const int64_t off = (int64_t)page * p.page_stride + (int64_t)(t & page_mask) * D;
                dma16(kbase + off + (key_off[j] / 2 - in * D), kdst + j * 1024);
                dma16(vbase + off + (value_off / 2 - in * D), kdst + kTileBytes + j * 1024);
            }
        }
    };

    float16v o[kDt];
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
    Softmax<T> sm;
    if (tid < kEdges) sh.partly[tid] = 0;
    if (tid == 0) sh.bad = 0;
    int edges = 0;

    // LDS addresses in buffer 0.  A key piece's place depends on the piece and the
    // token modulo 16, a value's on its 64 bytes and the token modulo 4, so that
    // everything else of an address is an instruction's own offset.
    uint32_t ka[kKs], va[kDt];
#pragma unroll
    for (int ks = 0; ks < kKs; ++ks) ka[ks] = lds0 + i * (D * 2) + ((2 * ks + h) ^ key_place<D>(i)) * 16;
    const int vr = (lane & 15) >> 2, vd = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;  // row of 4 and dim that the lane reads for a turned load
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) {
        const int d = dt * 32 + vd, t = h * 4 + vr;
        va[dt] = lds0 + kTileBytes + t * (D * 2) + ((d / 8) ^ value_place<D>(t)) * 16 + (d & 4) * 2;
    }

    // Values that no row sees are cleared in LDS, and so is what is not finite of
    // tokens that only some rows see: 0 times it would not be 0.  Such tokens are
    // noted; what was not finite is added at the end to the rows that see it.
    auto clean = [&](int t0, uint32_t at) {
        const int edge = min(edges++, kEdges - 1);
        if (tid == 0) sh.edge[edge] = t0;
#pragma unroll 1
        for (int x = tid; x < kTileTokens * kPieces; x += kThreads) {
            const int t = t0 + x / kPieces;
            if (t <= lo && (t < p.sinks || t > hi - p.window)) continue;
            const bool any = used(t);
            const u32x4 w = lds_read<u32x4>(at + x * 16);
            u32x4 f;
            bool same = true;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[e] = any ? finite_part<T>(w[e]) : 0u;
                same = same && f[e] == w[e];
            }
            if (same) continue;
            lds_write(at + x * 16, f);
            if (any) atomicOr(&sh.partly[edge], 1ull << (x / kPieces));
        }
        lds_barrier();
    };
    auto add_others = [&] {
        for (int e = 0; e < min(edges, kEdges); ++e) {
            uint64_t tokens = sh.partly[e];
            while (tokens) {
                const int t = sh.edge[e] + __builtin_ctzll(tokens);
                tokens &= tokens - 1;
                const uint16_t* src = vbase + (int64_t)checked(trow[t >> p.log2_page]) * p.page_stride + (int64_t)(t & page_mask) * D;
                if (!sees(p, place, t)) continue;
#pragma unroll
                for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4) {
                        const u32x2 w = *gbl(reinterpret_cast<const u32x2*>(src + dt * 32 + 8 * r4 + 4 * h));
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[dt][4 * r4 + r] += other_part<T>(w[r / 2] >> (16 * (r & 1)));
                    }
            }
        }
    };

    if (begin < end) fetch(begin, 0);
    for (int step = begin; step < end; ++step) {
        const int buffer = (step - begin) & 1;
        const int t0 = tiles.token(step);
        dma_done_and_barrier();  // the tile is there, and the other buffer no longer read
        if (step + 1 < end) fetch(step + 1, buffer ^ 1);
        const uint32_t at = buffer * 2 * kTileBytes;

        const int tl = t0 + kTileTokens - 1;
        const bool all = tl <= lo && (tl < p.sinks || t0 > hi - p.window);  // every row sees every token
        if (!all) clean(t0, lds0 + kTileBytes + at);

        // A tile that none of the wave's rows sees.
        if (idle || t0 > whi || (t0 >= p.sinks && tl <= wlo - p.window)) continue;
        float16v st[2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[tt][r] = 0.0f;
        // Products that follow each other are of different sums.
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
                st[tt] = Type<T>::mfma32(__builtin_bit_cast(Vec8, lds_read<u32x4>(ka[ks] + at + tt * 32 * (D * 2))), qf[ks], st[tt]);
        // Reads ahead of the products that use them.
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int x = 0; x < 2 * kKs - 6; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
        if (!(tl <= wlo && (tl < p.sinks || t0 > whi - p.window))) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!sees(p, place, t0 + tt * 32 + 8 * (r / 4) + 4 * h + r % 4)) st[tt][r] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[tt][r]);
        mx = pair_max<true>(mx);
        float f;
        if (sm.advance(mx, p.c, f)) {
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) o[dt] *= f;
        }
        const float shift = sm.shift(p.c);
        // Weights are rounded once to the values' type (their sum is of the unrounded ones):
        // against fp32 weights a prompt's error grows from 1.9e-4 to 2.5e-4 of the output's norm
        // in binary16, from 1.6e-3 to 2.0e-3 in bfloat16.  Multiplying what rounding takes, as
        // few_body does, would make the products of this kernel, which they bound, half as many
        // again.
        Vec8 pf[4];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = exp2_(fmaf(st[x / 2][(x & 1) * 8 + j], p.c, shift));
                sm.l += w;
                pf[x][j] = static_cast<T>(w);
            }
        // Product x takes tokens 16 x + {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3}.
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) {
                const u32x2 a = lds_read_turned(va[dt] + at + x * 16 * (D * 2)), b = lds_read_turned(va[dt] + at + (x * 16 + 8) * (D * 2));
                const u32x4 w = {a.x, a.y, b.x, b.y};
                o[dt] = Type<T>::mfma32(__builtin_bit_cast(Vec8, w), pf[x], o[dt]);
            }
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
        for (int x = 0; x < 4 * kDt - 4; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    }

    float l = pair_sum<true>(sm.l);
    // A page outside the cache, met by any wave: the sum of every row is NaN.
    if (bad) sh.bad = 1;
    lds_barrier();
    if (sh.bad) l = NAN;
    add_others();
    if (!row_ok) return;
    if (p.splits == 1) {
        write_rows<T, D>(p, out_row(p, q, kvh, row, D), o, l, h);
    } else {
        const int64_t slot = ((int64_t)(q.first + row / p.group) * p.hq + kvh * p.group + row % p.group) * p.splits + split;
        float* dst = p.tile_acc + slot * D;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *reinterpret_cast<float4v*>(dst + dt * 32 + r4 * 8 + h * 4) =
                    float4v{o[dt][r4 * 4], o[dt][r4 * 4 + 1], o[dt][r4 * 4 + 2], o[dt][r4 * 4 + 3]};
        if (h == 0) p.tile_ml[slot] = make_float2(sm.m, l);
    }
}

template <typename T, int D, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void tile_kernel(const Params p) {
    __shared__ __align__(16) TileShared<D> sh;
    tile_body<T, D, WHOLE>(p, blockIdx.x, sh);
}

// A mixed batch in one launch: row tiles, then units of few rows.  Neither waits
// for the other, and the units, which are bound by memory, run beside the row
// tiles.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, 2) void mixed_kernel(const Params p, int tile_blocks) {
    __shared__ __align__(16) union {
        TileShared<D> tile;
        FewShared<D, kWaves> few;
    } sh;
    if ((int)blockIdx.x < tile_blocks) tile_body<T, D, true>(p, blockIdx.x, sh.tile);
    else few_body<T, D, true, kWaves>(p, blockIdx.x - tile_blocks, sh.few);
}

// One workgroup per (token, query head) of the sequences that tile_kernel took.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void tile_merge_kernel(const Params p) {
    const int head = blockIdx.x % p.hq, token = blockIdx.x / p.hq, lane = threadIdx.x & 63;
    // The sequence: the last one that starts at or before the token.
    int s = -1;
    for (int s0 = 0; s0 < p.num_seqs; s0 += 64) {
        bool mine = false;
        if (s0 + lane < p.num_seqs) {
            const Seq q = seq_of(p, s0 + lane);
            mine = token >= q.first && token < q.first + q.n && !q.few(p) && !q.bad;
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(mine);
        if (m) {
            s = s0 + __builtin_ctzll(m);
            break;
        }
    }
    if (s < 0) return;
    merge_row<T, D>(p, p.tile_acc, p.tile_ml, ((int64_t)token * p.hq + head) * p.splits, 1, p.splits,
                    p.out + (int64_t)token * p.out_stride + (int64_t)head * D);
}

// ------------------------------------------------------------------ host

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kRound = 512;  // workgroups of few_kernel that run at once: two to a CU
// Steps up to which a sequence is not cut, where the sequences are few and where
// they give every CU a workgroup.
constexpr int64_t kWholeFew = 32, kWholeMany = 96;

struct Plan {
    bool few, tiles;
    int64_t units, round, few_slots, row_tiles, splits;
    size_t few_acc, few_ml, few_units, tile_acc, tile_ml, total;  // offsets of the parts of the workspace
};

Plan plan_of(int64_t seqs, int64_t tokens, int64_t max_query, int64_t hq, int64_t hkv, int64_t dim, int64_t max_len, int64_t window, int64_t sinks) {
    Plan pl{};
    const int64_t group = hq / hkv;
    pl.tiles = max_query * group > kFewRows;
    pl.few = !(pl.tiles && seqs == 1 && tokens * group > kFewRows);
    // Tokens that a sequence's few new ones see at most.
    const int64_t few_query = std::min(max_query, std::max<int64_t>(1, kFewRows / group));
    const int64_t steps = ceil_div(std::min(max_len, sinks + window + few_query), kFewTokens) + 2;
    pl.few_slots = std::min<int64_t>(kFewRows, max_query * group);
    pl.units = seqs;
    pl.round = std::max<int64_t>(1, kRound / hkv);
    // Two rounds of workgroups that take a sequence whole are not cut either.  24/8 heads
    // of 128: 128 sequences of 3000 to 4000 tokens take 298 us whole and 319 cut, of 4000
    // each 324 and 322.  Uneven ones lose by it: 256 of 200 to 8000 tokens 444 and 392, and
    // 128 with one of 30000 among 200 to 1000 325 and 82 (127 of them, which are cut: 82).
    if (steps > (seqs * hkv >= kRound / 2 ? kWholeMany : kWholeFew) && seqs * hkv < 2 * kRound) {
        const int64_t want = std::max(2 * pl.round, 2 * seqs);
        pl.units = std::max(std::min(want, seqs * ceil_div(steps, kWaves)), seqs + 1);
        pl.round = std::min(pl.round, pl.units);
    }
    pl.row_tiles = std::min(ceil_div(tokens * group, kTileRows) + seqs, seqs * ceil_div(std::min(max_query, tokens) * group, kTileRows));
    const int64_t groups = ceil_div(tokens * group, kTileRows) * hkv;
    const int64_t seen = ceil_div(std::min(max_len, sinks + window + kTileRows / group + 1), kTileTokens) + 1;
    // Launches that fill three quarters of a round are not split: 1540 new tokens of 16384,
    // 32/8 heads of 128 (392 workgroups), take 462 us in one part and 537 in two.  Below,
    // 1500 (376) take 460 and 475, 1100 (280) 410 and 444: the line could lie lower.
    pl.splits = groups >= 384 ? 1 : std::max<int64_t>(1, std::min<int64_t>({ceil_div(512, groups), seen / 16, 32}));
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += (size_t)ceil_div(bytes, 16) * 16;
        return here;
    };
    const int64_t few_parts = pl.few && pl.units > seqs ? pl.units * hkv * pl.few_slots : 0;
    const int64_t tile_parts = pl.tiles && pl.splits > 1 ? tokens * hq * pl.splits : 0;
    pl.few_acc = take(few_parts * dim * 4);
    pl.few_ml = take(few_parts * 8);
    pl.few_units = take(few_parts ? seqs * hkv * 8 : 0);
    pl.tile_acc = take(tile_parts * dim * 4);
    pl.tile_ml = take(tile_parts * 8);
    pl.total = at;
    return pl;
}

wq_status check_sizes(const char* fn, int64_t seqs, int64_t tokens, int64_t max_query, int64_t hq, int64_t hkv, int64_t dim, int64_t max_len,
                      int64_t window, int64_t sinks) {
    WQ_TRY(in_range(fn, "num_seqs", seqs, 1, WQ_WINDOW_MAX_SEQS));
    WQ_TRY(in_range(fn, "num_tokens", tokens, 1, WQ_WINDOW_MAX_TOKENS));
    WQ_TRY(in_range(fn, "max_query_len", max_query, 1, tokens));
    WQ_TRY(in_range(fn, "num_kv_heads", hkv, 1, WQ_WINDOW_MAX_KV_HEADS));
    if (hq < 1 || hq % hkv != 0)
        return err(WQ_ERR_INVALID_ARG, "%s: num_q_heads (%lld) must be a positive multiple of num_kv_heads (%lld)", fn, (long long)hq, (long long)hkv);
    if (hq / hkv > WQ_WINDOW_MAX_GROUP)
        return err(WQ_ERR_UNSUPPORTED, "%s: at most %d query heads per kv head (got %lld)", fn, WQ_WINDOW_MAX_GROUP, (long long)(hq / hkv));
    if (dim != 64 && dim != 128) return err(WQ_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128 (got %lld)", fn, (long long)dim);
    WQ_TRY(in_range(fn, "max_seq_len", max_len, 1, WQ_WINDOW_MAX_SEQ_LEN));
    WQ_TRY(in_range(fn, "window", window, 0, (int64_t)1 << 30));
    WQ_TRY(in_range(fn, "sinks", sinks, 0, (int64_t)1 << 30));
    const Plan pl = plan_of(seqs, tokens, max_query, hq, hkv, dim, max_len, window, sinks);
    if (pl.units * hkv > INT32_MAX || seqs * pl.few_slots * hkv > INT32_MAX || pl.row_tiles * pl.splits * hkv + pl.units * hkv > INT32_MAX || tokens * hq > INT32_MAX)
        return err(WQ_ERR_INVALID_ARG, "%s: too many workgroups for one launch", fn);
    return WQ_OK;
}

template <typename T, int D>
hipError_t launch(const Params& p, const Plan& pl, hipStream_t stream) {
    const int64_t tile_blocks = pl.tiles ? pl.row_tiles * pl.splits * p.hkv : 0, few_blocks = pl.few ? (int64_t)p.units * p.hkv : 0;
    const dim3 tiles((unsigned)tile_blocks), few((unsigned)few_blocks);
    const bool split = p.units > p.num_seqs;
    if (pl.tiles && pl.few && p.log2_page >= 4) {
        hipLaunchKernelGGL((mixed_kernel<T, D>), dim3((unsigned)(tile_blocks + few_blocks)), dim3(kThreads), 0, stream, p, (int)tile_blocks);
    } else {
        if (pl.tiles && p.log2_page >= 4) hipLaunchKernelGGL((tile_kernel<T, D, true>), tiles, dim3(kThreads), 0, stream, p);
        else if (pl.tiles) hipLaunchKernelGGL((tile_kernel<T, D, false>), tiles, dim3(kThreads), 0, stream, p);
        if (pl.few) {
            const bool whole = p.log2_page >= 3;
            if (whole && split) hipLaunchKernelGGL((few_kernel<T, D, true, 4>), few, dim3(256), 0, stream, p);
            else if (whole) hipLaunchKernelGGL((few_kernel<T, D, true, 8>), few, dim3(512), 0, stream, p);
            else if (split) hipLaunchKernelGGL((few_kernel<T, D, false, 4>), few, dim3(256), 0, stream, p);
            else hipLaunchKernelGGL((few_kernel<T, D, false, 8>), few, dim3(512), 0, stream, p);
        }
    }
    if (pl.tiles && pl.splits > 1) hipLaunchKernelGGL((tile_merge_kernel<T, D>), dim3((unsigned)(p.num_tokens * p.hq)), dim3(kThreads), 0, stream, p);
    if (pl.few && split) hipLaunchKernelGGL((few_merge_kernel<T, D>), dim3((unsigned)(p.num_seqs * p.few_slots * p.hkv)), dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace
}  // namespace window
}  // namespace wq

using namespace wq::window;
using wq::host::aligned;
using wq::host::err;
using wq::host::in_range;
using wq::host::overlaps;
using wq::host::span;
using wq::host::Span;

extern "C" {

wq_status wq_window_attention_workspace_size(int64_t num_seqs, int64_t num_tokens, int64_t max_query_len, int64_t num_q_heads,
                                             int64_t num_kv_heads, int64_t head_dim, int64_t max_seq_len, int64_t window, int64_t sinks,
                                             size_t* bytes) {
    static const char* fn = "wq_window_attention_workspace_size";
    if (!bytes) return err(WQ_ERR_INVALID_ARG, "%s: null output pointer", fn);
    WQ_TRY(check_sizes(fn, num_seqs, num_tokens, max_query_len, num_q_heads, num_kv_heads, head_dim, max_seq_len, window, sinks));
    *bytes = plan_of(num_seqs, num_tokens, max_query_len, num_q_heads, num_kv_heads, head_dim, max_seq_len, window, sinks).total;
    return WQ_OK;
}

wq_status wq_window_attention(const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache, const int32_t* block_table,
                              const int32_t* seq_lens, const int32_t* q_starts, uint16_t* out, int64_t num_seqs, int64_t num_tokens,
                              int64_t max_query_len, int64_t num_q_heads, int64_t num_kv_heads, int64_t head_dim, int64_t q_stride,
                              int64_t out_stride, int64_t page_size, int64_t num_pages, int64_t max_pages_per_seq, int64_t max_seq_len,
                              int64_t window, int64_t sinks, float scale, int64_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
    static const char* fn = "wq_window_attention";
    if (!q || !k_cache || !v_cache || !block_table || !seq_lens || !out) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(check_sizes(fn, num_seqs, num_tokens, max_query_len, num_q_heads, num_kv_heads, head_dim, max_seq_len, window, sinks));
    if (!wq::host::is_pow2(page_size) || page_size > WQ_WINDOW_MAX_PAGE_SIZE)
        return err(WQ_ERR_UNSUPPORTED, "%s: page_size must be a power of two in [1, %d] (got %lld)", fn, WQ_WINDOW_MAX_PAGE_SIZE, (long long)page_size);
    if (dtype != WQ_DTYPE_F16 && dtype != WQ_DTYPE_BF16)
        return err(WQ_ERR_UNSUPPORTED, "%s: dtype must be WQ_DTYPE_F16 or WQ_DTYPE_BF16 (got %lld)", fn, (long long)dtype);
    WQ_TRY(in_range(fn, "num_pages", num_pages, 1, INT32_MAX));
    WQ_TRY(in_range(fn, "max_pages_per_seq", max_pages_per_seq, 1, INT32_MAX));
    if (!q_starts && (num_tokens != num_seqs || max_query_len != 1))
        return err(WQ_ERR_INVALID_ARG, "%s: without q_starts there is one new token per sequence (%lld tokens, %lld sequences, max_query_len %lld)", fn,
                   (long long)num_tokens, (long long)num_seqs, (long long)max_query_len);
    const int64_t row = num_q_heads * head_dim;
    for (const int64_t stride : {q_stride, out_stride})
        if (stride < row || stride % 8 != 0 || stride > ((int64_t)1 << 32))
            return err(WQ_ERR_INVALID_ARG, "%s: strides must be multiples of 8 of at least num_q_heads * head_dim (got %lld)", fn, (long long)stride);
    if (!std::isfinite(scale)) return err(WQ_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16))
        return err(WQ_ERR_MISALIGNED, "%s: q, out, k_cache and v_cache must be 16-byte aligned", fn);
    if (!aligned(block_table, 4) || !aligned(seq_lens, 4) || !aligned(q_starts, 4))
        return err(WQ_ERR_MISALIGNED, "%s: block_table, seq_lens and q_starts must be 4-byte aligned", fn);

    const Plan pl = plan_of(num_seqs, num_tokens, max_query_len, num_q_heads, num_kv_heads, head_dim, max_seq_len, window, sinks);
    if (pl.total > 0) {
        if (!workspace || workspace_bytes < pl.total)
            return err(WQ_ERR_INVALID_ARG, "%s: a workspace of %zu bytes is needed (got %zu)", fn, pl.total, workspace ? workspace_bytes : (size_t)0);
        if (!aligned(workspace, 16)) return err(WQ_ERR_MISALIGNED, "%s: workspace must be 16-byte aligned", fn);
    }
    const uint64_t cache_bytes = (uint64_t)num_pages * num_kv_heads * page_size * head_dim * 2;
    const Span so = span(out, ((uint64_t)(num_tokens - 1) * out_stride + row) * 2), sw = span(workspace, pl.total);
    const Span inputs[] = {span(q, ((uint64_t)(num_tokens - 1) * q_stride + row) * 2), span(k_cache, cache_bytes), span(v_cache, cache_bytes),
                           span(block_table, (uint64_t)num_seqs * max_pages_per_seq * 4), span(seq_lens, (uint64_t)num_seqs * 4),
                           span(q_starts, q_starts ? (uint64_t)(num_seqs + 1) * 4 : 0)};
    for (const Span& in : inputs) {
        if (overlaps(so, in)) return err(WQ_ERR_INVALID_ARG, "%s: out overlaps an input", fn);
        if (overlaps(sw, in)) return err(WQ_ERR_INVALID_ARG, "%s: the workspace overlaps an input", fn);
    }
    if (overlaps(so, sw)) return err(WQ_ERR_INVALID_ARG, "%s: out overlaps the workspace", fn);

    Params p{};
    p.q = q;
    p.k = k_cache;
    p.v = v_cache;
    p.table = block_table;
    p.lens = seq_lens;
    p.starts = q_starts;
    p.out = out;
    p.max_pages = max_pages_per_seq;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.page_stride = num_kv_heads * page_size * head_dim;
    p.num_seqs = (int32_t)num_seqs;
    p.num_tokens = (int32_t)num_tokens;
    p.max_query = (int32_t)max_query_len;
    p.num_pages = (int32_t)num_pages;
    p.hq = (int32_t)num_q_heads;
    p.hkv = (int32_t)num_kv_heads;
    p.group = (int32_t)(num_q_heads / num_kv_heads);
    p.log2_page = wq::host::log2_of(page_size);
    p.max_seq_len = (int32_t)max_seq_len;
    p.window = (int32_t)window;
    p.sinks = (int32_t)sinks;
    p.c = scale == 0.0f ? 1.0f : (float)(std::fabs((double)scale) * 1.4426950408889634);  // log2(e)
    p.q_and = scale == 0.0f ? 0u : ~0u;
    p.q_xor = scale < 0.0f ? 0x80008000u : 0u;
    p.units = (int32_t)pl.units;
    p.round = (int32_t)pl.round;
    p.few_slots = (int32_t)pl.few_slots;
    char* ws = static_cast<char*>(workspace);
    p.few_acc = reinterpret_cast<float*>(ws + pl.few_acc);
    p.few_ml = reinterpret_cast<float2*>(ws + pl.few_ml);
    p.few_units = reinterpret_cast<int2*>(ws + pl.few_units);
    p.splits = (int32_t)pl.splits;
    p.tile_acc = reinterpret_cast<float*>(ws + pl.tile_acc);
    p.tile_ml = reinterpret_cast<float2*>(ws + pl.tile_ml);
    // (With one sequence, whose n may be below num_tokens, only one kernel is launched.)
    p.few_rows = !pl.tiles ? INT32_MAX : pl.few ? kFewRows : 0;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    hipError_t e;
    if (dtype == WQ_DTYPE_F16) e = head_dim == 128 ? launch<_Float16, 128>(p, pl, st) : launch<_Float16, 64>(p, pl, st);
    else e = head_dim == 128 ? launch<__bf16, 128>(p, pl, st) : launch<__bf16, 64>(p, pl, st);
    return wq::host::hip_result(fn, e);
}

}  // extern "C"
