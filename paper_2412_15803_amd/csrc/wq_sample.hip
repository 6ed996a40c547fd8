// The choice of the next word by chance (gfx950, wave64): temperature, top-k,
// top-p, min-p and a given random number.
//
// The words that stay are a beginning of the order (logit falling, word rising), so
// they are told by the last of them, the cut.
//   survey   a workgroup to a chunk of a row, which it reads into registers: the largest
//            logit, and what the row's settings ask for: the sum of the weights, or a
//            histogram over the distance from a reference near the row's largest logit
//            (of counts for top-k, of weights for top-p; bins as fine as 1/64 of the
//            distance).
//   plan     adds up a row's histograms, which tell the bin that the cut lies in.
//            Without top-k, top-p and min-p it chooses the word.
//   list     a workgroup to a chunk, read again from the caches: lists the words that may
//            be the cut; those that surely stay are listed too while they are few, or
//            else their weights summed.
//   finish   finds the cut in a row's list, the chunk that the random number falls into,
//            and in it the word.
// Few rows take two launches, as launches and waiting bound them: the second has the
// chunks' workgroups each make the plan for themselves, and the row's last one to be
// done with its list finish it (1 x 128256, top-k and top-p: 19 us; with a launch for plan 2.4 more).  In
// many rows plans by every chunk would read the histograms over and over, and finish,
// in the last of small workgroups with room for a whole list, kept others from their
// CUs: each has a launch (256 x 100277 fp32: 105 us; list and finish in one 10 more).
// Rows whose list would be too long (thousands of equal logits) are worked out by one
// workgroup, which then looks through the row instead of the list.
//
// A lane takes its words of a chunk at once and without branches: what bounds few rows is how
// long one workgroup takes (loads, then the chain of fp64 operations of a weight).  Many rows:
// survey, half of the time, is the loads, weights (16 us of 55) and LDS atomics (9) in turn;
// more or fewer waves to a workgroup or to a SIMD were no faster.
//
// Weights are formed in fp64 and held as whole multiples of 2^-s: their sums do
// not depend on the order in which they are added, so atomics may add them.
// A 32-bit weight would move the border between two words by up to 2^-24 of the
// total, which random numbers of 24 bits hit.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "wq_device.h"
#include "wq_host.h"
#include "wq_internal.h"
#include "wq_sample.h"

namespace wq {
namespace sample {
namespace {

using dev::gbl;
using dev::u32x4;
using namespace host;

constexpr int kChunk = 8192;    // words of a chunk
constexpr int kAbove = 512, kBelow = 1024, kBins = kAbove + kBelow;  // of a histogram, above and below its reference
constexpr int kList = 4096;     // words that are listed
constexpr int kStaged = 512;    // of a chunk's that are listed together
constexpr int kRanked = 256;    // words of a list that are put in order by comparing all with all
constexpr int kCompared = 64;   // numbers that are searched so, where their weights are read too (237: 15 us; by parts 4)
constexpr int kPartBits = 9, kParts = 1 << kPartBits;  // of a list's range
constexpr int kAhead = 16;      // histograms that are read at once

template <typename T>
constexpr int kPer = 16 / sizeof(T);  // words of a 16-byte load
template <typename T>
constexpr int kVectors = kChunk / kPer<T>;  // of a chunk

// What survey leaves of a chunk: its best word, the sum of its weights, and the bins
// [low, high) that are not empty.
struct Record {
    uint64_t sum;
    double offset;  // of its weights
    uint32_t key;
    int32_t word;
    int32_t low, high;
    float reference;  // of the row's bins
    int32_t unused;
};
// What is done with a row.
enum Way { kDone, kMinP, kCount, kWeight };
// What plan tells the others, and what a row's workgroups share.
struct Plan {
    double offset;              // of the weights
    uint64_t ahead, need;       // words, or weights, before the cut's bin, and of it up to the cut
    uint32_t best;              // key of the largest logit
    int32_t word;               // and its word
    float reference;
    int32_t way, cut_bin, few, alone;
    uint32_t done, listed;      // workgroups that are done, and words listed
    int32_t unused;
};

struct Params {
    wq_sample_call c;
    int32_t weight_bits;  // s
    int32_t has;          // which lists are given: 1 temperature, 2 top_p, 4 min_p, 8 top_k
    int32_t chunks;       // of a row
    int32_t list_size;    // words that a row's list holds
    Record* records;      // [rows][chunks]
    uint64_t* bins;       // [rows][chunks][kBins]
    uint64_t* sums;       // [rows][chunks] weights that surely stay
    uint64_t* list;       // [rows][list_size]
    Plan* plans;          // [rows]
};

// One row's logits: vector v holds the words v * kPer - lead .. + kPer - 1, so that whole vectors
// are aligned whatever word the row starts at.
template <typename T>
struct Row {
    typedef T vec __attribute__((ext_vector_type(kPer<T>)));
    const T* x;
    int vocab, lead, vectors;
    int inside, outside;  // vectors [inside, outside) lie in the row whole
    __device__ __forceinline__ Row(const Params& p, int64_t row) {
        x = static_cast<const T*>(p.c.logits) + row * p.c.logits_stride;
        vocab = (int)p.c.vocab;
        lead = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) % kPer<T>);
        vectors = (vocab + lead + kPer<T> - 1) / kPer<T>;
        inside = lead ? 1 : 0;
        outside = (vocab + lead) / kPer<T>;
    }
    __device__ __forceinline__ int chunk_of(int word) const { return (word + lead) / kChunk; }
    // The bits of vector v, or of one that lies in the row whole, if there is one, where v does not.  (No branch on v,
    // so that loads of several vectors do not wait for each other.)
    __device__ __forceinline__ u32x4 fetch(int v) const {
        if (outside <= inside) return u32x4{0, 0, 0, 0};
        return *gbl(reinterpret_cast<const u32x4*>(x + (min(max(v, inside), outside - 1) * kPer<T> - lead)));
    }
    // The words of vector v as fp32; NaN and what lies outside the row as -infinity.
    __device__ __forceinline__ void words(int v, u32x4 bits, float (&out)[kPer<T>]) const {
        const vec w = __builtin_bit_cast(vec, bits);
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i) out[i] = (float)w[i];
        if (v < inside || v >= outside) {
            const int first = v * kPer<T> - lead;
#pragma unroll
            for (int i = 0; i < kPer<T>; ++i) out[i] = first + i >= 0 && first + i < vocab ? (float)gbl(x)[first + i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i) out[i] = out[i] != out[i] ? -INFINITY : out[i] + 0.0f;  // -0 is 0
    }
    // f(logit, word) for the words of the vectors [from, end); words that take no part have -infinity.
    template <typename F>
    __device__ __forceinline__ void each(int from, int end, F f) const {
#pragma unroll 1
        for (int v = from + threadIdx.x; v < end; v += blockDim.x) {
            float y[kPer<T>];
            words(v, fetch(v), y);
#pragma unroll
            for (int i = 0; i < kPer<T>; ++i) f(y[i], v * kPer<T> - lead + i);
        }
    }
};
// Larger for larger logits.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __builtin_bit_cast(float, key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
constexpr uint32_t kNothing = 0x007FFFFFu;  // of -infinity
constexpr uint32_t kInfinity = 0xFF800000u;  // of +infinity

// 2^t for t <= 0, relative error below 2^-50: a polynomial in the fraction, |f| <= 1/2, the Chebyshev series of 2^f
// cut behind its eleventh term and written in powers of f (2^-51.5 from 2^f, and the roundings).
__device__ __forceinline__ double exp2_of(double t) {
    const double n = __builtin_rint(t), f = t - n;
    double r = 0x1.e6228bff026d1p-28;
    r = fma(r, f, 0x1.b675be272450dp-24);
    r = fma(r, f, 0x1.62bfc2c7ae40ep-20);
    r = fma(r, f, 0x1.ffcb54047bef3p-17);
    r = fma(r, f, 0x1.430913112cb56p-13);
    r = fma(r, f, 0x1.5d87fe9d7afb3p-10);
    r = fma(r, f, 0x1.3b2ab6fb9f1a3p-7);
    r = fma(r, f, 0x1.c6b08d703ce43p-5);
    r = fma(r, f, 0x1.ebfbdff82c5aep-3);
    r = fma(r, f, 0x1.62e42fefa3a19p-1);
    r = fma(r, f, 1.0);
    return __builtin_ldexp(r, (int)n);
}

// How a row's logits become weights: w = 2^(x log2(e) / temperature - offset), offset the whole number that
// brings the largest logit's to (1/2, 1].  So those of a chunk's largest logit and those of the row's differ by
// a whole power of two.  Formed as 2^((x - top) log2(e) / temperature + rest), top the largest logit, whose own
// weight takes `rest`: however large logits or small temperatures are, the difference keeps its digits.
struct Weights {
    double top, factor, rest;
    double low;      // smallest log2 w that min-p leaves
    double steps;    // 2^s
    bool infinite;   // the largest logit is +infinity: those that are weigh 1
    // log2 w; not below -2000, which weighs nothing, as -infinity does.  (So does what is no number: zero times infinity.)
    __device__ __forceinline__ double log2_of(float x) const {
        const double t = fmax(fma((double)x - top, factor, rest), -2000.0);
        return x == INFINITY ? 0.0 : t;
    }
    // A whole number of steps, rounded to nearest.  (Below 2^52, adding 2^52 leaves the number in the low bits.)
    __device__ __forceinline__ uint64_t of(double log2w) const {
        const double w = fma(exp2_of(log2w), steps, 4503599627370496.0);
        return __builtin_bit_cast(uint64_t, w) & 0xFFFFFFFFFFFFFull;
    }
};

// Words of the order up to and with this one.
struct Cut {
    uint32_t key;
    int word;
    __device__ __forceinline__ bool keeps(uint32_t k, int w) const { return k > key || (k == key && w <= word); }
};

// The whole part of share * total, 0 <= share < 1, and whether that leaves something.  Exactly: of equal words, the number
// that reaches top_p of their sum, or that a random number is passed by, does not depend on a rounding.
__device__ __forceinline__ uint64_t part_of(float share, uint64_t total, bool& more) {
    // (The same in all lanes, and so worked out once.)
    const uint32_t bits = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, share)), e = bits >> 23;
    const uint64_t m = (bits & 0x7FFFFF) | (e ? 0x800000 : 0);
    const int down = 150 - (int)max(e, 1u);  // share = m 2^-down, down >= 24; total < 2^63
    const uint64_t lo = m * total, hi = __umul64hi(m, total);
    if (down < 64) {
        more = (lo << (64 - down)) != 0;
        return hi << (64 - down) | lo >> down;
    }
    const uint64_t below = down - 64 < 24 ? ((uint64_t)1 << (down - 64)) - 1 : ~0ull;  // hi has 23 bits
    more = lo != 0 || (hi & below) != 0;
    return hi > below ? hi >> (down - 64) : 0;
}
// The least whole number of steps that reaches a share below 1 of the total, at least one.
__device__ __forceinline__ uint64_t share_of(float share, uint64_t total) {
    bool more;
    const uint64_t whole = part_of(share, total, more);
    return max(whole + (more ? 1 : 0), (uint64_t)1);
}

// A row's settings, those that change nothing left out.
struct Settings {
    double temperature;
    int top_k;      // 0: all
    float random;   // 1: the last word
    float top_p;    // 1: all
    float min_p;    // 0: all
    bool greedy;
    __device__ __forceinline__ Settings(const Params& p, int64_t r) {
        // (Lists that are not given point at the random numbers, so that no load waits behind a branch.)
        const wq_sample_call& c = p.c;
        const float u = gbl(c.random)[r], given_t = gbl(c.temperature)[r], given_p = gbl(c.top_p)[r], given_m = gbl(c.min_p)[r];
        const int given_k = gbl(c.top_k)[r];
        const float t = p.has & 1 ? given_t : 1.0f, tp = p.has & 2 ? given_p : 1.0f, mp = p.has & 4 ? given_m : 0.0f;
        const int k = p.has & 8 ? given_k : 0;
        temperature = t;
        greedy = !(t > 0.0f);
        top_k = k > 0 && k < c.vocab ? k : 0;
        top_p = tp < 1.0f ? fmaxf(tp, 0.0f) : 1.0f;
        min_p = mp > 0.0f ? fminf(mp, 1.0f) : 0.0f;
        random = u > 0.0f ? fminf(u, 1.0f) : 0.0f;
    }
    // The smallest offset with which no logit up to `top` weighs more than 1.
    __device__ __forceinline__ double offset_of(float top) const { return ceil((double)top * (1.44269504088896340736 / temperature)); }
    __device__ __forceinline__ Weights weights(const Params& p, float top, double offset) const {
        Weights w;
        w.infinite = top == INFINITY;
        w.top = top;
        w.factor = 1.44269504088896340736 / temperature;
        // (Past 2^52 the product has no fraction left, but then any other logit's weight is 0.)
        w.rest = fmin(fmax(fma(w.top, w.factor, -offset), -1.0), 0.0);
        w.steps = __builtin_ldexp(1.0, p.weight_bits);
        w.low = min_p > 0.0f ? w.log2_of(top) + log2((double)min_p) : -4000.0;
        return w;
    }
    __device__ __forceinline__ uint64_t goal(uint64_t total) const {
        bool more;
        return random < 1.0f ? part_of(random, total, more) : total - 1;
    }
};

// Bin of a logit by its distance from the reference, the largest logits in the lowest bins: 32 bins to an
// octave above it and 64 below, from 2^-5 to 2^11.  Larger logits are never in higher bins: the difference
// and its rounding keep their order.
__device__ __forceinline__ int bin_of(float x, float reference) {
    const float d = reference - x;
    const int bits = (int)(__builtin_bit_cast(uint32_t, d) & 0x7FFFFFFFu);
    if (d < 0.0f) return kAbove - 1 - min(max((bits >> 18) - ((127 - 5) << 5), 0), kAbove - 1);
    return kAbove + min(max((bits >> 17) - ((127 - 5) << 6), 0), kBelow - 1);
}
__device__ __forceinline__ Way way_of(const Settings& set) { return set.top_k ? kCount : set.top_p < 1.0f ? kWeight : set.min_p > 0.0f ? kMinP : kDone; }

// A listed word as a number, the smaller the earlier in the order of words; with its halves exchanged, the
// smaller the lower the word.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int word) { return (uint64_t)~key << 32 | (uint32_t)word; }
__device__ __forceinline__ uint64_t turned(uint64_t e) { return e << 32 | e >> 32; }
__device__ __forceinline__ float value_of_entry(uint64_t e) { return value_of(~(uint32_t)(e >> 32)); }

// Values that workgroups of one launch pass on: atomic accesses at the device's scope go past the XCDs'
// caches, so that no cache has to be written back or emptied for them (a release by every workgroup, which
// writes back the L2, made the launch take 80 us longer for 256 rows).
__device__ __forceinline__ void share_out(uint64_t* to, uint64_t v) { __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t share_in(const uint64_t* from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// What a listed word weighs in a search.
struct Weigh {
    Weights weights;
    uint64_t last;           // words after this one weigh nothing
    bool ones, by_word;      // each weighs 1; numbers are turned
    bool min_p;              // words that min-p leaves out weigh nothing
    __device__ __forceinline__ uint64_t operator()(uint64_t number) const {
        if (ones) return 1;
        const uint64_t e = by_word ? turned(number) : number;
        const double t = weights.log2_of(value_of_entry(e));
        const uint64_t w = weights.of(t);
        return e > last || (min_p && t < weights.low) ? 0 : w;
    }
};

template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) {  // 0 where no lane is read
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
    return (uint64_t)hi << 32 | lo;
}
// Over the lanes up to this one: their sum, or the largest of them.
template <typename F>
__device__ __forceinline__ uint64_t scan16(uint64_t v, F f) {  // of 16 lanes
    v = f(v, dpp64<0x111, 0xF>(v));  // row_shr:1
    v = f(v, dpp64<0x112, 0xF>(v));
    v = f(v, dpp64<0x114, 0xF>(v));
    return f(v, dpp64<0x118, 0xF>(v));
}
// The largest of each 4 or 16 lanes, in all of them.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_most(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true));
}
template <int LANES>
__device__ __forceinline__ uint32_t most_of_lanes(uint32_t v) {
    v = dpp_most<0x4E>(dpp_most<0xB1>(v));  // quad_perm [1,0,3,2], [2,3,0,1]
    if constexpr (LANES == 16) v = dpp_most<0x140>(dpp_most<0x141>(v));  // row_half_mirror, row_mirror
    return v;
}
template <typename F>
__device__ __forceinline__ uint64_t scan64(uint64_t v, F f) {
    v = scan16(v, f);
    v = f(v, dpp64<0x142, 0xA>(v));  // row_bcast:15 into rows 1, 3
    return f(v, dpp64<0x143, 0xC>(v));  // row_bcast:31 into rows 2, 3
}
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
struct Sum {
    __device__ __forceinline__ uint64_t operator()(uint64_t a, uint64_t b) const { return a + b; }
};
struct Most {
    __device__ __forceinline__ uint64_t operator()(uint64_t a, uint64_t b) const { return a > b ? a : b; }
};
__device__ __forceinline__ void add(uint64_t* at, uint64_t v) { atomicAdd(reinterpret_cast<unsigned long long*>(at), (unsigned long long)v); }

// What workgroups of kThreads lanes do.
template <int kThreads>
struct Block {
    static constexpr int kWaves = kThreads / 64;
    template <typename T>
    static constexpr int kEach = kVectors<T> / kThreads;  // vectors of a lane

    struct Small {  // what a block's lanes exchange
        uint64_t parts[2][kWaves];
        uint64_t before, found;
        uint32_t digit, base, count;
        int low, high;
        int turn[kWaves];  // of parts; each wave has its own
    };
    static __device__ __forceinline__ void begin(Small& s) {
        if (threadIdx.x % 64 == 0) s.turn[threadIdx.x / 64] = 0;
    }

    // A chunk's words of a lane.
    template <typename T>
    struct Chunk {
        u32x4 bits[kEach<T>];
        float x[kEach<T>][kPer<T>];
        int first;
        __device__ __forceinline__ Chunk(const Row<T>& row, int chunk) {
            first = chunk * kVectors<T> + threadIdx.x;
#pragma unroll
            for (int i = 0; i < kEach<T>; ++i) bits[i] = row.fetch(first + i * kThreads);
        }
        __device__ __forceinline__ void take(const Row<T>& row) {
#pragma unroll
            for (int i = 0; i < kEach<T>; ++i) row.words(first + i * kThreads, bits[i], x[i]);
        }
        template <typename F>
        __device__ __forceinline__ void each(const Row<T>& row, F f) const {
#pragma unroll
            for (int i = 0; i < kEach<T>; ++i)
#pragma unroll
                for (int j = 0; j < kPer<T>; ++j) f(x[i][j], (first + i * kThreads) * kPer<T> - row.lead + j);
        }
    };

    // Over the block: in the lanes before this one, and in all.  (Two places in turn, so that one barrier does.)
    template <typename F>
    static __device__ __forceinline__ uint64_t block_scan(Small& s, uint64_t v, uint64_t& all, F f) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
        uint64_t* const parts = s.parts[s.turn[wave]];
        const uint64_t up = scan64(v, f);
        if (lane == 63) parts[wave] = up, s.turn[wave] ^= 1;
        __syncthreads();
        const uint64_t waves = scan16(lane < kWaves ? parts[lane] : 0, f);
        all = lane_of(waves, kWaves - 1);
        const uint64_t before = wave ? lane_of(waves, wave - 1) : 0;
        const uint64_t mine = dpp64<0x138, 0xF>(up);  // wave_shr:1
        return f(before, mine);
    }
    // Sum of v in the lanes before this one; `total` that of all.
    static __device__ __forceinline__ uint64_t block_before(Small& s, uint64_t v, uint64_t& total) { return block_scan(s, v, total, Sum()); }
    static __device__ __forceinline__ uint64_t block_sum(Small& s, uint64_t v) {
        uint64_t total;
        block_scan(s, v, total, Sum());
        return total;
    }
    static __device__ __forceinline__ uint64_t block_most(Small& s, uint64_t v) {
        uint64_t most;
        block_scan(s, v, most, Most());
        return most;
    }
    // The best word of the block's words, the same in all lanes: the largest key, of equal ones the lowest word.
    static __device__ __forceinline__ void block_best(Small& s, uint32_t& key, int& word) {
        const uint64_t best = block_most(s, (uint64_t)key << 32 | ~(uint32_t)word);
        key = (uint32_t)(best >> 32), word = (int)~(uint32_t)best;
    }

    // The reference: the largest logit of the row's first vectors, the same for all of its chunks; 0 where that is no
    // logit that words worth choosing have (the lowest value of a type stands for a mask), as all of those would lie in
    // one bin.
    template <typename T>
    static __device__ __forceinline__ float reference_of(Small& s, const Row<T>& row, u32x4 bits) {
        uint32_t key = kNothing;
        int word = 0;
        float y[kPer<T>];
        row.words(threadIdx.x, bits, y);
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i) key = max(key, key_of(y[i]));
        block_best(s, key, word);
        const float most = value_of(key);
        return fabsf(most) < 1024.0f ? most : 0.0f;
    }

    // Workgroups of a row are `rows` apart, so that a row's run at the same time.
    template <typename T>
    static __device__ __forceinline__ void survey(const Params& p) {
        __shared__ struct : Small {
            uint64_t bins[kBins];
        } s;
        const int64_t r = blockIdx.x;
        const int chunk = blockIdx.y;
        const Row<T> row(p, r);
        begin(s);
        Chunk<T> x(row, chunk);
        const u32x4 ahead = row.fetch(threadIdx.x);
        const Settings set(p, r);
        const Way way = way_of(set);
        const bool binned = !set.greedy && (way == kCount || way == kWeight);
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.bins[i] = 0;
        if (threadIdx.x == 0) s.low = kBins, s.high = 0;
        x.take(row);
        uint32_t best = kNothing;
        int word = INT32_MAX;
        x.each(row, [&](float v, int w) {
            const uint32_t key = key_of(v);
            word = key > best ? w : word;  // (A lane's words rise.)
            best = max(best, key);
        });
        const uint32_t own = best;
        block_best(s, best, word);
        Record record{0, 0.0, best, word, 0, 0, reference_of(s, row, ahead), 0};
        const int64_t at = r * p.chunks + chunk;
        if (!set.greedy && best != kNothing && way != kMinP) {
            const bool infinite = best == kInfinity;
            record.offset = infinite ? 0.0 : set.offset_of(value_of(best));
            const Weights weights = set.weights(p, value_of(best), record.offset);
            uint64_t sum = 0;
            if (way == kCount) {
                // Where top_k groups of lanes have a word each that is no smaller than this, smaller ones are not among the
                // row's first top_k, and not counted.
                uint32_t least = own;
                if (set.top_k <= kThreads / 4) least = most_of_lanes<4>(least);
                if (set.top_k <= kThreads / 16) least = most_of_lanes<16>(least);
                least = set.top_k <= kThreads ? ~(uint32_t)block_most(s, (uint32_t)~least) : 0;
                x.each(row, [&](float v, int) {
                    if (v > -INFINITY && key_of(v) >= least) add(&s.bins[bin_of(v, record.reference)], 1);
                });
            } else {
                // A vector's weights first, so that their chains of operations run side by side.
#pragma unroll
                for (int i = 0; i < kEach<T>; ++i) {
                    uint64_t w[kPer<T>];
#pragma unroll
                    for (int j = 0; j < kPer<T>; ++j) w[j] = weights.of(weights.log2_of(x.x[i][j]));
#pragma unroll
                    for (int j = 0; j < kPer<T>; ++j) {
                        sum += w[j];
                        if (binned && w[j]) add(&s.bins[bin_of(x.x[i][j], record.reference)], w[j]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (binned) {
                __syncthreads();
                int low = kBins, high = 0;
                for (int i = threadIdx.x; i < kBins; i += kThreads)
                    if (s.bins[i]) low = min(low, i), high = max(high, i + 1);
                if (high) atomicMin(&s.low, low), atomicMax(&s.high, high);
                __syncthreads();
                record.low = s.low, record.high = s.high;
                for (int i = s.low + threadIdx.x; i < s.high; i += kThreads) gbl(p.bins)[at * kBins + i] = s.bins[i];
            } else {
                record.sum = block_sum(s, sum);
            }
        }
        if (threadIdx.x == 0) {
            p.records[at] = record;
            if (chunk == 0) p.plans[r].done = p.plans[r].listed = 0;
        }
    }

    // The word of a chunk at which the sum of weights passes `goal`.  Where it does not quite (the chunk's weight was
    // summed from other roundings than these), it is the chunk's best word, which stays if any of the chunk does.
    template <typename T, typename F>
    static __device__ __forceinline__ void choose_in_chunk(Small& s, const Params& p, int64_t r, const Row<T>& row, int chunk, uint64_t goal, double total, F weight) {
        // Words in their order are vector by vector, and the lanes of a round are consecutive ones.
        const Chunk<T> x(row, chunk);
#pragma unroll
        for (int i = 0; i < kEach<T>; ++i) {
            const int v = x.first + i * kThreads;
            float y[kPer<T>];
            row.words(v, x.bits[i], y);
            uint64_t w[kPer<T>], sum = 0, all;
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j) {
                w[j] = weight(y[j], v * kPer<T> + j - row.lead);
                sum += w[j];
            }
            uint64_t up = block_before(s, sum, all);
            if (goal < all) {
#pragma unroll
                for (int j = 0; j < kPer<T>; ++j) {
                    if (up <= goal && goal < up + w[j]) {
                        gbl(p.c.token)[r] = v * kPer<T> + j - row.lead;
                        if (p.c.share) gbl(p.c.share)[r] = (float)((double)w[j] / total);
                    }
                    up += w[j];
                }
                return;
            }
            goal -= all;
        }
        if (threadIdx.x == 0) {
            const Record& record = p.records[r * p.chunks + chunk];
            gbl(p.c.token)[r] = record.word;
            if (p.c.share) gbl(p.c.share)[r] = (float)((double)weight(value_of(record.key), record.word) / total);
        }
    }

    struct Survey : Small {  // what plan looks up of the chunks: their bins' first, end and shift
        uint32_t ranges[WQ_SAMPLE_MAX_VOCAB / kChunk + 1 + kAhead];
    };

    // What is to be done with a row, by a workgroup whose lanes are at least as many as the chunks.  Rows that need no
    // cut are answered here, where `answers`.
    template <typename T>
    static __device__ __forceinline__ Plan plan(Survey& s, const Params& p, int64_t r, const Row<T>& row, const Settings& set, bool answers) {
        // What survey left: thread i has chunk i's.
        const bool has = (int)threadIdx.x < p.chunks;
        Record record{0, 0.0, kNothing, INT32_MAX, 0, 0, 0.0f, 0};
        if (has) record = p.records[r * p.chunks + threadIdx.x];
        uint32_t best = record.key;
        int word = record.word;
        block_best(s, best, word);
        const float reference = p.records[r * p.chunks].reference;
        Plan plan{};
        plan.best = best, plan.word = word, plan.cut_bin = kBins, plan.reference = reference;
        plan.way = best == kNothing || set.greedy ? kDone : way_of(set);
        if (plan.way == kDone && !answers) return plan;
        if (best == kNothing || set.greedy) {
            if (threadIdx.x == 0) {
                gbl(p.c.token)[r] = best == kNothing ? -1 : word;
                if (p.c.share) gbl(p.c.share)[r] = best == kNothing ? 0.0f : 1.0f;
            }
        } else {
            // A chunk's offset differs from the row's by a whole number: by as many bits its weights are too large.  (Where the
            // largest logit is +infinity, only the chunks that have it weigh anything.)
            const bool infinite = best == kInfinity;
            plan.offset = infinite ? 0.0 : set.offset_of(value_of(best));
            const int over = record.key == kNothing || (infinite && record.key != kInfinity) ? 63 : (int)fmin(plan.offset - record.offset, 63.0);
            if (plan.way == kDone) {
                const uint64_t mine = record.sum >> over;
                uint64_t total;
                const uint64_t up = block_before(s, mine, total), goal = set.goal(total);
                if (up <= goal && goal < up + mine) s.digit = threadIdx.x, s.before = (goal - up) << over, s.base = record.key, s.ranges[0] = (uint32_t)over, s.found = __builtin_bit_cast(uint64_t, record.offset);
                __syncthreads();
                const Weights own = set.weights(p, value_of(s.base), __builtin_bit_cast(double, s.found));
                choose_in_chunk(s, p, r, row, (int)s.digit, s.before, __builtin_ldexp((double)total, (int)s.ranges[0]), [&](float v, int) { return own.of(own.log2_of(v)); });
            } else if (plan.way != kMinP) {
                // The bin that the cut lies in, and what lies before it.
                if ((int)threadIdx.x < p.chunks + kAhead)
                    s.ranges[threadIdx.x] = has ? (uint32_t)record.low | (uint32_t)record.high << 11 | (plan.way == kCount ? 0u : (uint32_t)over) << 22 : 0;
                __syncthreads();
                constexpr int kMine = 2;
                static_assert(kThreads * kMine >= kBins, "(Of the last lanes none.)");
                typedef uint64_t u64x2 __attribute__((ext_vector_type(kMine)));
                uint64_t v[kMine] = {}, sum = 0, total;
                const int first = threadIdx.x * kMine, wave_first = __builtin_amdgcn_readfirstlane(first);
#pragma unroll 1
                for (int c = 0; c < p.chunks; c += kAhead) {
                    // (One look into LDS for each wave; its broadcasts for every chunk took longer than the bins.)
                    const uint32_t ranges = s.ranges[c + threadIdx.x % kAhead];
                    u64x2 b[kAhead];
#pragma unroll
                    for (int a = 0; a < kAhead; ++a) {
                        // (Most waves have no bin of a chunk that was written, and need no load: those bounded this.)
                        const uint32_t range = (uint32_t)__builtin_amdgcn_readlane((int)ranges, a);
                        const int low = range & 0x7FF, high = range >> 11 & 0x7FF;
                        const uint64_t* const bins = p.bins + (r * p.chunks + c + a) * kBins + min(first, kBins - kMine);
                        b[a] = u64x2{0, 0};
                        if (wave_first + 64 * kMine > low && wave_first < high) b[a] = *gbl(reinterpret_cast<const u64x2*>(bins));
                    }
#pragma unroll
                    for (int a = 0; a < kAhead; ++a) {
                        const uint32_t range = (uint32_t)__builtin_amdgcn_readlane((int)ranges, a);
                        const int low = range & 0x7FF, high = range >> 11 & 0x7FF, by = (int)(range >> 22);
#pragma unroll
                        for (int i = 0; i < kMine; ++i) v[i] += first + i >= low && first + i < high ? b[a][i] >> by : 0;  // (What lies outside was not written.)
                    }
                }
#pragma unroll
                for (int i = 0; i < kMine; ++i) sum += v[i];
                uint64_t up = block_before(s, sum, total);
                const uint64_t target = plan.way == kCount ? std::min<uint64_t>(set.top_k, total) : share_of(set.top_p, total);
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    if (up < target && up + v[i] >= target) s.digit = first + i, s.before = up, s.found = v[i];
                    up += v[i];
                }
                __syncthreads();
                plan.cut_bin = (int)s.digit, plan.ahead = s.before, plan.need = target - s.before;
                // While all words that may stay are few, all are listed.  A long list, and top-p behind a long
                // top-k, are worked out by one workgroup.
                if (plan.way == kCount) {
                    plan.few = s.before + s.found <= (uint64_t)p.list_size;
                    plan.alone = !plan.few && (set.top_p < 1.0f || s.found > (uint64_t)p.list_size);
                }
            }
        }
        return plan;
    }

    template <typename T>
    static __device__ __forceinline__ void plan_rows(const Params& p) {
        __shared__ Survey s;
        const int64_t r = blockIdx.x;
        begin(s);
        const Plan made = plan(s, p, r, Row<T>(p, r), Settings(p, r), true);
        if (threadIdx.x == 0) p.plans[r] = made;
    }

    struct Listing : Small {
        uint64_t staged[kStaged];
    };
    struct Choice : Survey {
        uint64_t list[kList];
        uint64_t bins[kParts];
        uint64_t active[kRanked];
        uint64_t chunks[WQ_SAMPLE_MAX_VOCAB / kChunk + 1];
    };

    // f for every number of the list, or for every word of the row.
    template <typename T, typename F>
    static __device__ __forceinline__ void each_number(Choice& s, const Row<T>& row, bool of_row, int listed, F f) {
        if (of_row) {
            row.each(0, row.vectors, [&](float v, int w) {
                if (v > -INFINITY) f(entry_of(key_of(v), w));
            });
        } else {
#pragma unroll 1
            for (int i = threadIdx.x; i < listed; i += kThreads) f(s.list[i]);
        }
    }

    // The number up to which, in rising order, the numbers' weights reach `target` (which their sum does).  Their
    // range is cut into kParts; of the part that it lies in, the range again, until each lane has one number left
    // and can add up those below it.
    template <typename T>
    static __device__ __forceinline__ uint64_t find_number(Choice& s, const Row<T>& row, bool of_row, int listed, uint64_t target, const Weigh& weigh) {
        uint64_t low = 0, high = ~0ull;  // it lies in here
        const bool all_few = !of_row && listed <= kCompared;
        bool first = true;
#pragma unroll 1
        for (;;) {
            uint64_t least = ~0ull, most = 0;
            uint32_t total = listed;
            __syncthreads();
            if (!of_row && !first) {
                // Those that are left are put together, if they are few.
                if (threadIdx.x == 0) s.count = 0;
                __syncthreads();
                each_number(s, row, of_row, listed, [&](uint64_t e) {
                    if (e < low || e > high) return;
                    const uint32_t at = atomicAdd(&s.count, 1u);
                    if (at < kCompared) s.active[at] = e;
                });
                __syncthreads();
                total = s.count;
            }
            if (of_row || total > kCompared) {
                uint32_t left = 0;
                each_number(s, row, of_row, listed, [&](uint64_t e) {
                    if (e >= low && e <= high) least = std::min(least, e), most = std::max(most, e), ++left;
                });
                least = ~block_most(s, ~least);
                most = block_most(s, most);
                if (of_row) total = (uint32_t)block_sum(s, left);
            }
            first = false;
            if (total <= kCompared) {
                if (of_row) {
                    if (threadIdx.x == 0) s.count = 0;
                    __syncthreads();
                    each_number(s, row, of_row, listed, [&](uint64_t e) {
                        if (e >= low && e <= high) s.active[atomicAdd(&s.count, 1u)] = e;
                    });
                    __syncthreads();
                }
                const uint64_t* const numbers = all_few ? s.list : s.active;
                const bool mine = threadIdx.x < total;
                const uint64_t e = mine ? numbers[threadIdx.x] : 0, w = mine ? weigh(e) : 0;
                if (mine) s.bins[threadIdx.x] = w;
                __syncthreads();
                uint64_t below = 0;
                if (mine) {
#pragma unroll 8
                    for (uint32_t i = 0; i < total; ++i) below += numbers[i] < e ? s.bins[i] : 0;
                    if (below < target && below + w >= target) s.found = e;
                }
                __syncthreads();
                return s.found;
            }
            const int bits = 64 - __builtin_clzll(most - least), shift = bits > kPartBits ? bits - kPartBits : 0;
            for (int i = threadIdx.x; i < kParts; i += kThreads) s.bins[i] = 0;
            __syncthreads();
            each_number(s, row, of_row, listed, [&](uint64_t e) {
                if (e >= low && e <= high) add(&s.bins[(e - least) >> shift], weigh(e));
            });
            __syncthreads();
            constexpr int kMine = (kParts + kThreads - 1) / kThreads;
            uint64_t own[kMine], sum = 0, all;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int at = threadIdx.x * kMine + i;
                own[i] = at < kParts ? s.bins[at] : 0;
                sum += own[i];
            }
            uint64_t up = block_before(s, sum, all);
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                if (up < target && up + own[i] >= target) s.digit = threadIdx.x * kMine + i, s.before = up;
                up += own[i];
            }
            __syncthreads();
            low = least + ((uint64_t)s.digit << shift);
            high = low + (((uint64_t)1 << shift) - 1);
            target -= s.before;
        }
    }

    // The cut, from the listed words, and the word that the random number falls on.
    template <typename T>
    static __device__ __forceinline__ void finish(Choice& s, const Params& p, int64_t r, const Row<T>& row, const Settings& set, const Plan& plan) {
        const Way way = (Way)plan.way;
        Weigh weigh{set.weights(p, value_of(plan.best), plan.offset), ~0ull, false, false, false};
        const Weights& weights = weigh.weights;
        const uint64_t need = plan.need, ahead = plan.ahead;
        const bool few = plan.few, alone = plan.alone;
        const bool has = (int)threadIdx.x < p.chunks;
        int listed = alone ? 0 : (int)__hip_atomic_load(&p.plans[r].listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool of_row = alone || listed > p.list_size;  // no list, or one that did not hold all
        __syncthreads();
        if (!of_row)
            for (int i = threadIdx.x; i < listed; i += kThreads) s.list[i] = share_in(p.list + r * p.list_size + i);
        if (has) s.chunks[threadIdx.x] = few || of_row ? 0 : share_in(p.sums + r * p.chunks + threadIdx.x);
        __syncthreads();
        if (few && !of_row && listed <= kRanked) {
            // Each lane has a word, and finds by comparing it with all others its places in the order of words and by
            // number.
            const bool mine = (int)threadIdx.x < listed;
            const uint64_t e = mine ? s.list[threadIdx.x] : 0;
            const double t = mine ? weights.log2_of(value_of_entry(e)) : -2000.0;
            uint64_t w = mine ? weights.of(t) : 0, all;
            int rank = 0, place = 0;
            if (mine) {
#pragma unroll 8
                for (int i = 0; i < listed; ++i) {
                    const uint64_t other = s.list[i];
                    rank += other < e;
                    place += (uint32_t)other < (uint32_t)e;
                }
            }
            if (rank >= (int)(ahead + need)) w = 0;  // top-k
            if (mine) s.bins[rank] = w;
            __syncthreads();
            const uint64_t ordered = mine ? s.bins[threadIdx.x] : 0, before = block_before(s, ordered, all);
            if (mine) s.active[threadIdx.x] = before;
            __syncthreads();
            // A word stays for top-p while those before it do not weigh enough.
            if (mine && (t < weights.low || (set.top_p < 1.0f && s.active[rank] >= share_of(set.top_p, all)))) w = 0;
            if (mine) s.bins[place] = w;
            __syncthreads();
            const uint64_t placed = mine ? s.bins[threadIdx.x] : 0, up = block_before(s, placed, all), goal = set.goal(all);
            if (mine) s.active[threadIdx.x] = up;
            __syncthreads();
            if (mine && s.active[place] <= goal && goal < s.active[place] + w) {
                gbl(p.c.token)[r] = (int)(uint32_t)e;
                if (p.c.share) gbl(p.c.share)[r] = (float)((double)w / (double)all);
            }
            return;
        }
        // The searches: the last word that stays, by number for top-k and by weight for top-p; where all words that stay
        // are listed, then the word that the random number falls on, in the order of words.
        const bool complete = few || of_row;  // the list, or the row, holds what lies ahead of the cut's bin too
        uint64_t total = 0;
#pragma unroll 1
        for (int search = 0; search < 3; ++search) {
            uint64_t target;
            if (search == 0) {
                if (way != kCount) continue;
                weigh.ones = true;
                target = complete ? ahead + need : need;
            } else if (search == 1) {
                if (way == kMinP || set.top_p >= 1.0f) continue;
                weigh.ones = false;
                uint64_t sum = 0;
                each_number(s, row, of_row, listed, [&](uint64_t e) { sum += weigh(e); });
                sum = block_sum(s, sum);
                target = complete ? share_of(set.top_p, sum) : std::min(need, sum);
                if (target == 0) continue;  // words too light to weigh anything: it does not matter which stay
            } else {
                weigh.ones = false, weigh.min_p = true;
                if (!few || of_row) continue;
                uint64_t sum = 0;
                each_number(s, row, of_row, listed, [&](uint64_t e) { sum += weigh(e); });
                total = block_sum(s, sum);
                target = set.goal(total) + 1;
                for (int i = threadIdx.x; i < listed; i += kThreads) s.list[i] = turned(s.list[i]);
                weigh.by_word = true;
            }
            const uint64_t found = find_number(s, row, of_row, listed, target, weigh);
            if (search < 2) {
                weigh.last = found;
            } else {
                if (threadIdx.x == 0) {
                    gbl(p.c.token)[r] = (int)(found >> 32);
                    if (p.c.share) gbl(p.c.share)[r] = (float)((double)weigh(found) / (double)total);
                }
                return;
            }
        }
        // The chunks' weights, those of the list among them, and the chunk that the random number falls into.
        if (of_row) {
#pragma unroll 1
            for (int c = 0; c < p.chunks; ++c) {
                uint64_t sum = 0;
                row.each(c * kVectors<T>, min((c + 1) * kVectors<T>, row.vectors), [&](float v, int w) { sum += weigh(entry_of(key_of(v), w)); });
                if (sum) add(&s.chunks[c], sum);
            }
        } else {
            // (Lanes add to sums of their own where there is room, not to wait for each other.)
            const int copies = min(8, kParts / p.chunks), copy = threadIdx.x % copies * p.chunks;
            __syncthreads();
            for (int i = threadIdx.x; i < kParts; i += kThreads) s.bins[i] = 0;
            __syncthreads();
#pragma unroll 1
            for (int i = threadIdx.x; i < listed; i += kThreads) {
                const uint64_t w = weigh(s.list[i]);
                if (w) add(&s.bins[copy + row.chunk_of((int)(uint32_t)s.list[i])], w);
            }
            __syncthreads();
            if (has)
                for (int i = 0; i < copies; ++i) s.chunks[threadIdx.x] += s.bins[i * p.chunks + threadIdx.x];
        }
        __syncthreads();
        const uint64_t mine = has ? s.chunks[threadIdx.x] : 0, up = block_before(s, mine, total), goal = set.goal(total);
        if (up <= goal && goal < up + mine) s.digit = threadIdx.x, s.before = up;
        __syncthreads();
        const int target = (int)s.digit;
        const uint64_t within = goal - s.before;
        choose_in_chunk(s, p, r, row, target, within, (double)total, [&](float v, int w) { return weigh(entry_of(key_of(v), w)); });
    }

    // Lists a chunk's words that may be the cut (all that may stay, where they are few), and sums the weights of those
    // that surely stay.
    template <typename T>
    static __device__ __forceinline__ void list_chunk(Listing& s, const Params& p, int64_t r, int chunk, const Row<T>& row, Chunk<T>& x, const Settings& set, const Plan& plan) {
        const Way way = (Way)plan.way;
        const Weights weights = set.weights(p, value_of(plan.best), plan.offset);
        const float reference = plan.reference;
        const int cut_bin = plan.cut_bin;
        const bool few = plan.few;
        uint32_t* const listed = &p.plans[r].listed;
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
        x.take(row);
        uint64_t sum = 0;
        if (way == kWeight && set.min_p == 0.0f) {
            // Survey's histogram has the weights of the bins ahead of the cut's.
            const Record& record = p.records[r * p.chunks + chunk];
            const int over = (int)fmin(plan.offset - record.offset, 63.0);
            const uint64_t* const bins = p.bins + (r * p.chunks + chunk) * kBins;
            for (int i = record.low + threadIdx.x; i < min(record.high, cut_bin); i += kThreads) sum += gbl(bins)[i];
            sum = block_sum(s, sum) >> (weights.infinite && record.key != kInfinity ? 63 : over);
            sum = threadIdx.x == 0 ? sum : 0;
        } else if (!few) {
            x.each(row, [&](float v, int) {
                const double t = weights.log2_of(v);
                const uint64_t w = weights.of(t);
                sum += t >= weights.low && (way == kMinP || bin_of(v, reference) < cut_bin) ? w : 0;
            });
        }
        if (way != kMinP) {
            x.each(row, [&](float v, int w) {
                const int bin = v > -INFINITY ? bin_of(v, reference) : kBins;
                if (bin == cut_bin || (few && bin < cut_bin)) {
                    const uint64_t e = entry_of(key_of(v), w);
                    const uint32_t at = atomicAdd(&s.count, 1u);
                    if (at < kStaged) {
                        s.staged[at] = e;
                    } else {
                        const uint32_t to = atomicAdd(listed, 1u);
                        if (to < (uint32_t)p.list_size) share_out(p.list + r * p.list_size + to, e);
                    }
                }
            });
        }
        if (!few) {
            sum = block_sum(s, sum);
            if (threadIdx.x == 0) share_out(p.sums + r * p.chunks + chunk, sum);
        }
        __syncthreads();
        const uint32_t count = std::min<uint32_t>(s.count, kStaged);
        if (threadIdx.x == 0 && count) s.base = atomicAdd(listed, count);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < count; i += kThreads)
            if (s.base + i < (uint32_t)p.list_size) share_out(p.list + r * p.list_size + s.base + i, s.staged[i]);
    }

    // Few rows: a chunk's workgroup makes the row's plan for itself, and the last one of the row to be done goes on.
    template <typename T>
    static __device__ __forceinline__ void choose(const Params& p) {
        __shared__ struct {
            Listing listing;
            Choice choice;
        } s;
        const int64_t r = blockIdx.x;
        const int chunk = blockIdx.y;
        const Row<T> row(p, r);
        begin(s.listing);
        begin(s.choice);
        Chunk<T> x(row, chunk);
        const Settings set(p, r);
        const Plan made = plan(s.choice, p, r, row, set, chunk == 0);
        if (made.way == kDone || (made.alone && chunk != 0)) return;
        if (!made.alone) {
            list_chunk(s.listing, p, r, chunk, row, x, set, made);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what this wave shares has arrived
            __syncthreads();
            if (threadIdx.x == 0) s.listing.digit = __hip_atomic_fetch_add(&p.plans[r].done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == (uint32_t)p.chunks;
            __syncthreads();
            if (!s.listing.digit) return;
            asm volatile("" ::: "memory");
        }
        finish(s.choice, p, r, row, set, made);
    }

    // Many rows: a launch each.
    template <typename T>
    static __device__ __forceinline__ void list_chunks(const Params& p) {
        __shared__ Listing s;
        const int64_t r = blockIdx.x;
        const Plan& made = p.plans[r];
        if (made.way == kDone || made.alone) return;
        begin(s);
        const Row<T> row(p, r);
        Chunk<T> x(row, blockIdx.y);
        list_chunk(s, p, r, blockIdx.y, row, x, Settings(p, r), made);
    }
    template <typename T>
    static __device__ __forceinline__ void finish_rows(const Params& p) {
        __shared__ Choice s;
        const int64_t r = blockIdx.x;
        const Plan& made = p.plans[r];
        if (made.way == kDone) return;
        begin(s);
        finish(s, p, r, Row<T>(p, r), Settings(p, r), made);
    }
};

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void survey_kernel(const Params p) {
    Block<THREADS>::template survey<T>(p);
}
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void plan_kernel(const Params p) {
    Block<THREADS>::template plan_rows<T>(p);
}
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void list_kernel(const Params p) {
    Block<THREADS>::template list_chunks<T>(p);
}
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void finish_kernel(const Params p) {
    Block<THREADS>::template finish_rows<T>(p);
}
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void choose_kernel(const Params p) {
    Block<THREADS>::template choose<T>(p);
}

// ------------------------------------------------------------------ host

wq_status check_sizes(const char* fn, int64_t rows, int64_t vocab, int64_t dtype) {
    WQ_TRY(in_range(fn, "rows", rows, 1, WQ_SAMPLE_MAX_ROWS));
    WQ_TRY(in_range(fn, "vocab", vocab, 1, WQ_SAMPLE_MAX_VOCAB));
    if (dtype != WQ_DTYPE_F16 && dtype != WQ_DTYPE_BF16 && dtype != WQ_DTYPE_F32)
        return err(WQ_ERR_UNSUPPORTED, "%s: dtype must be one of WQ_DTYPE_* (got %lld)", fn, (long long)dtype);
    return WQ_OK;
}

// Chunks of a row, wherever in 16 bytes it starts.
int64_t chunks_of(int64_t vocab, int64_t dtype) {
    const int64_t lead = dtype == WQ_DTYPE_F32 ? 3 : 7;
    return (vocab + lead + kChunk - 1) / kChunk;
}
constexpr int kFewThreads = 1024, kManyThreads = 256;  // of a workgroup, in small batches and in large ones
static_assert(kBins < 1 << 11, "a range in 22 bits");
static_assert(WQ_SAMPLE_MAX_VOCAB / kChunk + 1 + kAhead <= kManyThreads && kRanked <= kManyThreads, "a lane for every chunk and for every word compared");

// The parts of the workspace, each a multiple of 16 bytes.
size_t round16(size_t n) { return (n + 15) / 16 * 16; }
size_t lay_out(Params& p, uint8_t* base) {
    const size_t rows = (size_t)p.c.rows, chunks = rows * p.chunks;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        uint8_t* const part = base ? base + at : nullptr;
        at += round16(bytes);
        return part;
    };
    p.records = reinterpret_cast<Record*>(take(chunks * sizeof(Record)));
    p.sums = reinterpret_cast<uint64_t*>(take(chunks * 8));
    p.plans = reinterpret_cast<Plan*>(take(rows * sizeof(Plan)));
    p.list = reinterpret_cast<uint64_t*>(take(rows * p.list_size * 8));
    p.bins = reinterpret_cast<uint64_t*>(take(chunks * kBins * 8));
    return at;
}

void set_sizes(Params& p) {
    p.chunks = (int32_t)chunks_of(p.c.vocab, p.c.dtype);
    p.list_size = (int32_t)std::min<int64_t>(kList, p.c.vocab);
    p.weight_bits = std::min(51, 62 - log2_of(p.c.vocab));
}
// Rows of one pair of launches: enough chunks to fill the CUs several times over; more rows take more
// launches, which share the workspace.
int64_t slab_of(const Params& p) { return std::max<int64_t>(1, 4096 / p.chunks); }

size_t workspace_of(int64_t rows, int64_t vocab, int64_t dtype) {
    Params p{};
    p.c.vocab = vocab;
    p.c.dtype = dtype;
    set_sizes(p);
    p.c.rows = std::min(rows, slab_of(p));
    return lay_out(p, nullptr);
}

template <typename T>
void launch(const Params& p, hipStream_t st) {
    const dim3 rows((unsigned)p.c.rows), chunks((unsigned)p.c.rows, (unsigned)p.chunks), few(kFewThreads), many(kManyThreads);
    // While each large workgroup has a CU of its own.  (128256 words, top-p and top-k with top-p: 16 rows 33 and 20 us,
    // in the launches of many rows 41 and 27; 24 rows 46 and 30, 43 and 27.)
    if (p.c.rows * p.chunks <= 256) {
        hipLaunchKernelGGL((survey_kernel<T, kFewThreads>), chunks, few, 0, st, p);
        hipLaunchKernelGGL((choose_kernel<T, kFewThreads>), chunks, few, 0, st, p);
    } else {
        hipLaunchKernelGGL((survey_kernel<T, kManyThreads>), chunks, many, 0, st, p);
        hipLaunchKernelGGL((plan_kernel<T, kFewThreads>), rows, few, 0, st, p);
        hipLaunchKernelGGL((list_kernel<T, kManyThreads>), chunks, many, 0, st, p);
        hipLaunchKernelGGL((finish_kernel<T, kFewThreads>), rows, few, 0, st, p);
    }
}

}  // namespace
}  // namespace sample
}  // namespace wq

using namespace wq::sample;

extern "C" {

wq_status wq_sample_logits_workspace_size(int64_t rows, int64_t vocab, int64_t dtype, size_t* bytes) {
    static const char* fn = "wq_sample_logits_workspace_size";
    if (!bytes) return err(WQ_ERR_INVALID_ARG, "%s: null output pointer", fn);
    WQ_TRY(check_sizes(fn, rows, vocab, dtype));
    *bytes = workspace_of(rows, vocab, dtype);
    return WQ_OK;
}

wq_status wq_sample_logits(const wq_sample_call* call, void* workspace, size_t workspace_bytes, void* stream) {
    static const char* fn = "wq_sample_logits";
    if (!call || !call->logits || !call->random || !call->token) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    Params p{};
    p.c = *call;
    const wq_sample_call& c = p.c;
    WQ_TRY(check_sizes(fn, c.rows, c.vocab, c.dtype));
    const int64_t size = c.dtype == WQ_DTYPE_F32 ? 4 : 2;
    WQ_TRY(in_range(fn, "logits_stride", c.logits_stride, c.vocab, (int64_t)1 << 32));
    if (!aligned(c.logits, size)) return err(WQ_ERR_MISALIGNED, "%s: logits must be aligned to their elements", fn);
    const void* const lists[] = {c.random, c.temperature, c.top_k, c.top_p, c.min_p, c.token, c.share};
    for (const void* l : lists)
        if (!aligned(l, 4)) return err(WQ_ERR_MISALIGNED, "%s: every list must be 4-byte aligned", fn);
    const size_t ws = workspace_of(c.rows, c.vocab, c.dtype);
    if (ws > 0) {
        if (!workspace || workspace_bytes < ws)
            return err(WQ_ERR_INVALID_ARG, "%s: a workspace of %zu bytes is needed (got %zu)", fn, ws, workspace ? workspace_bytes : (size_t)0);
        if (!aligned(workspace, 16)) return err(WQ_ERR_MISALIGNED, "%s: workspace must be 16-byte aligned", fn);
    }
    const uint64_t rows = (uint64_t)c.rows;
    const auto list = [&](const void* ptr) { return span(ptr, ptr ? rows * 4 : 0); };
    const Span token = list(c.token), share = list(c.share), work = span(workspace, ws);
    const Span inputs[] = {span(c.logits, ((rows - 1) * c.logits_stride + c.vocab) * size), list(c.random), list(c.temperature), list(c.top_k), list(c.top_p), list(c.min_p)};
    for (const Span& s : inputs)
        if (overlaps(s, token) || overlaps(s, share) || overlaps(s, work)) return err(WQ_ERR_INVALID_ARG, "%s: an output or the workspace overlaps an input", fn);
    if (overlaps(token, share) || overlaps(token, work) || overlaps(share, work))
        return err(WQ_ERR_INVALID_ARG, "%s: token, share and the workspace must not overlap", fn);
    set_sizes(p);
    p.has = (c.temperature ? 1 : 0) | (c.top_p ? 2 : 0) | (c.min_p ? 4 : 0) | (c.top_k ? 8 : 0);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const int64_t slab = slab_of(p);
    for (int64_t row = 0; row < call->rows; row += slab) {
        p.c = *call;
        p.c.rows = std::min(slab, call->rows - row);
        p.c.logits = static_cast<const uint8_t*>(call->logits) + row * call->logits_stride * size;
        p.c.random += row;
        p.c.token += row;
        p.c.temperature = call->temperature ? call->temperature + row : p.c.random;
        p.c.top_p = call->top_p ? call->top_p + row : p.c.random;
        p.c.min_p = call->min_p ? call->min_p + row : p.c.random;
        p.c.top_k = call->top_k ? call->top_k + row : reinterpret_cast<const int32_t*>(p.c.random);
        if (p.c.share) p.c.share += row;
        lay_out(p, static_cast<uint8_t*>(workspace));
        if (call->dtype == WQ_DTYPE_F16) launch<_Float16>(p, st);
        else if (call->dtype == WQ_DTYPE_BF16) launch<__bf16>(p, st);
        else launch<float>(p, st);
    }
    return wq::host::hip_result(fn, hipGetLastError());
}

}  // extern "C"
