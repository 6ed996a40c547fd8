// The choice of the next word by chance (gfx950, wave64): temperature, top-k,
// top-p, min-p and a given random number.
//
// The words that stay are a beginning of the order (logit falling, word rising), so
// they are told by the last of them, the cut.  It is found by digits of an
// order-preserving integer of the logit: a histogram of one digit (of counts for
// top-k, of weights for top-p) in LDS tells which value the cut's digit has, and the
// next pass looks only at words that share the digits found so far; equal logits
// are told apart by their words in the same way, where the cut falls among them.
//
// Weights are formed in fp64 and held as whole multiples of 2^-s: their sums do
// not depend on the order in which they are added, so LDS atomics may add them.
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

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;

struct Params {
    wq_sample_call c;
    int32_t weight_bits;  // s
};

template <typename T>
constexpr int kPer = 16 / sizeof(T);  // words of a 16-byte load

// One row's logits: vector v holds the words v * kPer - lead .. + kPer - 1, so that whole vectors
// are aligned whatever word the row starts at.
template <typename T>
struct Row {
    const T* x;
    int vocab, lead, vectors;
    __device__ __forceinline__ Row(const Params& p, int64_t row) {
        x = static_cast<const T*>(p.c.logits) + row * p.c.logits_stride;
        vocab = (int)p.c.vocab;
        lead = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) % kPer<T>);
        vectors = (vocab + lead + kPer<T> - 1) / kPer<T>;
    }
    // The words of vector v as fp32; NaN and what lies outside the row as -infinity.
    __device__ __forceinline__ void load(int v, float (&out)[kPer<T>]) const {
        const int first = v * kPer<T> - lead;
        if (first >= 0 && first + kPer<T> <= vocab) {
            typedef T vec __attribute__((ext_vector_type(kPer<T>)));
            const vec r = __builtin_bit_cast(vec, *gbl(reinterpret_cast<const u32x4*>(x + first)));
#pragma unroll
            for (int i = 0; i < kPer<T>; ++i) out[i] = (float)r[i];
        } else {
#pragma unroll
            for (int i = 0; i < kPer<T>; ++i) out[i] = first + i >= 0 && first + i < vocab ? (float)gbl(x)[first + i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i) out[i] = out[i] != out[i] ? -INFINITY : out[i] + 0.0f;  // -0 is 0
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

// 2^t for t <= 0, relative error below 2^-50: a Taylor series in the fraction's
// logarithm, |f ln 2| <= 0.347, whose first missing term is 0.347^14 / 14!.
__device__ __forceinline__ double exp2_of(double t) {
    const double n = __builtin_rint(t), y = (t - n) * 0.693147180559945309417;
    double r = 1.0 / 6227020800.0;
    r = fma(r, y, 1.0 / 479001600.0);
    r = fma(r, y, 1.0 / 39916800.0);
    r = fma(r, y, 1.0 / 3628800.0);
    r = fma(r, y, 1.0 / 362880.0);
    r = fma(r, y, 1.0 / 40320.0);
    r = fma(r, y, 1.0 / 5040.0);
    r = fma(r, y, 1.0 / 720.0);
    r = fma(r, y, 1.0 / 120.0);
    r = fma(r, y, 1.0 / 24.0);
    r = fma(r, y, 1.0 / 6.0);
    r = fma(r, y, 0.5);
    r = fma(r, y, 1.0);
    r = fma(r, y, 1.0);
    return __builtin_ldexp(r, (int)n);
}

// How a row's logits become weights.
struct Weights {
    double top, factor, low;  // largest logit; log2(e) / temperature; smallest log2 w that stays under min-p
    double steps;             // 2^s
    bool infinite;
    // log2 w; at most 0, not below -2000.
    __device__ __forceinline__ double log2_of(float x) const {
        if (infinite) return x == INFINITY ? 0.0 : -2000.0;
        return fmax(((double)x - top) * factor, -2000.0);
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

struct Shared {
    uint64_t bins[kBins];
    uint64_t tiles[WQ_SAMPLE_MAX_VOCAB / (kThreads * 4) + 2];
    uint64_t parts[kWaves];
    uint64_t before, found;
    uint32_t keys[kWaves];
    uint32_t digit;
    int words[kWaves];
};

__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor((unsigned long long)v, d);
    return v;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {  // inclusive
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t o = __shfl_up((unsigned long long)v, d);
        if ((int)(threadIdx.x % 64) >= d) v += o;
    }
    return v;
}
// Sum over the block of v in the lanes before this one; `total` the sum of all.
__device__ __forceinline__ uint64_t block_before(Shared& s, uint64_t v, uint64_t& total) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint64_t up = wave_scan(v);
    __syncthreads();
    if (lane == 63) s.parts[wave] = up;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
    for (int i = 0; i < kWaves; ++i) {
        const uint64_t part = s.parts[i];
        if (i < wave) before += part;
        total += part;
    }
    return before + up - v;
}

// Which bin, counted from `from_top` or from the bottom, the sum of bins reaches `target`
// in: the bin, what lies before it, and its own sum, the same in all lanes.
__device__ __forceinline__ void find_bin(Shared& s, bool from_top, uint64_t target, uint32_t& digit, uint64_t& before, uint64_t& own) {
    uint64_t v[kBins / kThreads], sum = 0, total;
#pragma unroll
    for (int i = 0; i < kBins / kThreads; ++i) {
        const int at = threadIdx.x * (kBins / kThreads) + i;
        v[i] = s.bins[from_top ? kBins - 1 - at : at];
        sum += v[i];
    }
    uint64_t up = block_before(s, sum, total);
#pragma unroll
    for (int i = 0; i < kBins / kThreads; ++i) {
        if (up < target && up + v[i] >= target) {
            const int at = threadIdx.x * (kBins / kThreads) + i;
            s.digit = from_top ? kBins - 1 - at : at;
            s.before = up;
            s.found = v[i];
        }
        up += v[i];
    }
    __syncthreads();
    digit = s.digit, before = s.before, own = s.found;
}

__device__ __forceinline__ void clear_bins(Shared& s) {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.bins[i] = 0;
    __syncthreads();
}
__device__ __forceinline__ void add(uint64_t* at, uint64_t v) { atomicAdd(reinterpret_cast<unsigned long long*>(at), (unsigned long long)v); }

template <typename T, typename F>
__device__ __forceinline__ void each_word(const Row<T>& row, F f) {
    for (int v = threadIdx.x; v < row.vectors; v += kThreads) {
        float x[kPer<T>];
        row.load(v, x);
#pragma unroll
        for (int i = 0; i < kPer<T>; ++i)
            if (x[i] != -INFINITY) f(x[i], v * kPer<T> + i - row.lead);
    }
}

// The cut at which the words kept by `in` reach the target: `share` of their weights (share > 0) or
// `count` of them (share = 0).
template <typename T>
__device__ Cut find_cut(Shared& s, const Row<T>& row, const Weights& weights, Cut in, double share, uint64_t count) {
    const bool by_weight = share > 0.0;
    uint64_t target = count, before = 0, own = 0;
    uint32_t prefix = 0, digit;
    // Digits of the logit, from the top: 11, 11 and 10 bits.  The integers of 16-bit logits end with the second.
    constexpr int kLevels = sizeof(T) == 2 ? 2 : 3;
#pragma unroll
    for (int level = 0; level < kLevels; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, above = level == 0 ? 32 : level == 1 ? 21 : 10;
        clear_bins(s);
        each_word(row, [&](float x, int word) {
            const uint32_t key = key_of(x);
            if ((level == 0 || key >> above % 32 == prefix >> above % 32) && in.keeps(key, word))
                add(&s.bins[(key >> shift) & ((1u << (above - shift)) - 1)], by_weight ? weights.of(weights.log2_of(x)) : 1);
        });
        __syncthreads();
        if (level == 0 && by_weight) {
            uint64_t sum = 0, total;
            for (int i = threadIdx.x; i < kBins; i += kThreads) sum += s.bins[i];
            block_before(s, sum, total);
            const double want = ceil(share * (double)total);
            target = want < 1.0 ? 1 : want >= (double)total ? total : (uint64_t)want;
        }
        uint64_t up;
        find_bin(s, true, target - before, digit, up, own);
        before += up;
        prefix |= digit << shift;
    }
    // What the 16-bit types' integers leave below the second digit: ten ones for negative logits, zeros for others.
    const uint32_t key = kLevels == 2 && !(prefix & 0x80000000u) ? prefix | 0x3FFu : prefix;
    // Of `own`, the words with this logit, the first few are needed.
    uint64_t each = 1;
    if (by_weight) {
        each = weights.of(weights.log2_of(value_of(key)));
        each = each ? each : 1;
    }
    const uint64_t need = (target - before + each - 1) / each, have = own / each;
    if (need >= have) return Cut{key, INT32_MAX};
    uint64_t passed = 0;
    int word = 0;
#pragma unroll
    for (int level = 0; level < 2; ++level) {
        clear_bins(s);
        each_word(row, [&](float x, int w) {
            if (key_of(x) == key && in.keeps(key, w) && (level == 0 || w >> 10 == word >> 10)) add(&s.bins[level == 0 ? w >> 10 : w & 1023], 1);
        });
        __syncthreads();
        uint64_t up;
        find_bin(s, false, need - passed, digit, up, own);
        passed += up;
        word |= digit << (level == 0 ? 10 : 0);
    }
    return Cut{key, word};
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const Params p) {
    __shared__ Shared s;
    const wq_sample_call& c = p.c;
    const int64_t r = blockIdx.x;
    const Row<T> row(p, r);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;

    // The best word.
    uint32_t best = kNothing;
    int word = INT32_MAX;
    each_word(row, [&](float x, int w) {
        const uint32_t key = key_of(x);
        if (key > best) best = key, word = w;  // (A lane's words rise.)
    });
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        const uint32_t k = __shfl_xor(best, d);
        const int w = __shfl_xor(word, d);
        if (k > best || (k == best && w < word)) best = k, word = w;
    }
    if (lane == 0) s.keys[wave] = best, s.words[wave] = word;
    __syncthreads();
    for (int i = 0; i < kWaves; ++i) {
        const uint32_t k = s.keys[i];
        const int w = s.words[i];
        if (k > best || (k == best && w < word)) best = k, word = w;
    }
    const float temperature = c.temperature ? gbl(c.temperature)[r] : 1.0f;
    if (best == kNothing || !(temperature > 0.0f)) {
        if (threadIdx.x == 0) {
            gbl(c.token)[r] = best == kNothing ? -1 : word;
            if (c.share) gbl(c.share)[r] = best == kNothing ? 0.0f : 1.0f;
        }
        return;
    }
    const int top_k = c.top_k ? gbl(c.top_k)[r] : 0;
    const float top_p = c.top_p ? gbl(c.top_p)[r] : 1.0f, min_p = c.min_p ? gbl(c.min_p)[r] : 0.0f;
    Weights weights;
    weights.infinite = best == kInfinity;
    weights.top = (double)value_of(best);
    weights.factor = 1.44269504088896340736 / (double)temperature;
    weights.low = min_p > 0.0f ? log2((double)fminf(min_p, 1.0f)) : -4000.0;
    weights.steps = __builtin_ldexp(1.0, p.weight_bits);

    Cut cut{kNothing, INT32_MAX};
    if (top_k > 0 && top_k < row.vocab) {
        uint64_t n = 0, total;
        each_word(row, [&](float, int) { ++n; });
        block_before(s, n, total);
        if ((uint64_t)top_k < total) cut = find_cut(s, row, weights, cut, 0.0, (uint64_t)top_k);
    }
    if (top_p < 1.0f) cut = top_p > 0.0f ? find_cut(s, row, weights, cut, (double)top_p, 0) : Cut{best, word};

    // The weights of the words that stay, by tiles of one vector per lane.
    auto weight = [&](float x, int w) -> uint64_t {
        if (x == -INFINITY || !cut.keeps(key_of(x), w)) return 0;
        const double t = weights.log2_of(x);
        return t >= weights.low ? weights.of(t) : 0;
    };
    const int tiles = (row.vectors + kThreads - 1) / kThreads;
    __syncthreads();
    for (int i = threadIdx.x; i < tiles; i += kThreads) s.tiles[i] = 0;
    __syncthreads();
    for (int tile = 0; tile < tiles; ++tile) {
        const int v = tile * kThreads + threadIdx.x;
        uint64_t sum = 0;
        if (v < row.vectors) {
            float x[kPer<T>];
            row.load(v, x);
#pragma unroll
            for (int i = 0; i < kPer<T>; ++i) sum += weight(x[i], v * kPer<T> + i - row.lead);
        }
        sum = wave_sum(sum);
        if (lane == 0 && sum) add(&s.tiles[tile], sum);
    }
    __syncthreads();
    // The tile in which the sum passes random * total, found by every lane for itself from its share of the tiles.
    uint64_t total;
    const uint64_t mine = (int)threadIdx.x < tiles ? s.tiles[threadIdx.x] : 0;
    const uint64_t up = block_before(s, mine, total);
    const float random = gbl(c.random)[r];
    const double u = random > 0.0f ? fmin((double)random, 0.99999999999999989) : 0.0;
    uint64_t goal = (uint64_t)(u * (double)total);
    goal = goal < total ? goal : total - 1;
    if (up <= goal && goal < up + mine) s.digit = threadIdx.x, s.before = up;
    __syncthreads();
    const int tile = (int)s.digit;
    goal -= s.before;
    // Its words.
    const int v = tile * kThreads + threadIdx.x;
    uint64_t w[kPer<T>], sum = 0;
    float x[kPer<T>];
    if (v < row.vectors) row.load(v, x);
#pragma unroll
    for (int i = 0; i < kPer<T>; ++i) {
        w[i] = v < row.vectors ? weight(x[i], v * kPer<T> + i - row.lead) : 0;
        sum += w[i];
    }
    uint64_t unused, at = block_before(s, sum, unused);
#pragma unroll
    for (int i = 0; i < kPer<T>; ++i) {
        if (at <= goal && goal < at + w[i]) {
            gbl(c.token)[r] = v * kPer<T> + i - row.lead;
            if (c.share) gbl(c.share)[r] = (float)((double)w[i] / (double)total);
        }
        at += w[i];
    }
}

// ------------------------------------------------------------------ host

wq_status check_sizes(const char* fn, int64_t rows, int64_t vocab, int64_t dtype) {
    WQ_TRY(in_range(fn, "rows", rows, 1, WQ_SAMPLE_MAX_ROWS));
    WQ_TRY(in_range(fn, "vocab", vocab, 1, WQ_SAMPLE_MAX_VOCAB));
    if (dtype != WQ_DTYPE_F16 && dtype != WQ_DTYPE_BF16 && dtype != WQ_DTYPE_F32)
        return err(WQ_ERR_UNSUPPORTED, "%s: dtype must be one of WQ_DTYPE_* (got %lld)", fn, (long long)dtype);
    return WQ_OK;
}

size_t workspace_of(int64_t, int64_t, int64_t) { return 0; }

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
    p.weight_bits = std::min(51, 62 - log2_of(c.vocab));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)c.rows), block(kThreads);
    (void)hipGetLastError();
    if (c.dtype == WQ_DTYPE_F16) hipLaunchKernelGGL((sample_kernel<_Float16>), grid, block, 0, st, p);
    else if (c.dtype == WQ_DTYPE_BF16) hipLaunchKernelGGL((sample_kernel<__bf16>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((sample_kernel<float>), grid, block, 0, st, p);
    return wq::host::hip_result(fn, hipGetLastError());
}

}  // extern "C"
