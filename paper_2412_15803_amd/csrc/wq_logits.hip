// From logits to the next token (gfx950, wave64): penalties for repeated words,
// biases, a grammar's mask and the best word, in one pass over the logits.
//
// The logits are read once and written once, which is what bounds large
// batches.  A workgroup takes a tile of one row's words.  What it has to know of
// the row's history is how often each word of its tile occurs, so it scans the
// history once (a few thousand words, from L2) into counters in LDS, marks the
// listed biases there, and then streams its tile: 16 bytes
// per lane and load, whatever word the row starts at, as long as input and
// output rows lie alike.  The best word of each tile goes to the workspace and
// pick_kernel takes the best of a row's.  Integer LDS atomics are the only
// ones, so results do not depend on the order they run in.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "wq_device.h"
#include "wq_host.h"
#include "wq_internal.h"
#include "wq_logits.h"

namespace wq {
namespace logits {
namespace {

using dev::gbl;
using dev::u32x4;
using namespace host;

constexpr int kPickThreads = 64;
// A word's counter: the times it was generated, and whether it occurs in the
// prompt and in the bias list.
constexpr uint32_t kPrompt = 0x80000000u, kListed = 0x40000000u, kTimes = kListed - 1;
constexpr int kTileBias = 256;  // biases of one tile that are kept in LDS
constexpr int kMinTile = 2048, kMaxTile = 8192;

typedef int int4v __attribute__((ext_vector_type(4)));

struct Params {
    wq_logits_call c;
    float* best;         // [rows][tiles] largest value of each tile
    int32_t* best_word;  // [rows][tiles], -1: none
    int32_t tile, tiles;
};

template <typename T>
struct Type;
template <>
struct Type<_Float16> {
    static constexpr int kPer = 8;
};
template <>
struct Type<__bf16> {
    static constexpr int kPer = 8;
};
template <>
struct Type<float> {
    static constexpr int kPer = 4;
};

// The larger of two candidates; the lower word where they are equal, and none
// (word -1) only where both are none.
__device__ __forceinline__ void better(float& v, int& w, float v2, int w2) {
    if (w2 >= 0 && (w < 0 || v2 > v || (v2 == v && w2 < w))) {
        v = v2;
        w = w2;
    }
}

template <int kCount>
__device__ __forceinline__ void best_of_wave(float& v, int& w) {
#pragma unroll
    for (int d = kCount / 2; d >= 1; d >>= 1) {
        const float v2 = __shfl_xor(v, d);
        const int w2 = __shfl_xor(w, d);
        better(v, w, v2, w2);
    }
}

// The words of 16 bytes of logits with those masked that `ok` does not allow,
// and the largest value left (NaN left out).
template <typename T>
__device__ __forceinline__ float mask_and_max(u32x4& w, uint32_t ok) {
    float m = -INFINITY;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const uint32_t v = ok >> d & 1 ? w[d] : 0xFF800000u;
            w[d] = v;
            m = fmaxf(m, __builtin_bit_cast(float, v));
        }
    } else {
        constexpr uint32_t kLowest = std::is_same_v<T, _Float16> ? 0xFC00FC00u : 0xFF80FF80u;  // two of -infinity
        dev::half2v pair = dev::as_h2(0xFC00FC00u);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const uint32_t lo = (uint32_t)((int)(ok << (31 - 2 * d)) >> 31), hi = (uint32_t)((int)(ok << (30 - 2 * d)) >> 31);
            const uint32_t keep = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
            w[d] = (w[d] & keep) | (kLowest & ~keep);
            if constexpr (std::is_same_v<T, _Float16>) {
                pair = __builtin_elementwise_max(pair, dev::as_h2(w[d]));
            } else {
                m = fmaxf(m, __builtin_bit_cast(float, w[d] << 16));
                m = fmaxf(m, __builtin_bit_cast(float, w[d] & 0xFFFF0000u));
            }
        }
        if constexpr (std::is_same_v<T, _Float16>) m = fmaxf((float)pair.x, (float)pair.y);
    }
    return m;
}

// Element e of 16 bytes of logits.
template <typename T>
__device__ __forceinline__ T element(const u32x4 w, int e) {
    const int d = sizeof(T) == 4 ? e : e / 2;
    const uint32_t v = d == 0 ? w.x : d == 1 ? w.y : d == 2 ? w.z : w.w;
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, v);
    else return __builtin_bit_cast(T, (uint16_t)(v >> (16 * (e & 1))));
}
template <typename T>
__device__ __forceinline__ void set_element(u32x4& w, int e, T x) {
    const int d = sizeof(T) == 4 ? e : e / 2;
    uint32_t bits, keep = 0;
    if constexpr (sizeof(T) == 4) {
        bits = __builtin_bit_cast(uint32_t, x);
    } else {
        bits = (uint32_t)__builtin_bit_cast(uint16_t, x) << (16 * (e & 1));
        keep = e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
    }
    w.x = d == 0 ? (w.x & keep) | bits : w.x;
    w.y = d == 1 ? (w.y & keep) | bits : w.y;
    w.z = d == 2 ? (w.z & keep) | bits : w.z;
    w.w = d == 3 ? (w.w & keep) | bits : w.w;
}

struct Row {
    float repetition, frequency, presence;
    // The row's bias list, and the part of it in this tile: (word, position).
    const int32_t* ids;
    const float* values;
    int listed;
    const int2* tile_bias;
    const int* tile_listed;
};

// The bias of a word that the row lists: that of its last position.  The tile's
// part of the list is looked through for each listed word, the whole list where the
// tile has more than kTileBias: a row of 128256 words takes 11 us without biases,
// 141 with 256 in one tile, 175 with 300, 1926 with 2000 and 65228 with 65536.
__device__ __forceinline__ float bias_of(int w, const Row& r) {
    int at = -1;
    const int n = *r.tile_listed;
    if (n <= kTileBias) {
        for (int i = 0; i < n; ++i)
            if (r.tile_bias[i].x == w) at = max(at, r.tile_bias[i].y);
    } else {
        for (int i = 0; i < r.listed; ++i)
            if (r.ids[i] == w) at = i;
    }
    return r.values[at];
}

// A word's value, `uses` being its counter.
__device__ __forceinline__ float adjusted(float x, uint32_t uses, int w, const Row& r) {
#pragma clang fp contract(off)
    if (uses & ~kListed) {
        x = x > 0.0f ? x / r.repetition : x * r.repetition;
        const uint32_t c = uses & kTimes;
        const float taken = r.frequency * (float)c;
        x = x - taken;
        if (c) x = x - r.presence;
    }
    if (uses & kListed) x = x + bias_of(w, r);
    return x;
}

template <typename T, bool HISTORY, bool BIAS, bool VECTOR, int THREADS>
__global__ __launch_bounds__(THREADS) void logits_kernel(const Params p) {
    constexpr int kThreads = THREADS, kWaves = THREADS / 64;
    extern __shared__ __align__(16) uint32_t smem[];
    constexpr int kPer = Type<T>::kPer;
    __shared__ float sh_v[kWaves];
    __shared__ int sh_w[kWaves];
    __shared__ int2 sh_bias[BIAS ? kTileBias : 1];
    __shared__ int sh_listed;
    constexpr bool COUNTS = HISTORY || BIAS;
    uint32_t* uses = smem;  // [tile + kPer] counters, where there are any
    const wq_logits_call& c = p.c;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.y;
    const T* x = reinterpret_cast<const T*>(c.logits) + row * c.logits_stride;
    T* y = reinterpret_cast<T*>(c.out) + row * c.out_stride;
    const uint32_t* mask = c.mask ? c.mask + row * c.mask_stride : nullptr;
    const int vocab = (int)c.vocab;

    // Words before the row's first 16-byte boundary belong to the first tile.
    const int head = VECTOR ? (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)) : 0;
    const int begin = blockIdx.x == 0 ? 0 : min(vocab, head + (int)blockIdx.x * p.tile);
    const int end = min(vocab, head + ((int)blockIdx.x + 1) * p.tile);
    // The word of LDS entry 0.  With vectors, the first whole vector has entry
    // kPer, so that a vector's counters are whole 16-byte pieces of LDS.
    const int from = VECTOR && blockIdx.x == 0 ? min(head, end) : begin;  // words from here on come in vectors
    const int base = VECTOR ? from - kPer : begin;

    Row r{1.0f, 0.0f, 0.0f, nullptr, nullptr, 0, sh_bias, &sh_listed};
    if constexpr (HISTORY) {
        if (c.repetition) r.repetition = c.repetition[row];
        if (c.frequency) r.frequency = c.frequency[row];
        if (c.presence) r.presence = c.presence[row];
    }
    // The first vectors and their mask words are on their way while the history is
    // counted.
    typedef T Vec __attribute__((ext_vector_type(kPer)));
    constexpr int kUnroll = 4;
    const int vectors = VECTOR ? (end - from) / kPer : 0;
    const int words = (vocab + 31) >> 5;
    struct Batch {
        Vec in[kUnroll];
        uint32_t lo[kUnroll], hi[kUnroll];
    } batch;
    auto load = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
            const int w = from + min(i0 + j * kThreads, vectors - 1) * kPer;
            batch.in[j] = __builtin_nontemporal_load(gbl(reinterpret_cast<const Vec*>(x + w)));
            if (mask) {
                batch.lo[j] = mask[w >> 5];
                batch.hi[j] = mask[min((w >> 5) + 1, words - 1)];
            }
        }
    };
    if (vectors > 0) load(tid);

    if constexpr (COUNTS) {
        const int entries = p.tile + kPer;
        if (BIAS && tid == 0) sh_listed = 0;
        for (int i = tid * 4; i < entries; i += kThreads * 4) *reinterpret_cast<u32x4*>(smem + i) = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    if constexpr (HISTORY) {
        const int32_t* h = c.history + row * c.history_size;
        int n = (int)c.history_size, prompt = 0;
        if (c.history_lens) n = min(max(c.history_lens[row], 0), n);
        if (c.prompt_lens) prompt = c.prompt_lens[row];
        auto use = [&](int i, int w) {
            if (w >= begin && w < end) {
                if (i < prompt) atomicOr(&uses[w - base], kPrompt);
                else atomicAdd(&uses[w - base], 1u);
            }
        };
        // Four words at a time from the first 16-byte boundary on, several loads in
        // flight.
        const int lead = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(h) & 15)) & 15) / 4);
        if (tid < lead) use(tid, h[tid]);
        const int whole = (n - lead) / 4;
        constexpr int kAhead = 4;
        for (int i0 = tid; i0 < whole; i0 += kThreads * kAhead) {
            int4v w[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) w[j] = *gbl(reinterpret_cast<const int4v*>(h + lead) + min(i0 + j * kThreads, whole - 1));
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = i0 + j * kThreads;
                if (i >= whole) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) use(lead + 4 * i + e, w[j][e]);
            }
        }
        const int rest = lead + 4 * whole + tid;
        if (rest < n) use(rest, h[rest]);
    }
    if constexpr (BIAS) {
        r.ids = c.bias_ids + row * c.bias_size;
        r.values = c.bias_values + row * c.bias_size;
        r.listed = (int)c.bias_size;
        if (c.bias_lens) r.listed = min(max(c.bias_lens[row], 0), r.listed);
        for (int i = tid; i < r.listed; i += kThreads) {
            const int w = r.ids[i];
            if (w >= begin && w < end) {
                atomicOr(&uses[w - base], kListed);
                const int at = atomicAdd(&sh_listed, 1);
                if (at < kTileBias) sh_bias[at] = make_int2(w, i);
            }
        }
    }
    if constexpr (COUNTS) __syncthreads();

    // The best word so far, or the first word of the vector `best` that holds it.
    float top = -INFINITY;
    int word = -1;
    Vec best = {};
    uint32_t best_ok = 0;
    // (Words come in any order.)
    auto take = [&](float v, int w, bool allowed) {
        if (allowed && v == v) better(top, word, v, w);
    };
    auto one = [&](int w) {
        const bool allowed = !mask || (mask[w >> 5] >> (w & 31) & 1);
        const float v = adjusted((float)x[w], COUNTS ? uses[w - base] : 0, w, r);
        y[w] = (T)(allowed ? v : -INFINITY);
        take(v, w, allowed);
    };
    if constexpr (!VECTOR) {
        for (int w = begin + tid; w < end; w += kThreads) one(w);
    } else {
        for (int i0 = tid; i0 < vectors; i0 += kThreads * kUnroll) {
            if (i0 != tid) load(i0);
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                const int i = i0 + j * kThreads, w = from + i * kPer;
                if (i >= vectors) break;
                const uint32_t ok = mask ? __builtin_amdgcn_alignbit(batch.hi[j], batch.lo[j], w & 31) : ~0u;
                u32x4 bits = __builtin_bit_cast(u32x4, batch.in[j]);
                uint32_t changed = 0;  // words that the history or the bias list changes
                if constexpr (COUNTS) {
                    u32x4 used[kPer / 4];
                    uint32_t any = 0;
#pragma unroll
                    for (int e = 0; e < kPer / 4; ++e) {
                        used[e] = *reinterpret_cast<const u32x4*>(uses + (w - base) + 4 * e);
                        any |= used[e].x | used[e].y | used[e].z | used[e].w;
                    }
                    if (any) {
#pragma unroll
                        for (int e = 0; e < kPer; ++e) changed |= used[e / 4][e % 4] ? 1u << e : 0u;
                    }
                }
                // The others stay as they are.
                float m = mask_and_max<T>(bits, ok & ~changed);
                // Few vectors have any, and those seldom more than one, which is taken
                // by itself; where some lane has several (common words lie together),
                // all eight are formed at once.
                if (__builtin_amdgcn_ballot_w64((changed & (changed - 1)) != 0)) {
                    if (changed) {
#pragma unroll
                        for (int e = 0; e < kPer; ++e) {
                            if (!(changed & ok & 1u << e)) continue;
                            const float v = adjusted((float)batch.in[j][e], uses[w - base + e], w + e, r);
                            m = fmaxf(m, v);
                            set_element<T>(bits, e, (T)v);
                        }
                    }
                } else if (changed & ok) {
                    const int e = __builtin_ctz(changed);
                    const float v = adjusted((float)element<T>(__builtin_bit_cast(u32x4, batch.in[j]), e), uses[w - base + e], w + e, r);
                    m = fmaxf(m, v);
                    set_element<T>(bits, e, (T)v);
                }
                if (m > top) {
                    top = m;
                    word = w;
                    best = batch.in[j];
                    best_ok = ok;
                }
                __builtin_nontemporal_store(bits, gbl(reinterpret_cast<u32x4*>(y + w)));
            }
        }
        if (blockIdx.x == 0 && tid < from) one(tid);
        const int rest = from + vectors * kPer + tid;
        if (rest < end) one(rest);
    }
    if (!c.token) return;
    auto best_of_block = [&] {
        best_of_wave<64>(top, word);
        if ((tid & 63) == 0) {
            sh_v[tid >> 6] = top;
            sh_w[tid >> 6] = word;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) better(top, word, sh_v[i], sh_w[i]);
    };
    const float my_top = top;
    const int my_word = word;
    best_of_block();
    bool mine = word >= 0 && my_word == word;
    if (mine && best_ok && my_word >= from && my_word < from + vectors * kPer) {
        // Which of the vector's words it is.
        for (int e = kPer - 1; e >= 0; --e)
            if (best_ok >> e & 1) {
                const float v = COUNTS ? adjusted((float)best[e], uses[my_word - base + e], my_word + e, r) : (float)best[e];
                if (v == my_top) word = my_word + e;
            }
    }
    if (word < 0) {
        // Nothing above -infinity: the first allowed word that is not NaN, from what
        // was written.
        __syncthreads();
        for (int w = begin + tid; w < end && word < 0; w += kThreads)
            if (!mask || (mask[w >> 5] >> (w & 31) & 1)) take((float)y[w], w, true);
        best_of_block();
        mine = tid == 0;
    }
    if (mine) {
        if (p.tiles == 1) {
            c.token[row] = word;
        } else {
            p.best[row * p.tiles + blockIdx.x] = top;
            p.best_word[row * p.tiles + blockIdx.x] = word;
        }
    }
}

// The best of a row's tiles; one wave per row.
__global__ __launch_bounds__(kPickThreads) void pick_kernel(const Params p) {
    const int64_t row = blockIdx.x;
    float top = -INFINITY;
    int word = -1;
    for (int i = threadIdx.x; i < p.tiles; i += kPickThreads) better(top, word, p.best[row * p.tiles + i], p.best_word[row * p.tiles + i]);
    best_of_wave<64>(top, word);
    if (threadIdx.x == 0) p.c.token[row] = word;
}

// ------------------------------------------------------------------ host

// Words of a tile: long ones scan a history less often, short ones give every
// CU some.
int64_t tile_of(int64_t rows, int64_t vocab) {
    int64_t t = kMaxTile;
    while (t > kMinTile && rows * ((vocab + t - 1) / t) < 1024) t /= 2;
    return t;
}
int64_t tiles_of(int64_t vocab, int64_t tile) { return (vocab + tile - 1) / tile; }

size_t workspace_of(int64_t rows, int64_t vocab) {
    const int64_t tiles = tiles_of(vocab, tile_of(rows, vocab));
    return tiles > 1 ? (size_t)(rows * tiles * 8 + 15) / 16 * 16 : 0;
}

wq_status check_sizes(const char* fn, int64_t rows, int64_t vocab, int64_t dtype) {
    WQ_TRY(in_range(fn, "rows", rows, 1, WQ_LOGITS_MAX_ROWS));
    WQ_TRY(in_range(fn, "vocab", vocab, 1, WQ_LOGITS_MAX_VOCAB));
    if (dtype != WQ_DTYPE_F16 && dtype != WQ_DTYPE_BF16 && dtype != WQ_DTYPE_F32)
        return err(WQ_ERR_UNSUPPORTED, "%s: dtype must be one of WQ_DTYPE_* (got %lld)", fn, (long long)dtype);
    return WQ_OK;
}

template <typename T, bool HISTORY, bool BIAS>
void launch_as(const Params& p, bool vector, hipStream_t stream) {
    const dim3 grid((unsigned)p.tiles, (unsigned)p.c.rows);
    const size_t lds = HISTORY || BIAS ? (size_t)(p.tile + Type<T>::kPer) * 4 : 0;
    // 32 KB of logits, which only the longest tiles of fp32 have, are four 16-byte loads
    // for each of 512 lanes (256 rows of 100277 words: 48.5 us with 256 lanes, 44.7 with
    // 512).
    if constexpr (kMaxTile * sizeof(T) >= 32768) {
        if (vector && p.tile == kMaxTile) {
            hipLaunchKernelGGL((logits_kernel<T, HISTORY, BIAS, true, 512>), grid, dim3(512), lds, stream, p);
            return;
        }
    }
    if (vector) hipLaunchKernelGGL((logits_kernel<T, HISTORY, BIAS, true, 256>), grid, dim3(256), lds, stream, p);
    else hipLaunchKernelGGL((logits_kernel<T, HISTORY, BIAS, false, 256>), grid, dim3(256), lds, stream, p);
}

template <typename T>
void launch_type(const Params& p, hipStream_t stream) {
    // 16-byte accesses need input and output rows that lie alike, row by row.
    const uintptr_t apart = reinterpret_cast<uintptr_t>(p.c.logits) - reinterpret_cast<uintptr_t>(p.c.out);
    const bool vector = apart % 16 == 0 && (p.c.rows == 1 || (p.c.logits_stride - p.c.out_stride) * (int64_t)sizeof(T) % 16 == 0);
    const bool history = p.c.history != nullptr, bias = p.c.bias_ids != nullptr;
    if (history && bias) launch_as<T, true, true>(p, vector, stream);
    else if (history) launch_as<T, true, false>(p, vector, stream);
    else if (bias) launch_as<T, false, true>(p, vector, stream);
    else launch_as<T, false, false>(p, vector, stream);
}

}  // namespace
}  // namespace logits
}  // namespace wq

using namespace wq::logits;
using wq::host::aligned;
using wq::host::err;
using wq::host::in_range;
using wq::host::overlaps;
using wq::host::span;
using wq::host::Span;

extern "C" {

wq_status wq_process_logits_workspace_size(int64_t rows, int64_t vocab, int64_t dtype, size_t* bytes) {
    static const char* fn = "wq_process_logits_workspace_size";
    if (!bytes) return err(WQ_ERR_INVALID_ARG, "%s: null output pointer", fn);
    WQ_TRY(check_sizes(fn, rows, vocab, dtype));
    *bytes = workspace_of(rows, vocab);
    return WQ_OK;
}

wq_status wq_process_logits(const wq_logits_call* call, void* workspace, size_t workspace_bytes, void* stream) {
    static const char* fn = "wq_process_logits";
    if (!call || !call->logits || !call->out) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    Params p{};
    p.c = *call;
    const wq_logits_call& c = p.c;
    WQ_TRY(check_sizes(fn, c.rows, c.vocab, c.dtype));
    const int64_t size = c.dtype == WQ_DTYPE_F32 ? 4 : 2, words = (c.vocab + 31) / 32;
    constexpr int64_t kMaxStride = (int64_t)1 << 32;
    WQ_TRY(in_range(fn, "logits_stride", c.logits_stride, c.vocab, kMaxStride));
    WQ_TRY(in_range(fn, "out_stride", c.out_stride, c.vocab, kMaxStride));
    if (c.mask) WQ_TRY(in_range(fn, "mask_stride", c.mask_stride, words, kMaxStride));
    if (c.history) {
        WQ_TRY(in_range(fn, "history_size", c.history_size, 1, WQ_LOGITS_MAX_HISTORY));
    } else if (c.history_lens || c.prompt_lens || c.repetition || c.frequency || c.presence) {
        return err(WQ_ERR_INVALID_ARG, "%s: lengths and penalties need a history", fn);
    }
    if (c.bias_ids) {
        WQ_TRY(in_range(fn, "bias_size", c.bias_size, 1, WQ_LOGITS_MAX_BIAS));
        if (!c.bias_values) return err(WQ_ERR_INVALID_ARG, "%s: bias_ids without bias_values", fn);
    } else if (c.bias_values || c.bias_lens) {
        return err(WQ_ERR_INVALID_ARG, "%s: bias values or lengths without bias_ids", fn);
    }
    if (!aligned(c.logits, size) || !aligned(c.out, size)) return err(WQ_ERR_MISALIGNED, "%s: logits and out must be aligned to their elements", fn);
    const void* const fours[] = {c.token, c.mask, c.history, c.history_lens, c.prompt_lens, c.repetition, c.frequency, c.presence, c.bias_ids, c.bias_values, c.bias_lens};
    for (const void* f : fours)
        if (!aligned(f, 4)) return err(WQ_ERR_MISALIGNED, "%s: every list must be 4-byte aligned", fn);

    const uint64_t rows = (uint64_t)c.rows;
    const size_t ws = c.token ? workspace_of(c.rows, c.vocab) : 0;
    if (ws > 0) {
        if (!workspace || workspace_bytes < ws)
            return err(WQ_ERR_INVALID_ARG, "%s: a workspace of %zu bytes is needed (got %zu)", fn, ws, workspace ? workspace_bytes : (size_t)0);
        if (!aligned(workspace, 16)) return err(WQ_ERR_MISALIGNED, "%s: workspace must be 16-byte aligned", fn);
    }
    const Span out = span(c.out, ((rows - 1) * c.out_stride + c.vocab) * size), in = span(c.logits, ((rows - 1) * c.logits_stride + c.vocab) * size);
    const Span token = span(c.token, c.token ? rows * 4 : 0), work = span(workspace, ws);
    auto list = [&](const void* ptr, uint64_t bytes) { return span(ptr, ptr ? bytes : 0); };
    const Span inputs[] = {list(c.mask, ((rows - 1) * c.mask_stride + words) * 4), list(c.history, rows * c.history_size * 4), list(c.history_lens, rows * 4),
                           list(c.prompt_lens, rows * 4), list(c.repetition, rows * 4), list(c.frequency, rows * 4), list(c.presence, rows * 4),
                           list(c.bias_ids, rows * c.bias_size * 4), list(c.bias_values, rows * c.bias_size * 4), list(c.bias_lens, rows * 4)};
    for (const Span& s : inputs)
        if (overlaps(s, out) || overlaps(s, token) || overlaps(s, work)) return err(WQ_ERR_INVALID_ARG, "%s: an output or the workspace overlaps an input", fn);
    const bool in_place = c.out == c.logits && (c.out_stride == c.logits_stride || c.rows == 1);
    if ((overlaps(out, in) && !in_place) || overlaps(out, token) || overlaps(out, work) || overlaps(in, token) || overlaps(in, work) || overlaps(token, work))
        return err(WQ_ERR_INVALID_ARG, "%s: out, token and the workspace must not overlap", fn);

    p.tile = (int32_t)tile_of(c.rows, c.vocab);
    p.tiles = (int32_t)tiles_of(c.vocab, p.tile);
    p.best = static_cast<float*>(workspace);
    p.best_word = ws ? reinterpret_cast<int32_t*>(p.best + rows * p.tiles) : nullptr;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    if (c.dtype == WQ_DTYPE_F16) launch_type<_Float16>(p, st);
    else if (c.dtype == WQ_DTYPE_BF16) launch_type<__bf16>(p, st);
    else launch_type<float>(p, st);
    if (c.token && p.tiles > 1) hipLaunchKernelGGL(pick_kernel, dim3((unsigned)c.rows), dim3(kPickThreads), 0, st, p);
    return wq::host::hip_result(fn, hipGetLastError());
}

}  // extern "C"
