// y = x W^T of microscaled matrices on the matrix cores (gfx950, wave64).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows of W by 16 rows of x over
// 128 elements and applies both block scales.  W is its first operand, so a lane
// ends up with four neighbouring outputs of one row of y:
//   FP4   lane l holds elements 32 (l / 16) .. + 31 of row l % 16 (16 bytes)
//   FP8   lane l holds elements 16 (l / 16) .. + 15, and the same 64 further on
//   scale lane l's byte is that of row l % 16, block l / 16
//   out   lane l holds y[row l % 16 of x][rows 4 (l / 16) .. + 3 of W]
// Both kernels read the matrices as they are defined, row by row: the four lanes
// of a row take 64 consecutive bytes.
//
//   few_kernel   up to 64 rows of x: bound by the bytes of W.  A workgroup takes
//                16 or 32 rows of W whole, its waves the 512-element steps of K in
//                turn, straight from memory into the matrix cores' registers;
//                the waves' sums are added in LDS.
//   tile_kernel  more rows: bound by the matrix cores.  Tiles of both matrices go
//                from memory straight into LDS, in the order in which lanes read
//                them (no bank conflicts), two steps ahead of the products.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "wq_host.h"
#include "wq_internal.h"
#include "wq_mx_device.h"

namespace wq {
namespace mxl {
namespace {

using namespace mx;
using namespace host;

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) uint8_t lds_u8;

constexpr int kStep = 128;   // elements of one matrix instruction
constexpr int kSuper = 512;  // elements whose scales are 16 bytes of a row
constexpr int kSteps = kSuper / kStep;
constexpr uint32_t kOne = 127;  // the scale 1

struct Params {
    const uint8_t *w_codes, *w_scales, *x_codes, *x_scales;
    void* y;
    int64_t n, m, y_stride, scale_stride;
    uint32_t k, blocks;             // blocks of 32 of a row
    uint32_t tiles_n, tiles_m;      // tile_kernel
};

template <int XF>
struct Piece {  // what a lane holds of 16 rows of x for one step
    static constexpr int kRegs = XF == WQ_MX_FP8 ? 2 : 1;
    u32x4 v[kRegs];
};

template <int XF, int BW, int BX>
__device__ __forceinline__ float4v mma(u32x4 w, const Piece<XF>& x, float4v c, uint32_t sw, uint32_t sx) {
    const int4v a = __builtin_bit_cast(int4v, w);
    const int8v wide = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    const int4v b = __builtin_bit_cast(int4v, x.v[0]);
    if constexpr (XF == WQ_MX_FP8) {
        const int4v b1 = __builtin_bit_cast(int4v, x.v[1]);
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide, __builtin_shufflevector(b, b1, 0, 1, 2, 3, 4, 5, 6, 7), c, 4, 0, BW, (int)sw, BX, (int)sx);
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide, __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1), c, 4, 4, BW, (int)sw, BX, (int)sx);
    }
}

// Four neighbouring outputs of one row, those below n, rounded once.
template <typename T>
__device__ __forceinline__ void store_outputs(const Params& p, int64_t row, int64_t col, float4v v, bool whole) {
    typedef T vec __attribute__((ext_vector_type(4)));
    T* const y = static_cast<T*>(p.y) + row * p.y_stride + col;
    const vec r = __builtin_convertvector(v, vec);
    if (whole) {
        *gbl(reinterpret_cast<u32x2*>(y)) = __builtin_bit_cast(u32x2, r);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < p.n) gbl(y)[i] = r[i];
    }
}

// ------------------------------------------------------------ up to 64 rows

// TN tiles of 16 rows of W and TM of x to a workgroup of up to WAVES waves.
template <typename T, int XF, int TN, int TM, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void few_kernel(const Params p) {
    __shared__ float4v sums[WAVES][TN * TM][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    const int r = lane % 16, q = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * (TN * 16);
    const uint8_t *w[TN], *ws[TN], *x[TM], *xs[TM];
    // Rows past the end stand in for the last one: every output has sums of its own.
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        const int64_t row = std::min(n0 + i * 16 + r, p.n - 1);
        w[i] = p.w_codes + row * (p.k / 2);
        ws[i] = p.w_scales + row * p.scale_stride;
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int64_t row = std::min((int64_t)(j * 16 + r), p.m - 1);
        x[j] = p.x_codes + row * (XF == WQ_MX_FP8 ? p.k : p.k / 2);
        xs[j] = p.x_scales + row * p.scale_stride;
    }
    float4v acc[TN][TM] = {};
    const uint32_t supers = (p.blocks + 15) / 16;
    for (uint32_t s = wave; s < supers; s += waves) {
        const uint32_t left = p.blocks - s * 16;
        u32x4 sw[TN], sx[TM], wv[kSteps][TN];
        Piece<XF> xv[kSteps][TM];
#pragma unroll
        for (int i = 0; i < TN; ++i) sw[i] = *gbl(reinterpret_cast<const u32x4*>(ws[i] + s * 16));
#pragma unroll
        for (int j = 0; j < TM; ++j) sx[j] = *gbl(reinterpret_cast<const u32x4*>(xs[j] + s * 16));
        if (left >= 16) {
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                const uint32_t e = s * kSuper + t * kStep;
#pragma unroll
                for (int i = 0; i < TN; ++i) wv[t][i] = *gbl(reinterpret_cast<const u32x4*>(w[i] + (e / 2 + q * 16)));
#pragma unroll
                for (int j = 0; j < TM; ++j) {
                    if constexpr (XF == WQ_MX_FP8) {
                        xv[t][j].v[0] = *gbl(reinterpret_cast<const u32x4*>(x[j] + (e + q * 16)));
                        xv[t][j].v[1] = *gbl(reinterpret_cast<const u32x4*>(x[j] + (e + 64 + q * 16)));
                    } else {
                        xv[t][j].v[0] = *gbl(reinterpret_cast<const u32x4*>(x[j] + (e / 2 + q * 16)));
                    }
                }
            }
        } else {
            // The last blocks of a row: what lies past them counts as zeros under a scale of 1, and
            // is read from the last block instead.
            const u32x4 zero = {0, 0, 0, 0};
            auto masked = [&](const uint8_t* row, uint32_t block, uint32_t at, uint32_t bytes) {
                const uint32_t b = block < left ? block : left - 1;
                const u32x4 v = *gbl(reinterpret_cast<const u32x4*>(row + (s * 16 + b) * bytes + at));
                return block < left ? v : zero;
            };
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
#pragma unroll
                for (int i = 0; i < TN; ++i) wv[t][i] = masked(w[i], t * 4 + q, 0, 16);
#pragma unroll
                for (int j = 0; j < TM; ++j) {
                    if constexpr (XF == WQ_MX_FP8) {
                        xv[t][j].v[0] = masked(x[j], t * 4 + q / 2, q % 2 * 16, 32);
                        xv[t][j].v[1] = masked(x[j], t * 4 + 2 + q / 2, q % 2 * 16, 32);
                    } else {
                        xv[t][j].v[0] = masked(x[j], t * 4 + q, 0, 16);
                    }
                }
#pragma unroll
                for (int i = 0; i < TN; ++i) sw[i][t] = t * 4 + q < left ? sw[i][t] : kOne << q * 8;
#pragma unroll
                for (int j = 0; j < TM; ++j) sx[j][t] = t * 4 + q < left ? sx[j][t] : kOne << q * 8;
            }
        }
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j) acc[i][j] = mma<XF, 0, 0>(wv[t][i], xv[t][j], acc[i][j], sw[i][t] >> q * 8, sx[j][t] >> q * 8);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) sums[wave][i * TM + j][lane] = acc[i][j];
    __syncthreads();
    const bool vector = p.y_stride % 4 == 0 && reinterpret_cast<uintptr_t>(p.y) % 8 == 0;
    for (int o = wave; o < TN * TM; o += waves) {
        float4v v = sums[0][o][lane];
        for (int i = 1; i < waves; ++i) v += sums[i][o][lane];
        const int64_t row = o % TM * 16 + r, col = n0 + o / TM * 16 + q * 4;
        if (row < p.m && col < p.n) store_outputs<T>(p, row, col, v, vector && col + 4 <= p.n);
    }
}

// ----------------------------------------------------------------- tiles

template <typename V>
__device__ __forceinline__ V lds_read(uint32_t addr) {
    return *reinterpret_cast<__attribute__((address_space(3))) V*>((lds_u8*)(size_t)addr);
}
template <typename V>
__device__ __forceinline__ void lds_write(uint32_t addr, V v) {
    *reinterpret_cast<__attribute__((address_space(3))) V*>((lds_u8*)(size_t)addr) = v;
}

// 16 bytes per lane from base + offset straight into LDS, lane after lane.  Written
// out because the compiler would wait for every load in flight before any LDS
// read that follows its own form; the waits are written out too.
__device__ __forceinline__ void dma16(const uint8_t* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds) : "memory");
}
// All but the newest N loads of this wave are done, its LDS writes too, and so for all waves.
template <int N>
__device__ __forceinline__ void arrive() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// How BM rows of x and BN of W are multiplied by WM x WN waves.
template <int XF, int BM_, int BN_, int WM_, int WN_>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kWaves = WM * WN;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;          // tiles of 16 of a wave
    static constexpr int kXRegs = Piece<XF>::kRegs;
    static constexpr int kWBytes = BN * 64, kXBytes = BM * 64 * kXRegs;  // of a step
    static constexpr int kStage = kWBytes + kXBytes, kStages = 3;
    static constexpr int kLoads = kStage / 1024, kEach = kLoads / kWaves;  // per stage and per wave
    static constexpr int kScaleBytes = (BM + BN) * 16;                   // of kSteps steps
    static constexpr int kScaleAt = kStages * kStage;
    static constexpr int kLds = kScaleAt + 2 * kScaleBytes;
    static_assert(kLoads % kWaves == 0 && (BM + BN) / 64 <= kWaves && kLds <= 160 * 1024, "");
};

// Workgroups are dealt to the 8 XCDs in turn; give each a run of tiles, so
// that its L2 holds what they share.
__device__ __forceinline__ uint32_t xcd_run(uint32_t b, uint32_t blocks) {
    const uint32_t xcd = b % 8, per = blocks / 8, more = blocks % 8;
    return xcd * per + std::min(xcd, more) + b / 8;
}

template <typename T, int XF, typename S>
__global__ __launch_bounds__(S::kWaves * 64, 1) void tile_kernel(const Params p) {
    __shared__ __align__(16) uint8_t memory[S::kLds];
    const uint32_t lds = (uint32_t)(size_t)(lds_u8*)memory;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int r = lane % 16, q = lane / 16;
    const int wm = wave % S::WM, wn = wave / S::WM;
    // Bands of 8 tiles along x, so that a run's tiles share rows of both matrices.
    uint32_t tm, tn;
    {
        const uint32_t b = xcd_run(blockIdx.x, gridDim.x), band = 8 * p.tiles_n, first = b / band * 8;
        const uint32_t high = std::min(p.tiles_m - first, 8u), in = b % band;
        tm = first + in % high;
        tn = in / high;
    }
    const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
    const uint32_t rows_m = (uint32_t)std::min<int64_t>(p.m - m0, S::BM), rows_n = (uint32_t)std::min<int64_t>(p.n - n0, S::BN);
    const uint32_t x_row = XF == WQ_MX_FP8 ? p.k : p.k / 2, w_row = p.k / 2;
    const uint8_t* const w_base = p.w_codes + n0 * w_row;
    const uint8_t* const x_base = p.x_codes + m0 * x_row;
    const uint32_t steps = (p.blocks + 3) / 4, supers = (p.blocks + 15) / 16, last = p.blocks % 4;

    // Load i of a stage fills its bytes [1024 i, + 1024): tile i of W, or tile and half (i - BN / 16)
    // of x.  Rows past the end stand in for the last one.
    uint32_t offset[S::kEach];
    bool of_w[S::kEach];
    uint32_t half[S::kEach];
#pragma unroll
    for (int i = 0; i < S::kEach; ++i) {
        const int load = wave * S::kEach + i, xl = load - S::BN / 16;
        of_w[i] = load < S::BN / 16;
        half[i] = of_w[i] ? 0 : xl % S::kXRegs;
        const uint32_t row = of_w[i] ? std::min<uint32_t>(load * 16 + r, rows_n - 1) : std::min<uint32_t>(xl / S::kXRegs * 16 + r, rows_m - 1);
        offset[i] = row * (of_w[i] ? w_row : x_row) + half[i] * 64 + q * 16;
    }
    auto load_stage = [&](uint32_t step) {
        const uint32_t to = lds + step % S::kStages * S::kStage + wave * (S::kEach * 1024);
        if (last == 0 || step + 1 < steps) {
#pragma unroll
            for (int i = 0; i < S::kEach; ++i)
                dma16((of_w[i] ? w_base : x_base) + (int64_t)step * (of_w[i] || XF == WQ_MX_FP4 ? 64 : 128), offset[i], to + i * 1024);
        } else {
            // The last blocks of a row: what lies past them counts as zeros, and is not read.
#pragma unroll
            for (int i = 0; i < S::kEach; ++i) {
                const bool fp4 = of_w[i] || XF == WQ_MX_FP4;
                u32x4 v = {0, 0, 0, 0};
                if ((fp4 ? (uint32_t)q : half[i] * 2 + q / 2) < last)
                    v = *gbl(reinterpret_cast<const u32x4*>((of_w[i] ? w_base : x_base) + (int64_t)step * (fp4 ? 64 : 128) + offset[i]));
                lds_write(to + i * 1024 + lane * 16, v);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
    };
    // The scales of four steps: 16 bytes of every row of W, then of x.
    constexpr int kScaleLoads = (S::BM + S::BN) / 64;
    const int scale_row = wave * 64 + lane;
    const bool scale_of_w = scale_row < S::BN;
    const uint8_t* const scale_base = wave * 64 < S::BN ? p.w_scales + n0 * p.scale_stride : p.x_scales + m0 * p.scale_stride;
    const uint32_t scale_offset = (scale_of_w ? std::min<uint32_t>(scale_row, rows_n - 1) : std::min<uint32_t>(scale_row - S::BN, rows_m - 1)) * (uint32_t)p.scale_stride;
    auto load_scales = [&](uint32_t super) {
        if (wave < kScaleLoads) dma16(scale_base + super * 16, scale_offset, lds + S::kScaleAt + super % 2 * S::kScaleBytes + wave * 1024);
    };
    // Turned, so that a lane's four bytes of a row, one for each step, lie in one word.
    auto turn_scales = [&](uint32_t super) {
        if (wave < kScaleLoads) {
            const uint32_t at = lds + S::kScaleAt + super % 2 * S::kScaleBytes + wave * 1024 + lane * 16;
            u32x4 v = lds_read<u32x4>(at);
            const uint32_t left = p.blocks - super * 16;
            if (left < 16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // Bytes past the last block stand for the scale 1.
                    const uint32_t keep = left >= 4u * i + 4 ? ~0u : left <= 4u * i ? 0u : (1u << (left - 4 * i) * 8) - 1;
                    v[i] = (v[i] & keep) | (0x7F7F7F7Fu & ~keep);
                }
            }
            const uint32_t a = __builtin_amdgcn_perm(v[1], v[0], 0x05010400u), b = __builtin_amdgcn_perm(v[3], v[2], 0x05010400u),
                           c = __builtin_amdgcn_perm(v[1], v[0], 0x07030602u), d = __builtin_amdgcn_perm(v[3], v[2], 0x07030602u);
            // a: bytes 0 of steps 0 and 1, then bytes 1 of them; b: the same of steps 2 and 3; c, d: bytes 2 and 3.
            lds_write(at, u32x4{__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x05040100u),
                                __builtin_amdgcn_perm(d, c, 0x07060302u)});
        }
    };

    float4v acc[S::FN][S::FM] = {};
    load_scales(0);
    load_stage(0);
    if (steps > 1) load_stage(1);
    // (With one step fewer loads are in flight than counted here; the wait is the stricter one then.)
    if (steps > 1) arrive<2 * S::kEach>();
    else arrive<0>();
    turn_scales(0);
    for (uint32_t super = 0; super < supers; ++super) {
        uint32_t sw[S::FN], sx[S::FM];
#pragma unroll
        for (int t = 0; t < kSteps; ++t) {
            const uint32_t step = super * kSteps + t;
            if (step >= steps) break;
            if (step + 1 < steps) arrive<S::kEach>();
            else arrive<0>();
            if (t == 0 && super + 1 < supers) load_scales(super + 1);
            if (step + 2 < steps) load_stage(step + 2);
            if (t == 0) {
                const uint32_t at = lds + S::kScaleAt + super % 2 * S::kScaleBytes + r * 16 + q * 4;
#pragma unroll
                for (int i = 0; i < S::FN; ++i) sw[i] = lds_read<uint32_t>(at + (wn * S::FN + i) * 256);
#pragma unroll
                for (int j = 0; j < S::FM; ++j) sx[j] = lds_read<uint32_t>(at + S::BN * 16 + (wm * S::FM + j) * 256);
            }
            if (t == kSteps - 1 && super + 1 < supers) turn_scales(super + 1);
            const uint32_t from = lds + step % S::kStages * S::kStage + lane * 16;
            Piece<XF> xv[S::FM];
            u32x4 wv[S::FN];
#pragma unroll
            for (int j = 0; j < S::FM; ++j)
#pragma unroll
                for (int h = 0; h < S::kXRegs; ++h) xv[j].v[h] = lds_read<u32x4>(from + S::kWBytes + ((wm * S::FM + j) * S::kXRegs + h) * 1024);
#pragma unroll
            for (int i = 0; i < S::FN; ++i) wv[i] = lds_read<u32x4>(from + (wn * S::FN + i) * 1024);
            auto products = [&](auto T_) {
#pragma unroll
                for (int i = 0; i < S::FN; ++i)
#pragma unroll
                    for (int j = 0; j < S::FM; ++j) acc[i][j] = mma<XF, decltype(T_)::value, decltype(T_)::value>(wv[i], xv[j], acc[i][j], sw[i], sx[j]);
            };
            if (t == 0) products(std::integral_constant<int, 0>());
            else if (t == 1) products(std::integral_constant<int, 1>());
            else if (t == 2) products(std::integral_constant<int, 2>());
            else products(std::integral_constant<int, 3>());
        }
    }
    const bool vector = p.y_stride % 4 == 0 && reinterpret_cast<uintptr_t>(p.y) % 8 == 0;
#pragma unroll
    for (int j = 0; j < S::FM; ++j) {
        const int64_t row = m0 + (wm * S::FM + j) * 16 + r;
        if (row < p.m) {
#pragma unroll
            for (int i = 0; i < S::FN; ++i) {
                const int64_t col = n0 + (wn * S::FN + i) * 16 + q * 4;
                if (col < p.n) store_outputs<T>(p, row, col, acc[i][j], vector && col + 4 <= p.n);
            }
        }
    }
}

// ------------------------------------------------------------------ host

constexpr int64_t kFewRows = 64;

template <typename T, int XF, int TN, int TM, int WAVES>
void launch_few_as(const Params& p, hipStream_t st) {
    const int supers = (int)((p.blocks + 15) / 16);
    // As many waves as take equal numbers of steps.
    const int rounds = (supers + WAVES - 1) / WAVES, waves = (supers + rounds - 1) / rounds;
    const dim3 grid((unsigned)((p.n + TN * 16 - 1) / (TN * 16)));
    hipLaunchKernelGGL((few_kernel<T, XF, TN, TM, WAVES>), grid, dim3(waves * 64), 0, st, p);
}

template <typename T, int XF>
void launch_few(const Params& p, hipStream_t st) {
    if (p.m <= 16) launch_few_as<T, XF, 1, 1, 8>(p, st);
    else if (p.m <= 32) launch_few_as<T, XF, 1, 2, 8>(p, st);
    else if (p.m <= 48) launch_few_as<T, XF, 1, 3, 8>(p, st);
    else launch_few_as<T, XF, 1, 4, 8>(p, st);
}

template <typename T, int XF, typename S>
void launch_tiles_as(Params p, hipStream_t st) {
    p.tiles_n = (uint32_t)((p.n + S::BN - 1) / S::BN);
    p.tiles_m = (uint32_t)((p.m + S::BM - 1) / S::BM);
    hipLaunchKernelGGL((tile_kernel<T, XF, S>), dim3(p.tiles_n * p.tiles_m), dim3(S::kWaves * 64), 0, st, p);
}

int64_t tiles(int64_t n, int64_t m, int64_t bn, int64_t bm) { return (n + bn - 1) / bn * ((m + bm - 1) / bm); }

template <typename T, int XF>
void launch_tiles(const Params& p, hipStream_t st) {
    if (tiles(p.n, p.m, 256, 256) >= 192) launch_tiles_as<T, XF, Shape<XF, 256, 256, 4, 2>>(p, st);
    else if (tiles(p.n, p.m, 128, 128) >= 192) launch_tiles_as<T, XF, Shape<XF, 128, 128, 2, 2>>(p, st);
    else launch_tiles_as<T, XF, Shape<XF, 64, 64, 2, 2>>(p, st);
}

template <typename T, int XF>
void launch(const Params& p, hipStream_t st) {
    if (p.m <= kFewRows) launch_few<T, XF>(p, st);
    else launch_tiles<T, XF>(p, st);
}

wq_status check_sizes(const char* fn, int64_t n, int64_t k, int64_t m, int64_t x_format) {
    WQ_TRY(in_range(fn, "N", n, 1, WQ_MX_MAX_ROWS));
    WQ_TRY(in_range(fn, "K", k, 1, WQ_MX_MAX_COLS));
    WQ_TRY(in_range(fn, "M", m, 1, WQ_MX_MAX_ROWS));
    if (k % kBlock) return err(WQ_ERR_UNSUPPORTED, "%s: K must be a multiple of %d (got %lld)", fn, kBlock, (long long)k);
    if (x_format != WQ_MX_FP4 && x_format != WQ_MX_FP8)
        return err(WQ_ERR_UNSUPPORTED, "%s: x_format must be WQ_MX_FP4 or WQ_MX_FP8 (got %lld)", fn, (long long)x_format);
    return WQ_OK;
}

size_t workspace_of(int64_t, int64_t, int64_t, int64_t) { return 0; }

}  // namespace
}  // namespace mxl
}  // namespace wq

using namespace wq::mxl;

extern "C" {

wq_status wq_mx_linear_workspace_size(int64_t N, int64_t K, int64_t M, int64_t x_format, size_t* bytes) {
    static const char* fn = "wq_mx_linear_workspace_size";
    if (!bytes) return err(WQ_ERR_INVALID_ARG, "%s: null output pointer", fn);
    WQ_TRY(check_sizes(fn, N, K, M, x_format));
    *bytes = workspace_of(N, K, M, x_format);
    return WQ_OK;
}

wq_status wq_mx_linear(const uint8_t* w_codes, const uint8_t* w_scales, const uint8_t* x_codes, const uint8_t* x_scales, void* y, int64_t N, int64_t K,
                       int64_t M, int64_t y_stride, int64_t x_format, int64_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
    static const char* fn = "wq_mx_linear";
    if (!w_codes || !w_scales || !x_codes || !x_scales || !y) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(check_sizes(fn, N, K, M, x_format));
    if (dtype != WQ_DTYPE_F16 && dtype != WQ_DTYPE_BF16)
        return err(WQ_ERR_UNSUPPORTED, "%s: dtype must be WQ_DTYPE_F16 or WQ_DTYPE_BF16 (got %lld)", fn, (long long)dtype);
    WQ_TRY(in_range(fn, "y_stride", y_stride, N, (int64_t)1 << 32));
    for (const void* ptr : {(const void*)w_codes, (const void*)w_scales, (const void*)x_codes, (const void*)x_scales})
        if (!aligned(ptr, 16)) return err(WQ_ERR_MISALIGNED, "%s: codes and scales must be 16-byte aligned", fn);
    if (!aligned(y, 2)) return err(WQ_ERR_MISALIGNED, "%s: y must be aligned to its elements", fn);
    const size_t ws = workspace_of(N, K, M, x_format);
    if (ws > 0) {
        if (!workspace || workspace_bytes < ws)
            return err(WQ_ERR_INVALID_ARG, "%s: a workspace of %zu bytes is needed (got %zu)", fn, ws, workspace ? workspace_bytes : (size_t)0);
        if (!aligned(workspace, 16)) return err(WQ_ERR_MISALIGNED, "%s: workspace must be 16-byte aligned", fn);
    }
    const uint64_t scale_stride = WQ_MX_SCALE_STRIDE(K);
    const Span out = span(y, ((uint64_t)(M - 1) * y_stride + N) * 2), work = span(workspace, ws);
    const Span inputs[] = {span(w_codes, (uint64_t)N * K / 2), span(w_scales, N * scale_stride), span(x_codes, (uint64_t)M * (x_format == WQ_MX_FP8 ? K : K / 2)),
                           span(x_scales, M * scale_stride)};
    for (const Span& s : inputs)
        if (overlaps(s, out) || overlaps(s, work)) return err(WQ_ERR_INVALID_ARG, "%s: y or the workspace overlaps an input", fn);
    if (overlaps(out, work)) return err(WQ_ERR_INVALID_ARG, "%s: y overlaps the workspace", fn);
    const Params p{w_codes, w_scales, x_codes, x_scales, y, N, M, y_stride, (int64_t)scale_stride, (uint32_t)K, (uint32_t)(K / kBlock), 0, 0};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const bool half = dtype == WQ_DTYPE_F16;
    if (x_format == WQ_MX_FP8) half ? launch<_Float16, WQ_MX_FP8>(p, st) : launch<__bf16, WQ_MX_FP8>(p, st);
    else half ? launch<_Float16, WQ_MX_FP4>(p, st) : launch<__bf16, WQ_MX_FP4>(p, st);
    return wq::host::hip_result(fn, hipGetLastError());
}

}  // extern "C"
