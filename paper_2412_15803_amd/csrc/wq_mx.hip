// Values to microscaled matrices and back (gfx950, wave64).
//
// Each value is read once and each code written once, which is all that bounds
// these kernels.  A lane takes a piece of 8 values, found from its number by a
// multiplication: many short workgroups keep more loads in flight than lanes with
// several pieces (2048 x 14336 gated fp16 to 8 bits: 24 us, 6.2 TB/s; 31 with four
// pieces; without non-temporal loads 25; 4096 x 14336 bf16 to 4 bits: 27.5, 32 and 29).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "wq_host.h"
#include "wq_internal.h"
#include "wq_mx_device.h"

namespace wq {
namespace mx {
namespace {

using namespace host;

constexpr int kThreads = 256;
constexpr int64_t kMaxPieces = 0x7FFFFFFF;    // of one launch

// n / d for n < 2^31: with m = ceil(2^(31 + l) / d), l = ceil(log2 d), the product
// n m is at most n / 2^(31 + l) <= 2^-l <= 1 / d above n / d in these units.
struct Divisor {
    uint32_t d, m, shift;
    explicit Divisor(uint32_t v) : d(v), m(0), shift(0) {
        while ((uint64_t(1) << shift) < v) ++shift;
        m = (uint32_t)(((uint64_t(1) << (31 + shift)) + v - 1) / v);
    }
    __device__ __forceinline__ uint32_t divide(uint32_t n) const { return (uint32_t)((uint64_t)n * m >> 31 >> shift); }
};

struct QuantizeParams {
    const void* x;
    uint8_t *codes, *scales;
    int64_t x_stride, code_stride, scale_stride;
    uint32_t cols, pieces;  // of this launch
    Divisor per_row;        // pieces of a row
};

// g / (1 + exp(-g)) u.  exp(-g) = 2^t e^r, t = -g log2(e) as it comes out and r = -g - t ln 2 what its rounding left out,
// up to 2^-18 far from 0, to first order.  Relative error in units of 2^-24: exp(-g) 7 (the hardware's exponential 2, the
// correction 1, the constant in r 4 at most), 1 + exp(-g) 1, the reciprocal 2, products 2: below 2^-20.  The exponent takes
// g in [-88, 128]: beyond, exp(-g) is 0 on one side, and on the other, from -87.34 on, the reciprocal is below the
// normal numbers, for which the hardware gives 0, and g times it -0.  (2048 x 14336 fp16
// to 8 bits, inputs from beyond the caches: 25.8 us, 25.4 with r left out.)
__device__ __forceinline__ float silu_mul(float g, float u) {
    const float a = __builtin_amdgcn_fmed3f(g, -88.0f, 128.0f), t = a * -0x1.715476p+0f, r = fmaf(t, -0x1.62e43p-1f, -a);
    const float p = __builtin_amdgcn_exp2f(t);
    return g * __builtin_amdgcn_rcpf(1.0f + fmaf(p, r, p)) * u;
}

template <typename T, int FMT, bool GATED>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const QuantizeParams p) {
    const uint32_t piece = blockIdx.x * kThreads + threadIdx.x;
    // (Pieces of a launch are a multiple of four: a block's lanes go on together.)
    if (piece >= p.pieces) return;
    const uint32_t row = p.per_row.divide(piece), col = (piece - row * p.per_row.d) * kPiece;
    const T* const x = static_cast<const T*>(p.x) + row * p.x_stride + col;
    Raw<T> a, b;
    a.load_once(x);
    if constexpr (GATED) b.load_once(x + p.cols);
    float8v f = a.f32();
    if constexpr (GATED) {
        const float8v u = b.f32();
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = silu_mul(f[j], u[j]);
    }
    store_mx<FMT>(p.codes + row * p.code_stride, p.scales + row * p.scale_stride, col, f);
}

struct DequantizeParams {
    const uint8_t *codes, *scales;
    void* out;
    int64_t out_stride, code_stride, scale_stride;
    uint32_t pieces;
    Divisor per_row;
};

template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(const DequantizeParams p) {
    const uint32_t piece = blockIdx.x * kThreads + threadIdx.x;
    if (piece >= p.pieces) return;
    const uint32_t row = p.per_row.divide(piece), col = (piece - row * p.per_row.d) * kPiece;
    const uint8_t* const at = p.codes + row * p.code_stride;
    u32x2 codes;
    if constexpr (FMT == WQ_MX_FP8) codes = *gbl(reinterpret_cast<const u32x2*>(at + col));
    else codes[0] = *gbl(reinterpret_cast<const uint32_t*>(at + col / 2));
    const uint32_t byte = *gbl(p.scales + row * p.scale_stride + col / kBlock);
    // 2^(byte - 127); that of byte 0 is a denormal, that of 255 a NaN.
    const float scale = __builtin_bit_cast(float, byte == 255 ? 0x7FC00000u : byte == 0 ? 0x00400000u : byte << 23);
    float8v f;
    if constexpr (FMT == WQ_MX_FP8) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[j], true);
            f[4 * j] = lo[0], f[4 * j + 1] = lo[1], f[4 * j + 2] = hi[0], f[4 * j + 3] = hi[1];
        }
    } else {
        const float2v q0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[0], 1.0f, 0), q1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[0], 1.0f, 1),
                      q2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[0], 1.0f, 2), q3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[0], 1.0f, 3);
        f = float8v{q0[0], q0[1], q1[0], q1[1], q2[0], q2[1], q3[0], q3[1]};
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= scale;
    store8(static_cast<T*>(p.out) + row * p.out_stride + col, f);
}

// ------------------------------------------------------------------ host

wq_status check_matrix(const char* fn, int64_t rows, int64_t cols, int64_t dtype, int64_t format) {
    WQ_TRY(in_range(fn, "rows", rows, 1, WQ_MX_MAX_ROWS));
    WQ_TRY(in_range(fn, "cols", cols, 1, WQ_MX_MAX_COLS));
    if (cols % kBlock) return err(WQ_ERR_UNSUPPORTED, "%s: cols must be a multiple of %d (got %lld)", fn, kBlock, (long long)cols);
    if (dtype != WQ_DTYPE_F16 && dtype != WQ_DTYPE_BF16 && dtype != WQ_DTYPE_F32)
        return err(WQ_ERR_UNSUPPORTED, "%s: dtype must be one of WQ_DTYPE_* (got %lld)", fn, (long long)dtype);
    if (format != WQ_MX_FP4 && format != WQ_MX_FP8) return err(WQ_ERR_UNSUPPORTED, "%s: format must be WQ_MX_FP4 or WQ_MX_FP8 (got %lld)", fn, (long long)format);
    return WQ_OK;
}

wq_status check_values(const char* fn, const char* name, const void* values, int64_t stride, int64_t least) {
    constexpr int64_t kMaxStride = (int64_t)1 << 32;
    if (stride < least || stride > kMaxStride || stride % 8)
        return err(WQ_ERR_INVALID_ARG, "%s: %s_stride must be a multiple of 8 in [%lld, 2^32] (got %lld)", fn, name, (long long)least, (long long)stride);
    if (!aligned(values, 16)) return err(WQ_ERR_MISALIGNED, "%s: %s must be 16-byte aligned", fn, name);
    return WQ_OK;
}

int64_t code_bytes(int64_t cols, int64_t format) { return format == WQ_MX_FP4 ? cols / 2 : cols; }

template <typename T>
void launch_quantize(const QuantizeParams& p, bool gated, int64_t format, hipStream_t st) {
    const dim3 grid((p.pieces + kThreads - 1) / kThreads), block(kThreads);
    if (format == WQ_MX_FP4) {
        if (gated) hipLaunchKernelGGL((quantize_kernel<T, WQ_MX_FP4, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((quantize_kernel<T, WQ_MX_FP4, false>), grid, block, 0, st, p);
    } else {
        if (gated) hipLaunchKernelGGL((quantize_kernel<T, WQ_MX_FP8, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((quantize_kernel<T, WQ_MX_FP8, false>), grid, block, 0, st, p);
    }
}

template <typename T>
void launch_dequantize(const DequantizeParams& p, int64_t format, hipStream_t st) {
    const dim3 grid((p.pieces + kThreads - 1) / kThreads), block(kThreads);
    if (format == WQ_MX_FP4) hipLaunchKernelGGL((dequantize_kernel<T, WQ_MX_FP4>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((dequantize_kernel<T, WQ_MX_FP8>), grid, block, 0, st, p);
}

}  // namespace
}  // namespace mx
}  // namespace wq

using namespace wq::mx;

extern "C" {

wq_status wq_mx_quantize(const void* x, uint8_t* codes, uint8_t* scales, int64_t rows, int64_t cols, int64_t x_stride, int64_t dtype, int64_t gated,
                         int64_t format, void* stream) {
    static const char* fn = "wq_mx_quantize";
    if (!x || !codes || !scales) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(check_matrix(fn, rows, cols, dtype, format));
    WQ_TRY(in_range(fn, "gated", gated, 0, 1));
    const int64_t width = gated ? 2 * cols : cols, size = dtype == WQ_DTYPE_F32 ? 4 : 2;
    WQ_TRY(check_values(fn, "x", x, x_stride, width));
    if (!aligned(codes, 16) || !aligned(scales, 16)) return err(WQ_ERR_MISALIGNED, "%s: codes and scales must be 16-byte aligned", fn);
    const int64_t code_stride = code_bytes(cols, format), scale_stride = WQ_MX_SCALE_STRIDE(cols);
    const Span in = span(x, (uint64_t)((rows - 1) * x_stride + width) * size), out = span(codes, (uint64_t)rows * code_stride),
               sc = span(scales, (uint64_t)rows * scale_stride);
    if (overlaps(in, out) || overlaps(in, sc) || overlaps(out, sc)) return err(WQ_ERR_INVALID_ARG, "%s: arrays overlap", fn);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    // Pieces are counted in 31 bits; a larger matrix takes more launches.
    const int64_t slab = kMaxPieces / (cols / kPiece);
    for (int64_t row = 0; row < rows; row += slab) {
        QuantizeParams p{static_cast<const uint8_t*>(x) + row * x_stride * size, codes + row * code_stride, scales + row * scale_stride, x_stride, code_stride,
                         scale_stride, (uint32_t)cols, (uint32_t)(std::min(slab, rows - row) * (cols / kPiece)), Divisor((uint32_t)(cols / kPiece))};
        if (dtype == WQ_DTYPE_F16) launch_quantize<_Float16>(p, gated, format, st);
        else if (dtype == WQ_DTYPE_BF16) launch_quantize<__bf16>(p, gated, format, st);
        else launch_quantize<float>(p, gated, format, st);
    }
    return hip_result(fn, hipGetLastError());
}

wq_status wq_mx_dequantize(const uint8_t* codes, const uint8_t* scales, void* out, int64_t rows, int64_t cols, int64_t out_stride, int64_t format,
                           int64_t dtype, void* stream) {
    static const char* fn = "wq_mx_dequantize";
    if (!codes || !scales || !out) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    WQ_TRY(check_matrix(fn, rows, cols, dtype, format));
    WQ_TRY(check_values(fn, "out", out, out_stride, cols));
    if (!aligned(codes, 16) || !aligned(scales, 16)) return err(WQ_ERR_MISALIGNED, "%s: codes and scales must be 16-byte aligned", fn);
    const int64_t code_stride = code_bytes(cols, format), scale_stride = WQ_MX_SCALE_STRIDE(cols), size = dtype == WQ_DTYPE_F32 ? 4 : 2;
    const Span to = span(out, (uint64_t)((rows - 1) * out_stride + cols) * size);
    if (overlaps(to, span(codes, (uint64_t)rows * code_stride)) || overlaps(to, span(scales, (uint64_t)rows * scale_stride)))
        return err(WQ_ERR_INVALID_ARG, "%s: out overlaps an input", fn);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    const int64_t slab = kMaxPieces / (cols / kPiece);
    for (int64_t row = 0; row < rows; row += slab) {
        DequantizeParams p{codes + row * code_stride, scales + row * scale_stride, static_cast<uint8_t*>(out) + row * out_stride * size, out_stride, code_stride,
                           scale_stride, (uint32_t)(std::min(slab, rows - row) * (cols / kPiece)), Divisor((uint32_t)(cols / kPiece))};
        if (dtype == WQ_DTYPE_F16) launch_dequantize<_Float16>(p, format, st);
        else if (dtype == WQ_DTYPE_BF16) launch_dequantize<__bf16>(p, format, st);
        else launch_dequantize<float>(p, format, st);
    }
    return hip_result(fn, hipGetLastError());
}

}  // extern "C"
