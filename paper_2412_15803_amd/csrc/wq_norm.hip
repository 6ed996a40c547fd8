// The residual's addition and the root-mean-square norm of the sum, into the next
// linear's input in 16 or 32 bits and / or as an MX matrix (gfx950, wave64).
//
// One pass: a workgroup holds a row in registers, 8 values to a piece, adds the
// squares over its waves (one barrier), and writes the sum and the normalised
// values.  Every array is read or written once, which bounds large calls (8192 rows
// of 4096 bf16 with residual, sum and 8-bit result: 39 us, 6.0 TB/s; x and residual
// read past the caches, with ordinary loads 42.6); a single row is launch and one
// memory round trip.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "wq_host.h"
#include "wq_internal.h"
#include "wq_mx_device.h"
#include "wq_norm.h"

namespace wq {
namespace norm {
namespace {

using namespace mx;
using namespace host;

constexpr int kMaxThreads = 1024;
constexpr int kMaxPieces = 4;
static_assert((int64_t)kMaxThreads * kMaxPieces * kPiece >= WQ_NORM_MAX_DIM, "the longest row fits the registers of a workgroup");

struct Params {
    wq_norm_call c;
    int64_t code_stride, scale_stride;
};

// Below this mean of squares (with eps), what fp32 drops of squares under its smallest number, 2^-150 of each, may
// count: it is less than 2^-40 of this.
constexpr float kLeastMean = 0x1p-110f;
constexpr int kScaledExponent = 50;  // of a row's largest magnitude where its squares are formed anew

// One row to a workgroup of blockDim.x lanes, each holding the pieces threadIdx.x
// + i * blockDim.x.  FMT 0: no MX result.
template <typename T, int FMT, int PIECES>
__global__ __launch_bounds__(kMaxThreads) void norm_kernel(const Params p) {
    __shared__ float parts[kMaxThreads / 64], tops[kMaxThreads / 64], sums[kMaxThreads / 64];
    const wq_norm_call& c = p.c;
    const int64_t row = blockIdx.x;
    const uint32_t threads = blockDim.x, pieces = (uint32_t)c.dim / kPiece;
    const T* const x = static_cast<const T*>(c.x) + row * c.x_stride;
    const T* const r = c.residual ? static_cast<const T*>(c.residual) + row * c.residual_stride : nullptr;
    // A long row's weight is read when its sum is known, and fp32 ones are read half by half: registers hold no more.
    // (1024 rows of 32768 fp32, residual, to 8 bits: 90 us; all at once, with up to 100 registers in scratch memory, 159.
    // 2048 of binary16: 96 and 169.)
    constexpr bool kLate = PIECES == kMaxPieces;
    constexpr int kAtOnce = kLate && sizeof(T) == 4 ? 2 : PIECES;
    Raw<T> rx[PIECES], rr[PIECES], rw[PIECES];
    float8v s[PIECES];
    float sum = 0.0f;
#pragma unroll
    for (int first = 0; first < PIECES; first += kAtOnce) {
#pragma unroll
        for (int i = first; i < first + kAtOnce; ++i) {
            const uint32_t at = threadIdx.x + i * threads;
            if (at < pieces) {
                rx[i].load_once(x + at * kPiece);
                if (r) rr[i].load_once(r + at * kPiece);
                if constexpr (!kLate) rw[i].load(static_cast<const T*>(c.weight) + at * kPiece);
            }
        }
#pragma unroll
        for (int i = first; i < first + kAtOnce; ++i) {
            if (threadIdx.x + i * threads < pieces) {
                s[i] = rx[i].f32();
                if (r) s[i] += rr[i].f32();
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fmaf(s[i][j], s[i][j], sum);
            }
        }
    }
    sum = dev::segment_sum<64>(sum);
    if (threadIdx.x % 64 == 63) parts[threadIdx.x / 64] = sum;
    __syncthreads();
    // Every wave adds the waves' sums in the same order.
    const uint32_t waves = (threads + 63) / 64;
    float total = 0.0f;
    for (uint32_t w = 0; w < waves; ++w) total += parts[w];
    float mean = total / (float)c.dim + c.eps;
    // Squares that leave fp32's range: they are formed anew of s 2^up, which brings the largest magnitude of the row
    // (or the root of eps) to 2^49 .. 2^50, and the mean and its root follow.  A row of zeros without eps, and one that
    // holds an infinity, stay as they are.  (All lanes have the same mean; binary16's squares lie well inside.)
    bool scaled = false;
    if constexpr (!std::is_same<T, _Float16>::value) {
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(mean < kLeastMean || mean == INFINITY), 0)) {
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                if (threadIdx.x + i * threads < pieces) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(s[i][j]));
                }
            }
            for (int lanes = 32; lanes > 0; lanes /= 2) top = fmaxf(top, __shfl_xor(top, lanes));
            if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
            __syncthreads();
            top = sqrtf(c.eps);
            for (uint32_t w = 0; w < waves; ++w) top = fmaxf(top, tops[w]);
            scaled = __builtin_amdgcn_readfirstlane(top > 0.0f && top < INFINITY);
            if (scaled) {
                const int up = __builtin_amdgcn_readfirstlane(kScaledExponent - __builtin_amdgcn_frexp_expf(top));
                sum = 0.0f;
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    const uint32_t at = threadIdx.x + i * threads;
                    if (at < pieces) {
                        if (c.total) store8(static_cast<T*>(c.total) + row * c.total_stride + at * kPiece, s[i]);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            s[i][j] = ldexpf(s[i][j], up);
                            sum = fmaf(s[i][j], s[i][j], sum);
                        }
                    }
                }
                sum = dev::segment_sum<64>(sum);
                if (threadIdx.x % 64 == 63) sums[threadIdx.x / 64] = sum;
                __syncthreads();
                total = 0.0f;
                for (uint32_t w = 0; w < waves; ++w) total += sums[w];
                mean = total / (float)c.dim + ldexpf(c.eps, 2 * up);
            }
        }
    }
    const float inv = 1.0f / sqrtf(mean);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const uint32_t at = threadIdx.x + i * threads;
        // (Four lanes of a block are in here together: a row's pieces are a multiple of four.)
        if (at < pieces) {
            if (c.total && !scaled) store8(static_cast<T*>(c.total) + row * c.total_stride + at * kPiece, s[i]);
            if constexpr (kLate) rw[i].load(static_cast<const T*>(c.weight) + at * kPiece);
            const float8v w = rw[i].f32();
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i][j] = s[i][j] * inv * w[j];
            if (c.out) store8(static_cast<T*>(c.out) + row * c.out_stride + at * kPiece, s[i]);
            if constexpr (FMT != 0) store_mx<FMT>(c.codes + row * p.code_stride, c.scales + row * p.scale_stride, at * kPiece, s[i]);
        }
    }
}

// ------------------------------------------------------------------ host

template <typename T, int FMT>
void launch_as(const Params& p, hipStream_t stream) {
    const uint32_t pieces = (uint32_t)p.c.dim / kPiece;
    const auto threads_of = [&](uint32_t each) { return ((pieces + each - 1) / each + 63) / 64 * 64; };
    const dim3 grid((unsigned)p.c.rows);
    if (pieces <= kMaxThreads) hipLaunchKernelGGL((norm_kernel<T, FMT, 1>), grid, dim3(threads_of(1)), 0, stream, p);
    else if (pieces <= 2 * kMaxThreads) hipLaunchKernelGGL((norm_kernel<T, FMT, 2>), grid, dim3(threads_of(2)), 0, stream, p);
    else hipLaunchKernelGGL((norm_kernel<T, FMT, kMaxPieces>), grid, dim3(threads_of(kMaxPieces)), 0, stream, p);
}

template <typename T>
void launch_type(const Params& p, hipStream_t stream) {
    if (!p.c.codes) launch_as<T, 0>(p, stream);
    else if (p.c.format == WQ_MX_FP4) launch_as<T, WQ_MX_FP4>(p, stream);
    else launch_as<T, WQ_MX_FP8>(p, stream);
}

}  // namespace
}  // namespace norm
}  // namespace wq

using namespace wq::norm;

extern "C" wq_status wq_add_rmsnorm(const wq_norm_call* call, void* stream) {
    static const char* fn = "wq_add_rmsnorm";
    if (!call) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    Params p{};
    p.c = *call;
    const wq_norm_call& c = p.c;
    if (!c.x || !c.weight) return err(WQ_ERR_INVALID_ARG, "%s: null pointer", fn);
    if (!c.out && !c.codes) return err(WQ_ERR_INVALID_ARG, "%s: out or codes must be given", fn);
    if ((c.codes == nullptr) != (c.scales == nullptr)) return err(WQ_ERR_INVALID_ARG, "%s: codes and scales go together", fn);
    WQ_TRY(in_range(fn, "rows", c.rows, 1, WQ_NORM_MAX_ROWS));
    WQ_TRY(in_range(fn, "dim", c.dim, 1, WQ_NORM_MAX_DIM));
    if (c.dim % kBlock) return err(WQ_ERR_UNSUPPORTED, "%s: dim must be a multiple of %d (got %lld)", fn, kBlock, (long long)c.dim);
    if (c.dtype != WQ_DTYPE_F16 && c.dtype != WQ_DTYPE_BF16 && c.dtype != WQ_DTYPE_F32)
        return err(WQ_ERR_UNSUPPORTED, "%s: dtype must be one of WQ_DTYPE_* (got %lld)", fn, (long long)c.dtype);
    if (c.codes && c.format != WQ_MX_FP4 && c.format != WQ_MX_FP8)
        return err(WQ_ERR_UNSUPPORTED, "%s: format must be WQ_MX_FP4 or WQ_MX_FP8 (got %lld)", fn, (long long)c.format);
    if (!(std::isfinite(c.eps) && c.eps >= 0.0f)) return err(WQ_ERR_INVALID_ARG, "%s: eps must be finite and not negative", fn);
    constexpr int64_t kMaxStride = (int64_t)1 << 32;
    const struct {
        const char* name;
        const void* ptr;
        int64_t stride;
    } arrays[] = {{"x", c.x, c.x_stride}, {"residual", c.residual, c.residual_stride}, {"total", c.total, c.total_stride}, {"out", c.out, c.out_stride}};
    for (const auto& a : arrays) {
        if (!a.ptr) continue;
        if (a.stride < c.dim || a.stride > kMaxStride || a.stride % 8)
            return err(WQ_ERR_INVALID_ARG, "%s: the stride of %s must be a multiple of 8 in [dim, 2^32] (got %lld)", fn, a.name, (long long)a.stride);
        if (!aligned(a.ptr, 16)) return err(WQ_ERR_MISALIGNED, "%s: %s must be 16-byte aligned", fn, a.name);
    }
    if (!aligned(c.weight, 16) || !aligned(c.codes, 16) || !aligned(c.scales, 16))
        return err(WQ_ERR_MISALIGNED, "%s: weight, codes and scales must be 16-byte aligned", fn);
    p.code_stride = c.format == WQ_MX_FP4 ? c.dim / 2 : c.dim;
    p.scale_stride = WQ_MX_SCALE_STRIDE(c.dim);
    const uint64_t size = c.dtype == WQ_DTYPE_F32 ? 4 : 2, rows = (uint64_t)c.rows;
    const auto matrix = [&](const void* ptr, int64_t stride) { return span(ptr, ptr ? ((rows - 1) * stride + c.dim) * size : 0); };
    const Span x = matrix(c.x, c.x_stride), r = matrix(c.residual, c.residual_stride), weight = span(c.weight, c.dim * size);
    const Span outs[] = {matrix(c.total, c.total_stride), matrix(c.out, c.out_stride), span(c.codes, c.codes ? rows * p.code_stride : 0),
                         span(c.scales, c.scales ? rows * p.scale_stride : 0)};
    for (int i = 0; i < 4; ++i) {
        if (overlaps(outs[i], weight)) return err(WQ_ERR_INVALID_ARG, "%s: an output overlaps weight", fn);
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i], outs[j])) return err(WQ_ERR_INVALID_ARG, "%s: outputs overlap", fn);
        // A row's workgroup has read all of it before it writes: total and out may take an
        // input's place, row by row.
        const int64_t stride = i == 0 ? c.total_stride : c.out_stride;
        const void* const ptr = i == 0 ? c.total : i == 1 ? c.out : nullptr;
        const auto in_place = [&](const void* in, int64_t in_stride) { return ptr && ptr == in && (stride == in_stride || rows == 1); };
        if ((overlaps(outs[i], x) && !in_place(c.x, c.x_stride)) || (overlaps(outs[i], r) && !in_place(c.residual, c.residual_stride)))
            return err(WQ_ERR_INVALID_ARG, "%s: an output overlaps an input", fn);
    }
    const hipStream_t st = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    if (c.dtype == WQ_DTYPE_F16) launch_type<_Float16>(p, st);
    else if (c.dtype == WQ_DTYPE_BF16) launch_type<__bf16>(p, st);
    else launch_type<float>(p, st);
    return hip_result(fn, hipGetLastError());
}
