// Device-side building blocks of the microscaled (MX) formats: loads of eight
// values of any type, rounding of a block to E2M1 or E4M3 under a power-of-two
// scale (gfx950, wave64).
//
// A lane holds 8 consecutive elements ("piece"), four neighbouring lanes a block
// of 32, so a block's largest magnitude takes two DPP steps.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "wq_device.h"
#include "wq_mx.h"

namespace wq {
namespace mx {

using dev::gbl;
using dev::u32x4;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));

constexpr int kPiece = 8;
constexpr int kBlock = WQ_MX_BLOCK;

// Eight values as they lie in memory, and as fp32.  load_once leaves no room in the caches to what is not read again.
template <typename T>
struct Raw;
template <>
struct Raw<_Float16> {
    u32x4 v;
    __device__ __forceinline__ void load(const _Float16* p) { v = *gbl(reinterpret_cast<const u32x4*>(p)); }
    __device__ __forceinline__ void load_once(const _Float16* p) { v = __builtin_nontemporal_load(gbl(reinterpret_cast<const u32x4*>(p))); }
    __device__ __forceinline__ float8v f32() const { return __builtin_convertvector(__builtin_bit_cast(half8v, v), float8v); }
};
template <>
struct Raw<__bf16> {
    u32x4 v;
    __device__ __forceinline__ void load(const __bf16* p) { v = *gbl(reinterpret_cast<const u32x4*>(p)); }
    __device__ __forceinline__ void load_once(const __bf16* p) { v = __builtin_nontemporal_load(gbl(reinterpret_cast<const u32x4*>(p))); }
    __device__ __forceinline__ float8v f32() const {
        float8v f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, v[i] << 16);
            f[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xFFFF0000u);
        }
        return f;
    }
};
template <>
struct Raw<float> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = gbl(reinterpret_cast<const u32x4*>(p))[0];
        b = gbl(reinterpret_cast<const u32x4*>(p))[1];
    }
    __device__ __forceinline__ void load_once(const float* p) {
        a = __builtin_nontemporal_load(gbl(reinterpret_cast<const u32x4*>(p)));
        b = __builtin_nontemporal_load(gbl(reinterpret_cast<const u32x4*>(p)) + 1);
    }
    __device__ __forceinline__ float8v f32() const {
        const float4v x = __builtin_bit_cast(float4v, a), y = __builtin_bit_cast(float4v, b);
        return float8v{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    }
};

// Eight fp32 values rounded to T (nearest, ties to even) and stored.
__device__ __forceinline__ void store8(_Float16* p, float8v f) {
    *gbl(reinterpret_cast<u32x4*>(p)) = __builtin_bit_cast(u32x4, __builtin_convertvector(f, half8v));
}
__device__ __forceinline__ void store8(__bf16* p, float8v f) {
    *gbl(reinterpret_cast<u32x4*>(p)) = __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf8v));
}
__device__ __forceinline__ void store8(float* p, float8v f) {
    gbl(reinterpret_cast<u32x4*>(p))[0] = __builtin_bit_cast(u32x4, float4v{f[0], f[1], f[2], f[3]});
    gbl(reinterpret_cast<u32x4*>(p))[1] = __builtin_bit_cast(u32x4, float4v{f[4], f[5], f[6], f[7]});
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t t = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
    return v > t ? v : t;
}

// Largest magnitude of the block that this lane and its three neighbours hold,
// as the bits of an fp32 number: those of NaN and infinity are above all others.
__device__ __forceinline__ uint32_t block_max(float8v f) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = f[i];  // (The cast of a vector's element itself would be that of its first.)
        const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu;
        m = b > m ? b : m;
    }
    m = dpp_max<0xB1>(m);  // quad_perm [1,0,3,2]
    return dpp_max<0x4E>(m);  // quad_perm [2,3,0,1]
}

// The scale byte: the smallest power of two, from 2^-127 on, that brings the
// largest magnitude to 1.5 * 2^2 (FP4) or 1.75 * 2^8 (FP8) or below.  Adding what
// the type's largest mantissa lacks of the next power of two carries into the
// exponent exactly when the mantissa is larger.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t max_bits) {
    if (max_bits >= 0x7F800000u) return 255;
    const int e = (int)((max_bits + (FMT == WQ_MX_FP4 ? 0x3FFFFFu : 0x1FFFFFu)) >> 23) - (FMT == WQ_MX_FP4 ? 2 : 8);
    return (uint32_t)(e > 0 ? e : 0);
}

// 1 / scale as an exact fp32 number; 0 for a NaN scale.  Bytes come from
// scale_byte: at most 253, so the result is no denormal.
__device__ __forceinline__ float scale_inverse(uint32_t byte) {
    return byte == 255 ? 0.0f : __builtin_bit_cast(float, (254u - byte) << 23);
}

// Eight elements of one block rounded to nearest, ties to even, by the
// conversions of the hardware.  Multiplying by a power of two is exact (what
// becomes an fp32 denormal is far below half of the smallest element).  With a NaN scale
// all elements are +0.
__device__ __forceinline__ u32x2 to_fp8(float8v f, uint32_t byte) {
    const float inv = scale_inverse(byte);
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * inv, f[1] * inv, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * inv, f[3] * inv, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * inv, f[5] * inv, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6] * inv, f[7] * inv, hi, true);
    return byte == 255 ? u32x2{0, 0} : u32x2{(uint32_t)lo, (uint32_t)hi};
}
__device__ __forceinline__ uint32_t to_fp4(float8v f, uint32_t byte) {
    const float inv = scale_inverse(byte);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[0] * inv, f[1] * inv, 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[2] * inv, f[3] * inv, 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[4] * inv, f[5] * inv, 1.0f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[6] * inv, f[7] * inv, 1.0f, 3);
    return byte == 255 ? 0u : r;
}

// Rounds the lane's piece of an MX row and stores it: element `col` (a multiple
// of 8) is the piece's first.  All four lanes of a block call this together.
template <int FMT>
__device__ __forceinline__ void store_mx(uint8_t* code_row, uint8_t* scale_row, uint32_t col, float8v f) {
    const uint32_t byte = scale_byte<FMT>(block_max(f));
    if constexpr (FMT == WQ_MX_FP8) *gbl(reinterpret_cast<u32x2*>(code_row + col)) = to_fp8(f, byte);
    else *gbl(reinterpret_cast<uint32_t*>(code_row + col / 2)) = to_fp4(f, byte);
    if (col % kBlock == 0) *gbl(scale_row + col / kBlock) = (uint8_t)byte;
}

}  // namespace mx
}  // namespace wq
