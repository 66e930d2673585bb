// qmm_mx.cuh -- microscaled 4-bit floating point: the packed operand and the quantisation of one block,
// shared by the quantiser, the few-token product and the gated product's epilogue.
//
// Packed operand: units of 128 rows x 256 k, one unit = the codes (16 KB, K-major rows of 128 bytes with the
// 16-byte chunks of row r permuted by r % 8: the 128-byte swizzle of the tensor core's shared-memory
// operands) followed by the scales (512-byte groups of 128 rows x 4 blocks, row r at 16 (r % 32) +
// 4 (r / 32): the order that one copy into tensor memory takes).  A unit therefore goes from HBM to the
// tensor core as one contiguous bulk copy, without tensor maps and without a pass over the scales.
#pragma once

#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "qmm_common.cuh"
#include <cuda_bf16.h>

namespace qmm {
namespace mx {

constexpr int kUnitRows = 128;
constexpr int kUnitK = 256;
constexpr int kCodeBytes = kUnitRows * kUnitK / 2;

__host__ __device__ constexpr int scale_bytes(int fmt) { return kUnitRows * kUnitK / fmt; }      // fmt = block length
__host__ __device__ constexpr int unit_bytes(int fmt) { return kCodeBytes + scale_bytes(fmt); }
__host__ __device__ inline int64_t k_units(int64_t K) { return (K + kUnitK - 1) / kUnitK; }

// Byte offset inside a unit of the 16-byte code chunk c (32 elements) of row r, and of the 4-byte scale word of
// row r in scale group j.
__device__ __forceinline__ uint32_t chunk_offset(uint32_t r, uint32_t c) { return r * 128u + ((c ^ (r & 7u)) << 4); }
__device__ __forceinline__ uint32_t scale_offset(uint32_t r, uint32_t j)
{
    return (uint32_t)kCodeBytes + j * 512u + ((r & 31u) << 4) + ((r >> 5) << 2);
}

// ------------------------------------------------------- data types

template <typename T> struct Dt;
template <> struct Dt<__half> {
    static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
    static __device__ __forceinline__ uint32_t down2(float a, float b)
    {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ float2 up2(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
};
template <> struct Dt<__nv_bfloat16> {
    static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
    static __device__ __forceinline__ uint32_t down2(float a, float b)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ float2 up2(uint32_t u)                 // a bf16 is the upper half of its fp32
    {
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
    }
};
template <> struct Dt<float> {
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};

// ------------------------------------------------------- quantisation of one block

// Two fp32 -> two e2m1 codes in a byte (first in the low nibble): nearest, ties to the even code, saturating at 6.
__device__ __forceinline__ uint32_t codes2(float a, float b)
{
    return (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest);
}

__device__ __forceinline__ float e8m0_value(uint32_t b)                       // 2^(b - 127); b = 0 is a subnormal fp32
{
    return b == 255u ? __int_as_float(0x7FFFFFFF) : __uint_as_float(b == 0u ? 0x00400000u : b << 23);
}
__device__ __forceinline__ float e4m3_value(uint32_t b)
{
    const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)b, __NV_E4M3);
    return __half2float(__half(h));
}

// Scale byte of a block from its largest magnitude, given as fp32 bits (sign cleared; a NaN's bits exceed every
// finite value's, so the integer maximum of the elements' bits is the right reduction for both).
template <int FMT> __device__ __forceinline__ uint32_t block_scale(uint32_t amax_bits, float g6)
{
    if (FMT == QMM_MXFP4) {
        const uint32_t e = amax_bits >> 23;                                    // 127 + floor(log2 amax); 0: zero or subnormal
        return e == 255u ? 255u : e < 2u ? 0u : e - 2u;
    }
    if (amax_bits >= 0x7F800000u) return 0x7Fu;
    return (uint32_t)__nv_cvt_float_to_fp8(fminf(__uint_as_float(amax_bits) / g6, 448.0f), __NV_SATFINITE, __NV_E4M3);
}

// Codes of a block: FMT elements v -> FMT / 8 words, returns the scale byte.  g = the tensor's scale, g6 = 6 g in fp32.
//
// MXFP4: the quotient by a power of two is a product by its reciprocal, exactly.
// NVFP4: x / D in fp32 has to be the correctly rounded quotient, because ties are common (D has few significant
// bits) and a product by 1 / D would break them the wrong way.  One division per block gives r = rn(1 / D); then
// q0 = x r, e = x - q0 D (exact in one FMA), q = q0 + e r is the correctly rounded quotient (P. W. Markstein,
// "Computation of elementary functions on the IBM RISC System/6000 processor", IBM J. Res. Dev. 34, 1990), three
// operations per element.  That needs D and the quotients away from the ends of the exponent range; a block with D
// outside [2^-80, 2^80] or a quotient beyond 2^80 takes true divisions (a quotient that underflows is code 0 either way).
template <int FMT> __device__ __forceinline__ uint32_t quantize_block(const float (&v)[FMT], float g, float g6, uint32_t (&out)[FMT / 8])
{
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < FMT; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    const uint32_t sb = block_scale<FMT>(amax, g6);
    if (FMT == QMM_MXFP4) {
        if (sb == 255u) {
#pragma unroll
            for (int w = 0; w < FMT / 8; ++w) out[w] = 0u;
            return sb;
        }
        const float inv = __uint_as_float((254u - sb) << 23);                  // 2^(127 - sb), sb in 0 .. 252
#pragma unroll
        for (int w = 0; w < FMT / 8; ++w) {
            uint32_t c = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) c |= codes2(v[8 * w + 2 * i] * inv, v[8 * w + 2 * i + 1] * inv) << (8 * i);
            out[w] = c;
        }
        return sb;
    }
    const float D = e4m3_value(sb) * g;
    if (sb == 0x7Fu || !(D > 0.0f)) {
#pragma unroll
        for (int w = 0; w < FMT / 8; ++w) out[w] = 0u;
        return sb;
    }
    const float r = 1.0f / D;
    const bool plain = D >= 0x1p-80f && D <= 0x1p80f && __uint_as_float(amax) * r <= 0x1p80f;
#pragma unroll
    for (int w = 0; w < FMT / 8; ++w) {
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = v[8 * w + 2 * i], b = v[8 * w + 2 * i + 1];
            float qa, qb;
            if (plain) {
                qa = a * r, qb = b * r;
                qa = fmaf(fmaf(-qa, D, a), r, qa);
                qb = fmaf(fmaf(-qb, D, b), r, qb);
            } else {
                qa = a / D, qb = b / D;
            }
            c |= codes2(qa, qb) << (8 * i);
        }
        out[w] = c;
    }
    return sb;
}

}  // namespace mx
}  // namespace qmm
