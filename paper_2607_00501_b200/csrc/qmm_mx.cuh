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
#include <type_traits>

namespace qmm {
namespace mx {

constexpr int kUnitRows = 128;
constexpr int kUnitK = 256;
constexpr int kCodeBytes = kUnitRows * kUnitK / 2;

// Workspace of a product: status word; counters of tiles whose K is shared between blocks (two blocks per tile at least, so at most 74), 16 bits each; from kMxHeader
// partial sums.  The header is zero between calls.  The counters lie in the 256 bytes that every workspace with a status word keeps for it: the data of another
// operator that has used the same workspace begins behind them.
constexpr int kMxCounters = 64, kMxHeader = 1024;
static_assert(kMxCounters + 2 * (kNumSMs / 2) <= 256, "the counters share the status word's 256 bytes");

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

// 32 consecutive elements at p as fp32.  VEC: bytes per load that the row's alignment allows (32, 16, or 0: element
// by element); n < 32 elements exist (the rest read as zero).
template <typename T, int VEC> __device__ __forceinline__ void load32(const T* p, int n, float (&v)[32])
{
    constexpr int BYTES = 32 * (int)sizeof(T);
    if (VEC >= 16 && n >= 32) {
        uint32_t u[BYTES / 4];
        if (VEC == 32) {
#pragma unroll
            for (int i = 0; i < BYTES / 32; ++i) {
                const u32x8 w = ld_stream_256(reinterpret_cast<const uint8_t*>(p) + 32 * i);
#pragma unroll
                for (int k = 0; k < 8; ++k) u[8 * i + k] = w.v[k];
            }
        } else {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const uint4 w = __ldg(reinterpret_cast<const uint4*>(p) + i);
                u[4 * i] = w.x, u[4 * i + 1] = w.y, u[4 * i + 2] = w.z, u[4 * i + 3] = w.w;
            }
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 f = Dt<T>::up2(u[i]);
                v[2 * i] = f.x, v[2 * i + 1] = f.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = i < n ? Dt<T>::up(p[i]) : 0.0f;
}

// ------------------------------------------------------- quantisation of one block

// Eight fp32 -> eight e2m1 codes, first in the low nibble: nearest, ties to the even code, saturating at 6.
__device__ __forceinline__ uint32_t codes8(const float2 (&v)[4])
{
    uint32_t w;
    asm("{\n\t"
        ".reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t"
        "}\n"
        : "=r"(w)
        : "f"(v[0].x), "f"(v[0].y), "f"(v[1].x), "f"(v[1].y), "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y));
    return w;
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t as_u64(float2 v) { return *reinterpret_cast<uint64_t*>(&v); }
__device__ __forceinline__ float2 as_f2(uint64_t u) { return *reinterpret_cast<float2*>(&u); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(as_u64(a)), "l"(as_u64(b)));
    return as_f2(d);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(as_u64(a)), "l"(as_u64(b)), "l"(as_u64(c)));
    return as_f2(d);
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// max(m, |x|) that keeps a NaN.
__device__ __forceinline__ float maxabs(float m, float x)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(m), "f"(fabsf(x)));
    return d;
}
template <int N> __device__ __forceinline__ float block_amax(const float (&v)[N])
{
    float m[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < N; ++i) m[i & 3] = maxabs(m[i & 3], v[i]);
    return maxabs(maxabs(m[0], m[1]), maxabs(m[2], m[3]));
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

// Tensor scale g of an NVFP4 operand: 6 g in fp32 and its reciprocal (prepared once per thread).
struct TensorScale {
    float g, g6, r6;
    bool plain;                                            // g6 is far from the ends of the exponent range
    __device__ __forceinline__ explicit TensorScale(float scale) : g(scale), g6(6.0f * scale)
    {
        r6 = 1.0f / g6;
        plain = g6 >= 0x1p-40f && g6 <= 0x1p40f;
    }
};

// The two tensor scales a, b of a product (positive, finite) as factors of its fp32 sum, applied one after the other: sum * first * second.  Their product is one
// factor (first = 1) where it is far from the ends of the exponent range.  Elsewhere it could be infinite or lose its bits although a b sum is an fp32
// number -- sums of codes and block scales run from 2^-20 to about 2^43 -- and the two are applied in the order that keeps the step between inside the range.
struct ProductScale {
    float first, second;
    __device__ __forceinline__ ProductScale(float a, float b) : first(1.0f), second(a * b)
    {
        if (second >= 0x1p-100f && second <= 0x1p100f) return;
        const bool small = second < 1.0f;
        first = small ? fmaxf(a, b) : fminf(a, b);
        second = small ? fminf(a, b) : fmaxf(a, b);
    }
    // the first factor, on accumulators (bits of fp32)
    template <int N> __device__ __forceinline__ void apply_first(uint32_t (&v)[N]) const
    {
        if (first == 1.0f) return;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * first);
    }
};

// Correctly rounded a / b from r = rn(1 / b): q0 = a r, e = a - q0 b (exact in one FMA), q = q0 + e r; and rn(1 / b) itself from an
// approximation within an ulp, by one such step, unless b's significand is all ones (P. W. Markstein, "Computation of elementary
// functions on the IBM RISC System/6000 processor", IBM J. Res. Dev. 34, 1990).  Need b and the quotient away from the ends of the
// exponent range (a quotient that underflows is a zero code here either way).
__device__ __forceinline__ float quotient(float a, float b, float r)
{
    const float q = a * r;
    return fmaf(fmaf(-q, b, a), r, q);
}
__device__ __forceinline__ float2 quotient2(float2 a, float nb, float r)           // nb = -b
{
    const float2 q = mul2(a, both(r));
    return fma2(fma2(q, both(nb), a), both(r), q);
}
__device__ __forceinline__ float reciprocal(float b)
{
    if ((__float_as_uint(b) & 0x007FFFFFu) == 0x007FFFFFu) return 1.0f / b;
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(b));
    return fmaf(fmaf(-b, r, 1.0f), r, r);
}

// Codes of a block whose largest magnitude is amax (NaN if it holds one): FMT elements v -> FMT / 8 words, returns the scale byte.
//
// MXFP4: the quotient by a power of two is a product by its reciprocal, exactly.
// NVFP4: x / D in fp32 has to be the correctly rounded quotient, because ties are common (D has few significant
// bits) and a product by 1 / D would break them the wrong way: three operations per element, two elements per instruction.  With
// 2^-40 <= 6 g <= 2^40 and amax <= 2^40 nothing comes near the ends of the exponent range (2^-52 <= D <= 2^47 or D = 0); every other
// block takes true divisions.  8192 x 8192 bf16: 35 us, against 37.4 with a division per block and 27.8 for MXFP4.
template <int FMT> __device__ __forceinline__ uint32_t quantize_block(const float (&v)[FMT], float amax, const TensorScale& ts, uint32_t (&out)[FMT / 8])
{
    if (FMT == QMM_MXFP4) {
        const uint32_t e = __float_as_uint(amax) >> 23;                            // 127 + floor(log2 amax); 0: zero or subnormal
        const uint32_t sb = e == 255u ? 255u : e < 2u ? 0u : e - 2u;
        const float inv = sb == 255u ? 0.0f : __uint_as_float((254u - sb) << 23);  // 2^(127 - sb), sb in 0 .. 252
#pragma unroll
        for (int w = 0; w < FMT / 8; ++w) {
            float2 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = mul2(make_float2(v[8 * w + 2 * i], v[8 * w + 2 * i + 1]), both(inv));
            const uint32_t c = codes8(q);
            out[w] = sb == 255u ? 0u : c;
        }
        return sb;
    }
    if (ts.plain && amax <= 0x1p40f) {
        const uint32_t sb = (uint32_t)__nv_cvt_float_to_fp8(fminf(quotient(amax, ts.g6, ts.r6), 448.0f), __NV_SATFINITE, __NV_E4M3);
        const float D = e4m3_value(sb) * ts.g;
        const float r = D > 0.0f ? reciprocal(D) : 0.0f;                           // (D = 0: codes 0)
#pragma unroll
        for (int w = 0; w < FMT / 8; ++w) {
            float2 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = quotient2(make_float2(v[8 * w + 2 * i], v[8 * w + 2 * i + 1]), -D, r);
            out[w] = codes8(q);
        }
        return sb;
    }
    const bool finite = amax < __int_as_float(0x7F800000);
    const uint32_t sb = finite ? (uint32_t)__nv_cvt_float_to_fp8(fminf(amax / ts.g6, 448.0f), __NV_SATFINITE, __NV_E4M3) : 0x7Fu;
    const float D = e4m3_value(sb) * ts.g;
#pragma unroll 1
    for (int w = 0; w < FMT / 8; ++w) {
        float2 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = 0.0f, b = 0.0f;                                              // (v stays in registers: no indexing by the loop variable)
#pragma unroll
            for (int k = 0; k < FMT / 8; ++k)
                if (k == w) a = v[8 * k + 2 * i], b = v[8 * k + 2 * i + 1];
            q[i] = finite && D > 0.0f ? make_float2(a / D, b / D) : make_float2(0.0f, 0.0f);
        }
        const uint32_t c = codes8(q);
#pragma unroll
        for (int k = 0; k < FMT / 8; ++k)
            if (k == w) out[k] = c;
    }
    return sb;
}

// 32 elements (one MXFP4 block or two NVFP4 blocks) -> 16 bytes of codes and the scale byte(s).
template <int FMT> __device__ __forceinline__ uint4 quantize32(const float (&v)[32], const float (&amax)[32 / FMT], const TensorScale& ts, uint32_t& sb)
{
    if constexpr (FMT == QMM_MXFP4) {
        uint32_t w[4];
        sb = quantize_block<32>(v, amax[0], ts, w);
        return make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        float a[16], b[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) a[i] = v[i], b[i] = v[16 + i];
        uint32_t wa[2], wb[2];
        sb = quantize_block<16>(a, amax[0], ts, wa);
        sb |= quantize_block<16>(b, amax[1], ts, wb) << 8;
        return make_uint4(wa[0], wa[1], wb[0], wb[1]);
    }
}
template <int FMT> __device__ __forceinline__ uint4 quantize32(const float (&v)[32], const TensorScale& ts, uint32_t& sb)
{
    float m[32 / FMT];
#pragma unroll
    for (int b = 0; b < 32 / FMT; ++b) {
        float part[FMT];
#pragma unroll
        for (int i = 0; i < FMT; ++i) part[i] = v[b * FMT + i];
        m[b] = block_amax(part);
    }
    return quantize32<FMT>(v, m, ts, sb);
}

}  // namespace mx
}  // namespace qmm
