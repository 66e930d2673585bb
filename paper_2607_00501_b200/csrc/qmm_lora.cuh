// qmm_lora.cuh -- low-rank adapters beside a shared projection: rows of any mixture of adapters, forward and backward.
//
//   forward   s = A[a] x,        y  = y0  + scale[a] * B[a] s          A [n, r, K], B [n, N, r], a = idx[row]
//   backward  ds = scale[a] * B[a]^T dy,  dx = dx0 + A[a]^T ds,  dA[a] = sum ds x^T,  dB[a] = scale[a] * sum dy s^T
//
// The forward pass and dx are the same two products, a narrowing one over a row's K elements and a widening one over its N outputs, on weights laid out with either
// axis contiguous ("LAY" below).  All of them move far more bytes than the tensor cores have work (r = 16: 16 multiply-adds per element read), so what counts is that x and
// y pass through once, in wide accesses.  Few rows (lora_small_kernel): they go from global memory straight into the fragments of mma.sync; which k (n) stands at which place of a
// fragment is free as long as both operands agree, and with the orders below a lane's share of a row is one 16-byte access, without shared memory or
// transposition.  Many rows: stages of shared memory, copied asynchronously, so that more bytes are in flight than registers hold (2048 x 4096 x 28672: 85 us from registers,
// 58 from stages).  The warp-level products' rate (540 TFLOP/s measured) leaves the products 2 to 30 % of the time that the bytes take, except in the weight gradients from r = 32
// on; tcgen05 would take fp32 sums through tensor memory for a k or an n of 8 to 128, and s would still have to be split into parts by the warps.
//
// Sums are fp32.  s enters the widening product as the sum of two 16-bit numbers (high and low part) and the weight gradients as three bf16 or two tf32 ones, so that no bits of
// it are lost that matter beside fp32 sums; for fp16 the rows of s are scaled by a power of two first, or the product is one of tf32 halves (weight gradients), so that fp16's
// range does not bound s.
#pragma once

#include "qmm_async.cuh"
#include "qmm_launch.cuh"
#include "qmm_mx.cuh"

namespace qmm {
namespace lora {

using namespace mx;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kSmallRows = 512;                            // up to here the one-launch form finds an adapter's rows by itself
constexpr int kSmallBlocks = 8;                            // blocks of its clusters at most
constexpr int kTileRows = 64;                              // rows of a tile of the two-launch form (half a unit of the sort)

// ---------------------------------------------------------------- products of fragments

template <typename T> __device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d = a . b
template <typename T> __device__ __forceinline__ void mma16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma8_tf32_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma8_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// acc += d.  The tensor cores cut what does not fit a sum instead of rounding it; over a long chain of products into one accumulator that adds up (2048 rows: 2e-6 of the
// result), so short chains are added up here, where every addition is rounded to nearest.
__device__ __forceinline__ void add4(float (&acc)[4], const float (&d)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += d[i];
}
__device__ __forceinline__ uint32_t tf32(float v)
{
    uint32_t u;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(u) : "f"(v));
    return u;
}
// The halves of two registers that hold elements i and i + 1 of two rows: element (i & 1) of both, the first row's in the low half.
__device__ __forceinline__ uint32_t pair_of(uint32_t first, uint32_t second, int odd) { return __byte_perm(first, second, odd ? 0x7632 : 0x5410); }

// (hi, lo) 16-bit parts of two fp32 values.
template <typename T> __device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo)
{
    hi = Dt<T>::down2(a, b);
    const float2 f = Dt<T>::up2(hi);
    lo = Dt<T>::down2(a - f.x, b - f.y);
}

// Three bf16 parts of two fp32 values: all 24 bits.
__device__ __forceinline__ void split3(float a, float b, uint32_t& hi, uint32_t& mid, uint32_t& lo)
{
    hi = Dt<__nv_bfloat16>::down2(a, b);
    const float2 f = Dt<__nv_bfloat16>::up2(hi);
    split2<__nv_bfloat16>(a - f.x, b - f.y, mid, lo);
}

// ------------------------------------------------------------------ loads

template <bool NC> __device__ __forceinline__ uint32_t ld32(const void* p)
{
    return NC ? __ldg(reinterpret_cast<const uint32_t*>(p)) : *reinterpret_cast<const uint32_t*>(p);
}
// Eight consecutive elements of a row, from element `at` on, as four registers of T pairs; elements from `left` on are zero.  VEC: rows are 16-byte aligned and a
// multiple of 8 long, one access.  Otherwise rows start at any element: whole words with a shift by half a word where that stays inside the row, else (its ends) element by
// element.  NC: nobody writes the row meanwhile (y0 may be y).
template <typename T, bool VEC, bool NC = true> __device__ __forceinline__ void load8(const T* row, int64_t at, int left, uint32_t (&u)[4])
{
    const T* p = row + at;
    u[0] = u[1] = u[2] = u[3] = 0u;
    if (VEC) {
        if (left > 0) {
            const uint4 q = NC ? __ldg(reinterpret_cast<const uint4*>(p)) : *reinterpret_cast<const uint4*>(p);
            u[0] = q.x, u[1] = q.y, u[2] = q.z, u[3] = q.w;
        }
        return;
    }
    if (left <= 0) return;
    const bool odd = reinterpret_cast<uintptr_t>(p) & 2;
    if (left > 8 || (left == 8 && !odd)) {
        if (!odd || at > 0) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(p - (odd ? 1 : 0));
            uint32_t v[5];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = ld32<NC>(w + i);
            v[4] = odd ? ld32<NC>(w + 4) : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = __funnelshift_r(v[i], v[i + 1], odd ? 16 : 0);
            return;
        }
    }
    const unsigned short* e = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t a = 0u, b = 0u;
        if (2 * i < left) a = NC ? __ldg(e + 2 * i) : e[2 * i];
        if (2 * i + 1 < left) b = NC ? __ldg(e + 2 * i + 1) : e[2 * i + 1];
        u[i] = a | (b << 16);
    }
}
// R8 consecutive elements (1, 2, 4, 8 or 16) of a weight row of r contiguous ones; (R8 + 1) / 2 registers, a single element in the low half.
template <typename T, int R8, bool VEC> __device__ __forceinline__ void load_r(const T* p, bool there, uint32_t (&u)[(R8 + 1) / 2])
{
#pragma unroll
    for (int i = 0; i < (R8 + 1) / 2; ++i) u[i] = 0u;
    if (!there) return;
    const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
    if constexpr (R8 == 1) {
        u[0] = __ldg(s);
    } else if (!VEC) {
#pragma unroll
        for (int i = 0; i < R8 / 2; ++i) u[i] = (uint32_t)__ldg(s + 2 * i) | ((uint32_t)__ldg(s + 2 * i + 1) << 16);
    } else if constexpr (R8 == 2) {
        u[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
    } else if constexpr (R8 == 4) {
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
        u[0] = q.x, u[1] = q.y;
    } else {
#pragma unroll
        for (int i = 0; i < R8 / 8; ++i) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(p) + i);
            u[4 * i] = q.x, u[4 * i + 1] = q.y, u[4 * i + 2] = q.z, u[4 * i + 3] = q.w;
        }
    }
}

// Four codes of a row of 8 bits as two registers of T pairs: exact in both types.
template <typename T> __device__ __forceinline__ void values4(uint32_t w, int int8, uint32_t& lo, uint32_t& hi)
{
    __half2 a, b;
    if (int8) {
        __half2 q[2];
        q8_word_to_h2(w ^ 0x80808080u, q);
        a = q[0], b = q[1];
    } else {
        uint32_t x, y;
        asm("{\n\t.reg .b16 p, q;\n\tmov.b32 {p, q}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, p;\n\tcvt.rn.f16x2.e4m3x2 %1, q;\n\t}" : "=r"(x), "=r"(y) : "r"(w));
        a = as_h2(x), b = as_h2(y);
    }
    if constexpr (std::is_same<T, __half>::value) {
        lo = as_u32(a), hi = as_u32(b);
    } else {
        const float2 f = __half22float2(a), g = __half22float2(b);
        lo = Dt<T>::down2(f.x, f.y), hi = Dt<T>::down2(g.x, g.y);
    }
}
// A lane's eight elements of x as loaded: 16-bit pairs, or eight codes.
template <typename T, bool X8, bool VEC> struct XPiece {
    uint32_t u[X8 ? 2 : 4];
    __device__ __forceinline__ void load(const void* row, int64_t k, int left)                // row: null reads as zero
    {
        if (!row) left = 0;
        if constexpr (!X8) {
            load8<T, VEC>((const T*)row, k, left, u);
        } else if (VEC) {
            const uint2 q = left > 0 ? __ldg(reinterpret_cast<const uint2*>((const uint8_t*)row + k)) : make_uint2(0u, 0u);
            u[0] = q.x, u[1] = q.y;
        } else {
            const uint8_t* e = (const uint8_t*)row + k;
            const int off = (int)(reinterpret_cast<uintptr_t>(e) & 3);
            u[0] = u[1] = 0u;
            if (off == 0 ? left >= 8 : left >= 12 && k >= 4) {                 // words that lie inside the row
                const uint32_t* w = reinterpret_cast<const uint32_t*>(e - off);
                const uint32_t v[3] = {ld32<true>(w), ld32<true>(w + 1), off ? ld32<true>(w + 2) : 0u};
                u[0] = __funnelshift_r(v[0], v[1], 8 * off), u[1] = __funnelshift_r(v[1], v[2], 8 * off);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) u[i >> 2] |= (uint32_t)__ldg(e + i) << (8 * (i & 3));
            }
        }
    }
    __device__ __forceinline__ void pairs(int int8, uint32_t (&v)[4]) const
    {
        if constexpr (X8) {
            values4<T>(u[0], int8, v[0], v[1]);
            values4<T>(u[1], int8, v[2], v[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = u[i];
        }
    }
};

// ------------------------------------------------------------------ the narrowing product

// acc += rows . w1 over the chunks c0, c0 + step, ... < c1 of 32 elements, for MW tiles of 16 rows.  Lane (g, t) = (lane / 4, lane % 4) holds elements 8 t .. 8 t + 7 of
// a chunk for rows g and g + 8 of each tile: two k-steps of the MMA.
//   LAY 0: w1 [R, K], column c of accumulator tile i = rank 8 i + c;  LAY 1: w1 [K, R], rank c (R / 8) + i
// row[m][h]: row g + 8 h of tile m, or null.
template <typename T, bool X8, int R, int LAY, bool VEC, int MW>
__device__ __forceinline__ void narrow(float (&acc)[MW][R / 8][4], const void* const (&row)[MW][2], const T* __restrict__ w1, int K, int int8, int c0, int c1, int step,
                                       int lane)
{
    constexpr int R8 = R / 8;
    // chunks a round; the next round's are on their way during the products of this one
    constexpr int U = MW == 1 ? (R <= 64 ? 4 : 2) : (R <= 32 ? 2 : 1);
    const int g = lane >> 2, t = lane & 3;
    XPiece<T, X8, VEC> x[U][MW][2];
    auto fetch = [&](int c) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (c + u * step) * 32 + 8 * t;
            const int left = c + u * step < c1 ? K - k : 0;
#pragma unroll
            for (int m = 0; m < MW; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) x[u][m][h].load(row[m][h], k, left);
        }
    };
    fetch(c0);
    for (int c = c0; c < c1; c += step * U) {
        XPiece<T, X8, VEC> now[U][MW][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < MW; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) now[u][m][h] = x[u][m][h];
        fetch(c + step * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (c + u * step) * 32 + 8 * t;
            const int left = c + u * step < c1 ? K - k : 0;
            uint32_t a[MW][2][4];
#pragma unroll
            for (int m = 0; m < MW; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) now[u][m][h].pairs(int8, a[m][h]);
            if constexpr (LAY == 0) {
#pragma unroll
                for (int i = 0; i < R8; ++i) {
                    uint32_t w[4];
                    load8<T, VEC>(w1 + (int64_t)(8 * i + g) * K, k, left, w);
#pragma unroll
                    for (int m = 0; m < MW; ++m)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t f[4] = {a[m][0][2 * j], a[m][1][2 * j], a[m][0][2 * j + 1], a[m][1][2 * j + 1]};
                            mma16<T>(acc[m][i], f, w[2 * j], w[2 * j + 1]);
                        }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t w[4][(R8 + 1) / 2];
#pragma unroll
                    for (int q = 0; q < 4; ++q) load_r<T, R8, VEC>(w1 + (int64_t)(k + 4 * j + q) * R + g * R8, 4 * j + q < left, w[q]);
#pragma unroll
                    for (int i = 0; i < R8; ++i) {
                        const uint32_t b0 = pair_of(w[0][i >> 1], w[1][i >> 1], i & 1), b1 = pair_of(w[2][i >> 1], w[3][i >> 1], i & 1);
#pragma unroll
                        for (int m = 0; m < MW; ++m) {
                            const uint32_t f[4] = {a[m][0][2 * j], a[m][1][2 * j], a[m][0][2 * j + 1], a[m][1][2 * j + 1]};
                            mma16<T>(acc[m][i], f, b0, b1);
                        }
                    }
                }
            }
        }
    }
}
// The accumulators of one tile into shared memory [16][R].
template <int R, int LAY> __device__ __forceinline__ void put_narrow(const float (&acc)[R / 8][4], float* out, int lane)
{
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int i = 0; i < R / 8; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int j = LAY == 0 ? 8 * i + 2 * t + c : (2 * t + c) * (R / 8) + i;
            out[g * R + j] = acc[i][c];
            out[(g + 8) * R + j] = acc[i][2 + c];
        }
}

// ------------------------------------------------------------------ the widening product

// Rows of u = scale * s as two 16-bit parts in shared memory, for the fragments below: [rows][R] each, rows padded by 16 bytes.
template <int R> constexpr int u_pitch = 2 * R + 16;

// One row's share of four ranks j .. j + 3 (R / 4 neighbouring lanes hold a row): parts into shared memory, the row's factor into `back`.
// fp16: the row is scaled by a power of two so that its largest element lies in [1, 2).  bf16 has fp32's range.
template <typename T, int R> __device__ __forceinline__ void put_u(const float (&v)[4], uint8_t* hi, uint8_t* lo, float* back, int row, int j)
{
    float f[4] = {v[0], v[1], v[2], v[3]};
    if constexpr (std::is_same<T, __half>::value) {
        float m = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));
#pragma unroll
        for (int o = 1; o < R / 4; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const int e = min(max((int)(__float_as_uint(m) >> 23), 2), 252);                      // biased exponent, so that both factors are ordinary numbers
        const float down = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] *= down;
        if (j == 0) back[row] = __uint_as_float((uint32_t)e << 23);
    } else if (j == 0) {
        back[row] = 1.0f;
    }
    uint2 h, l;
    split2<T>(f[0], f[1], h.x, l.x);
    split2<T>(f[2], f[3], h.y, l.y);
    *reinterpret_cast<uint2*>(hi + row * u_pitch<R> + 2 * j) = h;
    *reinterpret_cast<uint2*>(lo + row * u_pitch<R> + 2 * j) = l;
}

// Fragments of u for k-step ks (16 ranks) of tile m.  LAY 0: lane t holds ranks 4 t .. 4 t + 3 of the step (R >= 32: of 8 t .. 8 t + 7 of two steps, the first four in the
// even one); LAY 1: ranks 2 t, 2 t + 1 and 2 t + 8, 2 t + 9.  R = 8: the missing ranks are zero.
template <int R, int LAY> __device__ __forceinline__ void get_u(const uint8_t* part, int m, int ks, int lane, uint32_t (&a)[4])
{
    const int g = lane >> 2, t = lane & 3;
    const uint8_t* r0 = part + (m * 16 + g) * u_pitch<R>;
    const uint8_t* r1 = r0 + 8 * u_pitch<R>;
    if constexpr (LAY == 0) {
        int at = 16 * ks + 4 * t;
        if (R >= 32) at = 32 * (ks >> 1) + 8 * t + 4 * (ks & 1);
        if (R == 8) {
            const bool in = t < 2;
            const uint2 p = in ? *reinterpret_cast<const uint2*>(r0 + 2 * at) : make_uint2(0u, 0u);
            const uint2 q = in ? *reinterpret_cast<const uint2*>(r1 + 2 * at) : make_uint2(0u, 0u);
            a[0] = p.x, a[2] = p.y, a[1] = q.x, a[3] = q.y;
        } else {
            const uint2 p = *reinterpret_cast<const uint2*>(r0 + 2 * at), q = *reinterpret_cast<const uint2*>(r1 + 2 * at);
            a[0] = p.x, a[2] = p.y, a[1] = q.x, a[3] = q.y;
        }
    } else {
        a[0] = *reinterpret_cast<const uint32_t*>(r0 + 2 * (16 * ks + 2 * t));
        a[1] = *reinterpret_cast<const uint32_t*>(r1 + 2 * (16 * ks + 2 * t));
        a[2] = R == 8 ? 0u : *reinterpret_cast<const uint32_t*>(r0 + 2 * (16 * ks + 2 * t + 8));
        a[3] = R == 8 ? 0u : *reinterpret_cast<const uint32_t*>(r1 + 2 * (16 * ks + 2 * t + 8));
    }
}

// Column groups of the widening product: 32 (LAY 0) or 64 (LAY 1) columns.  A lane ends up with OWN consecutive columns of a row, from OWN t on.
//   LAY 0: w2 [N, R]; column c of tile i (of 4) = 8 (c / 2) + 2 i + c % 2;   LAY 1: w2 [R, N]; column c of tile i (of 8) = 8 c + i
template <int LAY> struct Wide {
    static constexpr int cols = LAY == 0 ? 32 : 64;
    static constexpr int tiles = LAY == 0 ? 4 : 8;
    static constexpr int own = cols / 4;
};

// Weights of a column group for one block of ranks: two k-steps (LAY 0, R >= 32) or one.
template <typename T, int R, int LAY, bool VEC> struct WideBlock {
    static constexpr int steps = LAY == 0 && R >= 32 ? 2 : 1;
    static constexpr int blocks = (R < 16 ? 16 : R) / 16 / steps;
    uint32_t b[steps][Wide<LAY>::tiles][2];
    // column group from column n0; w2 of the adapter, N columns; q: which block
    __device__ __forceinline__ void load(const T* __restrict__ w2, int n0, int N, int q, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
        if constexpr (LAY == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = n0 + 8 * (g >> 1) + 2 * i + (g & 1);
                const T* p = w2 + (int64_t)n * R;
                const bool there = n < N;
                if constexpr (R >= 32) {
                    uint32_t u[4];
                    load8<T, VEC>(p, 32 * q + 8 * t, there ? R - (32 * q + 8 * t) : 0, u);
                    b[0][i][0] = u[0], b[0][i][1] = u[1];
                    b[1][i][0] = u[2], b[1][i][1] = u[3];
                } else {
                    uint32_t u[2];
                    load_r<T, 4, VEC>(p + 4 * t, there && (R == 16 || t < 2), u);
                    b[0][i][0] = u[0], b[0][i][1] = u[1];
                }
            }
        } else {
            uint32_t u[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int j = 16 * q + 2 * t + (k & 1) + 8 * (k >> 1);
                const int left = j < R ? N - (n0 + 8 * g) : 0;
                load8<T, VEC>(w2 + (int64_t)j * N, n0 + 8 * g, left, u[k]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                b[0][i][0] = pair_of(u[0][i >> 1], u[1][i >> 1], i & 1);
                b[0][i][1] = pair_of(u[2][i >> 1], u[3][i >> 1], i & 1);
            }
        }
    }
};
// All of a group's weights in registers, or, for high ranks, none of them: each row tile reads them again (from L1) block by block.
template <typename T, int R, int LAY, bool VEC> struct WideWeights {
    using Block = WideBlock<T, R, LAY, VEC>;
    static constexpr bool held = LAY == 0 ? R <= 64 : R <= 32;
    Block block[held ? Block::blocks : 1];
    const T* w2;
    int n0, N;
    __device__ __forceinline__ void load(const T* __restrict__ w, int first, int width, int lane)
    {
        w2 = w, n0 = first, N = width;
        if constexpr (held) {
#pragma unroll
            for (int q = 0; q < Block::blocks; ++q) block[q].load(w, first, width, q, lane);
        }
    }
};

// A lane's share of two rows (g, g + 8) of y0 as loaded.
template <typename T, int LAY, bool VEC> struct YPiece {
    static constexpr int regs = Wide<LAY>::own / 2;
    uint32_t u[2][regs];
    __device__ __forceinline__ void load(const T* y0, int64_t ld, const int (&row)[2], int n, int N)           // n: first column of the lane
    {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < regs; i += 4) {
                uint32_t v[4];
                load8<T, VEC, false>(y0 + row[h] * ld, n + 2 * i, y0 && row[h] >= 0 ? N - (n + 2 * i) : 0, v);
#pragma unroll
                for (int k = 0; k < 4; ++k) u[h][i + k] = v[k];
            }
    }
};
template <typename T, bool VEC> __device__ __forceinline__ void store8(T* p, int left, const uint32_t (&u)[4])
{
    if (VEC) {
        if (left > 0) *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
        return;
    }
    unsigned short* s = reinterpret_cast<unsigned short*>(p);
    if (left >= 8 && !(reinterpret_cast<uintptr_t>(p) & 2)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(p)[i] = u[i];
    } else if (left >= 8) {                                // an element, three words, an element
        s[0] = (unsigned short)u[0];
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<uint32_t*>(s + 1 + 2 * i) = __funnelshift_r(u[i], u[i + 1], 16);
        s[7] = (unsigned short)(u[3] >> 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) s[i] = (unsigned short)(u[i >> 1] >> (16 * (i & 1)));
    }
}

// y = rn(y0 + back * (u . w2)) for the 16 rows of tile m and one column group; to: the lane's columns of rows g and g + 8 of the tile (null: none), `left` columns from there.
template <typename T, int R, int LAY, bool VEC>
__device__ __forceinline__ void widen_at(WideWeights<T, R, LAY, VEC>& w, const YPiece<T, LAY, VEC>& y0, const uint8_t* hi, const uint8_t* lo, const float* back, int m,
                                         T* const (&to)[2], int left, int lane)
{
    using W = WideWeights<T, R, LAY, VEC>;
    constexpr int tiles = Wide<LAY>::tiles, steps = W::Block::steps;
    float acc[tiles][4];
#pragma unroll
    for (int i = 0; i < tiles; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;
    auto product = [&](const typename W::Block& b, int q) {
#pragma unroll
        for (int s = 0; s < steps; ++s) {
            uint32_t a[4];
            get_u<R, LAY>(lo, m, q * steps + s, lane, a);
#pragma unroll
            for (int i = 0; i < tiles; ++i) mma16<T>(acc[i], a, b.b[s][i][0], b.b[s][i][1]);
            get_u<R, LAY>(hi, m, q * steps + s, lane, a);
#pragma unroll
            for (int i = 0; i < tiles; ++i) mma16<T>(acc[i], a, b.b[s][i][0], b.b[s][i][1]);
        }
    };
    if constexpr (W::held) {
#pragma unroll
        for (int q = 0; q < W::Block::blocks; ++q) product(w.block[q], q);
    } else {
#pragma unroll 1
        for (int q = 0; q < W::Block::blocks; ++q) {
            w.block[0].load(w.w2, w.n0, w.N, q, lane);
            product(w.block[0], q);
        }
    }
    const int g = lane >> 2;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float f = back[m * 16 + g + 8 * h];
        if (!to[h]) continue;
#pragma unroll
        for (int i = 0; i < YPiece<T, LAY, VEC>::regs; i += 4) {
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 b = Dt<T>::up2(y0.u[h][i + k]);
                // columns 2 (i + k), 2 (i + k) + 1 of the lane's share
                float c0, c1;
                if constexpr (LAY == 0) c0 = acc[k][2 * h], c1 = acc[k][2 * h + 1];
                else c0 = acc[2 * k][2 * h + (i >> 2)], c1 = acc[2 * k + 1][2 * h + (i >> 2)];
                o[k] = Dt<T>::down2(fmaf(f, c0, b.x), fmaf(f, c1, b.y));
            }
            store8<T, VEC>(to[h] + 2 * i, left - 2 * i, o);
        }
    }
}
template <typename T, int R, int LAY, bool VEC>
__device__ __forceinline__ void widen(WideWeights<T, R, LAY, VEC>& w, const YPiece<T, LAY, VEC>& y0, const uint8_t* hi, const uint8_t* lo, const float* back, int m,
                                      T* y, int64_t ld, const int (&row)[2], int n, int N, int lane)
{
    T* const to[2] = {row[0] >= 0 ? y + row[0] * ld + n : nullptr, row[1] >= 0 ? y + row[1] * ld + n : nullptr};
    widen_at<T, R, LAY, VEC>(w, y0, hi, lo, back, m, to, N - n, lane);
}

// ------------------------------------------------------------------ copies into shared memory

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// ------------------------------------------------------------------ kernels

struct LoraP {
    const void* x;
    int64_t ldx;
    const float* x_scale;                                  // of rows of 8 bits, null: x has type T
    int int8;
    const int *idx, *order, *offsets, *units;
    int T, n, K, N;
    const void *w1, *w2;
    const float* scale;                                    // [n] or null
    const void* y0;                                        // null: zeros
    int64_t ldy0;
    void* y;
    int64_t ldy;
    float* s;                                              // [T, R]
    int s_scaled;                                          // what s keeps: 0 the narrowing product, 1 that times scale
    int rest;                                              // rows without an adapter get y0 (0: they have it already)
    int words;                                             // operands whose rows begin at whole words: 1 x, 2 w1, 4 y0, 8 w2
};
// A piece of 16 bytes of which `bytes` exist, by words: for rows that begin at whole words.  safe: any valid address of a whole word (a copy of no bytes needs an aligned one too).
__device__ __forceinline__ void async_words(uint32_t to, const void* from, int bytes, const void* safe)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = min(max(bytes - 4 * i, 0), 4);
        async4(to + 4 * i, n ? (const char*)from + 4 * i : safe, n);
    }
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float4 remote4(const float* p, int rank)
{
    uint32_t at = (uint32_t)__cvta_generic_to_shared(p), there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(there) : "memory");
    return v;
}

__device__ __forceinline__ void send4(float* p, int rank, float4 v)
{
    uint32_t at = (uint32_t)__cvta_generic_to_shared(p), there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(there), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// The blocks' four numbers at p (shared memory), added in block order; up to 16 blocks, the loads of eight in flight at once.
__device__ __forceinline__ float4 cluster_sum4(const float* p, int size)
{
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (8 * half >= size) break;
        float4 r[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) r[k] = 8 * half + k < size ? remote4(p, 8 * half + k) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < 8; ++k) v.x += r[k].x, v.y += r[k].y, v.z += r[k].z, v.w += r[k].w;
    }
    return v;
}

__device__ __forceinline__ float cluster_sum1(const float* p, int size)
{
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(p);
    float r[8], v = 0.0f;                                  // (weight gradients: eight blocks at most)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        r[k] = 0.0f;
        if (k < size) {
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(k));
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(r[k]) : "r"(there) : "memory");
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v += r[k];
    return v;
}

// Part `rank` of `size` of n things: [first, last).
__device__ __forceinline__ void share_of(int n, int rank, int size, int& first, int& last)
{
    first = (int)((int64_t)n * rank / size);
    last = (int)((int64_t)n * (rank + 1) / size);
}

// Shares of a long line: the first n % size are one longer.  One division for all of them.
struct LineShares {
    int64_t each;
    int more;
    __device__ __forceinline__ LineShares(int64_t n, int size)
    {
        each = n <= 0xFFFFFFFFll ? (int64_t)((uint32_t)n / (uint32_t)size) : n / size;
        more = (int)(n - each * size);
    }
    __device__ __forceinline__ int64_t begin(int k) const { return each * k + min(k, more); }
};

// Copies columns [n0, n1) of a row of y0 (null: zeros) to y, by one warp.
template <typename T, bool VEC> __device__ __forceinline__ void copy_row(const LoraP& p, int row, int n0, int n1, int lane)
{
    for (int n = n0 + 8 * lane; n < n1; n += 256) {
        uint32_t u[4];
        load8<T, VEC, false>((const T*)p.y0 + row * p.ldy0, n, p.y0 ? n1 - n : 0, u);
        store8<T, VEC>((T*)p.y + row * p.ldy + n, n1 - n, u);
    }
}

// Bound by latency: the adapter's rows, x and the weights, the meeting (behind which the second product's weights are asked for where R > 32), y.  16 x 8192 x 2048 of 16 adapters 6.6 us
// on the GPU (5 MB: 0.8 us), 77 x 2048 x 2048 of five at r = 64 10.2 us.
// Both products of up to 16 rows of one adapter by a cluster of blocks: each takes a share of K, the shares' sums meet through distributed shared memory, and each takes
// a share of N.  One launch: for a decode step two, and a sort before them, would cost as much as all their work.
//   groups 0: cluster b is there for row b; it does something if row b is the first, 17th, ... of its adapter's rows, and then takes 16 of them
//   groups > 0 (so many clusters, fewer than rows): cluster c takes the c-th group of 16 rows in the order of the adapters, which it counts
template <typename T, bool X8, int R, int LAY, bool VEC>
__global__ void __launch_bounds__(kThreads) lora_small_kernel(const LoraP p, int groups)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(128) uint8_t smem[];
    float* part = reinterpret_cast<float*>(smem);          // [kWarps][16][R]
    float* shares = part + kWarps * 16 * R;                // [kSmallBlocks][16][R]: the blocks' sums over their shares of K
    uint8_t* hi = reinterpret_cast<uint8_t*>(shares + kSmallBlocks * 16 * R);
    uint8_t* lo = hi + 16 * u_pitch<R>;
    constexpr int Q = kSmallRows / kThreads;               // rows of a thread: tid + q kThreads
    __shared__ float back[16];
    __shared__ int rows[16], before[Q * kWarps], first_of, adapter;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_rank(), size = (int)cluster_size();
    const int b = blockIdx.x / size;
    cluster_arrive();                                      // (the others' shared memory may be written once they have all begun)
    int n0, n1;
    constexpr int G = Wide<LAY>::cols;
    share_of((p.N + G - 1) / G, rank, size, n0, n1);
    if (!p.y) n1 = n0;                                     // s alone is wanted
    int id[Q], a = -1, first = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        id[q] = tid + q * kThreads < p.T ? __ldg(p.idx + tid + q * kThreads) : -1;
        if (id[q] >= p.n) id[q] = -1;
    }
    if (tid < 16) rows[tid] = -1;
    if (groups == 0) {
        a = __ldg(p.idx + b);
        if (a < 0 || a >= p.n) {                           // (the whole cluster)
            if (p.rest)
                for (int c = n0 + warp; c < n1; c += kWarps) copy_row<T, VEC>(p, b, c * G, min(c * G + G, p.N), lane);
            cluster_wait();
            return;
        }
    } else {
        int* count = reinterpret_cast<int*>(smem);         // rows of each adapter (4 KB, over the parts)
        for (int i = tid; i < 1024; i += kThreads) count[i] = 0;
        if (tid == 0) adapter = -1;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (id[q] >= 0) atomicAdd(&count[id[q]], 1);   // (a count: order does not matter)
        __syncthreads();
        const int4 c = reinterpret_cast<const int4*>(count)[tid];
        const int g0 = (c.x + 15) >> 4, g1 = g0 + ((c.y + 15) >> 4), g2 = g1 + ((c.z + 15) >> 4), g3 = g2 + ((c.w + 15) >> 4);
        int end = g3;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, end, o);
            if (lane >= o) end += v;
        }
        if (lane == 31) before[warp] = end;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            if (w < warp) end += before[w];
        const int at = b - (end - g3);                     // group b among this thread's
        if (at >= 0 && at < g3) {
            const int k = at < g0 ? 0 : at < g1 ? 1 : at < g2 ? 2 : 3;
            adapter = 4 * tid + k;
            first_of = 16 * (at - (k == 0 ? 0 : k == 1 ? g0 : k == 2 ? g1 : g2));
        }
        if (p.rest) {                                      // the rows without an adapter, dealt to the clusters
            for (int r = b; r < p.T; r += groups) {
                const int e = __ldg(p.idx + r);
                if (e < 0 || e >= p.n)
                    for (int cc = n0 + warp; cc < n1; cc += kWarps) copy_row<T, VEC>(p, r, cc * G, min(cc * G + G, p.N), lane);
            }
        }
        __syncthreads();
        a = adapter;
        if (a < 0) {                                       // (the whole cluster)
            cluster_wait();
            return;
        }
        first = first_of;
    }
    // the rows' places among their adapter's
    int mine[Q];
    unsigned same[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        same[q] = __ballot_sync(0xFFFFFFFFu, id[q] == a);
        if (lane == 0) before[q * kWarps + warp] = __popc(same[q]);
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        mine[q] = __popc(same[q] & ((1u << lane) - 1u));
#pragma unroll
        for (int w = 0; w < Q * kWarps; ++w)
            if (w < q * kWarps + warp) mine[q] += before[w];
    }
    if (groups == 0) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
            if (tid + q * kThreads == b) first_of = mine[q];
        __syncthreads();
        first = first_of;
        if (first & 15) {                                  // (the whole cluster)
            cluster_wait();
            return;
        }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
        if (id[q] == a && mine[q] >= first && mine[q] < first + 16) rows[mine[q] - first] = tid + q * kThreads;
    __syncthreads();

    const int g = lane >> 2, t = lane & 3;
    const int row[2] = {rows[g], rows[g + 8]};
    const T* w1 = (const T*)p.w1 + (int64_t)a * R * p.K;
    const T* w2 = (const T*)p.w2 + (int64_t)a * R * p.N;
    int c0, c1;
    share_of((p.K + 31) / 32, rank, size, c0, c1);
    const char* xb = (const char*)p.x;
    const int xs = X8 ? 1 : 2;
    const void* const xr[1][2] = {{row[0] >= 0 ? xb + row[0] * p.ldx * xs : nullptr, row[1] >= 0 ? xb + row[1] * p.ldx * xs : nullptr}};
    float acc[1][R / 8][4];
#pragma unroll
    for (int i = 0; i < R / 8; ++i) acc[0][i][0] = acc[0][i][1] = acc[0][i][2] = acc[0][i][3] = 0.0f;
    narrow<T, X8, R, LAY, VEC, 1>(acc, xr, w1, p.K, p.int8, c0 + warp, c1, kWarps, lane);
    // the first column group is on its way while the shares meet
    WideWeights<T, R, LAY, VEC> w;
    YPiece<T, LAY, VEC> y0;
    const int own = Wide<LAY>::own * t;
    int c = n0 + warp;
    if (c < n1) {
        if (R <= 32) w.load(w2, c * G, p.N, lane);
        y0.load((const T*)p.y0, p.ldy0, row, c * G + own, p.N);
    }
    put_narrow<R, LAY>(acc[0], part + warp * 16 * R, lane);
    __syncthreads();
    cluster_wait();
    for (int i = tid; i < 16 * R / 4; i += kThreads) {     // this block's sum goes to every block of the cluster
        float4 v = reinterpret_cast<float4*>(part)[i];
#pragma unroll
        for (int k = 1; k < kWarps; ++k) {
            const float4 q = reinterpret_cast<float4*>(part + k * 16 * R)[i];
            v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
        }
        for (int k = 0; k < size; ++k) send4(shares + rank * 16 * R + 4 * i, k, v);
    }
    cluster_arrive();
    cluster_wait();                                        // (the last that the blocks have to do with one another)
    const float sc = p.scale ? __ldg(p.scale + a) : 1.0f;
    constexpr int rounds = 16 * R / 4 < kThreads ? 1 : 16 * R / 4 / kThreads;
#pragma unroll
    for (int q = 0; q < rounds; ++q) {
        const int i = tid + q * kThreads;
        if (16 * R / 4 >= kThreads || warp < (16 * R / 4 + 31) / 32) {        // whole warps: put_u shuffles
            float4 v = reinterpret_cast<const float4*>(shares)[i];
            for (int k = 1; k < size; ++k) {
                const float4 r = reinterpret_cast<const float4*>(shares + k * 16 * R)[i];
                v.x += r.x, v.y += r.y, v.z += r.z, v.w += r.w;
            }
            const int m = 4 * i / R, j = 4 * i % R, to = rows[m];
            float f[4] = {v.x, v.y, v.z, v.w};
            if (X8 && to >= 0) {
                const float xsc = __ldg(p.x_scale + to);
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] *= xsc;
            }
            const float4 raw = make_float4(f[0], f[1], f[2], f[3]);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[k] *= sc;
            if (p.s && to >= 0 && rank == 0)
                *reinterpret_cast<float4*>(p.s + (int64_t)to * R + j) = p.s_scaled ? make_float4(f[0], f[1], f[2], f[3]) : raw;
            put_u<T, R>(f, hi, lo, back, m, j);
        }
    }
    __syncthreads();
    while (c < n1) {
        if (R > 32) w.load(w2, c * G, p.N, lane);
        widen<T, R, LAY, VEC>(w, y0, hi, lo, back, 0, (T*)p.y, p.ldy, row, c * G + own, p.N, lane);
        c += kWarps;
        if (c < n1) {
            if (R <= 32) w.load(w2, c * G, p.N, lane);
            y0.load((const T*)p.y0, p.ldy0, row, c * G + own, p.N);
        }
    }
}

// Which adapter a tile belongs to: the last a with starts[a] <= v, of n + 1 ascending numbers, by a warp.
__device__ __forceinline__ int find_part(const int* __restrict__ starts, int n, int v, int lane)
{
    // 32 samples, then the 32 (at most 33) numbers from the last sample that is not above v
    const int stride = (n + 32) / 32;
    const int at = min(lane * stride, n);
    const unsigned below = __ballot_sync(0xFFFFFFFFu, __ldg(starts + at) <= v && lane * stride < n);
    const int from = (31 - __clz(below | 1u)) * stride;
    int found = from;
    if (stride == 1) return found;
    for (int o = 0; o < stride; o += 32) {
        const int i = from + o + lane;
        const unsigned m = __ballot_sync(0xFFFFFFFFu, i < n && o + lane < stride && __ldg(starts + min(i, n)) <= v);
        if (m) found = from + o + 31 - __clz(m);
    }
    return found;
}

// Rows of tile `tile` (64 of a unit of 128 of the sort): adapter, first sorted row, number of rows; false if there are none, as in every tile behind the last unit (which
// counts to the last adapter, behind its rows).
__device__ __forceinline__ bool tile_rows(const LoraP& p, int tile, int lane, int& a, int& first, int& count)
{
    a = find_part(p.units, p.n, tile >> 1, lane);
    first = __ldg(p.offsets + a) + 128 * ((tile >> 1) - __ldg(p.units + a)) + kTileRows * (tile & 1);
    const int end = min(__ldg(p.offsets + a + 1), p.T);
    count = min(end - first, kTileRows);
    return count > 0;
}

// Shapes of the narrowing product of a tile of 64 rows: x and w1 come in stages of 128 elements of K.
template <bool X8, int R> struct NarrowShape {
    static constexpr int MW = R <= 64 ? 2 : 1;             // row tiles of a warp
    static constexpr int RG = kTileRows / 16 / MW, KP = kWarps / RG;          // row groups x shares of K
    static constexpr int K = 128, chunks = K / 32 / KP;    // elements of a stage; 32-element chunks of a warp
    static constexpr int xbytes = kTileRows * K * (X8 ? 1 : 2), wbytes = K * R * 2, stage = xbytes + wbytes;
    static constexpr int stages = R == 32 ? 4 : R <= 64 ? 3 : 2;              // (r = 32: three 221.5 us instead of 219.7 for the call below)
    static constexpr int sums = KP * kTileRows * R * 4;
    static constexpr int smem = stages * stage > sums ? stages * stage : sums;
    // Per SM, as shared memory allows; r = 32 needs the registers more (8192 x 2048 x 8192 with gradients: 220 us with two, 235 with three), r = 16 the blocks (2048 x 4096 x 28672: 71
    // and 67).
    static constexpr int blocks = R <= 16 ? 3 : 2;
};

// Places of 16-byte pieces in a stage: conflict-free both for eight rows' pieces at one k (ldmatrix) and for two rows' four neighbouring ones.
__device__ __forceinline__ uint32_t piece_in_row(int r, int c) { return (uint32_t)((c ^ (((r & 1) << 2) | ((r >> 1) & 3))) << 4); }
template <int R> __device__ __forceinline__ uint32_t piece_of_k(int k, int c)                 // row k of w1 [K, R]
{
    const int f = R >= 64 ? k & 7 : R == 32 ? (k >> 1) & 3 : R == 16 ? (k >> 2) & 1 : 0;
    return (uint32_t)(k * 2 * R + ((c ^ f) << 4));
}

// acc += tile . w1 over the stages [st0, st1) of K, rows[64] in shared memory.  VEC: whole pieces of 16 bytes, copied asynchronously.  Otherwise rows begin at whole words, which
// are copied one by one (p.words), or anywhere: then a stage's pieces are put together in registers, which wait there during the products of the stage that is there.
template <typename T, bool X8, int R, int LAY, bool VEC>
__device__ __forceinline__ void narrow_stages(float (&acc)[NarrowShape<X8, R>::MW][R / 8][4], const LoraP& p, const T* __restrict__ w1, const int* rows, uint8_t* smem, int st0,
                                              int st1)
{
    using S = NarrowShape<X8, R>;
    constexpr int MW = S::MW;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int rg = warp % S::RG, kp = warp / S::RG;
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem);
    constexpr int XP = X8 ? 8 : 16, XN = kTileRows * XP / kThreads, WN = 16 * R / kThreads ? 16 * R / kThreads : 1;      // pieces of a row of x; pieces of a thread
    const int xr = tid / XP, xc = tid % XP;
    const char* from[XN];
#pragma unroll
    for (int q = 0; q < XN; ++q) {
        const int r = rows[xr + q * (kThreads / XP)];
        from[q] = r >= 0 ? (const char*)p.x + (int64_t)r * p.ldx * (X8 ? 1 : 2) : nullptr;
    }
    auto x_at = [&](int q) -> uint32_t {
        const int r = xr + q * (kThreads / XP);
        return X8 ? (uint32_t)(r * S::K + ((xc ^ ((r & 3) << 1)) << 4)) : (uint32_t)(r * 2 * S::K) + piece_in_row(r, xc);
    };
    // piece i of w1: LAY 0 rank i / 16, elements 8 (i % 16) of the stage; LAY 1 element i / (R / 8) of the stage, ranks 8 (i % (R / 8))
    auto w_at = [&](int i) -> uint32_t { return S::xbytes + (LAY == 0 ? (uint32_t)(i / 16 * 2 * S::K) + piece_in_row(i / 16, i % 16) : piece_of_k<R>(i / (R / 8), i % (R / 8))); };
    uint4 held_x[VEC ? 1 : XN], held_w[VEC ? 1 : WN];
    auto fetch = [&](int st, int buf) {
        if (st < st1) {
            const uint32_t to = base + buf * S::stage;
            const int k0 = st * S::K, kx = k0 + 16 * xc / (X8 ? 1 : 2), left = p.K - kx;                                 // first element of this thread's pieces of x
#pragma unroll
            for (int q = 0; q < XN; ++q) {
                if constexpr (VEC) {
                    const int n = from[q] ? min(max(left * (X8 ? 1 : 2), 0), 16) : 0;
                    async16(to + x_at(q), n ? from[q] + (int64_t)kx * (X8 ? 1 : 2) : (const char*)p.x, n);
                } else if (p.words & 1) {
                    async_words(to + x_at(q), from[q] + (int64_t)kx * (X8 ? 1 : 2), from[q] ? left * (X8 ? 1 : 2) : 0, p.x);
                } else if constexpr (X8) {
                    XPiece<T, true, false> a, b;
                    a.load(from[q], kx, left);
                    b.load(from[q], kx + 8, left - 8);
                    held_x[q] = make_uint4(a.u[0], a.u[1], b.u[0], b.u[1]);
                } else {
                    uint32_t u[4];
                    load8<T, false>((const T*)from[q], kx, from[q] ? left : 0, u);
                    held_x[q] = make_uint4(u[0], u[1], u[2], u[3]);
                }
            }
#pragma unroll
            for (int q = 0; q < WN; ++q) {
                const int i = tid + q * kThreads;
                if (16 * R < kThreads && i >= 16 * R) break;
                const int k = k0 + (LAY == 0 ? i % 16 * 8 : i / (R / 8));
                const T* row = LAY == 0 ? w1 + (int64_t)(i / 16) * p.K : w1 + (int64_t)k * R;
                const int at = LAY == 0 ? k : i % (R / 8) * 8;
                if constexpr (VEC) {
                    const int n = k < p.K ? 16 : 0;
                    async16(to + w_at(i), n ? row + at : w1, n);
                } else if (p.words & 2) {
                    async_words(to + w_at(i), row + at, k < p.K ? 2 * ((LAY == 0 ? p.K : R) - at) : 0, w1);
                } else {
                    uint32_t u[4];
                    load8<T, false>(row, at, k < p.K ? (LAY == 0 ? p.K : R) - at : 0, u);
                    held_w[q] = make_uint4(u[0], u[1], u[2], u[3]);
                }
            }
        }
        async_commit();
    };
    auto put = [&](int st, int buf) {
        if constexpr (!VEC) {
            if (st >= st1) return;
            uint8_t* to = smem + buf * S::stage;
            if (!(p.words & 1)) {
#pragma unroll
                for (int q = 0; q < XN; ++q) *reinterpret_cast<uint4*>(to + x_at(q)) = held_x[q];
            }
            if (!(p.words & 2)) {
#pragma unroll
                for (int q = 0; q < WN; ++q) {
                    const int i = tid + q * kThreads;
                    if (16 * R < kThreads && i >= 16 * R) break;
                    *reinterpret_cast<uint4*>(to + w_at(i)) = held_w[q];
                }
            }
        }
    };
#pragma unroll
    for (int i = 0; i < S::stages - 1; ++i) {
        fetch(st0 + i, i);
        put(st0 + i, i);
    }
    int buf = 0;
    for (int st = st0; st < st1; ++st) {
        async_wait<S::stages - 2>();
        __syncthreads();                                   // the stage is there; the one before it is free
        const int next = buf == 0 ? S::stages - 1 : buf - 1;
        fetch(st + S::stages - 1, next);
        const uint8_t* xs = smem + buf * S::stage;
        const uint32_t xb = base + buf * S::stage, wb = xb + S::xbytes;
#pragma unroll
        for (int ch = 0; ch < S::chunks; ++ch) {
            const int c32 = kp * S::chunks + ch;           // 32 elements: pieces 4 c32 .. 4 c32 + 3 of a 16-bit row
            if constexpr (LAY == 0) {                      // lane's elements 8 t .. 8 t + 7 of the chunk, as in narrow()
                uint32_t a[MW][2][4];
#pragma unroll
                for (int m = 0; m < MW; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int r = (rg * MW + m) * 16 + g + 8 * h;
                        if constexpr (X8) {
                            XPiece<T, true, true> x;
                            const uint2 q = *reinterpret_cast<const uint2*>(xs + r * S::K + (((2 * c32 + (t >> 1)) ^ ((r & 3) << 1)) << 4) + 8 * (t & 1));
                            x.u[0] = q.x, x.u[1] = q.y;
                            x.pairs(p.int8, a[m][h]);
                        } else {
                            const uint4 q = *reinterpret_cast<const uint4*>(xs + r * 2 * S::K + piece_in_row(r, 4 * c32 + t));
                            a[m][h][0] = q.x, a[m][h][1] = q.y, a[m][h][2] = q.z, a[m][h][3] = q.w;
                        }
                    }
#pragma unroll
                for (int i = 0; i < R / 8; ++i) {
                    const int r = 8 * i + g;
                    const uint4 q = *reinterpret_cast<const uint4*>(xs + S::xbytes + r * 2 * S::K + piece_in_row(r, 4 * c32 + t));
#pragma unroll
                    for (int m = 0; m < MW; ++m) {
                        const uint32_t f0[4] = {a[m][0][0], a[m][1][0], a[m][0][1], a[m][1][1]}, f1[4] = {a[m][0][2], a[m][1][2], a[m][0][3], a[m][1][3]};
                        float d[4];
                        mma16_first<T>(d, f0, q.x, q.y);
                        mma16<T>(d, f1, q.z, q.w);
                        add4(acc[m][i], d);
                    }
                }
            } else {                                       // fragments in the MMA's own order; accumulator tile i has ranks 8 i .. 8 i + 7
                uint32_t a[MW][2][4];
#pragma unroll
                for (int m = 0; m < MW; ++m)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = (rg * MW + m) * 16 + (lane & 15);
                        ldmatrix4(a[m][j], xb + r * 2 * S::K + piece_in_row(r, 4 * c32 + 2 * j + (lane >> 4)));
                    }
#pragma unroll
                for (int i = 0; i < R / 8; i += 2) {
                    uint32_t b[2][4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) ldmatrix4t(b[j], wb + piece_of_k<R>(32 * c32 + 16 * j + (lane & 15), R == 8 ? 0 : i + (lane >> 4)));
#pragma unroll
                    for (int m = 0; m < MW; ++m)
#pragma unroll
                        for (int h = 0; h < (R > 8 ? 2 : 1); ++h) {
                            float d[4];
                            mma16_first<T>(d, a[m][0], b[0][2 * h], b[0][2 * h + 1]);
                            mma16<T>(d, a[m][1], b[1][2 * h], b[1][2 * h + 1]);
                            add4(acc[m][i + h], d);
                        }
                }
            }
        }
        put(st + S::stages - 1, next);
        buf = buf == S::stages - 1 ? 0 : buf + 1;
    }
    async_wait<0>();
    __syncthreads();
}

// The narrowing product of tiles of 64 rows, a tile per cluster whose blocks share K.  -> s [T, R].
// Bound by HBM (x once; w1 comes from L2) and the fill of its stages: 8192 x 8192 bf16 at r = 32, 134 MB in 32 us (4.2 TB/s; 64 us without stages), 8192 x 2048 e4m3 14 to 16 us,
// 2048 x 4096 fp16 at r = 16 12 us.
template <typename T, bool X8, int R, int LAY, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? NarrowShape<X8, R>::blocks : 2) lora_narrow_kernel(const LoraP p)
{
    pdl_launch_dependents();
    pdl_wait();
    using S = NarrowShape<X8, R>;
    constexpr int MW = S::MW, RG = S::RG, KP = S::KP;
    extern __shared__ __align__(128) uint8_t smem[];
    float* part = reinterpret_cast<float*>(smem);          // [KP][64][R], over the stages; share 0 holds the block's sum in the end
    __shared__ int rows[kTileRows];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_rank(), size = (int)cluster_size();
    int a, first, count;
    if (!tile_rows(p, blockIdx.x / size, lane, a, first, count)) return;      // (the whole cluster)
    if (tid < kTileRows) {
        const int r = tid < count ? __ldg(p.order + first + tid) : -1;
        rows[tid] = r >= 0 && r < p.T ? r : -1;
    }
    __syncthreads();
    const int rg = warp % RG, kp = warp / RG;
    const T* w1 = (const T*)p.w1 + (int64_t)a * R * p.K;
    float acc[MW][R / 8][4];
#pragma unroll
    for (int m = 0; m < MW; ++m)
#pragma unroll
        for (int i = 0; i < R / 8; ++i) acc[m][i][0] = acc[m][i][1] = acc[m][i][2] = acc[m][i][3] = 0.0f;
    int c0, c1;
    share_of((p.K + S::K - 1) / S::K, rank, size, c0, c1);
    narrow_stages<T, X8, R, LAY, VEC>(acc, p, w1, rows, smem, c0, c1);
#pragma unroll
    for (int m = 0; m < MW; ++m) put_narrow<R, 0>(acc[m], part + (kp * kTileRows + (rg * MW + m) * 16) * R, lane);
    __syncthreads();
    for (int i = tid; i < kTileRows * R / 4; i += kThreads) {
        float4 v = reinterpret_cast<float4*>(part)[i];
#pragma unroll
        for (int k = 1; k < KP; ++k) {
            const float4 q = reinterpret_cast<float4*>(part + k * kTileRows * R)[i];
            v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
        }
        reinterpret_cast<float4*>(part)[i] = v;
    }
    cluster_arrive();
    cluster_wait();
    const float sc = p.s_scaled && p.scale ? __ldg(p.scale + a) : 1.0f;
    int i0, i1;
    share_of(kTileRows * R / 4, rank, size, i0, i1);       // each block adds and stores its share of the tile's sums
    for (int i = i0 + tid; i < i1; i += kThreads) {
        const int to = rows[4 * i / R];
        float4 v = cluster_sum4(part + 4 * i, size);
        if (to < 0) continue;
        const float f = X8 ? __ldg(p.x_scale + to) : 1.0f;
        if (X8) v.x *= f, v.y *= f, v.z *= f, v.w *= f;
        if (p.s_scaled) v.x *= sc, v.y *= sc, v.z *= sc, v.w *= sc;
        *reinterpret_cast<float4*>(p.s + (int64_t)to * R + 4 * i % R) = v;
    }
    cluster_arrive();                                      // (a block's shared memory stays until the others have read it)
    cluster_wait();
}

// Stages of the widening product: 64 rows x 128 columns of y0 and the weights of these columns.
template <int R, int LAY> struct WideShape {
    static constexpr int cols = 128;
    static constexpr int ybytes = kTileRows * cols * 2, wbytes = cols * R * 2, stage = ybytes + wbytes;
    static constexpr int stages = R <= 32 ? 3 : 2;
    // Per SM: the products need the registers more than another block (three: 2048 x 4096 x 28672 at r = 16 67 us instead of 58, 8192 x 2048 x 8192 at r = 32 219 instead of 214).
    static constexpr int blocks = R <= 64 ? 2 : 1;
};
// 16-byte piece c of row r of y0 lies at place c ^ 4 (r % 2), so that two rows' shares of a column group do not meet in a bank.
__device__ __forceinline__ uint32_t y_place(int r, int c) { return (uint32_t)(r * 256 + ((c ^ ((r & 1) << 2)) << 4)); }

// y = rn(y0 + back * (u . w2)) over the stages [s0, s1) of 128 columns.  y0 and w2 come by cp.async in whole pieces of rows; a warp takes one column group of a stage and MU of its
// row tiles, and stores y from its fragments.  parts_of_s: what fills hi, lo and back, while the first stages are on their way.
template <typename T, int R, int LAY, bool VEC, typename F>
__device__ __forceinline__ void widen_stages(const LoraP& p, const T* __restrict__ w2, const int* rows, const uint8_t* hi, const uint8_t* lo, const float* back, uint8_t* stages,
                                             int count, int s0, int s1, F parts_of_s)
{
    using S = WideShape<R, LAY>;
    constexpr int G = Wide<LAY>::cols, GS = S::cols / G, MU = GS * 4 / kWarps, tiles = Wide<LAY>::tiles, steps = R < 16 ? 1 : R / 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int cw = warp % GS, m0 = warp / GS * MU;
    const int fr = tid >> 4, fc = tid & 15;                // piece fc of rows fr + 16 q of y0
    const T* from[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int r = rows[fr + 16 * q];
        from[q] = r >= 0 && p.y0 ? (const T*)p.y0 + (int64_t)r * p.ldy0 : nullptr;
    }
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(stages);
    constexpr int WN = 16 * R / kThreads ? 16 * R / kThreads : 1;             // pieces of w2 of a thread
    // piece i of w2.  LAY 0: row n = i / (R / 8) of 2 R bytes, at the row that its fragment has: column c of tile t of a group at 8 t + c.  LAY 1: rank i / 16, columns 8 (i % 16)
    auto w_at = [&](int i) -> uint32_t {
        if (LAY == 0) {
            const int n = i / (R / 8), at_row = (n & ~31) + ((n & 6) << 2) + ((n >> 3 & 3) << 1) + (n & 1);
            return S::ybytes + piece_of_k<R>(at_row, i % (R / 8));
        }
        const int j = i / 16;
        return S::ybytes + j * 256 + ((i % 16 ^ (((j >> 1) & 3) << 1)) << 4);
    };
    uint4 held_y[VEC ? 1 : 4], held_w[VEC ? 1 : WN];       // as in narrow_stages
    auto fetch = [&](int st, int buf) {
        if (st < s1) {
            const uint32_t at = base + buf * S::stage;
            const int n0 = st * S::cols, left = p.N - (n0 + 8 * fc);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (VEC) {
                    const bool in = left > 0 && from[q];
                    async16(at + y_place(fr + 16 * q, fc), in ? from[q] + n0 + 8 * fc : w2, in ? 16 : 0);
                } else if (p.words & 4) {
                    async_words(at + y_place(fr + 16 * q, fc), from[q] + n0 + 8 * fc, from[q] ? 2 * left : 0, p.s);
                } else {
                    uint32_t u[4];
                    load8<T, false, false>(from[q], n0 + 8 * fc, from[q] ? left : 0, u);
                    held_y[q] = make_uint4(u[0], u[1], u[2], u[3]);
                }
            }
#pragma unroll
            for (int q = 0; q < WN; ++q) {
                const int i = tid + q * kThreads;
                if (16 * R < kThreads && i >= 16 * R) break;
                const int n = n0 + (LAY == 0 ? i / (R / 8) : i % 16 * 8), col = LAY == 0 ? i % (R / 8) * 8 : n;
                const T* row = LAY == 0 ? w2 + (int64_t)n * R : w2 + (int64_t)(i / 16) * p.N;
                if constexpr (VEC) {
                    const bool in = n < p.N;
                    async16(at + w_at(i), in ? row + col : w2, in ? 16 : 0);
                } else if (p.words & 8) {
                    async_words(at + w_at(i), row + col, n < p.N ? 2 * ((LAY == 0 ? R : p.N) - col) : 0, w2);
                } else {
                    uint32_t u[4];
                    load8<T, false>(row, col, n < p.N ? (LAY == 0 ? R : p.N) - col : 0, u);
                    held_w[q] = make_uint4(u[0], u[1], u[2], u[3]);
                }
            }
        }
        async_commit();
    };
    auto put = [&](int st, int buf) {
        if constexpr (!VEC) {
            if (st >= s1) return;
            uint8_t* at = stages + buf * S::stage;
            if (!(p.words & 4)) {
#pragma unroll
                for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(at + y_place(fr + 16 * q, fc)) = held_y[q];
            }
            if (!(p.words & 8)) {
#pragma unroll
                for (int q = 0; q < WN; ++q) {
                    const int i = tid + q * kThreads;
                    if (16 * R < kThreads && i >= 16 * R) break;
                    *reinterpret_cast<uint4*>(at + w_at(i)) = held_w[q];
                }
            }
        }
    };
#pragma unroll
    for (int i = 0; i < S::stages - 1; ++i) {
        fetch(s0 + i, i);
        put(s0 + i, i);
    }
    parts_of_s();
    __syncthreads();
    T* to[MU][2];
    float factor[MU][2];
#pragma unroll
    for (int m = 0; m < MU; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = (m0 + m) * 16 + g + 8 * h, r = rows[at];
            to[m][h] = r >= 0 ? (T*)p.y + (int64_t)r * p.ldy + cw * G + Wide<LAY>::own * t : nullptr;
            factor[m][h] = back[at];
        }
    int buf = 0;
    for (int st = s0; st < s1; ++st) {
        async_wait<S::stages - 2>();
        __syncthreads();                                   // the stage is there; the one before it is free
        const int next = buf == 0 ? S::stages - 1 : buf - 1;
        fetch(st + S::stages - 1, next);
        const uint8_t* ys = stages + buf * S::stage;
        const uint32_t ws = base + buf * S::stage + S::ybytes;
        float acc[MU][tiles][4];
#pragma unroll
        for (int s = 0; s < steps; ++s) {
            uint32_t b[tiles][2];
            if constexpr (LAY == 0 && R == 8) {            // one piece per row: two tiles' rows at a time, their missing ranks zero
#pragma unroll
                for (int i = 0; i < 4; i += 4) {
                    uint32_t q[4];
                    ldmatrix4(q, ws + piece_of_k<8>(32 * cw + lane, 0));
                    b[0][0] = q[0], b[1][0] = q[1], b[2][0] = q[2], b[3][0] = q[3];
                    b[0][1] = b[1][1] = b[2][1] = b[3][1] = 0u;
                }
            } else if constexpr (LAY == 0) {
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    uint32_t q[4];
                    ldmatrix4(q, ws + piece_of_k<R>(32 * cw + 8 * i + (lane & 7) + 8 * (lane >> 4), 2 * s + ((lane >> 3) & 1)));
                    b[i][0] = q[0], b[i][1] = q[1], b[i + 1][0] = q[2], b[i + 1][1] = q[3];
                }
            } else {
                uint32_t u[4][4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int j = 16 * s + 2 * t + (k & 1) + 8 * (k >> 1);
                    uint4 q = make_uint4(0u, 0u, 0u, 0u);
                    if (R >= 16 || k < 2) q = *reinterpret_cast<const uint4*>(ys + S::ybytes + j * 256 + (((8 * cw + g) ^ (((j >> 1) & 3) << 1)) << 4));
                    u[k][0] = q.x, u[k][1] = q.y, u[k][2] = q.z, u[k][3] = q.w;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    b[i][0] = pair_of(u[0][i >> 1], u[1][i >> 1], i & 1);
                    b[i][1] = pair_of(u[2][i >> 1], u[3][i >> 1], i & 1);
                }
            }
#pragma unroll
            for (int m = 0; m < MU; ++m) {
                if ((m0 + m) * 16 >= count) continue;
#pragma unroll
                for (int part = 0; part < 2; ++part) {     // the low part first
                    uint32_t a[4];
                    get_u<R, 1>(part ? hi : lo, m0 + m, s, lane, a);          // (ranks in the MMA's own order)
#pragma unroll
                    for (int i = 0; i < tiles; ++i) {
                        if (s == 0 && part == 0) mma16_first<T>(acc[m][i], a, b[i][0], b[i][1]);
                        else mma16<T>(acc[m][i], a, b[i][0], b[i][1]);
                    }
                }
            }
        }
        const int n0 = st * S::cols, left = p.N - (n0 + cw * G + Wide<LAY>::own * t);
#pragma unroll
        for (int m = 0; m < MU; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!to[m][h]) continue;
                const float2 f = both(factor[m][h]);
#pragma unroll
                for (int v = 0; v < Wide<LAY>::own; v += 8) {
                    const uint4 q = *reinterpret_cast<const uint4*>(ys + y_place((m0 + m) * 16 + g + 8 * h, (cw * G + Wide<LAY>::own * t + v) >> 3));
                    const uint32_t y0[4] = {q.x, q.y, q.z, q.w};
                    uint32_t o[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float2 c;
                        if constexpr (LAY == 0) c = make_float2(acc[m][k][2 * h], acc[m][k][2 * h + 1]);
                        else c = make_float2(acc[m][2 * k][2 * h + (v >> 3)], acc[m][2 * k + 1][2 * h + (v >> 3)]);
                        const float2 r = fma2(f, c, Dt<T>::up2(y0[k]));
                        o[k] = Dt<T>::down2(r.x, r.y);
                    }
                    store8<T, VEC>(to[m][h] + n0 + v, left - v, o);
                }
            }
        put(st + S::stages - 1, next);
        buf = buf == S::stages - 1 ? 0 : buf + 1;
    }
}

// The widening product: a block takes a tile of 64 rows and `span` column groups.  blockIdx.x = tile * spans + span; blocks from `tile_blocks` on copy the rows without an adapter.
// Bound by HBM (y0 and y once): 2048 x 28672 fp16 at r = 16, 235 MB in 47 us (5.0 TB/s) on rows used before, 57 on others, 8192 x 8192 bf16 at r = 32, 268 MB in 55 to 58 us (4.9); a copy in tiles of this shape reaches
// 5.3 to 6.0 TB/s.  The rest is each block's chain of loads to its first rows, and the warps' waits for a stage.
template <typename T, int R, int LAY, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC ? WideShape<R, LAY>::blocks : R <= 64 ? 2 : 1) lora_widen_kernel(const LoraP p, int spans, int per_span, int tile_blocks)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(128) uint8_t smem[];
    uint8_t *hi = smem, *lo = smem + kTileRows * u_pitch<R>, *stages = smem + 2 * kTileRows * u_pitch<R>;
    __shared__ float back[kTileRows];
    __shared__ int rows[kTileRows];
    constexpr int G = Wide<LAY>::cols;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int groups = (p.N + G - 1) / G;
    if ((int)blockIdx.x >= tile_blocks) {                  // rows without an adapter among 64, the columns of a span
        const int id = (int)blockIdx.x - tile_blocks, t0 = id / spans * kTileRows, n0 = (id - id / spans * spans) * per_span * G;
        if (tid < kTileRows) {
            const int e = t0 + tid < p.T ? __ldg(p.idx + t0 + tid) : 0;
            rows[tid] = e < 0 || e >= p.n;
        }
        __syncthreads();
        const int n1 = min(n0 + per_span * G, p.N);
        for (int r = warp; r < kTileRows; r += kWarps)
            if (rows[r]) copy_row<T, VEC>(p, t0 + r, n0, n1, lane);
        return;
    }
    const int tile = blockIdx.x / spans, span = blockIdx.x - tile * spans;
    int a, first, count;
    if (!tile_rows(p, tile, lane, a, first, count)) return;
    if (tid < kTileRows) {
        const int r = tid < count ? __ldg(p.order + first + tid) : -1;
        rows[tid] = r >= 0 && r < p.T ? r : -1;
    }
    __syncthreads();
    const float sc = !p.s_scaled && p.scale ? __ldg(p.scale + a) : 1.0f;
    auto parts_of_s = [&] {
        for (int i = tid; i < kTileRows * R / 4; i += kThreads) {
            const int m = 4 * i / R, j = 4 * i % R, from = rows[m];
            const float4 v = from >= 0 ? *reinterpret_cast<const float4*>(p.s + (int64_t)from * R + j) : make_float4(0.f, 0.f, 0.f, 0.f);
            const float f[4] = {v.x * sc, v.y * sc, v.z * sc, v.w * sc};
            put_u<T, R>(f, hi, lo, back, m, j);
        }
    };
    const T* w2 = (const T*)p.w2 + (int64_t)a * R * p.N;
    const int last = min((span + 1) * per_span, groups);
    constexpr int per_stage = WideShape<R, LAY>::cols / G;
    widen_stages<T, R, LAY, VEC>(p, w2, rows, hi, lo, back, stages, count, span * per_span / per_stage, (last + per_stage - 1) / per_stage, parts_of_s);
}

// ------------------------------------------------------------------ weight gradients

struct WgradP {
    const void* v;                                         // rows [T, ldv] of W elements: x for dA, dy for dB
    int64_t ldv;
    const float* v_scale;                                  // of rows of 8 bits
    int int8;
    const float* s;                                        // [T, R]: ds for dA, s for dB
    const float* scale;                                    // [n] or null, applied to s
    const int *order, *offsets, *units;
    int T, n, W;
    float* out;                                            // [n, R, W] or, TRANS, [n, W, R]
    float* part;                                           // null: a cluster per adapter and 128 columns; else `blocks` share all rows, [blocks][2][R x 128] sums of shared adapters
    int blocks;
    int words;                                             // v's rows begin at whole words
};

// out[a] = sum over the adapter's rows of s (R) x v (W).  A block takes 128 columns of one adapter and 64 rows a stage, two or three stages in flight (cp.async).  Two forms:
//   few rows (kSmallRows): the blocks of a cluster share an adapter's rows and add their sums; nothing but one launch
//   many rows: the line of all adapters' rows, once for each 128 columns, is cut into as many equal pieces as blocks run at once, so that adapters with many rows do not end last;
//   what two blocks have of one adapter meets in the workspace, and a short launch adds it
//   (both passes of 1000 x 1000 x 1500 at r = 16: by clusters 52.7 us, 49.9 so; 8192 x 2048 x 8192 at r = 32: 254 and 234; 500 x 1001 x 700 at r = 8: 38 and 50.  Measured when the
//   two gradients were launches of their own.)
// A warp has all R ranks of 64, 32 or 16 columns (R x columns = 2048 where R >= 32: 64 accumulators a lane), the warps of a column group share the stage's
// rows.  k of the products is the row: v comes out of shared memory transposed (ldmatrix.trans; codes of 8 bits by words and byte permutes), s is brought into
// [rank][row] once per stage, split into 16-bit or tf32 parts:
//   bf16 products of three parts of s (all of its bits: with two, dA is off by 1.5e-6, with three by 1.6e-7); fp16 rows: tf32 products of two parts, whose exponent
//   holds any s (a gradient's 1e-7 is below fp16's normal numbers).
// The parts of a sum are added in a fixed order: warps, then blocks.
// Bound by HBM where R <= 16; from R = 32 on by the warps' chains of barriers, splits and warp-level tensor products of the parts (3 or 4 for each of s), two blocks per SM:
// 8192 rows, 8192 columns of bf16 and 2048 of e4m3 at r = 32: 83 us together (153 MB: 23 us; the products alone 32 us).
template <typename T, bool X8, int R> struct WgradShape {
    static constexpr bool tf32 = std::is_same<T, __half>::value && !X8;
    static constexpr int cols = 128, rows = 64, stages = R == 64 ? 2 : 3;      // (two blocks per SM up to R = 64)
    static constexpr int RT = R < 16 ? 16 : R;             // ranks, as whole tiles of 16
    static constexpr int MT = RT / 16;
    static constexpr int WC = R <= 32 ? 64 : R == 64 ? 32 : 16;               // columns of a warp
    static constexpr int CG = cols / WC, RG = kWarps / CG, NT = WC / 8;
    static constexpr int vpitch = X8 ? cols : 2 * cols;
    static constexpr int vbytes = rows * vpitch, sbytes = rows * R * 4;
    static constexpr int part = tf32 ? RT * rows * 4 : RT * rows * 2;
    static constexpr int parts = tf32 ? 2 : 3;
    static constexpr int stage = vbytes + sbytes;
    static constexpr int ahead = R <= 32 ? 2 : 1;          // sets of parts: with two, a stage's s is split during the products of the one before
    static constexpr int pitch = cols + 8;                 // floats of a row of the sums (8 apart: no bank conflicts)
    static constexpr int sums = RG * RT * pitch * 4;
    static constexpr int front = stages * stage > sums ? stages * stage : sums;
    static constexpr int smem = front + ahead * parts * part + stages * rows * 4;
};

// Block `block` of the `blocks` that work on one gradient.
template <typename T, bool X8, int R, bool TRANS, bool VEC> __device__ __forceinline__ void wgrad(const WgradP& p, int block, int blocks, uint8_t* smem)
{
    using S = WgradShape<T, X8, R>;
    constexpr int MT = S::MT, NT = S::NT, WC = S::WC, RG = S::RG, RT = S::RT;
    uint8_t* s_part = smem + S::front;
    float* s_scale = reinterpret_cast<float*>(s_part + S::ahead * S::parts * S::part);
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem), part0 = base + S::front;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int rank = (int)cluster_rank(), size = (int)cluster_size();
    const int chunks = (p.W + S::cols - 1) / S::cols;
    // what the block works on: rows [first, end) of an adapter, of them the stages [st0, st1), columns from vcol on
    int first, end, st0, st1, vcol, vleft;
    float sc;
    // The blocks' shares of the line: adapter by adapter in units of 128 rows, the line again for the next 128 columns.  The next segment's beginning and what is left of the share
    // wait in shared memory, as what is needed again at a segment's end does: the products need the registers.
    __shared__ int at_chunk, at_unit, at_left, seg_a, seg_col, seg_slot;      // seg_slot: -1, or where the segment's part goes
    if (p.part) {
        const int line = max(__ldg(p.units + p.n), 0);
        const LineShares shares((int64_t)chunks * line, blocks);
        const int64_t from = shares.begin(block), to = shares.begin(block + 1);
        if (to <= from) at_left = 0;
        else if (tid == 0) at_left = (int)(to - from), at_chunk = (int)(from / line), at_unit = (int)(from - from / line * line), seg_slot = -2;
        // adapters without rows
        for (int64_t e = (int64_t)block * kWarps + warp; e < (int64_t)p.n * chunks; e += (int64_t)blocks * kWarps) {
            const int c = (int)(e / p.n), none = (int)(e - (int64_t)c * p.n);
            if (__ldg(p.units + none) != __ldg(p.units + none + 1)) continue;
            const int wide = min(S::cols, p.W - c * S::cols);
            for (int i = lane; i < wide * R; i += 32) {
                const int j = i / wide;
                p.out[TRANS ? ((int64_t)none * p.W + c * S::cols) * R + i : ((int64_t)none * R + j) * p.W + c * S::cols + i - j * wide] = 0.0f;
            }
        }
    }
    const int cg = warp / RG, rg = warp % RG;
    const int es = X8 ? 1 : 2;

    // this thread's part of a stage: VN pieces of 16 bytes of v, rows vr + q VS; SN pieces of s, rows sr + q SS
    constexpr int VPR = S::vpitch / 16, VS = kThreads / VPR, VN = S::rows / VS;              // pieces per row
    constexpr int SPR = R * 4 / 16, SS = kThreads / SPR >= S::rows ? S::rows : kThreads / SPR, SN = S::rows / SS;
    const int vr = tid / VPR, vc = tid % VPR, sr = tid / SPR, sp = tid % SPR;
    const bool s_mine = tid < SS * SPR;
    int vrow[VN], srow[SN], xrow = -1;
    auto rows_of = [&](int stage) {                        // order of the stage's rows that this thread loads
        const int r0 = first + stage * S::rows;
        const int n = stage < st1 ? end - r0 : 0;
        auto at = [&](int i) {
            const int r = i < n ? __ldg(p.order + r0 + i) : -1;
            return r < p.T ? r : -1;
        };
#pragma unroll
        for (int q = 0; q < VN; ++q) vrow[q] = at(vr + q * VS);
#pragma unroll
        for (int q = 0; q < SN; ++q) srow[q] = s_mine ? at(sr + q * SS) : -1;
        if (X8 && tid < S::rows) xrow = at(tid);
    };
    auto v_place = [&](int r, int c) -> uint32_t {         // of 16-byte piece c of row r
        return (uint32_t)(r * S::vpitch) + (uint32_t)(X8 ? c ^ (((r >> 1) & 3) << 1) : c ^ (r & 7)) * 16u;
    };
    uint32_t held[VEC ? 1 : VN][4];                        // rows that are not 16-byte aligned come through registers
    auto fetch = [&](int buf) {
        const uint32_t to = base + buf * S::stage;
#pragma unroll
        for (int q = 0; q < VN; ++q) {
            const char* row = vrow[q] >= 0 ? (const char*)p.v + vrow[q] * p.ldv * es : nullptr;
            if constexpr (VEC) {
                const int bytes = row ? min(max(vleft * es, 0), 16) : 0;
                async16(to + v_place(vr + q * VS, vc), bytes ? row + (int64_t)vcol * es : p.v, bytes);
            } else if (p.words) {
                async_words(to + v_place(vr + q * VS, vc), row + (int64_t)vcol * es, row ? vleft * es : 0, p.v);
            } else if constexpr (!X8) {
                load8<T, false>((const T*)row, vcol, row ? vleft : 0, held[q]);
            } else {
                XPiece<T, true, false> lo, hi;
                lo.load(row, vcol, vleft);
                hi.load(row, vcol + 8, vleft - 8);
                held[q][0] = lo.u[0], held[q][1] = lo.u[1], held[q][2] = hi.u[0], held[q][3] = hi.u[1];
            }
        }
        if (s_mine) {
#pragma unroll
            for (int q = 0; q < SN; ++q)
                async16(to + S::vbytes + (sr + q * SS) * (R * 4) + sp * 16, srow[q] >= 0 ? p.s + (int64_t)srow[q] * R + sp * 4 : p.s, srow[q] >= 0 ? 16 : 0);
        }
        if (X8 && tid < S::rows)
            async4((uint32_t)__cvta_generic_to_shared(s_scale + buf * S::rows + tid), xrow >= 0 ? p.v_scale + xrow : p.v_scale, xrow >= 0 ? 4 : 0);
    };
    auto put_held = [&](int buf) {
        if (!VEC && !p.words) {
#pragma unroll
            for (int q = 0; q < VN; ++q)
                *reinterpret_cast<uint4*>(smem + buf * S::stage + v_place(vr + q * VS, vc)) = make_uint4(held[VEC ? 0 : q][0], held[VEC ? 0 : q][1], held[VEC ? 0 : q][2], held[VEC ? 0 : q][3]);
        }
    };

    float acc[MT][NT][4];
    if (R == 8)                                            // ranks 8 .. 15 of the tile
        for (int i = tid; i < S::ahead * S::parts * S::part / 4; i += kThreads) reinterpret_cast<uint32_t*>(s_part)[i] = 0u;
    // s of a stage into [rank][row] parts: eight rows of a rank per thread
    auto split = [&](int buf, int set) {
        const float* ss = reinterpret_cast<const float*>(smem + buf * S::stage + S::vbytes);
        uint8_t* pt = s_part + set * S::parts * S::part;
        for (int i = tid; i < 8 * R; i += kThreads) {
            const int j = i % R, c = i / R;
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                f[k] = ss[(8 * c + k) * R + j] * sc;
                if (X8) f[k] *= s_scale[buf * S::rows + 8 * c + k];
            }
            if constexpr (S::tf32) {
                uint32_t h[8], l[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    h[k] = tf32(f[k]);
                    l[k] = tf32(f[k] - __uint_as_float(h[k]));
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    uint8_t* to = pt + j * 256 + (((2 * c + q) ^ ((j & 7) << 1)) << 4);
                    *reinterpret_cast<uint4*>(to) = make_uint4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
                    *reinterpret_cast<uint4*>(to + S::part) = make_uint4(l[4 * q], l[4 * q + 1], l[4 * q + 2], l[4 * q + 3]);
                }
            } else {
                uint4 h, m, l;
                split3(f[0], f[1], h.x, m.x, l.x);
                split3(f[2], f[3], h.y, m.y, l.y);
                split3(f[4], f[5], h.z, m.z, l.z);
                split3(f[6], f[7], h.w, m.w, l.w);
                uint8_t* to = pt + j * 128 + ((c ^ (j & 7)) << 4);
                *reinterpret_cast<uint4*>(to) = h;
                *reinterpret_cast<uint4*>(to + S::part) = m;
                *reinterpret_cast<uint4*>(to + 2 * S::part) = l;
            }
        }
    };
    auto product = [&](int buf, int set) {
        const uint32_t vb = base + buf * S::stage;
        const uint8_t* pt = s_part + set * S::parts * S::part;
        constexpr int TN = NT < 4 ? NT : 4;                // column tiles at a time
#pragma unroll
        for (int k0 = 0; k0 < S::rows / RG; k0 += 16) {
            const int r0 = rg * (S::rows / RG) + k0;       // 16 rows of the stage
#pragma unroll
            for (int i0 = 0; i0 < NT; i0 += TN) {
                uint32_t b[TN][2];                         // pairs of rows (2 t, 2 t + 1) and (2 t + 8, 2 t + 9) of column g of the tile
                if constexpr (!X8) {
#pragma unroll
                    for (int i = 0; i < TN; i += 2) {
                        uint32_t q[4];
                        const int r = r0 + (lane & 15);
                        ldmatrix4t(q, vb + v_place(r, cg * (WC / 8) + i0 + i + (lane >> 4)));
                        b[i][0] = q[0], b[i][1] = q[1], b[i + 1][0] = q[2], b[i + 1][1] = q[3];
                    }
                } else {                                   // tile i has column NT g + i at place g: TN codes of a row per lane
                    uint32_t x[4][2];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int r = r0 + 2 * t + (q & 1) + 8 * (q >> 1), at = cg * WC + NT * g + i0;
                        const uint8_t* c = smem + buf * S::stage + v_place(r, at >> 4) + (at & 15);
                        const uint32_t w = TN == 4 ? *reinterpret_cast<const uint32_t*>(c) : *reinterpret_cast<const unsigned short*>(c);
                        values4<__nv_bfloat16>(w, p.int8, x[q][0], x[q][1]);
                    }
#pragma unroll
                    for (int i = 0; i < TN; ++i) {
                        b[i][0] = pair_of(x[0][i >> 1], x[1][i >> 1], i & 1);
                        b[i][1] = pair_of(x[2][i >> 1], x[3][i >> 1], i & 1);
                    }
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    float d[TN][4];
                    if constexpr (S::tf32) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {      // rows 2 t + 8 h and the next: k = t and t + 4
                            uint32_t f[2][4];
#pragma unroll
                            for (int q = 0; q < 2; ++q)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int j = 16 * m + g + 8 * e, r = r0 + 2 * t + 8 * h;
                                    const uint2 z = *reinterpret_cast<const uint2*>(pt + q * S::part + j * 256 + (((r >> 2) ^ ((j & 7) << 1)) << 4) + (r & 3) * 4);
                                    f[q][e] = z.x, f[q][2 + e] = z.y;
                                }
#pragma unroll
                            for (int i = 0; i < TN; ++i) {
                                const float2 x = Dt<__half>::up2(b[i][h]);
                                if (h == 0) mma8_tf32_first(d[i], f[1], __float_as_uint(x.x), __float_as_uint(x.y));
                                else mma8_tf32(d[i], f[1], __float_as_uint(x.x), __float_as_uint(x.y));
                                mma8_tf32(d[i], f[0], __float_as_uint(x.x), __float_as_uint(x.y));
                            }
                        }
                    } else {
#pragma unroll
                        for (int q = 2; q >= 0; --q) {     // smallest part first
                            uint32_t f[4];
                            const int j = 16 * m + (lane & 15), c = (r0 >> 3) + (lane >> 4);
                            ldmatrix4(f, part0 + set * S::parts * S::part + q * S::part + j * 128 + ((c ^ (j & 7)) << 4));
#pragma unroll
                            for (int i = 0; i < TN; ++i) {
                                if (q == 2) mma16_first<__nv_bfloat16>(d[i], f, b[i][0], b[i][1]);
                                else mma16<__nv_bfloat16>(d[i], f, b[i][0], b[i][1]);
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < TN; ++i) add4(acc[m][i0 + i], d[i]);
                }
            }
        }
    };
    for (;;) {
    int a, col0;
    if (p.part) {
        __syncthreads();
        const int line = __ldg(p.units + p.n), chunk = at_chunk, unit = at_unit, left = at_left, slot = seg_slot;
        if (left <= 0) break;
        __syncthreads();
        a = find_part(p.units, p.n, unit, lane);
        const int u0 = __ldg(p.units + a), u1 = __ldg(p.units + a + 1), some = max(min(min(u1, line) - unit, left), 1);
        first = max(__ldg(p.offsets + a) + 128 * (unit - u0), 0);
        end = min(min(__ldg(p.offsets + a + 1), p.T), first + 128 * some);
        st0 = 0, st1 = end > first ? (end - first + S::rows - 1) / S::rows : 0;
        col0 = chunk * S::cols;
        if (tid == 0) {
            const bool wrap = unit + some >= line;
            at_left = left - some, at_unit = wrap ? 0 : unit + some, at_chunk = chunk + wrap;
            seg_slot = some == u1 - u0 ? -1 : slot == -2 ? 0 : 1;              // the block's first segment has the first place
        }
    } else {
        const int64_t id = block / size;
        a = (int)(id / chunks), col0 = (int)(id - (int64_t)a * chunks) * S::cols;
        first = max(__ldg(p.offsets + a), 0), end = min(__ldg(p.offsets + a + 1), p.T);
        share_of(end > first ? (end - first + S::rows - 1) / S::rows : 0, rank, size, st0, st1);
        if (tid == 0) seg_slot = -1;
    }
    if (tid == 0) seg_a = a, seg_col = col0;
    vcol = col0 + vc * 16 / es, vleft = p.W - vcol;
    sc = p.scale ? __ldg(p.scale + a) : 1.0f;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[m][i][0] = acc[m][i][1] = acc[m][i][2] = acc[m][i][3] = 0.0f;
    rows_of(st0);
#pragma unroll
    for (int i = 0; i < S::stages - 1; ++i) {
        if (st0 + i < st1) fetch(i);
        async_commit();
        if (st0 + i < st1) put_held(i);
        rows_of(st0 + i + 1);
    }
    int buf = 0;
    if constexpr (S::ahead == 2) {
        static_assert(S::stages == 3, "a stage in use, one being split, one on its way");
        async_wait<1>();
        __syncthreads();
        if (st0 < st1) split(0, 0);
        for (int st = st0; st < st1; ++st) {
            const int set = (st - st0) & 1, after = buf == 2 ? 0 : buf + 1, next = buf == 0 ? 2 : buf - 1;
            async_wait<0>();
            __syncthreads();                               // the next stage is there and this one is split; the one before it is free
            const bool more = st + 2 < st1;
            if (more) fetch(next);
            async_commit();
            rows_of(st + 3);
            // half of the warps of a scheduler begin with the products
            if (!(warp & 4) && st + 1 < st1) split(after, set ^ 1);
            product(buf, set);
            if ((warp & 4) && st + 1 < st1) split(after, set ^ 1);
            if (more) put_held(next);
            buf = after;
        }
    } else {
        for (int st = st0; st < st1; ++st) {
            async_wait<S::stages - 2>();
            __syncthreads();                               // the stage is there; the one before it and the parts are free
            const int next = buf == 0 ? S::stages - 1 : buf - 1;
            const bool more = st + S::stages - 1 < st1;
            if (more) fetch(next);
            async_commit();
            rows_of(st + S::stages);
            split(buf, 0);
            __syncthreads();
            product(buf, 0);
            if (more) put_held(next);
            buf = buf == S::stages - 1 ? 0 : buf + 1;
        }
    }
    async_wait<0>();
    __syncthreads();
    // the warps' sums into shared memory [row group][rank][column], over the stages
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float* to = sums + (rg * RT + 16 * m + g + 8 * h) * S::pitch + cg * WC;
            if constexpr (X8) {                            // NT consecutive columns
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < NT; i += 2) *reinterpret_cast<float2*>(to + NT * (2 * t + c) + i) = make_float2(acc[m][i][2 * h + c], acc[m][i + 1][2 * h + c]);
            } else {
#pragma unroll
                for (int i = 0; i < NT; ++i) *reinterpret_cast<float2*>(to + 8 * i + 2 * t) = make_float2(acc[m][i][2 * h], acc[m][i][2 * h + 1]);
            }
        }
    __syncthreads();
    constexpr int Q = S::cols / 4;                         // pieces of a rank's columns
    if (RG > 1) {
        for (int i = tid; i < R * Q; i += kThreads) {
            float* at = sums + i / Q * S::pitch + i % Q * 4;
            float4 v = *reinterpret_cast<float4*>(at);
#pragma unroll
            for (int k = 1; k < RG; ++k) {
                const float4 q = *reinterpret_cast<const float4*>(at + k * RT * S::pitch);
                v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
            }
            *reinterpret_cast<float4*>(at) = v;
        }
    }
    if (size > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    // each block adds and stores its share of the sums, or, of an adapter that other blocks have a share of, its part of them: first the block's first one
    int i0, i1;
    share_of(R * S::cols / 4, rank, size, i0, i1);
    float* out;
    int wide, pitch = p.W;
    const int slot = seg_slot;
    if (slot < 0) {
        out = p.out + (TRANS ? ((int64_t)seg_a * p.W + seg_col) * R : (int64_t)seg_a * R * p.W + seg_col), wide = p.W - seg_col;
    } else {
        out = p.part + ((int64_t)block * 2 + slot) * (R * S::cols), wide = pitch = S::cols;
    }
    if constexpr (TRANS) {                                 // [column][rank]
        for (int i = i0 + tid; i < i1; i += kThreads) {    // four ranks of one column
            const int c = i / (R / 4), j = 4 * (i % (R / 4));
            float f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) f[k] = size > 1 ? cluster_sum1(sums + (j + k) * S::pitch + c, size) : sums[(j + k) * S::pitch + c];
            if (c < wide) *reinterpret_cast<float4*>(out + c * R + j) = make_float4(f[0], f[1], f[2], f[3]);
        }
    } else {
        for (int i = i0 + tid; i < i1; i += kThreads) {    // four columns of one rank
            const int j = i / Q, c = 4 * (i % Q);
            float* at = sums + j * S::pitch + c;
            const float4 v = size > 1 ? cluster_sum4(at, size) : *reinterpret_cast<float4*>(at);
            float* to = out + (int64_t)j * pitch + c;
            const float f[4] = {v.x, v.y, v.z, v.w};
            if (VEC) {
                if (c < wide) *reinterpret_cast<float4*>(to) = v;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < wide) to[k] = f[k];
            }
        }
    }
    if (!p.part) break;                                    // (else the next segment's stages take the sums' place, after a barrier)
    }
    if (size > 1) {
        cluster_arrive();                                  // (a block's shared memory stays until the others have read it)
        cluster_wait();
    }
}

// Both gradients as one grid, dB's blocks first: they run beside one another, behind one wait for all that they read.
// VB, VA: dY's and X's rows are whole pieces of 16 bytes; X8: X has 8 bits.
template <typename T, bool X8, int R, bool VB, bool VA>
__global__ void __launch_bounds__(kThreads, R >= 128 ? 1 : 2) lora_wgrad_kernel(const WgradP b, const WgradP a, int of_b)
{
    pdl_launch_dependents();
    pdl_wait();
    // (a 16-byte copy moves a sector of 32 bytes in one piece only where source and target lie alike in it: at 48 bytes past a 128-byte line the copies read everything twice, dB of
    // 8192 x 8192 81 us instead of 74)
    extern __shared__ __align__(128) uint8_t smem[];
    if ((int)blockIdx.x < of_b) wgrad<T, false, R, true, VB>(b, blockIdx.x, of_b, smem);
    else wgrad<T, X8, R, false, VA>(a, blockIdx.x - of_b, gridDim.x - of_b, smem);
}

// What the blocks of one weight gradient left in parts.
struct WgradParts {
    const float* part;
    float* out;
    int W, blocks, trans;
};
// Adds the parts of the adapters that several blocks had a share of, in the blocks' order.  blockIdx.x: a border between two blocks of g[0] or g[1]; the first border inside an
// adapter's segment (of one group of 128 columns) does it.  blockIdx.y: 256 of its pieces of 16 bytes.  Bound by latency: 8192 x 2048 x 8192 at r = 32, 6 us.
template <int R> __global__ void __launch_bounds__(kThreads) lora_wgrad_join_kernel(const int* __restrict__ units, int n, const WgradParts g0, const WgradParts g1)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int cols = 128;
    const bool second = (int)blockIdx.x >= g0.blocks - 1;
    const WgradParts& g = second ? g1 : g0;
    const int b = second ? blockIdx.x - (g0.blocks - 1) + 1 : blockIdx.x + 1;                 // block b begins at the border
    const int line = __ldg(units + n), chunks = (g.W + cols - 1) / cols;
    const int64_t total = (int64_t)line * chunks;
    const LineShares shares(total, g.blocks);
    auto begin = [&](int k) { return shares.begin(k); };
    const int64_t here = begin(b);
    if (here >= total) return;
    const int chunk = here <= 0xFFFFFFFFll ? (int)((uint32_t)here / (uint32_t)line) : (int)(here / line);
    const int a = find_part(units, n, (int)(here - (int64_t)chunk * line), threadIdx.x & 31);
    const int64_t from = (int64_t)chunk * line + __ldg(units + a), to = (int64_t)chunk * line + __ldg(units + a + 1);
    if (here == from || begin(b - 1) == here) return;
    if (b > 1 && begin(b - 1) > from) return;
    const int i = blockIdx.y * kThreads + threadIdx.x;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int k0 = b - 1; k0 < g.blocks && begin(k0) < to; k0 += 4) {           // (four loads at a time; a block may have nothing)
        float4 q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = k0 + e;
            const int64_t at = begin(k);
            q[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (k < g.blocks && at < to && at < begin(k + 1)) q[e] = reinterpret_cast<const float4*>(g.part + ((int64_t)k * 2 + (at < from)) * (R * cols))[i];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v.x += q[e].x, v.y += q[e].y, v.z += q[e].z, v.w += q[e].w;
    }
    const int left = g.W - chunk * cols;
    if (g.trans) {
        if (i / (R / 4) < left) reinterpret_cast<float4*>(g.out + ((int64_t)a * g.W + chunk * cols) * R)[i] = v;
    } else {
        const int j = i / (cols / 4), c = 4 * (i % (cols / 4));
        float* out = g.out + ((int64_t)a * R + j) * g.W + chunk * cols + c;
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k < left) out[k] = f[k];
    }
}

// ------------------------------------------------------------------ launches

template <typename F> static qmm_status by_rank(int r, F f)
{
    switch (r) {
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    case 32: return f(std::integral_constant<int, 32>());
    case 64: return f(std::integral_constant<int, 64>());
    default: return f(std::integral_constant<int, 128>());
    }
}

// Blocks of a cluster that share a length of `parts` pieces: a power of two up to `most`, each with at least one piece.
static int cluster_for(int64_t parts, int most)
{
    int c = 1;
    while (c < most && 2 * c <= parts) c *= 2;
    return c;
}

// Tiles that any distribution of T rows over n adapters can need.
static int64_t most_tiles(int64_t T, int64_t n)
{
    const int64_t used = T < n ? T : n;
    return 2 * ((T + 127 * used) / 128);
}

// vx, vy: x and w1, y and w2 have rows of whole 16-byte pieces.
template <typename T, int LAY> static qmm_status launch_pair(const LoraP& p, int r, bool x8, bool vx, bool vy, cudaStream_t st)
{
    return by_rank(r, [&](auto rank) {
        constexpr int R = decltype(rank)::value;
        constexpr int G = Wide<LAY>::cols;
        auto narrowed = [&](auto e8, auto vec) {
            constexpr bool X8 = decltype(e8)::value, VEC = decltype(vec)::value;
            if (p.T <= kSmallRows) {
                constexpr int smem = (kWarps + kSmallBlocks) * 16 * R * 4 + 2 * 16 * u_pitch<R>;              // (at least the 4 KB of the counts)
                static std::atomic<uint64_t> configured{0};
                auto kern = lora_small_kernel<T, X8, R, LAY, VEC>;
                const qmm_status s = configure_once(configured, kern, smem, false, "adapter attributes");
                if (s != QMM_OK) return s;
                // groups of 16 rows that any distribution can need, where they are fewer than the rows; blocks of 256 elements of K or N each, of 64 where that
                // leaves SMs without one (clusters of 16 were slower: 16 x 8192 x 2048 8.8 us against 7.0)
                const int64_t need = (p.T + 15 * (int64_t)(p.T < p.n ? p.T : p.n)) / 16, clusters = need < p.T ? need : p.T;
                const int64_t longest = p.K > p.N ? p.K : p.N;
                const bool grouped = need < p.T && p.T > 16;                  // (up to 16 rows a cluster for each runs at once)
                int size = cluster_for(longest / 256, kSmallBlocks);
                while (size < kSmallBlocks && 2 * size <= longest / 64 && clusters * size * 2 <= 2 * kNumSMs) size *= 2;
                return launch_pdl(kern, dim3((unsigned)((grouped ? clusters : p.T) * size)), kThreads, smem, size, st, "adapter launch", p, (int)(grouped ? need : 0));
            }
            constexpr int smem = NarrowShape<X8, R>::smem;
            static std::atomic<uint64_t> configured{0};
            auto kern = lora_narrow_kernel<T, X8, R, LAY, VEC>;
            const qmm_status s = configure_once(configured, kern, smem, false, "adapter attributes");
            if (s != QMM_OK) return s;
            const int64_t tiles = (p.T + kTileRows - 1) / kTileRows;
            int size = 1;                                  // blocks that share a tile's K: as many as run at once in all, 128 elements each at least
            // (528 blocks where 264 run at once: 24 us against 18.5 for 6000 x 2048 at r = 64)
            const int64_t most = tiles + (p.T < p.n ? p.T : p.n) / 2;
            while (size < 8 && 2 * most * size <= (VEC ? NarrowShape<X8, R>::blocks : 2) * kNumSMs && p.K / (2 * size) >= 128) size *= 2;
            return launch_pdl(kern, dim3((unsigned)(most_tiles(p.T, p.n) * size)), kThreads, smem, size, st, "adapter narrowing launch", p);
        };
        auto first = [&](auto vec) {
            if constexpr (LAY == 0) return x8 ? narrowed(std::true_type(), vec) : narrowed(std::false_type(), vec);
            else return narrowed(std::false_type(), vec);
        };
        const bool small = p.T <= kSmallRows, v1 = small ? vx && vy : vx;
        const qmm_status s = v1 ? first(std::true_type()) : first(std::false_type());
        if (s != QMM_OK || small || !p.y) return s;
        const int groups = (p.N + G - 1) / G;
        // column groups of a block: 1024 columns, fewer where that leaves less than two blocks per SM (always whole stages of 128 columns).  2048 x 4096 x 28672, replayed on the same
        // rows: 512 columns 68.6 us, 1024 58.5, 2048 58.0; on other rows from call to call 1024 68, 2048 78 (the last round is longer).
        int per_span = 1024 / G;
        while (per_span > 256 / G && (int64_t)((p.T + kTileRows - 1) / kTileRows) * ((groups + per_span - 1) / per_span) < 2 * kNumSMs) per_span /= 2;
        const int spans = (groups + per_span - 1) / per_span;
        const int64_t blocks = most_tiles(p.T, p.n) * spans, rest = p.rest ? (int64_t)((p.T + kTileRows - 1) / kTileRows) * spans : 0;
        if (blocks + rest > 0x7FFFFFFF) return fail(QMM_ERR_UNSUPPORTED, "adapters: %lld blocks are too many for one launch", (long long)(blocks + rest));
        auto widened = [&](auto vec) {
            constexpr bool VEC = decltype(vec)::value;
            constexpr int smem = 2 * kTileRows * u_pitch<R> + WideShape<R, LAY>::stages * WideShape<R, LAY>::stage;
            static std::atomic<uint64_t> configured{0};
            auto kern = lora_widen_kernel<T, R, LAY, VEC>;
            const qmm_status c = configure_once(configured, kern, smem, false, "adapter attributes");
            if (c != QMM_OK) return c;
            return launch_pdl(kern, dim3((unsigned)(blocks + rest)), kThreads, smem, 1, st, "adapter widening launch", p, spans, per_span, (int)blocks);
        };
        return vy ? widened(std::true_type()) : widened(std::false_type());
    });
}

// dB (b.out null: not wanted) and dA (a.out null).
template <typename T, bool X8> static qmm_status launch_wgrads(const WgradP& b, const WgradP& a, int r, bool vb, bool va, cudaStream_t st)
{
    return by_rank(r, [&](auto rank) {
        constexpr int R = decltype(rank)::value;
        using SB = WgradShape<T, false, R>;
        using SA = WgradShape<T, X8, R>;
        auto go = [&](auto vec_b, auto vec_a) {
            constexpr int most = SB::smem > SA::smem ? SB::smem : SA::smem;
            static std::atomic<uint64_t> configured{0};
            auto kern = lora_wgrad_kernel<T, X8, R, decltype(vec_b)::value, decltype(vec_a)::value>;
            const qmm_status s = configure_once(configured, kern, most, false, "adapter gradient attributes");
            if (s != QMM_OK) return s;
            const WgradP& any = b.out ? b : a;
            const int smem = b.out ? most : SA::smem;
            if (any.part) return launch_pdl(kern, dim3((unsigned)(b.blocks + a.blocks)), kThreads, smem, 1, st, "adapter gradient launch", b, a, b.blocks);
            const int64_t of_b = b.out ? (int64_t)b.n * ((b.W + SB::cols - 1) / SB::cols) : 0, of_a = a.out ? (int64_t)a.n * ((a.W + SA::cols - 1) / SA::cols) : 0;
            const int64_t columns = of_b + of_a;
            // blocks that share a column's rows: as many as make about two per SM in all, 128 rows each at least if one adapter had them all, 96 up to r = 16, where a stage's products
            // are short (dS, dA and dB of 500 x 1001 x 700 at r = 8: 17.3 us with 96, 19.8 with 128; 390 x 512 x 2048 at r = 64: 29.2 and 27.2)
            int size = 1;
            while (size < 8 && columns * size < 3 * kNumSMs / 2 && (int64_t)any.T >= (R <= 16 ? 192 : 256) * size) size *= 2;
            if (columns * size > 0x7FFFFFFF) return fail(QMM_ERR_UNSUPPORTED, "adapter gradients: %lld blocks are too many for one launch", (long long)(columns * size));
            return launch_pdl(kern, dim3((unsigned)(columns * size)), kThreads, smem, size, st, "adapter gradient launch", b, a, (int)(of_b * size));
        };
        if (vb) return va ? go(std::true_type(), std::true_type()) : go(std::true_type(), std::false_type());
        return va ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
    });
}

// Blocks of both weight gradients that run at once.
static inline int wgrad_blocks(int r) { return (r >= 128 ? 1 : 2) * kNumSMs; }
// Of `blocks`, those of a gradient of `W` columns beside one of `other` (0: none): by their columns, tf32 products counted 1.5 times (6000 rows of fp16 codes at r = 64 with
// 2048 columns each: 73 us by tf32, 49 by bf16, with 148 blocks), and no more than there are units of 128 rows.
static inline int wgrad_share(int blocks, int64_t T, int64_t W, bool tf32, int64_t other, bool other_tf32)
{
    const int64_t columns = (W + 127) / 128, units = columns * ((T + 127) / 128), mine = columns * (tf32 ? 3 : 2), theirs = (other + 127) / 128 * (other_tf32 ? 3 : 2);
    int64_t b = theirs ? (2 * blocks * mine + mine + theirs) / (2 * (mine + theirs)) : blocks;
    b = b < 1 ? 1 : theirs && b > blocks - 1 ? blocks - 1 : b;
    return (int)(b < units ? b : units);
}

}  // namespace lora

// forward: both products of x with (A, B); backward: of dy with (B, A)
#define QMM_LORA_TYPE(NAME, TYPE)                                                                                                                          \
    qmm_status launch_lora_##NAME(const lora::LoraP& p, int r, bool x8, bool back, bool vx, bool vy, cudaStream_t st)                                      \
    {                                                                                                                                                      \
        return back ? lora::launch_pair<TYPE, 1>(p, r, false, vx, vy, st) : lora::launch_pair<TYPE, 0>(p, r, x8, vx, vy, st);                              \
    }
#define QMM_LORA_WGRAD_TYPE(NAME, TYPE, X8)                                                                                                                \
    qmm_status launch_lora_wgrad_##NAME(const lora::WgradP& b, const lora::WgradP& a, int r, bool vb, bool va, cudaStream_t st)                            \
    {                                                                                                                                                      \
        return lora::launch_wgrads<TYPE, X8>(b, a, r, vb, va, st);                                                                                         \
    }

// The parts of one or two (g1.blocks > 0) weight gradients.
#define QMM_LORA_JOIN                                                                                                                                      \
    qmm_status launch_lora_join(int r, const int* units, int n, const lora::WgradParts& g0, const lora::WgradParts& g1, cudaStream_t st)                   \
    {                                                                                                                                                      \
        const int borders = g0.blocks - 1 + (g1.blocks > 0 ? g1.blocks - 1 : 0);                                                                           \
        if (borders == 0) return QMM_OK;                                                                                                                   \
        return lora::by_rank(r, [&](auto rank) {                                                                                                           \
            constexpr int R = decltype(rank)::value;                                                                                                       \
            return launch_pdl(lora::lora_wgrad_join_kernel<R>, dim3((unsigned)borders, R / 8), lora::kThreads, 0, 1, st, "adapter gradient parts launch", units, n, g0, g1); \
        });                                                                                                                                                \
    }

}  // namespace qmm
