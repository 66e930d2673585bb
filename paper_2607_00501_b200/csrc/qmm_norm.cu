// qmm_norm.cu -- root-mean-square norm with the residual's addition, into rows of the input's type and / or rows of 8 bits with a scale
// each, its gradient, and the 8-bit rows by themselves.
//
//   h = rn(x + residual);  rstd = (mean h^2 + eps)^-1/2;  y = h * rstd * w
//   8 bits: t = fp32(h * w), amax = max |t|, code = rn8(fp32(t * fp32(L / amax))), scale = amax * rstd / L, L = 448 (e4m3) or 127 (int8)
//
// The codes are those of t, not of y: rstd is one factor of the whole row, so it cancels in t / amax, and a code does not depend on the order in
// which the squares were added.  Every element is read once and written once: a row lives in the registers of its threads.
#include "qmm_async.cuh"
#include "qmm_launch.cuh"
#include "qmm_mx.cuh"

#include <float.h>

namespace qmm {

using namespace mx;

// V elements of a row as loaded.
template <typename T, int V> struct Piece {
    static constexpr int B = V * (int)sizeof(T);
    static constexpr int W = B >= 4 ? B / 4 : 1;
    uint32_t u[W];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (B == 16) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            u[0] = q.x, u[1] = q.y, u[2] = q.z, u[3] = q.w;
        } else if constexpr (B == 4) {
            u[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            u[0] = *reinterpret_cast<const unsigned short*>(p);
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (B == 16) *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
        else if constexpr (B == 4) *reinterpret_cast<uint32_t*>(p) = u[0];
        else *reinterpret_cast<unsigned short*>(p) = (unsigned short)u[0];
    }
    __device__ __forceinline__ void fill(uint32_t v)
    {
#pragma unroll
        for (int i = 0; i < W; ++i) u[i] = v;
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(u[i]);
        } else {
            const float2 f = Dt<T>::up2(u[i >> 1]);
            return i & 1 ? f.y : f.x;
        }
    }
    __device__ __forceinline__ void set(const float (&f)[V])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] = __float_as_uint(f[i]);
        } else if constexpr (V == 1) {
            u[0] = Dt<T>::down2(f[0], 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) u[i] = Dt<T>::down2(f[2 * i], f[2 * i + 1]);
        }
    }
};

// Sum of a and largest magnitude of b (a NaN stays) over the `threads` threads of a row; the same value, added in the same order, on each.  `red`: two floats per warp.
__device__ __forceinline__ void row_reduce(float& a, float& b, int threads, int barrier, int tid, float* red)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        b = maxabs(b, __shfl_xor_sync(0xFFFFFFFFu, b, o));
    }
    if (threads == 32) return;
    const int warps = threads >> 5;
    if ((tid & 31) == 0) {
        red[2 * (tid >> 5)] = a;
        red[2 * (tid >> 5) + 1] = b;
    }
    asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory");
    const int at = (tid & 31) < warps ? tid & 31 : 0;
    a = (tid & 31) < warps ? red[2 * at] : 0.0f;
    b = red[2 * at + 1];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        b = maxabs(b, __shfl_xor_sync(0xFFFFFFFFu, b, o));
    }
    asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory");      // red may be written again
}

// 1 / sqrt(mean + eps) of a sum of squares.
__device__ __forceinline__ float rstd_of(float ss, int K, float eps) { return 1.0f / sqrtf(ss / (float)K + eps); }
// Sums of squares outside this range have lost values to fp32's ends and are formed again with scaled elements: by 2^64 in small rows, by 2^-80 in large ones, so that the sum
// of 32768 squares of the type's largest number is 2^111.
__device__ __forceinline__ bool off_range(float ss) { return !(ss < FLT_MAX) || ss < 0x1p-90f; }
__device__ __forceinline__ float square_scale(bool small) { return small ? 0x1p64f : 0x1p-80f; }
// Their rstd is up * the returned number: that of a large row alone would be below fp32's normal numbers.
__device__ __forceinline__ float rstd_scaled(float ss, int K, float eps, bool small, float& up)
{
    up = small ? 1.0f : 0x1p-64f;
    return (float)((small ? 1.0 : 0x1p64) / sqrt((double)ss / K * (small ? 0x1p-128 : 0x1p160) + (double)eps));
}

struct NormP {
    int64_t rows, ldx, ldr, ldh, ldy, ldc;
    int K, nv, tpr;                                        // nv: vectors per row; tpr: threads per row
    const void *x, *res, *w;                               // w null: 1
    void *h, *y;                                           // optional
    uint8_t* codes;                                        // optional
    float* scales;
    int int8, norm;                                        // norm 0: rstd = 1
    float eps;
};

__device__ __forceinline__ uint32_t code8(float a, int int8)
{
    if (int8) return (uint32_t)__float2int_rn(fminf(fmaxf(a, -127.0f), 127.0f)) & 0xFFu;
    return (uint32_t)__nv_cvt_float_to_fp8(a, __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t code8x2(float a, float b, int int8)
{
    if (int8) return code8(a, 1) | (code8(b, 1) << 8);
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// A row by p.tpr threads, NV vectors of V elements each; blocks of several rows where a row needs fewer than the block's threads.
// Bound by HBM: 8192 x 8192 bf16 with a residual into h and e4m3 rows, 470 MB in 77 us (6.1 TB/s); 8192 x 4096 into h and y, 268 MB in 48 us (5.6 TB/s).  With few rows bound by
// the launch and two dependent loads: 4 x 2048 in 2.0 us.
template <typename T, int V, int NV>
__global__ void __launch_bounds__(1024) rms_norm_kernel(const NormP p)
{
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float red[64];
    const int tpr = p.tpr, group = threadIdx.x / tpr, tid = threadIdx.x - group * tpr;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / tpr) + group;
    if (row >= p.rows) return;                             // (a whole row group leaves: its barrier is its own)
    const T* x = (const T*)p.x + row * p.ldx;
    const T* res = p.res ? (const T*)p.res + row * p.ldr : nullptr;
    Piece<T, V> h[NV], w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        h[i].fill(0u);
        w[i].fill(0u);
        const int v = tid + i * tpr;
        if (v < p.nv) h[i].load(x + v * V);
    }
    if (res) {
        Piece<T, V> r[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            r[i].fill(0u);
            const int v = tid + i * tpr;
            if (v < p.nv) r[i].load(res + v * V);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float f[V];
#pragma unroll
            for (int k = 0; k < V; ++k) f[k] = h[i].get(k) + r[i].get(k);
            h[i].set(f);
        }
    }
    if (p.w) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * tpr;
            if (v < p.nv) w[i].load((const T*)p.w + v * V);
        }
    } else {
        float one[V];
#pragma unroll
        for (int k = 0; k < V; ++k) one[k] = 1.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) w[i].set(one);
    }
    if (p.h) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * tpr;
            if (v < p.nv) h[i].store((T*)p.h + row * p.ldh + v * V);
        }
    }
    float ss = 0.0f, amax = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float f = h[i].get(k);
            ss = fmaf(f, f, ss);
            if (p.codes) amax = maxabs(amax, f * w[i].get(k));
        }
    row_reduce(ss, amax, tpr, 1 + group, tid, red + 2 * (group * (tpr >> 5)));
    float rstd = 1.0f, up = 1.0f;                          // (the row's rstd is up * rstd; up is 1 but for the largest rows)
    if (p.norm) {
        rstd = rstd_of(ss, p.K, p.eps);
        if (off_range(ss)) {                               // (the same on every thread of the row)
            const bool small = ss < 1.0f;
            const float f = square_scale(small);
            float again = 0.0f, none = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float e = h[i].get(k) * f;
                    again = fmaf(e, e, again);
                }
            row_reduce(again, none, tpr, 1 + group, tid, red + 2 * (group * (tpr >> 5)));
            rstd = rstd_scaled(again, p.K, p.eps, small, up);
        }
    }
    if (p.y) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * tpr;
            float f[V];
#pragma unroll
            for (int k = 0; k < V; ++k) f[k] = h[i].get(k) * up * rstd * w[i].get(k);
            Piece<T, V> o;
            o.set(f);
            if (v < p.nv) o.store((T*)p.y + row * p.ldy + v * V);
        }
    }
    if (p.codes) {
        const float top = p.int8 ? 127.0f : 448.0f;
        const bool fine = amax < INFINITY, zero = amax < 0x1p-118f;         // (a NaN is neither)
        const float inv = fine && !zero ? top / amax : 0.0f;
        if (tid == 0) p.scales[row] = !fine ? __int_as_float(0x7FC00000) : zero ? 0.0f : amax / top * up * rstd;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * tpr;
            if (v >= p.nv) continue;
            uint8_t* o = p.codes + row * p.ldc + v * V;
            uint32_t c[V > 4 ? 2 : 1] = {};
            if (fine && !zero) {
                if constexpr (V == 1) c[0] = code8(h[i].get(0) * w[i].get(0) * inv, p.int8);
                else {
#pragma unroll
                    for (int k = 0; k < V; k += 2)
                        c[k >> 2] |= code8x2(h[i].get(k) * w[i].get(k) * inv, h[i].get(k + 1) * w[i].get(k + 1) * inv, p.int8) << (8 * (k & 2));
                }
            }
            if constexpr (V == 8) *reinterpret_cast<uint2*>(o) = make_uint2(c[0], c[1]);
            else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(o) = c[0];
            else *o = (uint8_t)c[0];
        }
    }
}

// ------------------------------------------------------------------ gradient
//
//   xhat = h * rstd;  dx = rstd * (w dy - xhat * mean(w dy xhat)) (+ dh);  dw = sum over rows of dy * xhat
//
// One pass over h and dy.  A block takes every gridDim-th row and keeps its part of dw in registers, which it writes once; the parts are added by a second launch in
// block order: the same bits on every call.

struct NormGradP {
    int64_t rows, lddy, ldh, lddh, lddx;
    int K, nv;
    const void *dy, *h, *w, *dh;                           // w null: 1; dh optional
    void* dx;                                              // optional
    float* part;                                           // [gridDim, K], null: dw is not wanted
    float eps;
};

// Sums of a and b over the block, the same on every thread, added in a fixed order.
__device__ __forceinline__ void block_sum2(float& a, float& b, float (*red)[64])
{
    const int tid = threadIdx.x, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
    }
    if (warps == 1) return;
    __syncthreads();                                       // the sums before these have been read
    if ((tid & 31) == 0) red[0][tid >> 5] = a, red[1][tid >> 5] = b;
    __syncthreads();
    const bool mine = (tid & 31) < warps;
    a = mine ? red[0][tid & 31] : 0.0f;
    b = mine ? red[1][tid & 31] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        b += __shfl_xor_sync(0xFFFFFFFFu, b, o);
    }
}

//   dx = rstd (w dy - xhat mean(w dy xhat)) + dh, xhat = h rstd;   dw = sum over the rows of dy xhat
// A block takes every gridDim.x-th row and keeps its share of dw in registers; the parts are added by rms_norm_dw_kernel.  Bound by HBM: 8192 x 4096 bf16 with dh, 268 MB in
// 45 us (6.0 TB/s), straight into registers 77 us.
// RING > 0: the rows of h, dy and dh come through shared memory, RING rows in flight (cp.async; a thread reads what it copied itself, so the rows need no
// barrier).  RING 0: straight into registers, for rows that are not 16-byte aligned or too long for that.
template <typename T, int V, int NV, int RING>
__global__ void __launch_bounds__(NV <= 4 ? 512 : 1024) rms_norm_grad_kernel(const NormGradP p)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ __align__(16) uint8_t ring[];        // [RING][h, dy, dh][NV][threads] pieces of 16 bytes
    __shared__ float red[2][64];
    const int tpr = blockDim.x, tid = threadIdx.x;
    Piece<T, V> w[NV];
    float dw[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = tid + i * tpr;
        float one[V];
#pragma unroll
        for (int k = 0; k < V; ++k) one[k] = 1.0f, dw[i][k] = 0.0f;
        w[i].set(one);
        if (p.w && v < p.nv) w[i].load((const T*)p.w + v * V);
    }
    const int parts = p.dh ? 3 : 2;
    auto place = [&](int slot, int which, int i) { return ((slot * parts + which) * NV + i) * tpr * 16 + tid * 16; };
    auto fetch = [&](int64_t row, int slot) {
        if constexpr (RING > 0) {
            if (row < p.rows) {
                const uint32_t base = (uint32_t)__cvta_generic_to_shared(ring);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int v = tid + i * tpr, n = v < p.nv ? 16 : 0, at = v < p.nv ? v * V : 0;
                    async16(base + place(slot, 0, i), (const T*)p.h + row * p.ldh + at, n);
                    async16(base + place(slot, 1, i), (const T*)p.dy + row * p.lddy + at, n);
                    if (p.dh) async16(base + place(slot, 2, i), (const T*)p.dh + row * p.lddh + at, n);
                }
            }
            async_commit();
        }
    };
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) fetch(blockIdx.x + (int64_t)i * gridDim.x, i);
    int slot = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        Piece<T, V> h[NV], dy[NV];
        if constexpr (RING > 0) {
            fetch(row + (int64_t)(RING - 1) * gridDim.x, slot == 0 ? RING - 1 : slot - 1);
            async_wait<RING - 1>();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                h[i].load(reinterpret_cast<const T*>(ring + place(slot, 0, i)));
                dy[i].load(reinterpret_cast<const T*>(ring + place(slot, 1, i)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                h[i].fill(0u);
                dy[i].fill(0u);
                const int v = tid + i * tpr;
                if (v < p.nv) {
                    h[i].load((const T*)p.h + row * p.ldh + v * V);
                    dy[i].load((const T*)p.dy + row * p.lddy + v * V);
                }
            }
        }
        float ss = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float f = h[i].get(k);
                ss = fmaf(f, f, ss);
                dot = fmaf(w[i].get(k) * dy[i].get(k), f, dot);
            }
        block_sum2(ss, dot, red);
        float rstd = rstd_of(ss, p.K, p.eps), c = rstd * (rstd * dot / (float)p.K), up = 1.0f;         // rstd * mean(w dy xhat); rstd and c are times up
        if (off_range(ss)) {                               // (the same on every thread)
            const bool small = ss < 1.0f;
            const float f = square_scale(small);
            float again = 0.0f, none = 0.0f, mean = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float e = h[i].get(k) * f;
                    again = fmaf(e, e, again);
                }
            block_sum2(again, none, red);
            rstd = rstd_scaled(again, p.K, p.eps, small, up);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k) mean = fmaf(w[i].get(k) * dy[i].get(k), h[i].get(k) * up * rstd, mean);
            block_sum2(mean, none, red);
            c = rstd * (mean / (float)p.K);
        }
        auto put = [&](auto largest) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = tid + i * tpr;
                Piece<T, V> dh;
                dh.fill(0u);
                if constexpr (RING > 0) {
                    if (p.dh) dh.load(reinterpret_cast<const T*>(ring + place(slot, 2, i)));
                } else {
                    if (p.dh && v < p.nv) dh.load((const T*)p.dh + row * p.lddh + v * V);
                }
                float f[V];
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float g = w[i].get(k) * dy[i].get(k);
                    float xhat;
                    if constexpr (decltype(largest)::value) {
                        xhat = h[i].get(k) * up * rstd;
                        f[k] = fmaf(up, fmaf(rstd, g, -c * xhat), dh.get(k));
                    } else {
                        xhat = h[i].get(k) * rstd;
                        f[k] = fmaf(rstd, g, fmaf(-c, xhat, dh.get(k)));
                    }
                    dw[i][k] = fmaf(dy[i].get(k), xhat, dw[i][k]);
                }
                Piece<T, V> o;
                o.set(f);
                if (p.dx && v < p.nv) o.store((T*)p.dx + row * p.lddx + v * V);
            }
        };
        if (up == 1.0f) put(std::false_type());
        else put(std::true_type());
        if (RING > 0) slot = slot == RING - 1 ? 0 : slot + 1;
    }
    if (RING > 0) async_wait<0>();
    if (p.part) {
        float* part = p.part + (int64_t)blockIdx.x * p.K;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = tid + i * tpr;
            if (v >= p.nv) continue;
            if constexpr (V >= 4) {
#pragma unroll
                for (int k = 0; k < V; k += 4) *reinterpret_cast<float4*>(part + v * V + k) = make_float4(dw[i][k], dw[i][k + 1], dw[i][k + 2], dw[i][k + 3]);
            } else {
                part[v] = dw[i][0];
            }
        }
    }
}

// The blocks' parts of dw in a fixed order: 32 columns by 32 shares of the parts per block (all of a share's loads are in flight at once up to 512 parts).  Bound by latency:
// 592 parts of 4096 columns, 9.7 MB out of L2, 6.6 us; a thread for each column's parts took 16.5.
constexpr int kColThreads = 1024;
__global__ void __launch_bounds__(kColThreads) rms_norm_dw_kernel(const float* __restrict__ part, int parts, int K, float* __restrict__ dw)
{
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float red[32][33];
    const int lane = threadIdx.x & 31, share = threadIdx.x >> 5, k = blockIdx.x * 32 + lane;
    float s = 0.0f;
    for (int i0 = share; i0 < parts; i0 += 512) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = k < K && i0 + 32 * i < parts ? part[(int64_t)(i0 + 32 * i) * K + k] : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += v[i];
    }
    red[share][lane] = s;
    __syncthreads();
    s = red[lane][share];                                  // warp `share`: column `share` of the block
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0 && blockIdx.x * 32 + share < K) dw[blockIdx.x * 32 + share] = s;
}

// ------------------------------------------------------- 8-bit rows back to values

// Thread = V codes of a row.  Bound by HBM: 8192 x 8192 into bf16, 201 MB in 35 us (5.7 TB/s; the measured copy rate is 6.6).
template <typename T, int V>
__global__ void __launch_bounds__(256) rows8_dequantize_kernel(const uint8_t* __restrict__ codes, int64_t ldc, const float* __restrict__ scales, int int8, int64_t rows, int nv,
                                                               T* __restrict__ out, int64_t ldo)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = id / nv;
    if (row >= rows) return;
    const int64_t k = (id - row * nv) * V;
    const uint8_t* c = codes + row * ldc + k;
    uint32_t u[V >= 4 ? V / 4 : 1];
    if constexpr (V == 16) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(c));
        u[0] = q.x, u[1] = q.y, u[2] = q.z, u[3] = q.w;
    } else if constexpr (V == 8) {
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(c));
        u[0] = q.x, u[1] = q.y;
    } else {
        u[0] = __ldg(c);
    }
    const float s = __ldg(scales + row);
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t b = u[i >> 2] >> (8 * (i & 3)) & 0xFFu;
        f[i] = s * (int8 ? (float)(int8_t)b : __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)b, __NV_E4M3))));
    }
    constexpr int S = V * (int)sizeof(T) >= 16 ? 16 / (int)sizeof(T) : V;     // elements per store
#pragma unroll
    for (int i = 0; i < V; i += S) {
        Piece<T, S> o;
        float g[S];
#pragma unroll
        for (int j = 0; j < S; ++j) g[j] = f[i + j];
        o.set(g);
        o.store(out + row * ldo + k + i);
    }
}

// ------------------------------------------------------------------ launches

static uintptr_t norm_bits(const void* p, int64_t ld, int size) { return p ? reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size) : 0; }

// Threads per row and vectors per thread of a row of nv vectors.  Many rows: four vectors a thread keep more bytes in flight per warp and meet in fewer barriers;
// few rows (less than a warp per scheduler): one vector a thread, for latency.  In us, GPU time of the whole call:
//                                          one    two   four  eight vectors
//   4 x 2048 fp16                          2.0    2.1    2.6    5.2
//   500 x 1001 fp32, with gradients       14.2   12.2    9.7   10.8        (rows that begin anywhere: single elements)
//   8192 x 8192 bf16 to e4m3 and back      153    133    110    174
//   8192 x 4096 bf16, with gradients       102     98    101    135
struct NormShape {
    int tpr, per;
};
static NormShape norm_shape(int nv, int64_t rows, int most_threads)
{
    int per = rows * ((nv + 127) / 128) >= 4 * kNumSMs ? 4 : 1;
    while (per < 4 && (nv + per - 1) / per > most_threads) per *= 2;
    while (per < 32 && (nv + per - 1) / per > 1024) per *= 2;
    int tpr = 32;
    while (tpr * per < nv) tpr *= 2;
    while (per > 1 && tpr * (per / 2) >= nv) per /= 2;
    return {tpr, per};
}

template <typename F> static qmm_status norm_by_shape(int dtype, bool vec, int per, F f)
{
    auto by_per = [&](auto type, auto v) {
        if (per <= 1) return f(type, v, std::integral_constant<int, 1>());
        if (per <= 2) return f(type, v, std::integral_constant<int, 2>());
        if (per <= 4) return f(type, v, std::integral_constant<int, 4>());
        if constexpr (decltype(v)::value > 1) {            // 1024 threads of 8 vectors cover 32768 elements of either size
            return f(type, v, std::integral_constant<int, 8>());
        } else {
            if (per <= 8) return f(type, v, std::integral_constant<int, 8>());
            return f(type, v, std::integral_constant<int, 32>());
        }
    };
    if (dtype == QMM_F32) return vec ? by_per(float(), std::integral_constant<int, 4>()) : by_per(float(), std::integral_constant<int, 1>());
    if (dtype == QMM_F16) return vec ? by_per(__half(), std::integral_constant<int, 8>()) : by_per(__half(), std::integral_constant<int, 1>());
    return vec ? by_per(__nv_bfloat16(), std::integral_constant<int, 8>()) : by_per(__nv_bfloat16(), std::integral_constant<int, 1>());
}

qmm_status launch_rms_norm(int dtype, const void* x, int64_t ldx, const void* res, int64_t ldr, const void* w, float eps, int64_t rows, int K, void* h, int64_t ldh,
                           void* y, int64_t ldy, int row8, void* codes, int64_t ldc, float* scales, int norm, cudaStream_t st)
{
    const int size = dtype == QMM_F32 ? 4 : 2, V = 16 / size;
    const uintptr_t bits = norm_bits(x, ldx, size) | norm_bits(res, ldr, size) | norm_bits(w, 0, size) | norm_bits(h, ldh, size) | norm_bits(y, ldy, size);
    const bool vec = K % V == 0 && bits % 16 == 0 && norm_bits(codes, ldc, 1) % V == 0;
    const int nv = vec ? K / V : K;
    const NormShape s = norm_shape(nv, rows, 1024);
    NormP p = {rows, ldx, ldr, ldh, ldy, ldc, K, nv, s.tpr, x, res, w, h, y, (uint8_t*)codes, scales, row8, norm, eps};
    const int threads = s.tpr < 128 ? 128 : s.tpr;
    const int per_block = threads / s.tpr;
    const dim3 grid((unsigned)((rows + per_block - 1) / per_block));
    return norm_by_shape(dtype, vec, s.per, [&](auto type, auto v, auto n) {
        return launch_pdl(rms_norm_kernel<decltype(type), decltype(v)::value, decltype(n)::value>, grid, threads, 0, 1, st, "root-mean-square norm launch", p);
    });
}

// Blocks of the gradient: as many as run at once (two per SM of up to 512 threads, four of up to 256); each writes a part of dw.  (500 rows of 1001: a block for each 5 us
// and 5 for the sum of the parts; 148 blocks 9.7 and 5.)
constexpr int kGradBlocks = 4 * kNumSMs;
static int norm_grad_blocks(int64_t rows, int tpr)
{
    const int64_t most = tpr > 512 ? kNumSMs : tpr > 256 ? 2 * kNumSMs : kGradBlocks;
    return (int)(rows < most ? rows : most);
}
size_t rms_norm_grad_workspace_bytes(int64_t rows, int K) { return (size_t)(rows < kGradBlocks ? rows : kGradBlocks) * (size_t)K * 4; }

qmm_status launch_rms_norm_grad(int dtype, const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* w, float eps, int64_t rows, int K, const void* dh,
                                int64_t lddh, void* dx, int64_t lddx, float* dw, void* ws, cudaStream_t st)
{
    const int size = dtype == QMM_F32 ? 4 : 2, V = 16 / size;
    const uintptr_t bits = norm_bits(dy, lddy, size) | norm_bits(h, ldh, size) | norm_bits(w, 0, size) | norm_bits(dh, lddh, size) | norm_bits(dx, lddx, size);
    const bool vec = K % V == 0 && bits % 16 == 0;
    const int nv = vec ? K / V : K;
    // vectors per thread: two with rows in a ring (few registers, many threads), as in the forward pass without
    const int stage = (dh ? 3 : 2) * 16;                   // bytes of a row in the ring, per vector
    int tpr = 32, per = 2;
    while (tpr < 512 && 2 * tpr < nv) tpr *= 2;
    if (2 * tpr < nv) per = 4;
    bool in_ring = vec && per * tpr >= nv && (size_t)per * tpr * stage * 2 <= 200 * 1024;
    NormShape s = {tpr, per};
    if (!in_ring) {
        s = norm_shape(nv, rows, 512);                     // (the kernels of up to four vectors are built for 512 threads)
        if (s.per <= 4 && s.tpr > 512) s.per = 8;
    }
    const int blocks = norm_grad_blocks(rows, s.tpr);
    NormGradP p = {rows, lddy, ldh, lddh, lddx, K, nv, dy, h, w, dh, dx, dw ? (float*)ws : nullptr, eps};
    const size_t row_bytes = (size_t)s.per * s.tpr * stage;
    const bool three = row_bytes * 3 <= 72 * 1024 || (row_bytes * 3 <= 200 * 1024 && s.tpr > 256);
    const qmm_status e = norm_by_shape(dtype, vec, s.per, [&](auto type, auto v, auto n) {
        using D = decltype(type);
        constexpr int VV = decltype(v)::value, NV = decltype(n)::value;
        if constexpr (VV > 1 && (NV == 2 || NV == 4)) {
            if (in_ring) {
                auto go = [&](auto rows_in_flight) {
                    constexpr int RING = decltype(rows_in_flight)::value;
                    auto kern = rms_norm_grad_kernel<D, VV, NV, RING>;
                    static std::atomic<uint64_t> configured{0};
                    const qmm_status c = configure_once(configured, kern, 200 * 1024, false, "norm gradient attributes");
                    if (c != QMM_OK) return c;
                    return launch_pdl(kern, dim3((unsigned)blocks), s.tpr, row_bytes * RING, 1, st, "root-mean-square norm gradient launch", p);
                };
                return three ? go(std::integral_constant<int, 3>()) : go(std::integral_constant<int, 2>());
            }
        }
        return launch_pdl(rms_norm_grad_kernel<D, VV, NV, 0>, dim3((unsigned)blocks), s.tpr, 0, 1, st, "root-mean-square norm gradient launch", p);
    });
    if (e != QMM_OK || !dw) return e;
    return launch_pdl(rms_norm_dw_kernel, dim3((unsigned)((K + 31) / 32)), kColThreads, 0, 1, st, "norm weight gradient launch", (const float*)ws, blocks, K, dw);
}

template <typename T, int V>
static qmm_status dequantize_t(const void* codes, int64_t ldc, const float* scales, int int8, int64_t rows, int K, void* out, int64_t ldo, cudaStream_t st)
{
    const int nv = K / V;
    const int64_t blocks = (rows * nv + 255) / 256;
    if (blocks > 0x7FFFFFFF) return fail(QMM_ERR_UNSUPPORTED, "%lld row vectors are too many for one launch", (long long)(rows * nv));
    return launch_pdl(rows8_dequantize_kernel<T, V>, dim3((unsigned)blocks), 256, 0, 1, st, "8-bit rows launch", (const uint8_t*)codes, ldc, scales, int8, rows, nv, (T*)out,
                      ldo);
}
template <typename T> static qmm_status dequantize_v(const void* codes, int64_t ldc, const float* scales, int int8, int64_t rows, int K, void* out, int64_t ldo, cudaStream_t st)
{
    const bool wide = norm_bits(out, ldo, (int)sizeof(T)) % 16 == 0;
    const uintptr_t bits = norm_bits(codes, ldc, 1) | (uintptr_t)K;
    if (wide && bits % 16 == 0) return dequantize_t<T, 16>(codes, ldc, scales, int8, rows, K, out, ldo, st);
    if (wide && bits % 8 == 0) return dequantize_t<T, 8>(codes, ldc, scales, int8, rows, K, out, ldo, st);
    return dequantize_t<T, 1>(codes, ldc, scales, int8, rows, K, out, ldo, st);
}
qmm_status launch_rows8_dequantize(int row8, const void* codes, int64_t ldc, const float* scales, int64_t rows, int K, int dtype, void* out, int64_t ldo, cudaStream_t st)
{
    if (dtype == QMM_F16) return dequantize_v<__half>(codes, ldc, scales, row8, rows, K, out, ldo, st);
    if (dtype == QMM_BF16) return dequantize_v<__nv_bfloat16>(codes, ldc, scales, row8, rows, K, out, ldo, st);
    return dequantize_v<float>(codes, ldc, scales, row8, rows, K, out, ldo, st);
}

}  // namespace qmm
