// qmm_mx_quant.cu -- microscaled 4-bit floating point: canonical -> packed, quantisation (plain, and of
// tokens into the experts' row order) and dequantisation.  All are bound by HBM: one pass over the data, a thread
// per 32 elements.
#include "qmm_mx.cuh"

namespace qmm {

using namespace mx;

constexpr int kQuantThreads = 256;

// Where a token's pairs go (grouped rows), or nothing (plain rows).
struct MxRows {
    const int *idx, *place, *offsets, *units;
    int topk, E;
};

// Rows that 16-byte accesses cannot reach: the warp's 32 chunks are read or written one after the other through shared memory, 4 bytes per
// lane (VEC 4: 16-bit elements two chunks at a time) or one element (VEC 2) -- an access then covers consecutive elements of a row instead
// of one element of each of 32 places.  Shared memory of a warp: a chunk per row, rows of W words one word apart.
template <typename T> struct AnyRows {
    static constexpr int W = 8 * (int)sizeof(T);
    uint32_t w[kQuantThreads / 32][32 * (W + 1)];
};
template <typename T> __device__ __forceinline__ T* shfl_ptr(T* p, int lane)
{
    return reinterpret_cast<T*>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(p), lane));
}
template <typename T, int VEC> __device__ __forceinline__ void load32_any(AnyRows<T>& sm, const T* src, int n, float (&v)[32])
{
    constexpr int W = AnyRows<T>::W;
    const int lane = threadIdx.x & 31;
    uint32_t* rows = sm.w[threadIdx.x >> 5];
    if constexpr (sizeof(T) == 2 && VEC == 4) {
        const int l = lane & 15;
#pragma unroll 8
        for (int i = 0; i < 16; ++i) {
            const int j = 2 * i + (lane >> 4);
            const T* p = shfl_ptr(src, j);
            const int nj = __shfl_sync(0xFFFFFFFFu, n, j);
            uint32_t u = 0;
            if (2 * l + 1 < nj) u = __ldg(reinterpret_cast<const uint32_t*>(p) + l);
            else if (2 * l < nj) u = __ldg(reinterpret_cast<const unsigned short*>(p) + 2 * l);
            rows[j * (W + 1) + l] = u;
        }
    } else
#pragma unroll 8
    for (int j = 0; j < 32; ++j) {
        const T* p = shfl_ptr(src, j);
        const int nj = __shfl_sync(0xFFFFFFFFu, n, j);
        T e = T(0.0f);
        if (lane < nj) e = p[lane];
        reinterpret_cast<T*>(rows + j * (W + 1))[lane] = e;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const uint32_t u = rows[lane * (W + 1) + i];
        if constexpr (sizeof(T) == 2) {
            const float2 f = Dt<T>::up2(u);
            v[2 * i] = f.x, v[2 * i + 1] = f.y;
        } else {
            v[i] = __uint_as_float(u);
        }
    }
}
template <typename T, int VEC> __device__ __forceinline__ void store32_any(AnyRows<T>& sm, T* dst, int n, const float (&v)[32])
{
    constexpr int W = AnyRows<T>::W;
    const int lane = threadIdx.x & 31;
    uint32_t* rows = sm.w[threadIdx.x >> 5];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if constexpr (sizeof(T) == 2) rows[lane * (W + 1) + i] = Dt<T>::down2(v[2 * i], v[2 * i + 1]);
        else rows[lane * (W + 1) + i] = __float_as_uint(v[i]);
    }
    __syncwarp();
    if constexpr (sizeof(T) == 2 && VEC == 4) {
        const int l = lane & 15;
#pragma unroll 8
        for (int i = 0; i < 16; ++i) {
            const int j = 2 * i + (lane >> 4);
            T* p = shfl_ptr(dst, j);
            const int nj = __shfl_sync(0xFFFFFFFFu, n, j);
            const uint32_t u = rows[j * (W + 1) + l];
            if (2 * l + 1 < nj) reinterpret_cast<uint32_t*>(p)[l] = u;
            else if (2 * l < nj) reinterpret_cast<unsigned short*>(p)[2 * l] = (unsigned short)u;
        }
    } else
#pragma unroll 8
    for (int j = 0; j < 32; ++j) {
        T* p = shfl_ptr(dst, j);
        const int nj = __shfl_sync(0xFFFFFFFFu, n, j);
        if (lane < nj) p[lane] = reinterpret_cast<const T*>(rows + j * (W + 1))[lane];
    }
}

// Thread = one 32-element chunk of one row; chunks run over the padded K (a multiple of 256), so the padding of the last
// unit is written as zeros.  Consecutive lanes hold consecutive chunks of a row (a row has a multiple of 8):
// 4 (MXFP4) or 2 (NVFP4) neighbouring lanes join their scale bytes into one 4-byte store.
// EXPERTS: the row is a token, quantised once and stored at the row of each of its pairs.
// 8192 x 8192 -> MXFP4: fp16 24 us, bf16 26, fp32 49 (6.2 to 7.2 TB/s, part of the codes still in L2: bound by HBM); -> NVFP4: 35, 35, 51 (16-bit values:
// 4.9 TB/s, bound by instruction issue -- the quotients' correct rounding, beside the 64-bit division for a chunk's place that every form issues).
template <int FMT, typename T, int VEC, bool EXPERTS>
__global__ void __launch_bounds__(kQuantThreads)
mx_quantize_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows, int64_t K, const float* __restrict__ tensor_scale,
                   uint8_t* __restrict__ packed, const MxRows m, int early)
{
    if (early) pdl_launch_dependents();
    pdl_wait();
    const int64_t KU = k_units(K);
    const int64_t chunks = KU * (kUnitK / 32);
    int64_t id = (int64_t)blockIdx.x * kQuantThreads + threadIdx.x;
    const bool live = id < rows * chunks;                  // (whole quads: rows * chunks is a multiple of 8)
    if (!live) id = 0;                                     // (stays: whole warps meet below)
    const int64_t row = id / chunks;
    const int c = (int)(id - row * chunks);
    const TensorScale ts(tensor_scale ? __ldg(tensor_scale) : 1.0f);
    const int64_t left = K - (int64_t)c * 32;
    const T* src = x + row * ldx + (int64_t)c * 32;
    const int n = (int)(left < 0 || !live ? 0 : left < 32 ? left : 32);
    float v[32];
    if constexpr (VEC >= 16) {
        load32<T, VEC>(src, n, v);
    } else {
        __shared__ AnyRows<T> sm;
        load32_any<T, VEC>(sm, src, n, v);
    }
    uint32_t sb;
    const uint4 codes = quantize32<FMT>(v, ts, sb);
    // scale bytes of the group of four blocks, assembled in its first lane
    constexpr int LANES = FMT == QMM_MXFP4 ? 4 : 2;
    const uint32_t sub = (uint32_t)c & (LANES - 1);
    uint32_t word = sb << (sub * (32 / LANES));
    if (left <= 0) word = 0;
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) word |= __shfl_xor_sync(0xFFFFFFFFu, word, o);       // whole warps, whatever branches their lanes came by
    if (!live) return;
    const uint32_t group = (uint32_t)(c & 7) / LANES;
    auto store = [&](int64_t slot) {
        uint8_t* unit = packed + ((slot >> 7) * KU + (c >> 3)) * unit_bytes(FMT);
        const uint32_t r = (uint32_t)(slot & 127);
        *reinterpret_cast<uint4*>(unit + chunk_offset(r, c & 7)) = codes;
        if (sub == 0) *reinterpret_cast<uint32_t*>(unit + scale_offset(r, group)) = word;
    };
    if constexpr (!EXPERTS) {
        store(row);
    } else {
        for (int j = 0; j < m.topk; ++j) {
            const int64_t p = row * m.topk + j;
            const int r = m.place[p];
            if (r < 0) continue;
            const int e = m.idx[p];
            if ((unsigned)e >= (unsigned)m.E) continue;    // idx is the caller's: no row where it is not what was sorted
            const int first = m.offsets[e];
            if (r < first || r >= m.offsets[e + 1]) continue;
            store((int64_t)m.units[e] * 128 + (r - first));
        }
    }
}

// Elements per thread of the dequantisation, for rows of VEC-byte alignment.
template <typename T> __host__ __device__ constexpr int dequantize_elements(int vec) { return vec == 32 && sizeof(T) == 4 ? 8 : 32; }

// value = code * D in fp32 (rounded once), D = scale * g in fp32.  Thread = one 16-byte chunk of codes, 32 values.  Rows of fp32 that 32-byte
// stores reach: thread = one such store, 8 values, so that a warp's store covers whole lines (8192 x 8192 MXFP4 51.7 us, 5.9 TB/s, against 63.2;
// 16-bit values gain nothing from it: 30.3 against 29.9 us, 5.7 TB/s).  Bound by the writes.
template <int FMT, typename T, int VEC>
__global__ void __launch_bounds__(kQuantThreads)
mx_dequantize_kernel(const uint8_t* __restrict__ packed, int64_t rows, int64_t K, const float* __restrict__ tensor_scale,
                     T* __restrict__ out, int64_t ldo)
{
    pdl_wait();
    constexpr int V = dequantize_elements<T>(VEC);
    const int64_t pieces = (K + V - 1) / V;
    int64_t id = (int64_t)blockIdx.x * kQuantThreads + threadIdx.x;
    const bool live = id < rows * pieces;
    if (VEC >= 16 && !live) return;
    if (!live) id = 0;
    const int64_t row = (uint64_t)(rows * pieces) >> 32 ? id / pieces : (int64_t)((uint32_t)id / (uint32_t)pieces);
    const int64_t k = (id - row * pieces) * V;
    const float g = tensor_scale ? __ldg(tensor_scale) : 1.0f;
    const uint8_t* unit = packed + ((row >> 7) * k_units(K) + k / kUnitK) * unit_bytes(FMT);
    const uint32_t r = (uint32_t)(row & 127), in = (uint32_t)(k & (kUnitK - 1));
    const uint8_t* codes = unit + chunk_offset(r, in >> 5) + ((in & 31) >> 1);
    uint32_t w[V / 8];
    if constexpr (V == 32) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(codes));
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else {
        w[0] = __ldg(reinterpret_cast<const uint32_t*>(codes));
    }
    constexpr int BLOCKS = V > FMT ? V / FMT : 1;
    float D[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
        const uint32_t b = in / FMT + i;
        const uint8_t s = __ldg(unit + scale_offset(r, b >> 2) + (b & 3));
        D[i] = FMT == QMM_MXFP4 ? e8m0_value(s) : e4m3_value(s) * g;
    }
    float v[V];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(w[i >> 2] >> (8 * (i & 3))), __NV_E2M1);
        const float2 f = __half22float2(__half2(h));
        v[2 * i] = f.x * D[2 * i / (V / BLOCKS)];
        v[2 * i + 1] = f.y * D[2 * i / (V / BLOCKS)];
    }
    T* o = out + row * ldo + k;
    const int64_t left = K - k;
    if constexpr (VEC < 16) {
        __shared__ AnyRows<T> sm;
        store32_any<T, VEC>(sm, o, live ? (int)(left < 32 ? left : 32) : 0, v);
    } else if (left >= V) {
        constexpr int W = V * (int)sizeof(T) / 4;
        uint32_t u[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(T) == 2) u[i] = Dt<T>::down2(v[2 * i], v[2 * i + 1]);
            else u[i] = __float_as_uint(v[i]);
        }
#pragma unroll
        for (int i = 0; i < W / 4; ++i)
            if (VEC == 32) {
                if (i % 2 == 0) st_global_256(reinterpret_cast<uint4*>(o) + i, u + 4 * i);
            } else {
                reinterpret_cast<uint4*>(o)[i] = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
            }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) o[i] = Dt<T>::down(v[i]);
    }
}

// Canonical codes and scales -> packed.  Thread = one 16-byte chunk (and the scales of its 32 elements).
template <int FMT>
__global__ void __launch_bounds__(kQuantThreads)
mx_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t rows, int64_t K, uint8_t* __restrict__ packed)
{
    const int64_t KU = k_units(K), chunks = KU * (kUnitK / 32);
    const int64_t id = (int64_t)blockIdx.x * kQuantThreads + threadIdx.x;
    if (id >= rows * chunks) return;
    const int64_t row = id / chunks;
    const int c = (int)(id - row * chunks);
    const int64_t blocks = (K + FMT - 1) / FMT, pitch = blocks * (FMT / 2);
    uint8_t* unit = packed + ((row >> 7) * KU + (c >> 3)) * unit_bytes(FMT);
    const uint32_t r = (uint32_t)(row & 127);
    uint32_t w[4] = {0, 0, 0, 0};
    const uint8_t* src = codes + row * pitch + (int64_t)c * 16;
    const int64_t left = pitch - (int64_t)c * 16;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < left) w[i >> 2] |= (uint32_t)src[i] << (8 * (i & 3));
    *reinterpret_cast<uint4*>(unit + chunk_offset(r, c & 7)) = make_uint4(w[0], w[1], w[2], w[3]);
    constexpr int PER = 32 / FMT;                          // blocks per chunk
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int64_t b = (int64_t)c * PER + i;
        const uint32_t in_unit = (uint32_t)((c & 7) * PER + i);
        unit[scale_offset(r, in_unit >> 2) + (in_unit & 3)] = b < blocks ? scales[row * blocks + b] : (uint8_t)0;
    }
}

// ------------------------------------------------------------ launches

static qmm_status launch_grid(int64_t threads, dim3* grid)
{
    const int64_t blocks = (threads + kQuantThreads - 1) / kQuantThreads;
    if (blocks > 0x7FFFFFFF) return fail(QMM_ERR_UNSUPPORTED, "matrix of %lld 32-element chunks is too large for one launch", (long long)threads);
    *grid = dim3((unsigned)blocks);
    return QMM_OK;
}

template <typename... P, typename... A>
static qmm_status launch_pdl(void (*kern)(P...), dim3 grid, int threads, cudaStream_t st, const char* what, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, args...), what);
}

// `early`: let the next kernel in the stream start its prologue at once.  Only for activations on their way into a
// product of the same call: that product reads its weights before it waits, and the rows quantised here could be a caller's weights.
template <int FMT, typename T>
static qmm_status quantize_t(const void* x, int64_t ldx, int64_t rows, int64_t K, const float* ts, void* packed, const MxRows* m, bool early, cudaStream_t st)
{
    dim3 grid;
    const qmm_status s = launch_grid(rows * k_units(K) * (kUnitK / 32), &grid);
    if (s != QMM_OK) return s;
    const uintptr_t a = reinterpret_cast<uintptr_t>(x) | (rows > 1 ? (uintptr_t)(ldx * (int64_t)sizeof(T)) : 0);
    const int vec = a % 32 == 0 ? 32 : a % 16 == 0 ? 16 : a % 4 == 0 ? 4 : 2;     // (fp32 rows: 4 at least)
    const MxRows none = {nullptr, nullptr, nullptr, nullptr, 0, 0};
    auto go = [&](auto kern, const MxRows& r) {
        return launch_pdl(kern, grid, kQuantThreads, st, "microscaled quantisation launch", (const T*)x, ldx, rows, K, ts, (uint8_t*)packed, r, (int)early);
    };
    if (m) {
        if (vec == 32) return go(mx_quantize_kernel<FMT, T, 32, true>, *m);
        if (vec == 16) return go(mx_quantize_kernel<FMT, T, 16, true>, *m);
        return vec == 4 ? go(mx_quantize_kernel<FMT, T, 4, true>, *m) : go(mx_quantize_kernel<FMT, T, 2, true>, *m);
    }
    if (vec == 32) return go(mx_quantize_kernel<FMT, T, 32, false>, none);
    if (vec == 16) return go(mx_quantize_kernel<FMT, T, 16, false>, none);
    return vec == 4 ? go(mx_quantize_kernel<FMT, T, 4, false>, none) : go(mx_quantize_kernel<FMT, T, 2, false>, none);
}

static qmm_status quantize_any(int fmt, int dtype, const void* x, int64_t ldx, int64_t rows, int64_t K, const float* ts, void* packed,
                               const MxRows* m, bool early, cudaStream_t st)
{
    if (fmt == QMM_MXFP4) {
        if (dtype == QMM_F16) return quantize_t<QMM_MXFP4, __half>(x, ldx, rows, K, ts, packed, m, early, st);
        if (dtype == QMM_BF16) return quantize_t<QMM_MXFP4, __nv_bfloat16>(x, ldx, rows, K, ts, packed, m, early, st);
        return quantize_t<QMM_MXFP4, float>(x, ldx, rows, K, ts, packed, m, early, st);
    }
    if (dtype == QMM_F16) return quantize_t<QMM_NVFP4, __half>(x, ldx, rows, K, ts, packed, m, early, st);
    if (dtype == QMM_BF16) return quantize_t<QMM_NVFP4, __nv_bfloat16>(x, ldx, rows, K, ts, packed, m, early, st);
    return quantize_t<QMM_NVFP4, float>(x, ldx, rows, K, ts, packed, m, early, st);
}

qmm_status launch_mx_quantize(int fmt, int dtype, const void* x, int64_t ldx, int64_t rows, int64_t K, const float* ts, void* packed,
                              bool early, cudaStream_t st)
{
    return quantize_any(fmt, dtype, x, ldx, rows, K, ts, packed, nullptr, early, st);
}

qmm_status launch_mx_quantize_experts(int fmt, int dtype, const void* x, int64_t ldx, int T, int topk, int E, int64_t K, const int* idx,
                                      const int* place, const int* offsets, const int* units, const float* ts, void* packed, bool early,
                                      cudaStream_t st)
{
    const MxRows m = {idx, place, offsets, units, topk, E};
    return quantize_any(fmt, dtype, x, ldx, T, K, ts, packed, &m, early, st);
}

template <int FMT, typename T>
static qmm_status dequantize_t(const void* packed, int64_t rows, int64_t K, const float* ts, void* out, int64_t ldo, cudaStream_t st)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(out) | (rows > 1 ? (uintptr_t)(ldo * (int64_t)sizeof(T)) : 0);
    const int per = dequantize_elements<T>(a % 32 == 0 ? 32 : 2);
    dim3 grid;
    const qmm_status s = launch_grid(rows * ((K + per - 1) / per), &grid);
    if (s != QMM_OK) return s;
    return launch_pdl(a % 32 == 0 ? mx_dequantize_kernel<FMT, T, 32> : a % 16 == 0 ? mx_dequantize_kernel<FMT, T, 16> : a % 4 == 0 ? mx_dequantize_kernel<FMT, T, 4> : mx_dequantize_kernel<FMT, T, 2>,
                      grid, kQuantThreads, st,
                      "microscaled dequantisation launch", (const uint8_t*)packed, rows, K, ts, (T*)out, ldo);
}

qmm_status launch_mx_dequantize(int fmt, int dtype, const void* packed, int64_t rows, int64_t K, const float* ts, void* out, int64_t ldo, cudaStream_t st)
{
    if (fmt == QMM_MXFP4) {
        if (dtype == QMM_F16) return dequantize_t<QMM_MXFP4, __half>(packed, rows, K, ts, out, ldo, st);
        if (dtype == QMM_BF16) return dequantize_t<QMM_MXFP4, __nv_bfloat16>(packed, rows, K, ts, out, ldo, st);
        return dequantize_t<QMM_MXFP4, float>(packed, rows, K, ts, out, ldo, st);
    }
    if (dtype == QMM_F16) return dequantize_t<QMM_NVFP4, __half>(packed, rows, K, ts, out, ldo, st);
    if (dtype == QMM_BF16) return dequantize_t<QMM_NVFP4, __nv_bfloat16>(packed, rows, K, ts, out, ldo, st);
    return dequantize_t<QMM_NVFP4, float>(packed, rows, K, ts, out, ldo, st);
}

qmm_status launch_mx_pack(int fmt, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t K, void* packed, cudaStream_t st)
{
    dim3 grid;
    const qmm_status s = launch_grid(rows * k_units(K) * (kUnitK / 32), &grid);
    if (s != QMM_OK) return s;
    if (fmt == QMM_MXFP4) mx_pack_kernel<QMM_MXFP4><<<grid, kQuantThreads, 0, st>>>(codes, scales, rows, K, (uint8_t*)packed);
    else mx_pack_kernel<QMM_NVFP4><<<grid, kQuantThreads, 0, st>>>(codes, scales, rows, K, (uint8_t*)packed);
    return check_cuda(cudaGetLastError(), "microscaled pack launch");
}

}  // namespace qmm
