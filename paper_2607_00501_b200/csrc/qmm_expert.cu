// qmm_expert.cu -- tokens sorted by expert and back: the stable counting sort of a router's choices, the row moves it
// implies, and their gradients.  The sort is bound by latency, the moves by HBM: they work from the token's side,
// so that a token's row is read once however many experts it goes to.
#include "qmm_mx.cuh"

#include <type_traits>

namespace qmm {

using namespace mx;

template <typename... P, typename... A>
static qmm_status launch_pdl(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, const char* what, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, args...), what);
}

// ------------------------------------------------------------------ sort

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortChunkItems = 4;                         // pairs per thread when several blocks share the work
constexpr int kSortOneBlock = 8 * kSortThreads;            // up to here one block does everything (one launch)

// Expert of pair p; anything outside [0, E) and pairs past the end of the chunk's data map to the last bucket E
// (dropped) and E + 1 (nothing).
__device__ __forceinline__ int bucket_of(const int* __restrict__ idx, int64_t p, int64_t P, int E)
{
    if (p >= P) return E + 1;
    const int e = idx[p];
    return e >= 0 && e < E ? e : E;
}

// Rows per bucket of chunk blockIdx.x -> counts[chunk][E + 1].
__global__ void __launch_bounds__(kSortThreads) expert_count_kernel(const int* __restrict__ idx, int64_t P, int E, int* __restrict__ counts)
{
    pdl_launch_dependents();
    pdl_wait();
    __shared__ int hist[1026];
    for (int e = threadIdx.x; e < E + 2; e += kSortThreads) hist[e] = 0;
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * (kSortThreads * kSortChunkItems);
#pragma unroll
    for (int i = 0; i < kSortChunkItems; ++i)
        atomicAdd(&hist[bucket_of(idx, p0 + i * kSortThreads + threadIdx.x, P, E)], 1);      // a count: order does not matter
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kSortThreads) counts[(int64_t)blockIdx.x * (E + 1) + e] = hist[e];
}

// Places of the pairs of one chunk.  A warp takes ITEMS * 32 consecutive pairs, 32 at a time: lanes with the same bucket find
// one another (match_any) and rank themselves by lane, the bucket's running count of this warp gives the rest.
// With `chunks` > 1 the rows before this chunk and the totals come from `counts`; else this block is all there is.
// Dynamic shared memory: [kSortWarps][E + 2] running counts.
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads)
expert_place_kernel(const int* __restrict__ idx, int64_t P, int E, int chunks, const int* __restrict__ counts, int* __restrict__ order,
                    int* __restrict__ place, int* __restrict__ offsets, int* __restrict__ units)
{
    pdl_launch_dependents();
    pdl_wait();
    extern __shared__ int run[];
    __shared__ int base[1026];                             // first row of each bucket's pairs of this chunk
    __shared__ int s_rows[kSortWarps], s_units[kSortWarps];
    const int B = E + 2, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < kSortWarps * B; i += kSortThreads) run[i] = 0;
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * (kSortThreads * ITEMS) + (int64_t)warp * (32 * ITEMS);
    int bucket[ITEMS], rank[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) bucket[i] = bucket_of(idx, p0 + i * 32 + lane, P, E);
    int* mine = run + warp * B;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const unsigned same = __match_any_sync(0xFFFFFFFFu, bucket[i]);
        const int before = __popc(same & ((1u << lane) - 1u));
        rank[i] = mine[bucket[i]] + before;
        __syncwarp();
        if (before == 0) mine[bucket[i]] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    // counts of the warps -> rows of the bucket before each warp; totals over this chunk or over all of them
    const int e = threadIdx.x;
    int total = 0, before_chunk = 0, dropped_before = 0;
    if (e < E) {
        int sum = 0;
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = run[w * B + e];
            run[w * B + e] = sum;
            sum += c;
        }
        total = sum;
        if (chunks > 1) {
            total = 0;
            for (int c = 0; c < chunks; ++c) {
                const int v = counts[(int64_t)c * (E + 1) + e];
                total += v;
                if (c < (int)blockIdx.x) before_chunk += v;
            }
        }
    }
    if (threadIdx.x == kSortThreads - 1) {                 // the dropped pairs' bucket
        int sum = 0;
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = run[w * B + E];
            run[w * B + E] = sum;
            sum += c;
        }
        if (chunks > 1)
            for (int c = 0; c < (int)blockIdx.x; ++c) dropped_before += counts[(int64_t)c * (E + 1) + E];
    }
    // exclusive scans over the experts of rows and of 128-row units
    const int nu = (total + 127) >> 7;
    int rows = total, us = nu;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int r = __shfl_up_sync(0xFFFFFFFFu, rows, o), u = __shfl_up_sync(0xFFFFFFFFu, us, o);
        if (lane >= o) {
            rows += r;
            us += u;
        }
    }
    if (lane == 31) {
        s_rows[warp] = rows;
        s_units[warp] = us;
    }
    __syncthreads();
    if (warp == 0) {
        int r = s_rows[lane], u = s_units[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int r2 = __shfl_up_sync(0xFFFFFFFFu, r, o), u2 = __shfl_up_sync(0xFFFFFFFFu, u, o);
            if (lane >= o) {
                r += r2;
                u += u2;
            }
        }
        s_rows[lane] = r;
        s_units[lane] = u;
    }
    __syncthreads();
    rows += (warp ? s_rows[warp - 1] : 0) - total;
    us += (warp ? s_units[warp - 1] : 0) - nu;
    if (e < E) {
        base[e] = rows + before_chunk;
        if (blockIdx.x == 0) {
            offsets[e] = rows;
            units[e] = us;
            if (e == E - 1) {
                offsets[E] = rows + total;
                units[E] = us + nu;
            }
        }
    }
    if (threadIdx.x == kSortThreads - 1) base[E] = s_rows[kSortWarps - 1] + dropped_before;      // dropped pairs: past the last row
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t p = p0 + i * 32 + lane;
        if (p >= P) continue;
        const int row = base[bucket[i]] + mine[bucket[i]] + rank[i];
        const bool kept = bucket[i] < E;
        place[p] = kept ? row : -1;
        order[row] = kept ? (int)p : -1;
    }
}

static int sort_chunks(int64_t P) { return P <= kSortOneBlock ? 1 : (int)((P + kSortThreads * kSortChunkItems - 1) / (kSortThreads * kSortChunkItems)); }

size_t expert_sort_workspace_bytes(int64_t P, int E) { return P <= kSortOneBlock ? 0 : (size_t)sort_chunks(P) * (size_t)(E + 1) * 4; }

qmm_status launch_expert_sort(const int* idx, int64_t P, int E, int* order, int* place, int* offsets, int* units, void* ws, cudaStream_t st)
{
    const size_t smem = (size_t)kSortWarps * (E + 2) * 4;
    const int chunks = sort_chunks(P);
    auto go = [&](auto kern) -> qmm_status {
        if (smem > 40 * 1024) {                            // E > 318: beyond the default dynamic shared memory beside the static arrays
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return check_cuda(e, "expert sort shared memory size");
        }
        return launch_pdl(kern, dim3(chunks), kSortThreads, smem, st, "expert sort launch", idx, P, E, chunks, (const int*)ws, order, place, offsets, units);
    };
    if (chunks > 1) {
        const qmm_status s = launch_pdl(expert_count_kernel, dim3(chunks), kSortThreads, 0, st, "expert count launch", idx, P, E, (int*)ws);
        if (s != QMM_OK) return s;
        return go(expert_place_kernel<kSortChunkItems>);
    }
    if (P <= kSortThreads) return go(expert_place_kernel<1>);
    return go(expert_place_kernel<8>);
}

// ------------------------------------------------------------- row moves

constexpr int kMoveThreads = 256;

// One vector of V elements of a row: V * sizeof(T) = 16 bytes, 4 bytes, or a single element, as the rows' alignment allows.
template <typename T, int V> struct Vec {
    float f[V];
    __device__ __forceinline__ void load(const T* p)
    {
        constexpr int B = V * (int)sizeof(T);
        if constexpr (B == 16) {
            const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
            unpack(w);
        } else if constexpr (B == 4 && sizeof(T) == 2) {
            const uint32_t w[1] = {__ldg(reinterpret_cast<const uint32_t*>(p))};
            unpack(w);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = Dt<T>::up(p[i]);
        }
    }
    template <int W> __device__ __forceinline__ void unpack(const uint32_t (&w)[W])
    {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (sizeof(T) == 2) {
                const float2 v = Dt<T>::up2(w[i]);
                f[2 * i] = v.x, f[2 * i + 1] = v.y;
            } else {
                f[i] = __uint_as_float(w[i]);
            }
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
        constexpr int B = V * (int)sizeof(T);
        if constexpr (B == 16) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) w[i] = Dt<T>::down2(f[2 * i], f[2 * i + 1]);
                else w[i] = __float_as_uint(f[i]);
            }
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else if constexpr (B == 4 && sizeof(T) == 2) {
            *reinterpret_cast<uint32_t*>(p) = Dt<T>::down2(f[0], f[1]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) p[i] = Dt<T>::down(f[i]);
        }
    }
    __device__ __forceinline__ Vec scaled(float s) const
    {
        Vec r;
#pragma unroll
        for (int i = 0; i < V; ++i) r.f[i] = f[i] * s;
        return r;
    }
};

// Thread = one vector of one token's row: read once, written at the row of each of the token's pairs.  The rows past the
// last (one per dropped pair) are dealt to the tokens by index and zeroed.
template <typename T, int V>
__global__ void __launch_bounds__(kMoveThreads)
expert_gather_kernel(const T* __restrict__ x, int64_t ldx, int tokens, int topk, int nv, const int* __restrict__ order, const int* __restrict__ place,
                     const float* __restrict__ weights, T* __restrict__ xs, int64_t ldxs)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t id = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x;
    const int64_t t = id / nv;
    if (t >= tokens) return;
    const int64_t h = (id - t * nv) * V;
    Vec<T, V> v;
    v.load(x + t * ldx + h);
    for (int j = 0; j < topk; ++j) {
        const int64_t p = t * topk + j;
        const int r = __ldg(place + p);
        if (r >= 0) {
            if (weights) v.scaled(__ldg(weights + p)).store(xs + r * ldxs + h);
            else v.store(xs + r * ldxs + h);
        }
        if (__ldg(order + p) < 0) {
            Vec<T, V> z;
#pragma unroll
            for (int i = 0; i < V; ++i) z.f[i] = 0.0f;
            z.store(xs + p * ldxs + h);
        }
    }
}

// Thread = one vector of one token's row; the rows of up to eight pairs are in flight at once, added in order.
template <typename T, int V>
__global__ void __launch_bounds__(kMoveThreads)
expert_combine_kernel(const T* __restrict__ ys, int64_t ldys, int tokens, int topk, int nv, const int* __restrict__ place,
                      const float* __restrict__ weights, T* __restrict__ y, int64_t ldy)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t id = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x;
    const int64_t t = id / nv;
    if (t >= tokens) return;
    const int64_t h = (id - t * nv) * V;
    Vec<T, V> acc;
#pragma unroll
    for (int i = 0; i < V; ++i) acc.f[i] = 0.0f;
    for (int j0 = 0; j0 < topk; j0 += 8) {
        Vec<T, V> v[8];
        float w[8];
        int r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            r[j] = j0 + j < topk ? __ldg(place + t * topk + j0 + j) : -1;
            w[j] = r[j] >= 0 && weights ? __ldg(weights + t * topk + j0 + j) : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (r[j] >= 0) v[j].load(ys + r[j] * ldys + h);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (r[j] >= 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) acc.f[i] = fmaf(w[j], v[j].f[i], acc.f[i]);
            }
    }
    acc.store(y + t * ldy + h);
}

// Block = one token: its row of dy against the rows of its pairs, eight pairs at a time.  A pair's dot product is
// added over the thread's vectors, the warp (shuffles) and the warps in a fixed order.
template <typename T, int V>
__global__ void __launch_bounds__(kMoveThreads)
expert_combine_grad_kernel(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ ys, int64_t ldys, int topk, int nv,
                           const int* __restrict__ order, const int* __restrict__ place, const float* __restrict__ weights, T* __restrict__ dys,
                           int64_t lddys, float* __restrict__ dw)
{
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float red[kMoveThreads / 32][8];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int j0 = 0; j0 < topk; j0 += 8) {
        int r[8];
        float w[8], dot[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t p = t * topk + j0 + j;
            r[j] = j0 + j < topk ? __ldg(place + p) : -1;
            w[j] = r[j] >= 0 && weights ? __ldg(weights + p) : 1.0f;
            dot[j] = 0.0f;
        }
        for (int i = threadIdx.x; i < nv; i += blockDim.x) {
            const int64_t h = (int64_t)i * V;
            Vec<T, V> d, v[8];
            d.load(dy + t * lddy + h);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (r[j] >= 0) v[j].load(ys + r[j] * ldys + h);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (r[j] >= 0) {
#pragma unroll
                    for (int k = 0; k < V; ++k) dot[j] = fmaf(d.f[k], v[j].f[k], dot[j]);
                    d.scaled(w[j]).store(dys + r[j] * lddys + h);
                }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], o);
            if (lane == 0) red[warp][j] = dot[j];
        }
        __syncthreads();
        if (threadIdx.x < 8 && j0 + (int)threadIdx.x < topk) {
            float s = 0.0f;
            for (int k = 0; k < warps; ++k) s += red[k][threadIdx.x];
            dw[t * topk + j0 + threadIdx.x] = s;           // (a dropped pair's sum is zero)
        }
        __syncthreads();
    }
    for (int j = 0; j < topk; ++j) {                       // rows past the last, as in the gather
        const int64_t row = t * topk + j;
        if (__ldg(order + row) >= 0) continue;
        Vec<T, V> z;
#pragma unroll
        for (int i = 0; i < V; ++i) z.f[i] = 0.0f;
        for (int i = threadIdx.x; i < nv; i += blockDim.x) z.store(dys + row * lddys + (int64_t)i * V);
    }
}

// ------------------------------------------------------------ launches

// Largest vector (elements) that every given address and row pitch allows and that divides H.
static int vector_of(int size, int64_t H, uintptr_t bits)
{
    bits |= (uintptr_t)(H * size);
    return bits % 16 == 0 ? 16 / size : (size == 2 && bits % 4 == 0) ? 2 : 1;
}

static uintptr_t bits_of(const void* p, int64_t ld, int size) { return reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size); }

static qmm_status move_grid(int64_t threads, dim3* grid)
{
    const int64_t blocks = (threads + kMoveThreads - 1) / kMoveThreads;
    if (blocks > 0x7FFFFFFF) return fail(QMM_ERR_UNSUPPORTED, "%lld row vectors are too many for one launch", (long long)threads);
    *grid = dim3((unsigned)blocks);
    return QMM_OK;
}

// Calls f with the kernel template arguments (type, vector length) for a data type and a vector.
template <typename F> static qmm_status by_type(int dtype, int V, F f)
{
    if (dtype == QMM_F32) return V == 4 ? f(float(), std::integral_constant<int, 4>()) : f(float(), std::integral_constant<int, 1>());
    if (dtype == QMM_F16)
        return V == 8 ? f(__half(), std::integral_constant<int, 8>()) : V == 2 ? f(__half(), std::integral_constant<int, 2>()) : f(__half(), std::integral_constant<int, 1>());
    return V == 8 ? f(__nv_bfloat16(), std::integral_constant<int, 8>())
                  : V == 2 ? f(__nv_bfloat16(), std::integral_constant<int, 2>()) : f(__nv_bfloat16(), std::integral_constant<int, 1>());
}

qmm_status launch_expert_gather(int dtype, const void* x, int64_t ldx, int T, int topk, int64_t H, const int* order, const int* place, const float* weights,
                                void* xs, int64_t ldxs, cudaStream_t st)
{
    const int size = dtype == QMM_F32 ? 4 : 2;
    const int V = vector_of(size, H, bits_of(x, ldx, size) | bits_of(xs, ldxs, size)), nv = (int)(H / V);
    dim3 grid;
    const qmm_status s = move_grid((int64_t)T * nv, &grid);
    if (s != QMM_OK) return s;
    return by_type(dtype, V, [&](auto type, auto v) {
        using D = decltype(type);
        return launch_pdl(expert_gather_kernel<D, decltype(v)::value>, grid, kMoveThreads, 0, st, "expert gather launch", (const D*)x, ldx, T, topk, nv, order, place,
                          weights, (D*)xs, ldxs);
    });
}

qmm_status launch_expert_combine(int dtype, const void* ys, int64_t ldys, int T, int topk, int64_t H, const int* place, const float* weights, void* y, int64_t ldy,
                                 cudaStream_t st)
{
    const int size = dtype == QMM_F32 ? 4 : 2;
    const int V = vector_of(size, H, bits_of(ys, ldys, size) | bits_of(y, ldy, size)), nv = (int)(H / V);
    dim3 grid;
    const qmm_status s = move_grid((int64_t)T * nv, &grid);
    if (s != QMM_OK) return s;
    return by_type(dtype, V, [&](auto type, auto v) {
        using D = decltype(type);
        return launch_pdl(expert_combine_kernel<D, decltype(v)::value>, grid, kMoveThreads, 0, st, "expert combine launch", (const D*)ys, ldys, T, topk, nv, place,
                          weights, (D*)y, ldy);
    });
}

qmm_status launch_expert_combine_grad(int dtype, const void* dy, int64_t lddy, const void* ys, int64_t ldys, int T, int topk, int64_t H, const int* order,
                                      const int* place, const float* weights, void* dys, int64_t lddys, float* dw, cudaStream_t st)
{
    const int size = dtype == QMM_F32 ? 4 : 2;
    const int V = vector_of(size, H, bits_of(dy, lddy, size) | bits_of(ys, ldys, size) | bits_of(dys, lddys, size)), nv = (int)(H / V);
    const int threads = nv <= 64 ? 64 : nv <= 128 ? 128 : kMoveThreads;
    return by_type(dtype, V, [&](auto type, auto v) {
        using D = decltype(type);
        return launch_pdl(expert_combine_grad_kernel<D, decltype(v)::value>, dim3((unsigned)T), threads, 0, st, "expert combine gradient launch", (const D*)dy, lddy,
                          (const D*)ys, ldys, topk, nv, order, place, weights, (D*)dys, lddys, dw);
    });
}

}  // namespace qmm
