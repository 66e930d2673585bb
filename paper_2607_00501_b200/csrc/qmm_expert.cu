// qmm_expert.cu -- tokens sorted by expert and back: the stable counting sort of a router's choices, the row moves it
// implies, and their gradients.  The sort is bound by latency, the moves by HBM: they work from the token's side,
// so that a token's row is read once however many experts it goes to.
#include "qmm_mx.cuh"

#include <atomic>
#include <type_traits>

namespace qmm {

using namespace mx;

template <typename... P, typename... A>
static qmm_status launch_pdl(void (*kern)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, const char* what, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, args...), what);
}

// ------------------------------------------------------------------ sort

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortCluster = 16;                           // blocks of the one-launch form beyond a block's worth of pairs (a non-portable cluster)
constexpr int kSortOneLaunch = 8 * kSortThreads * kSortCluster;   // up to here (131072 pairs) one launch does everything
constexpr int kSortChunkItems = 4;                         // pairs per thread of the two-launch form

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

// Places of the pairs of one block's chunk.  A warp takes ITEMS * 32 consecutive pairs, 32 at a time: lanes with the same
// bucket find one another (one ballot per bit of the bucket's number; a match instruction took three times as long) and rank
// themselves by lane, the bucket's running count of this warp gives the rest.
// The rows before this chunk and the totals come from the other blocks of the cluster, through distributed shared memory
// (CLUSTER: the whole sort is one launch of up to sixteen blocks), or from `counts` (many chunks).
// Dynamic shared memory: [kSortWarps][E + 2] running counts.
// s_place, s_offsets, s_units (optional, shared memory of one block): copies of place, offsets and units for what follows in the kernel.
template <int ITEMS, bool CLUSTER>
__device__ __forceinline__ void place_pairs(const int* __restrict__ idx, int64_t P, int E, int chunks, const int* __restrict__ counts, int* __restrict__ order,
                                            int* __restrict__ place, int* __restrict__ offsets, int* __restrict__ units, int* s_place, int* s_offsets, int* s_unit0)
{
    pdl_launch_dependents();
    extern __shared__ int run[];
    __shared__ int base[1026];                             // this chunk's rows per bucket, then the first row of each
    __shared__ int local[ITEMS > 1 ? 1026 : 1];            // first place of each bucket's pairs inside the chunk
    __shared__ int s_rows[kSortWarps], s_units[kSortWarps], s_local[kSortWarps];
    const int B = E + 2, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < kSortWarps * B; i += kSortThreads) run[i] = 0;
    pdl_wait();
    const int64_t p0 = (int64_t)blockIdx.x * (kSortThreads * ITEMS) + (int64_t)warp * (32 * ITEMS);
    int bucket[ITEMS], rank[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) bucket[i] = bucket_of(idx, p0 + i * 32 + lane, P, E);
    __syncthreads();
    int* mine = run + warp * B;
    const int bits = 32 - __clz(E + 1);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        unsigned same = 0xFFFFFFFFu;                       // lanes with this lane's bucket: agreement in every bit of its number
        for (int b = 0; b < bits; ++b) {
            const unsigned ones = __ballot_sync(0xFFFFFFFFu, (bucket[i] >> b) & 1);
            same &= (bucket[i] >> b) & 1 ? ones : ~ones;
        }
        const int before = __popc(same & ((1u << lane) - 1u));
        rank[i] = mine[bucket[i]] + before;
        __syncwarp();
        if (before == 0) mine[bucket[i]] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    // counts of the warps -> rows of the bucket before each warp (thread e: expert e; the last thread: the dropped pairs)
    const int e = threadIdx.x;
    auto over_warps = [&](int bkt) {
        int c[kSortWarps], sum = 0;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) c[w] = run[w * B + bkt];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            run[w * B + bkt] = sum;
            sum += c[w];
        }
        return sum;
    };
    int total = 0, before_chunk = 0, dropped_before = 0;
    if (e < E) base[e] = total = over_warps(e);
    const int in_chunk = total;
    if (threadIdx.x == kSortThreads - 1) base[E] = over_warps(E);
    if (CLUSTER && chunks > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        auto others = [&](int bkt, int& before) {
            int v[kSortCluster], all = 0;
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(&base[bkt]);
#pragma unroll
            for (int c = 0; c < kSortCluster; ++c) {
                uint32_t remote;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(at), "r"(c));
                asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v[c]) : "r"(remote) : "memory");
            }
#pragma unroll
            for (int c = 0; c < kSortCluster; ++c) {
                all += v[c];
                if (c < (int)blockIdx.x) before += v[c];
            }
            return all;
        };
        if (e < E) total = others(e, before_chunk);
        if (threadIdx.x == kSortThreads - 1) others(E, dropped_before);
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // base[] is overwritten below
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else if (!CLUSTER) {
        auto others = [&](int bkt, int& before) {
            int all = 0;
#pragma unroll 8
            for (int c = 0; c < chunks; ++c) {
                const int v = __ldg(counts + (int64_t)c * (E + 1) + bkt);
                all += v;
                before += c < (int)blockIdx.x ? v : 0;
            }
            return all;
        };
        if (e < E) total = others(e, before_chunk);
        if (threadIdx.x == kSortThreads - 1) others(E, dropped_before);
    }
    // exclusive scans over the experts of rows, of 128-row units and of this chunk's pairs
    const int nu = (total + 127) >> 7;
    int rows = total, us = nu, ls = in_chunk;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int r = __shfl_up_sync(0xFFFFFFFFu, rows, o), u = __shfl_up_sync(0xFFFFFFFFu, us, o), l = __shfl_up_sync(0xFFFFFFFFu, ls, o);
        if (lane >= o) {
            rows += r;
            us += u;
            ls += l;
        }
    }
    if (lane == 31) {
        s_rows[warp] = rows;
        s_units[warp] = us;
        s_local[warp] = ls;
    }
    __syncthreads();
    if (warp == 0) {
        int r = s_rows[lane], u = s_units[lane], l = s_local[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int r2 = __shfl_up_sync(0xFFFFFFFFu, r, o), u2 = __shfl_up_sync(0xFFFFFFFFu, u, o), l2 = __shfl_up_sync(0xFFFFFFFFu, l, o);
            if (lane >= o) {
                r += r2;
                u += u2;
                l += l2;
            }
        }
        s_rows[lane] = r;
        s_units[lane] = u;
        s_local[lane] = l;
    }
    __syncthreads();
    rows += (warp ? s_rows[warp - 1] : 0) - total;
    us += (warp ? s_units[warp - 1] : 0) - nu;
    ls += (warp ? s_local[warp - 1] : 0) - in_chunk;
    if (e < E) {
        base[e] = rows + before_chunk;
        if (ITEMS > 1) local[e] = ls;
        if (blockIdx.x == 0) {
            offsets[e] = rows;
            units[e] = us;
            if (s_offsets) s_offsets[e] = rows, s_unit0[e] = us;
            if (e == E - 1) {
                offsets[E] = rows + total;
                units[E] = us + nu;
            }
        }
    }
    if (threadIdx.x == kSortThreads - 1) {
        base[E] = s_rows[kSortWarps - 1] + dropped_before;  // dropped pairs: past the last row
        if (ITEMS > 1) local[E] = s_local[kSortWarps - 1];
    }
    __syncthreads();
    // place[] is written in pair order.  order[] is written in row order: the chunk's pairs are sorted in shared memory first,
    // so that a bucket's run is one contiguous store (65536 pairs: 12.9 us against 14.1 with scattered stores).
    // (One pair per thread: too few for that to pay.)
    int2* sorted = reinterpret_cast<int2*>(run + ((kSortWarps * B + 1) & ~1));
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t p = p0 + i * 32 + lane;
        if (p >= P) continue;
        const int in_bucket = mine[bucket[i]] + rank[i], row = base[bucket[i]] + in_bucket;
        const bool kept = bucket[i] < E;
        place[p] = kept ? row : -1;
        if (s_place) s_place[p] = kept ? row : -1;
        if (ITEMS > 1) sorted[local[bucket[i]] + in_bucket] = make_int2(row, kept ? (int)p : -1);
        else order[row] = kept ? (int)p : -1;
    }
    if (ITEMS > 1) {
        __syncthreads();
        const int64_t left = P - (int64_t)blockIdx.x * (kSortThreads * ITEMS);
        const int n = (int)(left < kSortThreads * ITEMS ? left : kSortThreads * ITEMS);
        for (int q = threadIdx.x; q < n; q += kSortThreads) order[sorted[q].x] = sorted[q].y;
    }
}

template <int ITEMS, bool CLUSTER>
__global__ void __launch_bounds__(kSortThreads)
expert_place_kernel(const int* __restrict__ idx, int64_t P, int E, int chunks, const int* __restrict__ counts, int* __restrict__ order,
                    int* __restrict__ place, int* __restrict__ offsets, int* __restrict__ units)
{
    place_pairs<ITEMS, CLUSTER>(idx, P, E, chunks, counts, order, place, offsets, units, nullptr, nullptr, nullptr);
}

// The sort of a few pairs and the quantisation of their tokens in one block: the front of a decode step's routed layer, one launch
// where two (each about as long as its latency) would follow one another.  A thread takes 32 elements of a token at a time and stores
// them at the row of each of the token's pairs.
template <int FMT, typename T>
__global__ void __launch_bounds__(kSortThreads)
expert_place_quantize_kernel(const int* __restrict__ idx, int P, int E, int topk, int* __restrict__ order, int* __restrict__ place, int* __restrict__ offsets,
                             int* __restrict__ units, const T* __restrict__ x, int64_t ldx, int x_vec, int64_t K, const float* __restrict__ tensor_scale,
                             uint8_t* __restrict__ packed)
{
    __shared__ int s_place[kSortThreads], s_offsets[1024], s_units[1024];
    place_pairs<1, true>(idx, P, E, 1, nullptr, order, place, offsets, units, s_place, s_offsets, s_units);
    __syncthreads();
    const TensorScale ts(tensor_scale ? __ldg(tensor_scale) : 1.0f);
    const int KU = (int)k_units(K), chunks = KU * (kUnitK / 32);
    for (int id = threadIdx.x; id < P / topk * chunks; id += kSortThreads) {
        const int t = id / chunks, c = id - t * chunks;
        const int64_t left = K - (int64_t)c * 32;
        const int n = (int)(left < 0 ? 0 : left < 32 ? left : 32);
        const T* src = x + t * ldx + (int64_t)c * 32;
        float v[32];
        if (x_vec == 32) load32<T, 32>(src, n, v);
        else if (x_vec == 16) load32<T, 16>(src, n, v);
        else load32<T, 0>(src, n, v);
        uint32_t sb;
        const uint4 codes = quantize32<FMT>(v, ts, sb);
        for (int j = 0; j < topk; ++j) {
            const int r = s_place[t * topk + j];
            if (r < 0) continue;
            const int e = __ldg(idx + t * topk + j), slot = s_units[e] * 128 + r - s_offsets[e];
            uint8_t* unit = packed + ((int64_t)(slot >> 7) * KU + (c >> 3)) * unit_bytes(FMT);
            *reinterpret_cast<uint4*>(unit + chunk_offset(slot & 127, c & 7)) = codes;
            if (FMT == QMM_MXFP4) unit[scale_offset(slot & 127, (c & 7) >> 2) + (c & 3)] = (uint8_t)sb;
            else *reinterpret_cast<uint16_t*>(unit + scale_offset(slot & 127, (c & 7) >> 1) + 2 * (c & 1)) = (uint16_t)sb;
        }
    }
}

static int sort_chunks(int64_t P) { return (int)((P + kSortThreads * kSortChunkItems - 1) / (kSortThreads * kSortChunkItems)); }

size_t expert_sort_workspace_bytes(int64_t P, int E) { return P <= kSortOneLaunch ? 0 : (size_t)sort_chunks(P) * (size_t)(E + 1) * 4; }

struct SortArgs {
    const int* idx;
    int64_t P;
    int E;
    int *order, *place, *offsets, *units;
    const int* counts;
};
template <int ITEMS, bool CLUSTER> static qmm_status launch_place(const SortArgs& a, int chunks, cudaStream_t st)
{
    auto kern = expert_place_kernel<ITEMS, CLUSTER>;
    auto smem_of = [](int E) { return (size_t)((kSortWarps * (E + 2) + 1) & ~1) * 4 + (ITEMS > 1 ? (size_t)ITEMS * kSortThreads * 8 : 0); };
    static std::atomic<uint64_t> configured{0};            // devices that have the attributes
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0;
    if (!(configured.load(std::memory_order_relaxed) & bit)) {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_of(1024));
        if (e == cudaSuccess && CLUSTER) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return check_cuda(e, "expert sort attributes");
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    return launch_pdl(kern, dim3(chunks), kSortThreads, smem_of(a.E), CLUSTER ? chunks : 1, st, "expert sort launch", a.idx, a.P, a.E, chunks, a.counts, a.order,
                      a.place, a.offsets, a.units);
}

qmm_status launch_expert_sort(const int* idx, int64_t P, int E, int* order, int* place, int* offsets, int* units, void* ws, cudaStream_t st)
{
    const SortArgs a = {idx, P, E, order, place, offsets, units, (const int*)ws};
    if (P > kSortOneLaunch) {
        const int chunks = sort_chunks(P);
        const qmm_status s = launch_pdl(expert_count_kernel, dim3(chunks), kSortThreads, 0, 1, st, "expert count launch", idx, P, E, (int*)ws);
        if (s != QMM_OK) return s;
        return launch_place<kSortChunkItems, false>(a, chunks, st);
    }
    if (P <= kSortThreads) return launch_place<1, true>(a, 1, st);
    // sixteen blocks, as few pairs per thread as that allows (65536 pairs: 9.2 us, against 12.9 with 8 blocks)
    const int64_t items = (P + kSortThreads * kSortCluster - 1) / (kSortThreads * kSortCluster);
    if (items <= 1) return launch_place<1, true>(a, kSortCluster, st);
    if (items <= 2) return launch_place<2, true>(a, kSortCluster, st);
    if (items <= 4) return launch_place<4, true>(a, kSortCluster, st);
    return launch_place<8, true>(a, kSortCluster, st);
}

// Whether sort and quantisation of a layer's tokens are one launch: one block's worth of pairs, and at most two passes of its threads over the
// tokens' 32-element chunks.
bool expert_sort_quantize_fits(int64_t P, int topk, int64_t K) { return P <= kSortThreads && P / topk * k_units(K) * (kUnitK / 32) <= 2 * kSortThreads; }

template <int FMT, typename T> static qmm_status sort_quantize_t(const SortArgs& a, int topk, const void* x, int64_t ldx, int64_t K, const float* ts, void* packed, cudaStream_t st)
{
    const size_t smem = (size_t)((kSortWarps * (a.E + 2) + 1) & ~1) * 4;
    auto kern = expert_place_quantize_kernel<FMT, T>;
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0;
    if (!(configured.load(std::memory_order_relaxed) & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortWarps * 1026 * 4);
        if (e != cudaSuccess) return check_cuda(e, "expert sort and quantisation attributes");
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    const uintptr_t bits = reinterpret_cast<uintptr_t>(x) | (uintptr_t)(ldx * (int64_t)sizeof(T));
    const int vec = bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : 0;
    return launch_pdl(kern, dim3(1), kSortThreads, smem, 1, st, "expert sort and quantisation launch", a.idx, (int)a.P, a.E, topk, a.order, a.place, a.offsets, a.units,
                      (const T*)x, ldx, vec, K, ts, (uint8_t*)packed);
}

qmm_status launch_expert_sort_quantize(int fmt, int dtype, const int* idx, int64_t P, int topk, int E, int* order, int* place, int* offsets, int* units,
                                       const void* x, int64_t ldx, int64_t K, const float* ts, void* packed, cudaStream_t st)
{
    const SortArgs a = {idx, P, E, order, place, offsets, units, nullptr};
    if (fmt == QMM_MXFP4) {
        if (dtype == QMM_F16) return sort_quantize_t<QMM_MXFP4, __half>(a, topk, x, ldx, K, ts, packed, st);
        if (dtype == QMM_BF16) return sort_quantize_t<QMM_MXFP4, __nv_bfloat16>(a, topk, x, ldx, K, ts, packed, st);
        return sort_quantize_t<QMM_MXFP4, float>(a, topk, x, ldx, K, ts, packed, st);
    }
    if (dtype == QMM_F16) return sort_quantize_t<QMM_NVFP4, __half>(a, topk, x, ldx, K, ts, packed, st);
    if (dtype == QMM_BF16) return sort_quantize_t<QMM_NVFP4, __nv_bfloat16>(a, topk, x, ldx, K, ts, packed, st);
    return sort_quantize_t<QMM_NVFP4, float>(a, topk, x, ldx, K, ts, packed, st);
}

// ------------------------------------------------------------- row moves

constexpr int kMoveThreads = 256;

// One vector of V elements of a row: V * sizeof(T) = 16 bytes, 4 bytes, or a single element, as the rows' alignment allows (8 bytes: 16-bit sums of
// fp32 rows).
// Raw<T, V> is the vector as loaded: several of them in flight cost half the registers of their fp32 form.
template <typename T, int V> struct Raw {
    static constexpr int B = V * (int)sizeof(T);
    static constexpr int W = B >= 4 ? B / 4 : 1;
    uint32_t u[W];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (B == 16) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
            u[0] = q.x, u[1] = q.y, u[2] = q.z, u[3] = q.w;
        } else if constexpr (B == 4) {
            u[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        } else {
            u[0] = __ldg(reinterpret_cast<const unsigned short*>(p));
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (B == 16) *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
        else if constexpr (B == 8) *reinterpret_cast<uint2*>(p) = make_uint2(u[0], u[1]);
        else if constexpr (B == 4) *reinterpret_cast<uint32_t*>(p) = u[0];
        else *reinterpret_cast<unsigned short*>(p) = (unsigned short)u[0];
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < W; ++i) u[i] = 0u;
    }
    __device__ __forceinline__ float get(int i) const                          // element i as fp32 (i a constant once unrolled)
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(u[i]);
        } else {
            const float2 f = Dt<T>::up2(u[i >> 1]);
            return i & 1 ? f.y : f.x;
        }
    }
};
template <typename T, int V> struct Vec {
    float f[V];
    __device__ __forceinline__ Raw<T, V> raw() const
    {
        Raw<T, V> r;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) r.u[i] = __float_as_uint(f[i]);
        } else if constexpr (V == 1) {
            r.u[0] = Dt<T>::down2(f[0], 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) r.u[i] = Dt<T>::down2(f[2 * i], f[2 * i + 1]);
        }
        return r;
    }
};
template <typename T, int V> __device__ __forceinline__ Raw<T, V> scaled(const Raw<T, V>& x, float s)
{
    Vec<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v.f[i] = x.get(i) * s;
    return v.raw();
}

// Thread = one vector of one token's row: read once, written at the row of each of the token's pairs.  The rows past the
// last (one per dropped pair) are dealt to the tokens by index and zeroed.
// Bound by HBM (one row read, topk written): 8192 tokens x 8, 2048 bf16 48.6 us, 6.2 TB/s (50.0 with weights); fp32 94.9, 6.4.
// 61 tokens: 2.6 us, a launch.
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
    Raw<T, V> v, z;
    v.load(x + t * ldx + h);
    z.zero();
    for (int j = 0; j < topk; ++j) {
        const int64_t p = t * topk + j;
        const int r = __ldg(place + p);
        if (r >= 0) {
            if (weights) scaled(v, __ldg(weights + p)).store(xs + r * ldxs + h);
            else v.store(xs + r * ldxs + h);
        }
        if (__ldg(order + p) < 0) z.store(xs + p * ldxs + h);
    }
}

// Thread = one vector of one token's row; the rows of up to eight pairs are in flight at once, added in order (fp32).
// Bound by HBM (topk rows read, one written): 8192 tokens x 8, 2048 bf16 48.6 us, 6.2 TB/s; fp32 93.4, 6.5.  61 tokens: 2.0 us.
// TO: type of the sums (fp32 rows may have 16-bit sums).
template <typename T, typename TO, int V>
__global__ void __launch_bounds__(kMoveThreads)
expert_combine_kernel(const T* __restrict__ ys, int64_t ldys, int tokens, int topk, int nv, const int* __restrict__ place,
                      const float* __restrict__ weights, TO* __restrict__ y, int64_t ldy)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t id = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x;
    const int64_t t = id / nv;
    if (t >= tokens) return;
    const int64_t h = (id - t * nv) * V;
    Vec<TO, V> acc;
#pragma unroll
    for (int i = 0; i < V; ++i) acc.f[i] = 0.0f;
    for (int j0 = 0; j0 < topk; j0 += 8) {
        Raw<T, V> v[8];
        float w[8];
        int r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            r[j] = j0 + j < topk ? __ldg(place + t * topk + j0 + j) : -1;
            w[j] = r[j] >= 0 && weights ? __ldg(weights + t * topk + j0 + j) : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j].load(ys + max(r[j], 0) * ldys + h);   // no branch around a load: all are in flight together (row 0 stands in)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool kept = r[j] >= 0;
#pragma unroll
            for (int i = 0; i < V; ++i) acc.f[i] = kept ? fmaf(w[j], v[j].get(i), acc.f[i]) : acc.f[i];
        }
    }
    acc.raw().store(y + t * ldy + h);
}

// Block = one token: its row of dy against the rows of its pairs, eight pairs at a time.  A pair's dot product is
// added over the thread's vectors, the warp (shuffles) and the warps in a fixed order.
// Bound by HBM (dy and topk rows read, topk written): 8192 tokens x 8, 2048 bf16 93.0 us, 6.1 TB/s; fp32 174.9, 6.5.  61 tokens: 3.4 us.
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
            Raw<T, V> d, v[8];
            d.load(dy + t * lddy + h);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j].load(ys + max(r[j], 0) * ldys + h);   // no branch around a load (row 0 stands in)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (r[j] >= 0) {
#pragma unroll
                    for (int k = 0; k < V; ++k) dot[j] = fmaf(d.get(k), v[j].get(k), dot[j]);
                    scaled(d, w[j]).store(dys + r[j] * lddys + h);
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
        Raw<T, V> z;
        z.zero();
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
        return launch_pdl(expert_gather_kernel<D, decltype(v)::value>, grid, kMoveThreads, 0, 1, st, "expert gather launch", (const D*)x, ldx, T, topk, nv, order, place,
                          weights, (D*)xs, ldxs);
    });
}

template <typename T, typename TO, int V>
static qmm_status combine_t(const void* ys, int64_t ldys, int T_, int topk, int64_t H, const int* place, const float* weights, void* y, int64_t ldy, cudaStream_t st)
{
    const int nv = (int)(H / V);
    dim3 grid;
    const qmm_status s = move_grid((int64_t)T_ * nv, &grid);
    if (s != QMM_OK) return s;
    return launch_pdl(expert_combine_kernel<T, TO, V>, grid, kMoveThreads, 0, 1, st, "expert combine launch", (const T*)ys, ldys, T_, topk, nv, place, weights, (TO*)y, ldy);
}

// rows_dtype: type of ys, that of y or fp32.
qmm_status launch_expert_combine(int rows_dtype, int dtype, const void* ys, int64_t ldys, int T, int topk, int64_t H, const int* place, const float* weights, void* y,
                                 int64_t ldy, cudaStream_t st)
{
    const int size = dtype == QMM_F32 ? 4 : 2;
    if (rows_dtype != dtype) {                             // fp32 rows, 16-bit sums: 16-byte loads, 8-byte stores
        const bool wide = vector_of(4, H, bits_of(ys, ldys, 4)) == 4 && bits_of(y, ldy, size) % 8 == 0;
        if (dtype == QMM_F16)
            return wide ? combine_t<float, __half, 4>(ys, ldys, T, topk, H, place, weights, y, ldy, st)
                        : combine_t<float, __half, 1>(ys, ldys, T, topk, H, place, weights, y, ldy, st);
        return wide ? combine_t<float, __nv_bfloat16, 4>(ys, ldys, T, topk, H, place, weights, y, ldy, st)
                    : combine_t<float, __nv_bfloat16, 1>(ys, ldys, T, topk, H, place, weights, y, ldy, st);
    }
    return by_type(dtype, vector_of(size, H, bits_of(ys, ldys, size) | bits_of(y, ldy, size)), [&](auto type, auto v) {
        using D = decltype(type);
        return combine_t<D, D, decltype(v)::value>(ys, ldys, T, topk, H, place, weights, y, ldy, st);
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
        return launch_pdl(expert_combine_grad_kernel<D, decltype(v)::value>, dim3((unsigned)T), threads, 0, 1, st, "expert combine gradient launch", (const D*)dy, lddy,
                          (const D*)ys, ldys, topk, nv, order, place, weights, (D*)dys, lddys, dw);
    });
}

}  // namespace qmm
