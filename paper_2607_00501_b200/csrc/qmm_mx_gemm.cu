// qmm_mx_gemm.cu -- products of packed microscaled 4-bit operands on the block-scaled tcgen05 MMA.
//
// Y[m, n] = sum_b sa[m, b] sw[n, b] sum_i a[m, i] w[n, i]: the tensor core multiplies codes and applies the block scales
// itself, so no CUDA core touches an element on the way in.  Tokens are the rows of the MMA (128 lanes of
// tensor memory, one token row each), weight rows its columns; a pipeline stage is one unit of K (256 k):
//   16 KB codes + 1 / 2 KB scales of the token rows, the same of 128 (or 2 x 128) weight rows,
// fetched as contiguous bulk copies -- the packed operand holds exactly what a stage needs, in the order the
// tensor core reads it.  Scales go from shared memory to tensor memory with tcgen05.cp, in the issuing thread's
// order with the MMAs that read them (two sets of columns in turn).
//
// Why tokens on the lanes: a thread of the epilogue then holds consecutive outputs of one token row,
// which makes 32 consecutive intermediate features -- the blocks of the next product's operand -- local to a
// thread (gate/up form), and rows of Y full sectors.  With few tokens most lanes idle, which costs nothing: the
// 128 x 128 x 256 step takes 256 cycles of the tensor pipe per 17 KB of weights, and HBM delivers 17 KB per SM in
// ~750 cycles.
//
// Roles: warp 0 loads (one lane), warp 1 issues copies of scales and MMAs (converged, one elected lane), warps 4.. run the
// epilogue (four lane quarters; twice that in the gate/up form).  The kernel is persistent over tiles, ring and
// barrier phases run on across them.  Tile t = (token tile t / n_tiles, weight tile t % n_tiles).
// Forms:
//   dense      tiles dealt round-robin;
//   split      few tiles: a cluster of up to 8 blocks per tile, each a share of K; partial sums in shared
//              memory, added in rank order through distributed shared memory (same bits on every call);
//   grouped    token tiles of the experts' rows, from the device arrays units[] / offsets[].
// Every mbarrier wait is bounded; on give-up the block records QMM_ERR_DEVICE_TIMEOUT, waits (bounded) for its copies
// in flight, frees its tensor memory and returns.
#include "qmm_mx.cuh"
#include "qmm_tc.cuh"

#include <atomic>
#include <cuda.h>

namespace qmm {

using namespace mx;

enum MxForm { kMxDense = 0, kMxSplit = 1, kMxGrouped = 2 };

struct MxGemmParams {
    const uint8_t* a;                // packed token rows
    const uint8_t* w[2];             // packed weights (expert 0): W, or W_gate and W_up
    int64_t w_stride;                // bytes between experts
    int M, N, KU;                    // token rows (dense), weight rows, k units
    int n_tiles;                     // weight tiles of 128 rows
    const int *offsets, *units;      // grouped: [E + 1] each
    int E;
    const float* a_scale;            // tensor scales, null = 1
    const float* w_scale[2];         // grouped: [E]
    const float* h_scale;            // gate/up: tensor scale of the output operand
    void* y;                         // [rows, ldy], or the packed output operand (gate/up)
    int64_t ldy;
    int vec;                         // widest aligned store of Y: 32, 16 or 0 (element by element)
    int* status;
};

constexpr int kMxMaxE = 1024;

// NB: weight units per tile (2: gate and up).
template <int FMT, int NB, bool GATEUP> struct MxGeom {
    static constexpr int kUnit = unit_bytes(FMT);
    static constexpr int kStage = (1 + NB) * kUnit;
    static constexpr int kEpiWarps = GATEUP ? 8 : 4;
    static constexpr int kThreads = (4 + kEpiWarps) * 32;
    static constexpr int kTail = 1024 + (GATEUP || NB == 1 ? (kMxMaxE + 1) * 4 : 0);   // barriers, the experts' unit index
    static constexpr int kFit = (227 * 1024 - 1024 - kTail) / kStage;
    static constexpr int kStages = kFit < 6 ? kFit : 6;
    static constexpr int kSmem = 1024 + kStages * kStage + kTail;
    // tensor memory: accumulators (two when they fit), then two sets of scale columns
    static constexpr int kDCols = NB * 128;
    static constexpr int kAccBufs = NB == 1 ? 2 : 1;
    static constexpr int kGroups = kUnitK / FMT / 4;                            // scale groups per unit: 2 or 4
    static constexpr int kSfCols = kGroups * 4 * (1 + NB);
    static constexpr int kSf0 = kAccBufs * kDCols;
    static constexpr int kTmemCols = 512;
    static_assert(kSf0 + 2 * kSfCols <= kTmemCols, "tensor memory over-subscribed");
    static_assert(kStages >= 3, "pipeline too shallow");
};

// One piece of work: a token tile against a weight tile over the units [k0, k1).
struct MxWork {
    int m_unit;                      // row unit of the token operand
    int rows;                        // token rows in it (1 .. 128)
    int row0;                        // first row of Y
    int n_tile, expert, k0, k1;
};

__device__ __forceinline__ float silu_f32(float g) { return __fdividef(g, 1.0f + __expf(-g)); }

// 32 consecutive outputs of one row; n = how many exist.  vec: widest store (bytes) that the rows' alignment allows; 32-byte
// stores write whole sectors (a lane's neighbours in a store are other rows).
__device__ __forceinline__ void st_global_256(void* p, const uint32_t* u)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]),
                 "r"(u[6]), "r"(u[7])
                 : "memory");
}
template <typename T> __device__ __forceinline__ void store32(T* o, const float (&v)[32], int n, int vec)
{
    if (vec && n >= 32) {
        constexpr int W = 8 * (int)sizeof(T);
        uint32_t u[W];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = Dt<T>::down2(v[2 * i], v[2 * i + 1]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) u[i] = __float_as_uint(v[i]);
        }
        if (vec == 32) {
#pragma unroll
            for (int i = 0; i < W / 8; ++i) st_global_256(reinterpret_cast<uint8_t*>(o) + 32 * i, u + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) reinterpret_cast<uint4*>(o)[i] = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < n) o[i] = Dt<T>::down(v[i]);
}

__device__ __forceinline__ void mx_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster_v4(uint32_t local_addr, int rank)
{
    float4 v;
    asm volatile(
        "{\n\t"
        ".reg .b32 a;\n\t"
        "mapa.shared::cluster.u32 a, %4, %5;\n\t"
        "ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t"
        "}\n"
        : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
        : "r"(local_addr), "r"(rank)
        : "memory");
    return v;
}

template <int FMT, int NB, bool GATEUP, typename T, int FORM>
__global__ void __launch_bounds__(MxGeom<FMT, NB, GATEUP>::kThreads, 1) mx_gemm_kernel(const MxGemmParams p)
{
    using namespace tc;
    using G = MxGeom<FMT, NB, GATEUP>;
    constexpr int S = G::kStages, AB = G::kAccBufs, NEPI = G::kEpiWarps;
    constexpr int LOAD_WARP = 0, MMA_WARP = 1, EPI_WARP0 = 4;

    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + S * G::kStage);       // [S] loads -> MMA
    uint64_t* empty = full + S;                                               // [S] MMA -> loads
    uint64_t* acc_full = empty + S;                                           // [2] MMA -> epilogue
    uint64_t* acc_empty = acc_full + 2;                                       // [2] epilogue -> MMA
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    int* s_units = reinterpret_cast<int*>(smem + S * G::kStage + 1024);       // [E + 1] (grouped)
    const uint32_t smem0 = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], NEPI);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == MMA_WARP) {
        tmem_alloc(tmem_slot, G::kTmemCols);
        tmem_relinquish();
    }
    if (FORM == kMxGrouped) {
        pdl_wait();                                                           // the rows' grouping is written upstream
        for (int e = threadIdx.x; e <= p.E; e += G::kThreads) s_units[e] = p.units[e];
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_launch_dependents();

    int splits = 1, rank = 0;
    if (FORM == kMxSplit) {
        asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(splits));
        asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    }
    const int m_tiles = FORM == kMxGrouped ? s_units[p.E] : (p.M + 127) >> 7;
    const int total = m_tiles * p.n_tiles;

    // i-th piece of work of this block (the same sequence for every role)
    auto get_work = [&](int i, MxWork& w) -> bool {
        int t;
        if (FORM == kMxSplit) {
            if (i > 0) return false;
            t = (int)blockIdx.x / splits;
            w.k0 = (int)((int64_t)p.KU * rank / splits);
            w.k1 = (int)((int64_t)p.KU * (rank + 1) / splits);
        } else {
            t = (int)blockIdx.x + i * (int)gridDim.x;
            if (t >= total) return false;
            w.k0 = 0;
            w.k1 = p.KU;
        }
        const int mt = t / p.n_tiles;
        w.n_tile = t - mt * p.n_tiles;
        w.m_unit = mt;
        if (FORM == kMxGrouped) {
            int lo = 0, hi = p.E - 1;                                         // first e with units[e + 1] > mt
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (s_units[mid + 1] > mt) hi = mid;
                else lo = mid + 1;
            }
            const int first = __ldg(p.offsets + lo), past = __ldg(p.offsets + lo + 1);
            w.expert = lo;
            w.row0 = first + 128 * (mt - s_units[lo]);
            w.rows = min(128, past - w.row0);
        } else {
            w.expert = 0;
            w.row0 = mt * 128;
            w.rows = min(128, p.M - w.row0);
        }
        return true;
    };

    if (warp == LOAD_WARP) {
        // ================= loads
        if (lane == 0) {
            bool ok = true;
            int g = 0, early = 0;
            MxWork w;
            auto load_w = [&](int s, int ku) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const uint8_t* src = p.w[GATEUP ? b : 0] + w.expert * p.w_stride + ((int64_t)(GATEUP ? w.n_tile : w.n_tile * NB + b) * p.KU + ku) * G::kUnit;
                    bulk_load(smem0 + s * G::kStage + (1 + b) * G::kUnit, src, G::kUnit, smem_u32(&full[s]));
                }
            };
            auto expect = [&](int s) {
                const uint32_t rows8 = (uint32_t)(w.rows + 7) & ~7u;
                mbar_arrive_expect_tx(&full[s], NB * G::kUnit + rows8 * 128u + (uint32_t)scale_bytes(FMT));
            };
            // weights do not depend on the previous kernel: the first ring of them is requested before the wait for it
            if (FORM != kMxGrouped) {
                if (get_work(0, w))
                    for (; early < S && early < w.k1 - w.k0; ++early) {
                        expect(early);
                        load_w(early, w.k0 + early);
                    }
                pdl_wait();
            }
            for (int i = 0; ok && get_work(i, w); ++i) {
                const uint32_t rows8 = (uint32_t)(w.rows + 7) & ~7u;
                for (int ku = w.k0; ku < w.k1; ++ku, ++g) {
                    const int s = g % S;
                    if (g >= S) ok = mbar_wait(&empty[s], ((g / S) - 1) & 1, abort_flag);
                    if (!ok) break;
                    if (g >= early) {
                        expect(s);
                        load_w(s, ku);
                    }
                    const uint8_t* src = p.a + ((int64_t)w.m_unit * p.KU + ku) * G::kUnit;
                    const uint32_t dst = smem0 + s * G::kStage;
                    bulk_load(dst, src, rows8 * 128u, smem_u32(&full[s]));
                    bulk_load(dst + kCodeBytes, src + kCodeBytes, (uint32_t)scale_bytes(FMT), smem_u32(&full[s]));
                }
            }
            if (!ok) {
                *abort_flag = 1;
                // let copies in flight land before the block's shared memory is released
                for (int q = max(0, g - S); q < g; ++q) {
                    const long long t0 = clock64();
                    while (!mbar_try_wait(&full[q % S], (q / S) & 1) && clock64() - t0 < (1LL << 22)) {}
                }
            }
        }
    } else if (warp == MMA_WARP) {
        // ================= MMA issuer (whole warp converged, one lane acts)
        const uint32_t sel = elect_one() ? 1u : 0u;
        bool ok = true;
        int g = 0;
        MxWork w;
        for (int it = 0; ok && get_work(it, w); ++it) {
            const int buf = it % AB;
            if (it >= AB) {
                ok = mbar_wait(&acc_empty[buf], ((it / AB) - 1) & 1, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
            }
            const uint32_t d = tmem_base + (uint32_t)(buf * G::kDCols);
            for (int ku = w.k0; ku < w.k1; ++ku, ++g) {
                const int s = g % S;
                ok = mbar_wait(&full[s], (g / S) & 1, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t stage = smem0 + s * G::kStage;
                const uint32_t sfa = tmem_base + (uint32_t)(G::kSf0 + (g & 1) * G::kSfCols);
                const uint32_t sfb = sfa + (uint32_t)(G::kGroups * 4);
#pragma unroll
                for (int j = 0; j < G::kGroups; ++j) {
                    tmem_copy_scales(sfa + 4 * j, smem_desc_scales(stage + kCodeBytes + 512 * j), sel);
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        tmem_copy_scales(sfb + 4 * (j * NB + b), smem_desc_scales(stage + (1 + b) * G::kUnit + kCodeBytes + 512 * j), sel);
                }
                if (NB == 1) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {                             // K = 64 steps: 32 bytes of a row's 128
                        const int grp = FMT == QMM_MXFP4 ? k >> 1 : k, id = FMT == QMM_MXFP4 ? (k & 1) * 2 : 0;
                        mma_fp4<FMT == QMM_MXFP4>(d, smem_desc_k_sw128(stage) + 2 * k, smem_desc_k_sw128(stage + G::kUnit) + 2 * k,
                                                  idesc_fp4(FMT == QMM_MXFP4, 128, 128, id), sfa + 4 * grp, sfb + 4 * grp, ku != w.k0 || k != 0, sel);
                    }
                } else {
                    // the two weight units are not adjacent in shared memory (scales lie between): one N = 128 MMA each
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int grp = FMT == QMM_MXFP4 ? k >> 1 : k, id = FMT == QMM_MXFP4 ? (k & 1) * 2 : 0;
#pragma unroll
                        for (int b = 0; b < NB; ++b)
                            mma_fp4<FMT == QMM_MXFP4>(d + 128 * b, smem_desc_k_sw128(stage) + 2 * k, smem_desc_k_sw128(stage + (1 + b) * G::kUnit) + 2 * k,
                                                      idesc_fp4(FMT == QMM_MXFP4, 128, 128, id), sfa + 4 * grp, sfb + 4 * (grp * NB + b), ku != w.k0 || k != 0, sel);
                    }
                }
                mma_commit_sel(&empty[s], sel);
                __syncwarp();
            }
            if (ok) mma_commit_sel(&acc_full[buf], sel);
            __syncwarp();
        }
        if (!ok) *abort_flag = 1;
    } else if (warp >= EPI_WARP0) {
        // ================= epilogue
        const int quarter = warp & 3;
        const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16);
        bool ok = true;
        MxWork w;
        // every global write below comes after the previous kernel has completed (its readers of this buffer included)
        if (FORM != kMxGrouped) pdl_wait();
        const float a_scale = p.a_scale ? __ldg(p.a_scale) : 1.0f;
        for (int it = 0; ok && get_work(it, w); ++it) {
            const int buf = it % AB;
            ok = mbar_wait(&acc_full[buf], (it / AB) & 1, abort_flag);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            tc_fence_after_sync();
            const int r = quarter * 32 + lane;                                // token row of the tile
            const bool warp_has_rows = quarter * 32 < w.rows;
            const uint32_t d = lanes + (uint32_t)(buf * G::kDCols);
            if constexpr (GATEUP) {
                const float ag = a_scale * (p.w_scale[0] ? __ldg(p.w_scale[0] + w.expert) : 1.0f);
                const float au = a_scale * (p.w_scale[1] ? __ldg(p.w_scale[1] + w.expert) : 1.0f);
                const float hs = p.h_scale ? __ldg(p.h_scale) : 1.0f, h6 = 6.0f * hs;
                const int half = (warp - EPI_WARP0) >> 2;                     // 64 of the tile's 128 columns
                const int hku = (p.n_tiles + 1) >> 1;                         // k units of the output operand
                const uint32_t hb = (uint32_t)w.n_tile & 1;                   // which half of its unit this tile fills
                const bool fill = hb == 0 && w.n_tile == p.n_tiles - 1;       // nobody else writes the unit's other half
                uint8_t* unit = reinterpret_cast<uint8_t*>(p.y) + ((int64_t)w.m_unit * hku + (w.n_tile >> 1)) * G::kUnit;
                if (warp_has_rows) {
                    uint32_t scales = 0;
#pragma unroll 1
                    for (int blk = 0; blk < 2; ++blk) {
                        const int c0 = half * 64 + blk * 32;
                        uint32_t gv[32], uv[32];
                        tmem_ld_32x32b_x32(d + (uint32_t)c0, gv);
                        tmem_ld_32x32b_x32(d + (uint32_t)(128 + c0), uv);
                        tmem_wait_ld();
                        const int left = p.N - (w.n_tile * 128 + c0);
                        float h[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            h[i] = i < left ? silu_f32(ag * __uint_as_float(gv[i])) * (au * __uint_as_float(uv[i])) : 0.0f;
                        uint4 codes;
                        if constexpr (FMT == QMM_MXFP4) {
                            uint32_t cw[4];
                            scales |= quantize_block<32>(h, hs, h6, cw) << (8 * blk);
                            codes = make_uint4(cw[0], cw[1], cw[2], cw[3]);
                        } else {
                            float h0[16], h1[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) h0[i] = h[i], h1[i] = h[16 + i];
                            uint32_t w0[2], w1[2];
                            scales |= quantize_block<16>(h0, hs, h6, w0) << (16 * blk);
                            scales |= quantize_block<16>(h1, hs, h6, w1) << (16 * blk + 8);
                            codes = make_uint4(w0[0], w0[1], w1[0], w1[1]);
                        }
                        if (r < w.rows) {
                            const uint32_t chunk = (uint32_t)(2 * half + blk);
                            *reinterpret_cast<uint4*>(unit + chunk_offset(r, 4 * hb + chunk)) = codes;
                            if (fill) *reinterpret_cast<uint4*>(unit + chunk_offset(r, 4 + chunk)) = make_uint4(0, 0, 0, 0);
                        }
                    }
                    if (r < w.rows) {
                        if (FMT == QMM_MXFP4) {                               // the tile's four blocks are one group: two bytes each warp
                            *reinterpret_cast<uint16_t*>(unit + scale_offset(r, hb) + 2 * half) = (uint16_t)scales;
                            if (fill) *reinterpret_cast<uint16_t*>(unit + scale_offset(r, 1) + 2 * half) = 0;
                        } else {
                            *reinterpret_cast<uint32_t*>(unit + scale_offset(r, 2 * hb + half)) = scales;
                            if (fill) *reinterpret_cast<uint32_t*>(unit + scale_offset(r, 2 + half)) = 0;
                        }
                    }
                }
            } else if constexpr (FORM == kMxSplit) {
                // partial sums -> this block's shared memory (the ring is idle: every load has landed and every MMA is done)
                if (warp_has_rows) {
                    float* part = reinterpret_cast<float*>(smem) + r * 132;
#pragma unroll 1
                    for (int c0 = 0; c0 < 128; c0 += 32) {
                        uint32_t v[32];
                        tmem_ld_32x32b_x32(d + (uint32_t)c0, v);
                        tmem_wait_ld();
                        if (r < w.rows) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                reinterpret_cast<uint4*>(part + c0)[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                        }
                    }
                }
            } else {
                const float alpha = a_scale * (p.w_scale[0] ? __ldg(p.w_scale[0] + w.expert) : 1.0f);
                if (warp_has_rows) {
#pragma unroll 1
                    for (int c0 = 0; c0 < NB * 128; c0 += 32) {
                        const int n0 = w.n_tile * (NB * 128) + c0;
                        uint32_t v[32];
                        tmem_ld_32x32b_x32(d + (uint32_t)c0, v);
                        tmem_wait_ld();
                        if (r < w.rows) {
                            float f[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) f[i] = alpha * __uint_as_float(v[i]);
                            store32<T>(reinterpret_cast<T*>(p.y) + (int64_t)(w.row0 + r) * p.ldy + n0, f, p.N - n0, p.vec);
                        }
                    }
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[buf]);
        }
        if (!ok) *abort_flag = 1;
    }

    if constexpr (FORM == kMxSplit) {
        // rank j adds columns [128 j / splits, 128 (j + 1) / splits) of every row, partial sums in rank order
        MxWork w;
        get_work(0, w);
        __syncwarp();
        mx_cluster_sync();
        const float alpha = (p.a_scale ? __ldg(p.a_scale) : 1.0f) * (p.w_scale[0] ? __ldg(p.w_scale[0]) : 1.0f);
        const int quads = 32 / splits;                                        // groups of four columns per rank
        if (!*abort_flag) {
            for (int i = threadIdx.x; i < w.rows * quads; i += G::kThreads) {
                const int r = i / quads, c = (rank * quads + (i - r * quads)) * 4;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int q = 0; q < splits; ++q) {
                    const float4 v = ld_cluster_v4(smem0 + (uint32_t)(r * 132 + c) * 4u, q);
                    acc.x += v.x;
                    acc.y += v.y;
                    acc.z += v.z;
                    acc.w += v.w;
                }
                const float f[4] = {alpha * acc.x, alpha * acc.y, alpha * acc.z, alpha * acc.w};
                const int n0 = w.n_tile * 128 + c;
                T* o = reinterpret_cast<T*>(p.y) + (int64_t)(w.row0 + r) * p.ldy + n0;
                if (p.vec && n0 + 4 <= p.N) {
                    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(o) = make_uint2(Dt<T>::down2(f[0], f[1]), Dt<T>::down2(f[2], f[3]));
                    else *reinterpret_cast<float4*>(o) = make_float4(f[0], f[1], f[2], f[3]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (n0 + k < p.N) o[k] = Dt<T>::down(f[k]);
                }
            }
        }
        mx_cluster_sync();                                                    // nobody leaves while its sums are being read
    }

    // ---- teardown
    tc_fence_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag && p.status != nullptr) atomicExch(p.status, (int)QMM_ERR_DEVICE_TIMEOUT);
    if (warp == MMA_WARP) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, G::kTmemCols);
    }
}

// ------------------------------------------------------------ many tokens: pairs of SMs

// 256 x 256 tiles by two blocks on neighbouring SMs (cta_group::2).  A block holds 128 of the tile's token rows and half
// of its weight rows; the pair's MMA (M = 256, N = 256) reads each half of the weights from the block that has it, so a
// K step moves 16 KB + 16 KB of codes per SM for 512 cycles of tensor pipe -- half the L2 and shared-memory traffic
// per flop of the 128 x 128 tile of one SM, which that traffic bounds at less than half of the tensor rate.
// Every block keeps the scales of its own token rows and of all 256 weight rows in tensor memory.
//
// The first block's MMA warp issues for both.  The loads of both blocks complete on the first block's barrier, which tiled TMA
// loads of a pair can do and plain bulk copies cannot (with bulk copies and a warp of the second block passing completions on,
// the ring's round trip bounded the kernel at 40 % of this form).  tcgen05.commit frees ring slots and hands over the
// accumulators in both blocks.  Tensor memory holds one 256-column accumulator beside two sets of scale columns: eight epilogue
// warps take it into registers at once (128 columns each), free it, and store while the next tile's MMAs run.
template <int FMT> struct MxPairGeom {
    static constexpr int kSc = scale_bytes(FMT);
    static constexpr int kA = 0, kB = unit_bytes(FMT), kSb = kB + kCodeBytes;              // A unit | B codes | scales of both B units
    static constexpr int kStage = kSb + 2 * kSc;
    static constexpr int kFit = (227 * 1024 - 2048) / kStage;
    static constexpr int kStages = kFit < 6 ? kFit : 6;
    static constexpr int kSmem = 2048 + kStages * kStage;
    static constexpr int kGroups = kUnitK / FMT / 4;
    static constexpr int kSf0 = 256, kSfCols = kGroups * 12;
    static constexpr int kThreads = 12 * 32;
    static_assert(kSf0 + 2 * kSfCols <= 512 && kStages >= 4, "tensor memory or shared memory over-subscribed");
};

struct MxPairMaps {
    CUtensorMap a, w_codes, w_scales;                                         // boxes: a unit | a unit's codes | its scales
};

// Tile t of the pair form: token tiles in groups of eight, inside a group token tile first, so that the tiles in flight at one
// time span about as many token tiles as weight tiles (fewest distinct units between L2 and the SMs).
__device__ __forceinline__ void pair_tile(int t, int m_tiles, int n_tiles, int& mt, int& nt)
{
    const int per = 8 * n_tiles, g = t / per, in = t - g * per;
    const int rows = min(8, m_tiles - 8 * g);
    nt = in / rows;
    mt = 8 * g + (in - nt * rows);
}

template <int FMT, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MxPairGeom<FMT>::kThreads, 1) mx_pair_kernel(const __grid_constant__ MxPairMaps maps, const MxGemmParams p)
{
    using namespace tc;
    using G = MxPairGeom<FMT>;
    constexpr int S = G::kStages, UNIT = unit_bytes(FMT);

    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + S * G::kStage);       // [S] loads of both blocks -> MMA (first block)
    uint64_t* empty = full + S;                                               // [S] MMA -> loads
    uint64_t* acc_full = empty + S;                                           // MMA -> epilogue
    uint64_t* acc_empty = acc_full + 1;                                       // epilogues of both blocks -> MMA (first block)
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t smem0 = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, 16);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc_pair(tmem_slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    mx_cluster_sync();                                                        // the other block's barriers exist
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_launch_dependents();

    const int a_units = (p.M + 127) >> 7, b_units = p.n_tiles;                // units of 128 rows
    const int n_tiles = (b_units + 1) >> 1, m_tiles = (a_units + 1) >> 1, total = n_tiles * m_tiles;
    const int pairs = (int)gridDim.x >> 1, first = (int)blockIdx.x >> 1;

    if (warp == 0) {
        // ================= loads
        if (lane == 0) {
            bool ok = true;
            int g = 0, early = 0;
            prefetch_tensormap(&maps.a);
            prefetch_tensormap(&maps.w_codes);
            prefetch_tensormap(&maps.w_scales);
            constexpr int ROWS = UNIT / 128;
            const uint32_t full0 = cluster_addr(full, 0);
            auto load_w = [&](int s, int mt, int nt, int ku) {                // (first block: expects the stage of both) requests the weights
                const int a0 = 2 * mt, b0 = 2 * nt, b = b0 + (int)rank;
                const int as = a0 + 1 < a_units ? 2 : 1, bs = b0 + 1 < b_units ? 2 : 1;
                const uint32_t dst = smem0 + s * G::kStage, bar = full0 + 8 * s;
                if (rank == 0) mbar_arrive_expect_tx(&full[s], as * UNIT + bs * kCodeBytes + 2 * bs * G::kSc);
                const int y = (b0 * p.KU + ku) * ROWS, next = p.KU * ROWS;
                if (b < b_units) tma_load_2d_pair(dst + G::kB, &maps.w_codes, 0, y + (int)rank * next, bar);
                tma_load_2d_pair(dst + G::kSb, &maps.w_scales, 0, y + 128, bar);
                if (bs == 2) tma_load_2d_pair(dst + G::kSb + G::kSc, &maps.w_scales, 0, y + next + 128, bar);
            };
            int mt, nt;
            pair_tile(first, m_tiles, n_tiles, mt, nt);
            for (; early < S && early < p.KU; ++early) load_w(early, mt, nt, early);
            pdl_wait();
            for (int t = first; ok && t < total; t += pairs) {
                pair_tile(t, m_tiles, n_tiles, mt, nt);
                const int a = 2 * mt + (int)rank;
                for (int ku = 0; ku < p.KU; ++ku, ++g) {
                    const int s = g % S;
                    if (g >= S) ok = mbar_wait(&empty[s], ((g / S) - 1) & 1, abort_flag);
                    if (!ok) break;
                    if (g >= early) load_w(s, mt, nt, ku);
                    if (a < a_units) tma_load_2d_pair(smem0 + s * G::kStage, &maps.a, 0, (a * p.KU + ku) * ROWS, full0 + 8 * s);
                }
            }
            if (!ok) {
                *abort_flag = 1;
                // let copies in flight land (both blocks' count on the first block's barriers; the second waits for it at the end)
                for (int q = max(0, g - S); rank == 0 && q < g; ++q) {
                    const long long t0 = clock64();
                    while (!mbar_try_wait(&full[q % S], (q / S) & 1) && clock64() - t0 < (1LL << 22)) {}
                }
            }
        }
    } else if (warp == 1 && rank == 1) {
        // (the second block's tensor memory was allocated by this warp; it frees it at the end)
    } else if (warp == 1) {
        // ================= MMA issuer for the pair
        const uint32_t sel = elect_one() ? 1u : 0u;
        const uint64_t desc_a = smem_desc_k_sw128(smem0 + G::kA), desc_b = smem_desc_k_sw128(smem0 + G::kB);
        const uint64_t desc_sa = smem_desc_scales(smem0 + G::kA + kCodeBytes), desc_sb = smem_desc_scales(smem0 + G::kSb);
        bool ok = true;
        int g = 0, it = 0;
        for (int t = first; ok && t < total; t += pairs, ++it) {
            if (it > 0) {
                ok = mbar_wait_cluster(acc_empty, (it - 1) & 1, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
            }
            for (int ku = 0; ku < p.KU; ++ku, ++g) {
                const int s = g % S;
                ok = mbar_wait(&full[s], (g / S) & 1, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
                const uint64_t at = (uint64_t)(s * (G::kStage >> 4));
                const uint32_t sfa = tmem_base + (uint32_t)(G::kSf0 + (g & 1) * G::kSfCols);
                const uint32_t sfb = sfa + (uint32_t)(G::kGroups * 4);
#pragma unroll
                for (int j = 0; j < G::kGroups; ++j) {
                    tmem_copy_scales_pair(sfa + 4 * j, desc_sa + at + 32 * j, sel);
                    tmem_copy_scales_pair(sfb + 8 * j, desc_sb + at + 32 * j, sel);
                    tmem_copy_scales_pair(sfb + 8 * j + 4, desc_sb + at + (G::kSc >> 4) + 32 * j, sel);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int grp = FMT == QMM_MXFP4 ? k >> 1 : k, id = FMT == QMM_MXFP4 ? (k & 1) * 2 : 0;
                    mma_fp4_pair<FMT == QMM_MXFP4>(tmem_base, desc_a + at + 2 * k, desc_b + at + 2 * k, idesc_fp4(FMT == QMM_MXFP4, 256, 256, id), sfa + 4 * grp,
                                                   sfb + 8 * grp, ku != 0 || k != 0, sel);
                }
                mma_commit_pair(&empty[s], sel);
                __syncwarp();
            }
            if (ok) mma_commit_pair(acc_full, sel);
            __syncwarp();
        }
        if (!ok) *abort_flag = 1;
    } else if (warp >= 4) {
        // ================= epilogue: 32 rows x 128 columns per warp
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t d = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
        bool ok = true;
        int it = 0;
        pdl_wait();
        const float alpha = (p.a_scale ? __ldg(p.a_scale) : 1.0f) * (p.w_scale[0] ? __ldg(p.w_scale[0]) : 1.0f);
        for (int t = first; ok && t < total; t += pairs, ++it) {
            ok = mbar_wait(acc_full, it & 1, abort_flag);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            tc_fence_after_sync();
            uint32_t v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(d + 32 * c, v[c]);
            tmem_wait_ld();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(acc_empty, 0);
            int mt, nt;
            pair_tile(t, m_tiles, n_tiles, mt, nt);
            const int row = 256 * mt + 128 * (int)rank + quarter * 32 + lane;
            const int n0 = 256 * nt + 128 * half;
            if (row < p.M) {
                T* o = reinterpret_cast<T*>(p.y) + (int64_t)row * p.ldy + n0;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float f[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) f[i] = alpha * __uint_as_float(v[c][i]);
                    store32<T>(o + 32 * c, f, p.N - n0 - 32 * c, p.vec);
                }
            }
        }
        if (!ok) *abort_flag = 1;
    }

    // ---- teardown
    tc_fence_before_sync();
    __syncthreads();
    mx_cluster_sync();                                                        // no arrival or MMA of the other block is still to come
    if (threadIdx.x == 0 && *abort_flag && p.status != nullptr) atomicExch(p.status, (int)QMM_ERR_DEVICE_TIMEOUT);
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

// ------------------------------------------------------------ launches

template <int FMT, int NB, bool GATEUP, typename T, int FORM>
static qmm_status launch_t(const MxGemmParams& p, int grid, int cluster, cudaStream_t st)
{
    auto kern = mx_gemm_kernel<FMT, NB, GATEUP, T, FORM>;
    constexpr int smem = MxGeom<FMT, NB, GATEUP>::kSmem;
    static std::atomic<uint64_t> configured{0};                               // devices that have the attribute
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0;
    if (!(configured.load(std::memory_order_relaxed) & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return check_cuda(e, "microscaled product shared memory size");
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(MxGeom<FMT, NB, GATEUP>::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (FORM == kMxSplit) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, p), "microscaled product launch");
}

template <typename T> static int row_vec(const void* y, int64_t ldy)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(y) | (uintptr_t)(ldy * (int64_t)sizeof(T));
    return a % 32 == 0 ? 32 : a % 16 == 0 ? 16 : 0;
}

qmm_status make_unit_map(CUtensorMap* map, const void* packed, int64_t rows128, int box_rows);

template <int FMT, typename T> static qmm_status launch_pair_t(const MxGemmParams& p, int tiles, cudaStream_t st)
{
    auto kern = mx_pair_kernel<FMT, T>;
    constexpr int smem = MxPairGeom<FMT>::kSmem, ROWS = unit_bytes(FMT) / 128;
    static std::atomic<uint64_t> configured{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0;
    if (!(configured.load(std::memory_order_relaxed) & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return check_cuda(e, "microscaled pair product shared memory size");
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    MxPairMaps maps;
    const int64_t a_rows = (int64_t)((p.M + 127) / 128) * p.KU * ROWS, w_rows = (int64_t)p.n_tiles * p.KU * ROWS;
    qmm_status s = make_unit_map(&maps.a, p.a, a_rows, ROWS);
    if (s == QMM_OK) s = make_unit_map(&maps.w_codes, p.w[0], w_rows, 128);
    if (s == QMM_OK) s = make_unit_map(&maps.w_scales, p.w[0], w_rows, ROWS - 128);
    if (s != QMM_OK) return s;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * (tiles < kNumSMs / 2 ? tiles : kNumSMs / 2)));
    cfg.blockDim = dim3(MxPairGeom<FMT>::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, maps, p), "microscaled pair product launch");
}

template <int FMT, typename T> static qmm_status dense_t(MxGemmParams p, cudaStream_t st)
{
    p.vec = row_vec<T>(p.y, p.ldy);
    const int pair_tiles = ((p.n_tiles + 1) / 2) * ((p.M + 255) / 256);
    // (the pair form's row coordinates are 32-bit: operands below 2^31 rows of 128 bytes)
    const bool fits = ((int64_t)p.n_tiles + (p.M + 127) / 128) * p.KU * (unit_bytes(FMT) / 128) < (1LL << 31);
    if (p.M > 128 && fits && g_knobs.mx_pair != 2 && (pair_tiles >= 32 || g_knobs.mx_pair == 1)) return launch_pair_t<FMT, T>(p, pair_tiles, st);
    const int64_t tiles = (int64_t)p.n_tiles * ((p.M + 127) / 128);
    int splits = 1;
    while (splits < 8 && splits * 2 <= p.KU && tiles * splits * 2 <= kNumSMs) splits *= 2;
    if (splits > 1) return launch_t<FMT, 1, false, T, kMxSplit>(p, (int)tiles * splits, splits, st);
    return launch_t<FMT, 1, false, T, kMxDense>(p, (int)(tiles < kNumSMs ? tiles : kNumSMs), 1, st);
}

qmm_status launch_mx_gemm(int fmt, const void* a, int64_t M, const void* w, int64_t N, int64_t K, const float* a_scale, const float* w_scale,
                          int dtype, void* y, int64_t ldy, int* status, cudaStream_t st)
{
    MxGemmParams p = {};
    p.a = (const uint8_t*)a;
    p.w[0] = (const uint8_t*)w;
    p.M = (int)M;
    p.N = (int)N;
    p.KU = (int)k_units(K);
    p.n_tiles = (int)((N + 127) / 128);
    p.a_scale = a_scale;
    p.w_scale[0] = w_scale;
    p.y = y;
    p.ldy = ldy;
    p.status = status;
    if (fmt == QMM_MXFP4)
        return dtype == QMM_F16 ? dense_t<QMM_MXFP4, __half>(p, st) : dtype == QMM_BF16 ? dense_t<QMM_MXFP4, __nv_bfloat16>(p, st) : dense_t<QMM_MXFP4, float>(p, st);
    return dtype == QMM_F16 ? dense_t<QMM_NVFP4, __half>(p, st) : dtype == QMM_BF16 ? dense_t<QMM_NVFP4, __nv_bfloat16>(p, st) : dense_t<QMM_NVFP4, float>(p, st);
}

// Most row units that P pairs over E experts can take.
int64_t mx_max_row_units(int64_t pairs, int E)
{
    const int64_t used = pairs < E ? pairs : E;
    return (pairs - used) / 128 + used;
}

static int grouped_grid(int64_t pairs, int E, int n_tiles)
{
    const int64_t t = mx_max_row_units(pairs, E) * n_tiles;
    return (int)(t < kNumSMs ? t : kNumSMs);
}

qmm_status launch_mx_experts_gate_up(int fmt, const void* a, int64_t pairs, int E, const int* offsets, const int* units, const void* w_gate,
                                     const void* w_up, int64_t N, int64_t K, const float* a_scale, const float* gate_scale, const float* up_scale,
                                     const float* h_scale, void* h, int* status, cudaStream_t st)
{
    MxGemmParams p = {};
    p.a = (const uint8_t*)a;
    p.w[0] = (const uint8_t*)w_gate;
    p.w[1] = (const uint8_t*)w_up;
    p.N = (int)N;
    p.KU = (int)k_units(K);
    p.n_tiles = (int)((N + 127) / 128);
    p.w_stride = (int64_t)p.n_tiles * p.KU * unit_bytes(fmt);
    p.offsets = offsets;
    p.units = units;
    p.E = E;
    p.a_scale = a_scale;
    p.w_scale[0] = gate_scale;
    p.w_scale[1] = up_scale;
    p.h_scale = h_scale;
    p.y = h;
    p.status = status;
    const int grid = grouped_grid(pairs, E, p.n_tiles);
    if (fmt == QMM_MXFP4) return launch_t<QMM_MXFP4, 2, true, __half, kMxGrouped>(p, grid, 1, st);
    return launch_t<QMM_NVFP4, 2, true, __half, kMxGrouped>(p, grid, 1, st);
}

template <int FMT, typename T> static qmm_status grouped_t(MxGemmParams p, int grid, cudaStream_t st)
{
    p.vec = row_vec<T>(p.y, p.ldy);
    return launch_t<FMT, 1, false, T, kMxGrouped>(p, grid, 1, st);
}

qmm_status launch_mx_experts_gemm(int fmt, const void* a, int64_t pairs, int E, const int* offsets, const int* units, const void* w, int64_t N,
                                  int64_t K, const float* a_scale, const float* w_scale, int dtype, void* y, int64_t ldy, int* status, cudaStream_t st)
{
    MxGemmParams p = {};
    p.a = (const uint8_t*)a;
    p.w[0] = (const uint8_t*)w;
    p.N = (int)N;
    p.KU = (int)k_units(K);
    p.n_tiles = (int)((N + 127) / 128);
    p.w_stride = (int64_t)p.n_tiles * p.KU * unit_bytes(fmt);
    p.offsets = offsets;
    p.units = units;
    p.E = E;
    p.a_scale = a_scale;
    p.w_scale[0] = w_scale;
    p.y = y;
    p.ldy = ldy;
    p.status = status;
    const int grid = grouped_grid(pairs, E, p.n_tiles);
    if (fmt == QMM_MXFP4)
        return dtype == QMM_F16 ? grouped_t<QMM_MXFP4, __half>(p, grid, st) : dtype == QMM_BF16 ? grouped_t<QMM_MXFP4, __nv_bfloat16>(p, grid, st) : grouped_t<QMM_MXFP4, float>(p, grid, st);
    return dtype == QMM_F16 ? grouped_t<QMM_NVFP4, __half>(p, grid, st) : dtype == QMM_BF16 ? grouped_t<QMM_NVFP4, __nv_bfloat16>(p, grid, st) : grouped_t<QMM_NVFP4, float>(p, grid, st);
}

}  // namespace qmm
