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
    int vec;                         // 16-byte stores of Y are aligned
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

// 32 consecutive outputs of one row; n = how many exist.
template <typename T> __device__ __forceinline__ void store32(T* o, const float (&v)[32], int n, bool vec)
{
    if (vec && n >= 32) {
        if constexpr (sizeof(T) == 2) {
            uint32_t u[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = Dt<T>::down2(v[2 * i], v[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) reinterpret_cast<uint4*>(o)[i] = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<float4*>(o)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
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
                            store32<T>(reinterpret_cast<T*>(p.y) + (int64_t)(w.row0 + r) * p.ldy + n0, f, p.N - n0, p.vec != 0);
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

template <typename T> static bool row_vec(const void* y, int64_t ldy)
{
    return ((reinterpret_cast<uintptr_t>(y) | (uintptr_t)(ldy * (int64_t)sizeof(T))) & 15) == 0;
}

template <int FMT, typename T> static qmm_status dense_t(MxGemmParams p, cudaStream_t st)
{
    p.vec = row_vec<T>(p.y, p.ldy);
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
