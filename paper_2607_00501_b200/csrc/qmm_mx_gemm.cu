// qmm_mx_gemm.cu -- products of packed microscaled 4-bit operands on the block-scaled tcgen05 MMA.
//
// Y[m, n] = sum_b sa[m, b] sw[n, b] sum_i a[m, i] w[n, i]: the tensor core multiplies codes and applies the block scales
// itself, so no CUDA core touches an element on the way in.  Tokens are the rows of the MMA (128 lanes of
// tensor memory, one token row each), weight rows its columns; a pipeline stage is one unit of K (256 k): the codes and scales of
// up to 128 token rows and of BN weight rows (of one matrix, or of two: gate and up), fetched as contiguous bulk copies
// -- the packed operand holds exactly what a stage needs, in the order the tensor core reads it.  Scales go from shared
// memory to tensor memory with tcgen05.cp, in the issuing thread's order with the MMAs that read them (two sets of columns in turn).
//
// Why tokens on the lanes: a thread of the epilogue then holds consecutive outputs of one token row,
// which makes 32 consecutive intermediate features -- the blocks of the next product's operand -- local to a
// thread (gate/up form), and rows of Y full sectors.  With few tokens most lanes idle, which costs nothing: the
// 128 x 128 x 256 step takes 256 cycles of the tensor pipe per 17 KB of weights, and HBM delivers 17 KB per SM in
// ~750 cycles.
//
// Roles: warps 0 and 2 load weights and tokens, warp 1 issues copies of scales and MMAs (converged, one elected lane), warps 4.. run
// the epilogue: they take the accumulators into registers at once, free them, then work and store while the next tile's
// MMAs run.  The kernel is persistent over tiles, ring and barrier phases run on across them.
// Tile t = (token tile t / n_tiles, weight tile t % n_tiles).  BN = 128; 64 in the gate/up form of few rows.
// Few rows, few tiles, long K: blocks share a tile's K (mx_splits) and meet through memory.  (Meeting through the shared memory of a cluster
// was slower: 8.8 us against 6 unshared for one token and a 2048 x 2048 matrix -- clusters of eight do not all fit the GPU at once, and their
// launch costs 3 us.)
// What bounds it: one token, 128256 x 2048 25 us (MXFP4; 140 MB, 5.6 TB/s), 2048 x 2048 4.1 us (launch, first loads, 1.4 us of quantising the row
// in every block); one token, 2048 x 8192 5.8 us.  Gate/up of 128 experts x 768 x 2048, 16384 pairs: 53 us, DRAM 56 % and tensor pipe 35 % busy:
// the 128-row tiles of one SM take 17 KB per 256 cycles each of tokens and weights from L2.
// Grouped: token tiles of the experts' rows, from the device arrays units[] / offsets[].
// Every mbarrier wait is bounded; on give-up the block records QMM_ERR_DEVICE_TIMEOUT, waits (bounded) for its copies
// in flight, frees its tensor memory and returns.
#include "qmm_mx.cuh"
#include "qmm_tc.cuh"

#include <atomic>

namespace qmm {

using namespace mx;

struct MxGemmParams {
    const uint8_t* a;                // packed token rows
    const uint8_t* w[2];             // packed weights (expert 0): W, or W_gate and W_up
    int64_t w_stride;                // bytes between experts
    int M, N, KU;                    // token rows (dense), weight rows, k units
    int n_tiles;                     // weight tiles of BN rows (pair form: of 128)
    const int *offsets, *units;      // grouped: [E + 1] each
    int E;
    int list_ready;                  // grouped: units[] and offsets[] were complete before this kernel could start (the kernel upstream lets its
                                     // dependents go only after its own wait for the sort): weights are requested while that kernel still runs
    const float* a_scale;            // tensor scales, null = 1
    const float* w_scale[2];         // grouped: [E]
    const float* h_scale;            // gate/up: tensor scale of the output operand
    void* y;                         // [rows, ldy], or the packed output operand (gate/up)
    int64_t ldy;
    int vec;                         // widest aligned store of Y: 32, 16, 4 or 2 bytes
    const void* x;                   // few: token rows as they come, [M, ldx] of Y's type
    int64_t ldx, K;
    int x_vec;                       // widest aligned load of x
    int atoms;                       // few: 8-row atoms per unit (1 or 2)
    int stages;                      // ring depth (what resident rows or staging leave)
    int* status;
    int splits;                      // dense, few: blocks that share a tile's K (1: none); then every block has one piece of work, and
    float* partial;                  // partial sums go here, [tile][split][rows, a multiple of 32][128 columns],
    int* counters;                   // 16 bits per tile, zero between calls: the block that comes last adds the partial sums
};

constexpr int kMxMaxE = 1024;

// Forms of the kernel of one SM: packed token rows; packed rows grouped by expert; a few rows as they come.
enum MxForm { kMxDense = 0, kMxGrouped = 1, kMxFew = 2 };

// Shared memory of an epilogue warp that writes rows of any alignment: 32 rows of 32 words, one word apart.
constexpr int kRowStaging = 32 * 33 * 4;

template <int FMT, int BN, bool GATEUP, int FORM> struct MxGeom {
    static constexpr int NB = GATEUP ? 2 : 1;                                   // weight matrices
    static constexpr int kUnit = unit_bytes(FMT), kSc = scale_bytes(FMT);
    static constexpr bool kWhole = BN == 128;                                   // a tile's weights are whole units
    static constexpr int kCodes = BN * 128;                                     // codes of one matrix in a stage
    static constexpr int kW = FORM == kMxFew ? 0 : kUnit;                       // stage: token unit (few: none) | codes of each matrix | scales of each
    static constexpr int kScW = kW + NB * kCodes;
    static constexpr int kStage = kScW + NB * kSc;
    static constexpr int kCodeStep = kCodes >> 4, kScStep = kSc >> 4;           // from matrix to matrix, in descriptor units
    static constexpr int kDCols = NB * BN;
    // columns per epilogue warp: 32 of each matrix in the gate/up form (its arithmetic wants warps), else up to 64
    static constexpr int kCols = GATEUP ? 32 : 64;
    static constexpr int kParts = BN / kCols, kEpiWarps = 4 * kParts;
    static constexpr int kThreads = (4 + kEpiWarps) * 32;
    static constexpr int kHead = 1024 + (FORM == kMxGrouped ? 9 * 1024 : 0);    // barriers, the experts' first units and rows
    static constexpr int kStaging = GATEUP ? 0 : kEpiWarps * kRowStaging;       // after the ring, for rows that 16-byte stores cannot reach
    static constexpr int kRoom = 227 * 1024 - 1024 - kHead;                     // for the ring (few: after the resident rows)
    static constexpr int kFit = kRoom / kStage;
    static constexpr int kStages = kFit < 10 ? kFit : 10;
    static constexpr int kSmem = GATEUP ? 1024 + kHead + kStages * kStage : 227 * 1024;
    static_assert(2 * (kMxMaxE + 32) * 4 <= 9 * 1024, "index area");
    // tensor memory: accumulators (two when they fit), then two sets of scale columns
    static constexpr int kAccBufs = kDCols > 128 ? 1 : 2;
    static constexpr int kGroups = kUnitK / FMT / 4;                            // scale groups per unit: 2 or 4
    static constexpr int kSfCols = kGroups * 4 * (1 + NB);
    static constexpr int kSf0 = kAccBufs * kDCols;
    static constexpr int kTmemCols = 512;
    static_assert(kSf0 + 2 * kSfCols <= kTmemCols && kStage % 1024 == 0, "tensor memory over-subscribed or stage misaligned");
    static_assert(kStages >= 3, "pipeline too shallow");
};

// One piece of work: a token tile against a weight tile.
struct MxWork {
    int m_unit;                      // row unit of the token operand
    int rows;                        // token rows in it (1 .. 128)
    int row0;                        // first row of Y
    int n_tile, expert;
    int k0, k1;                      // k units (K shared between blocks)
};

// silu(g) u = (g / (1 + 2^(-g log2 e))) u for two features at a time, g and u still to be multiplied by the factors a0 and a1.  2^x and 1 / x are the hardware's
// approximations (relative error of a few 2^-23 each); g << 0 gives 2^x = inf and silu = -0.  silu is complete before u comes in: g u may be beyond fp32 where
// silu(g) u is not.  The denominator is inverted times 2^-8: its own reciprocal may be a subnormal, which the approximation flushes, where silu is none.  (The
// factor is not taken into the exponent: x - 8 has fewer bits behind the point than x; of 10^8 NVFP4 codes of h 67 then were not those of the exact h, 55 are.)
__device__ __forceinline__ float ex2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 silu_mul2(float2 g, float2 u, float a0, float a1)
{
    g = mul2(g, both(a0));
    const float2 x = mul2(g, both(-1.44269504f));
    const float2 den = fma2(make_float2(ex2_approx(x.x), ex2_approx(x.y)), both(0x1p-8f), both(0x1p-8f));
    const float2 r = mul2(make_float2(rcp_approx(den.x), rcp_approx(den.y)), both(0x1p-8f));
    return mul2(mul2(g, r), mul2(u, both(a1)));
}

// 32 consecutive outputs of one row; n = how many exist.  vec: 32 or 16 byte stores (32 writes whole sectors: a lane's neighbours in a
// store are other rows).
template <typename T> __device__ __forceinline__ void store32(T* o, const float (&v)[32], int n, int vec)
{
    if (n >= 32) {
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

// 32 rows (a lane each, `rows` of them exist; y: row 0) x 32 columns from n0 of a matrix whose rows start anywhere: through shared memory, so that
// a store instruction writes consecutive elements of one row.  (Element by element from the row's own lane, 128 x 300 took 20 us, so 3.)
template <typename T>
__device__ __forceinline__ void store_rows_any(uint32_t* staging, T* y, int64_t ldy, const uint32_t (&v)[32], float alpha, int lane, int rows, int n0, int N, int vec)
{
    __syncwarp();                                                             // (the previous columns have been read)
    constexpr int W = 8 * (int)sizeof(T);                                     // words of a row
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if constexpr (sizeof(T) == 2) staging[lane * 33 + i] = Dt<T>::down2(alpha * __uint_as_float(v[2 * i]), alpha * __uint_as_float(v[2 * i + 1]));
        else staging[lane * 33 + i] = __float_as_uint(alpha * __uint_as_float(v[i]));
    }
    __syncwarp();
    const int left = min(32, N - n0);
    if (sizeof(T) == 2 && vec >= 4) {                                         // two elements per lane, two rows per instruction
        const int c = 2 * (lane & 15);
        for (int r = lane >> 4; r < rows; r += 2) {
            const uint32_t u = staging[r * 33 + (lane & 15)];
            T* o = y + r * ldy + n0 + c;
            if (c + 2 <= left) *reinterpret_cast<uint32_t*>(o) = u;
            else if (c < left) *reinterpret_cast<unsigned short*>(o) = (unsigned short)u;
        }
    } else if (lane < left) {
        for (int r = 0; r < rows; ++r) y[r * ldy + n0 + lane] = reinterpret_cast<const T*>(staging + r * 33)[lane];
    }
}

__device__ __forceinline__ void mx_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The epilogue's warps meet: whether all / any of their threads said so.
template <int THREADS> __device__ __forceinline__ bool epilogue_all(bool x)
{
    int r;
    asm volatile("{.reg .pred p, q; setp.ne.s32 p, %1, 0; barrier.cta.red.and.pred q, 2, %2, p; selp.s32 %0, 1, 0, q;}" : "=r"(r) : "r"((int)x), "n"(THREADS) : "memory");
    return r != 0;
}
template <int THREADS> __device__ __forceinline__ bool epilogue_any(bool x)
{
    int r;
    asm volatile("{.reg .pred p, q; setp.ne.s32 p, %1, 0; barrier.cta.red.or.pred q, 2, %2, p; selp.s32 %0, 1, 0, q;}" : "=r"(r) : "r"((int)x), "n"(THREADS) : "memory");
    return r != 0;
}

template <int FMT, int BN, bool GATEUP, typename T, int FORM, bool SPLIT>
__global__ void __launch_bounds__(MxGeom<FMT, BN, GATEUP, FORM>::kThreads, 1) mx_gemm_kernel(const MxGemmParams p)
{
    using namespace tc;
    using G = MxGeom<FMT, BN, GATEUP, FORM>;
    constexpr bool GROUPED = FORM == kMxGrouped, FEW = FORM == kMxFew;
    constexpr int AB = G::kAccBufs, NEPI = G::kEpiWarps, NB = G::NB;
    constexpr int W_WARP = 0, MMA_WARP = 1, A_WARP = 2, EPI_WARP0 = 4;         // loads of weights and of tokens are two warps

    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int S = p.stages;                                                   // ring depth, at most 10
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);                       // [S] loads -> MMA
    uint64_t* empty = full + 10;                                              // [S] MMA -> loads
    uint64_t* acc_full = empty + 10;                                          // [2] MMA -> epilogue
    uint64_t* acc_empty = acc_full + 2;                                       // [2] epilogue -> MMA
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    int* s_units = reinterpret_cast<int*>(smem + 1024);                       // [E + 1], then INT_MAX up to a multiple of 32 (grouped)
    int* s_first = s_units + kMxMaxE + 32;                                    // [E + 1]
    // few: the resident token rows, atoms of 8 rows x 128 bytes (p.atoms of them per k unit), then their scales, then the ring.  The MMA reads
    // 128 rows from a unit's first atom: the rows past its own are whatever follows (never stored), inside the block's memory.
    uint8_t* resident = smem + G::kHead;
    const int resident_units = !FEW ? 0 : SPLIT ? (p.KU + p.splits - 1) / p.splits : p.KU, resident_codes = resident_units * p.atoms * 1024;
    const uint32_t ring0 = smem_u32(resident) + resident_codes + resident_units * G::kSc;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&full[s], FEW ? 1 : 2);                                 // the loading warps (+ their bytes)
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
    const bool waited = GROUPED && !p.list_ready;
    if (waited) pdl_wait();                                                   // the rows' grouping is written upstream
    if (GROUPED) {
        for (int e = threadIdx.x; e < ((p.E + 32) & ~31); e += G::kThreads) {
            s_units[e] = e <= p.E ? __ldcg(p.units + e) : 0x7FFFFFFF;         // (from L2: with list_ready no wait of this kernel stands before the read)
            if (e <= p.E) s_first[e] = __ldcg(p.offsets + e);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_launch_dependents();

    const int m_tiles = GROUPED ? s_units[p.E] : (p.M + 127) >> 7;
    const int total = m_tiles * p.n_tiles;

    // the units of K of a piece of work
    auto K0 = [&](const MxWork& w) { return SPLIT ? w.k0 : 0; };
    auto K1 = [&](const MxWork& w) { return SPLIT ? w.k1 : p.KU; };
    // i-th piece of work of this block (the same sequence for every role; whole converged warps)
    auto get_work = [&](int i, MxWork& w) -> bool {
        int t = (int)blockIdx.x + i * (int)gridDim.x;
        if (SPLIT) {
            if (i > 0) return false;
            const int q = t % p.splits;
            t /= p.splits;
            w.k0 = p.KU * q / p.splits;
            w.k1 = p.KU * (q + 1) / p.splits;
        }
        if (t >= total) return false;
        const int mt = t / p.n_tiles;
        w.n_tile = t - mt * p.n_tiles;
        w.m_unit = mt;
        if (GROUPED) {
            // the expert that unit mt belongs to: the last e with units[e] <= mt.  Two rounds of 32 comparisons: which run of 32 experts,
            // then which of them (units[] ascends; an expert without rows starts where the next one does)
            const int runs = (p.E + 31) >> 5;
            const unsigned in_run = __ballot_sync(0xFFFFFFFFu, lane < runs && s_units[lane * 32] <= mt);
            const int run = 31 - __clz(in_run);
            const unsigned in = __ballot_sync(0xFFFFFFFFu, s_units[run * 32 + lane] <= mt);
            w.expert = run * 32 + 31 - __clz(in);
            w.row0 = s_first[w.expert] + 128 * (mt - s_units[w.expert]);
            w.rows = min(128, s_first[w.expert + 1] - w.row0);
        } else {
            w.expert = 0;
            w.row0 = mt * 128;
            w.rows = min(128, p.M - w.row0);
        }
        return true;
    };

    // few: the whole block quantises the token rows once (a thread per 32 elements), into the place and order in which a unit's codes and
    // scales would have arrived; the MMA warp goes on when everybody has
    auto load_tokens = [&]() {
        pdl_wait();
        if constexpr (FEW) {
            const TensorScale ts(p.a_scale ? __ldg(p.a_scale) : 1.0f);
            const int q = SPLIT ? (int)blockIdx.x % p.splits : 0;             // the block's units of K
            const int k0 = SPLIT ? p.KU * q / p.splits : 0, chunks = (SPLIT ? p.KU * (q + 1) / p.splits - k0 : p.KU) * (kUnitK / 32);
            const T* x = reinterpret_cast<const T*>(p.x) + (SPLIT ? k0 * kUnitK : 0);
            const int64_t K = SPLIT ? p.K - k0 * kUnitK : p.K;
            for (int id = threadIdx.x; id < p.M * chunks; id += G::kThreads) {
                const int r = id / chunks, c = id - r * chunks, ku = c >> 3;
                const int64_t left = K - (int64_t)c * 32;
                const int n = (int)(left < 0 ? 0 : left < 32 ? left : 32);
                const T* src = x + r * p.ldx + (int64_t)c * 32;
                float v[32];
                if (p.x_vec == 32) load32<T, 32>(src, n, v);
                else if (p.x_vec == 16) load32<T, 16>(src, n, v);
                else load32<T, 0>(src, n, v);
                uint32_t sb;
                const uint4 codes = quantize32<FMT>(v, ts, sb);
                *reinterpret_cast<uint4*>(resident + (ku * p.atoms + (r >> 3)) * 1024 + chunk_offset(r & 7, c & 7)) = codes;
                uint8_t* sc = resident + resident_codes + ku * G::kSc - kCodeBytes;
                if (FMT == QMM_MXFP4) sc[scale_offset(r, (c & 7) >> 2) + (c & 3)] = (uint8_t)sb;
                else *reinterpret_cast<uint16_t*>(sc + scale_offset(r, (c & 7) >> 1) + 2 * (c & 1)) = (uint16_t)sb;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // ordinary stores, read by the tensor core
            asm volatile("bar.sync 1, %0;" ::"n"(G::kThreads) : "memory");
        }
    };

    if (FEW && warp > A_WARP && warp < EPI_WARP0) {
        load_tokens();
    } else if (warp == W_WARP || warp == A_WARP) {
        // ================= loads (whole warps converged, one lane acts); each warp's part counts on the stage's barrier
        const uint32_t sel = elect_one() ? 1u : 0u, full0 = smem_u32(full);
        bool ok = true;
        int s = 0, round = 0, early = 0, g = 0;
        MxWork w = {};
        auto load_w = [&](int s, int ku) {
            const uint32_t bar = full0 + 8 * s, dst = ring0 + s * G::kStage + G::kW;
            const int r0 = w.n_tile * BN;
            const int64_t at = w.expert * p.w_stride + ((int64_t)(r0 >> 7) * p.KU + ku) * G::kUnit;
            mbar_arrive_expect_tx_sel(bar, NB * (G::kCodes + G::kSc), sel);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (G::kWhole && NB == 1) {                                   // codes and scales in one copy
                    bulk_load_sel(dst, p.w[b] + at, G::kUnit, bar, sel);
                } else {
                    bulk_load_sel(dst + b * G::kCodes, p.w[b] + at + (r0 & 127) * 128, G::kCodes, bar, sel);
                    bulk_load_sel(dst + NB * G::kCodes + b * G::kSc, p.w[b] + at + kCodeBytes, G::kSc, bar, sel);
                }
            }
        };
        // weights do not depend on the previous kernel: the first ring of them is requested before the wait for it
        if (!GROUPED) {
            if (warp == W_WARP && get_work(0, w))
                for (; early < S && early < K1(w) - K0(w); ++early) load_w(early, K0(w) + early);
        }
        if (FEW) load_tokens();
        else if (!waited && warp == A_WARP) pdl_wait();                       // weights go on; token rows are the previous kernel's
        for (int i = 0; (!FEW || warp == W_WARP) && ok && get_work(i, w); ++i) {
            const uint32_t rows8 = (uint32_t)(w.rows + 7) & ~7u;
            const uint8_t* src = p.a + (int64_t)w.m_unit * p.KU * G::kUnit;
            for (int ku = K0(w); ku < K1(w); ++ku, ++g, s + 1 == S ? (s = 0, ++round) : ++s) {
                if (round > 0) ok = mbar_wait(&empty[s], (round - 1) & 1, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                if (FEW || warp == W_WARP) {
                    if (g >= early) load_w(s, ku);
                    continue;
                }
                const uint32_t bar = full0 + 8 * s, dst = ring0 + s * G::kStage;
                mbar_arrive_expect_tx_sel(bar, rows8 * 128u + G::kSc, sel);
                if (rows8 == 128) {
                    bulk_load_sel(dst, src + (int64_t)ku * G::kUnit, G::kUnit, bar, sel);
                } else {
                    bulk_load_sel(dst, src + (int64_t)ku * G::kUnit, rows8 * 128u, bar, sel);
                    bulk_load_sel(dst + kCodeBytes, src + (int64_t)ku * G::kUnit + kCodeBytes, G::kSc, bar, sel);
                }
            }
        }
        // the MMA's last arrivals (one per stage of the last round) have come before the block's shared memory is released
        for (int q = max(0, g - S); ok && warp == W_WARP && q < g; ++q) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&empty[q % S], (q / S) & 1, abort_flag));
        if (!ok) {
            *abort_flag = 1;
            // let copies in flight land, too
            for (int q = max(0, g - S); q < g; ++q) {
                const long long t0 = clock64();
                while (!mbar_try_wait(&full[q % S], (q / S) & 1) && clock64() - t0 < (1LL << 22)) {}
            }
        }
    } else if (warp == MMA_WARP) {
        // ================= MMA issuer (whole warp converged, one lane acts)
        const uint32_t sel = elect_one() ? 1u : 0u;
        // token operand: in the stage, or resident (then a k unit is atoms * 1024 bytes of codes and kSc of scales further)
        const uint64_t desc_a = smem_desc_k_sw128(FEW ? smem_u32(resident) : ring0), desc_w = smem_desc_k_sw128(ring0 + G::kW);
        const uint64_t desc_sa = smem_desc_scales(FEW ? smem_u32(resident) + resident_codes : ring0 + kCodeBytes), desc_sw = smem_desc_scales(ring0 + G::kScW);
        bool ok = true;
        int s = 0;
        uint32_t par = 0, set = 0;                                            // parity of the ring's round; set of scale columns
        MxWork w;
        if (FEW) load_tokens();
        for (int it = 0; ok && get_work(it, w); ++it) {
            const int buf = it % AB;
            if (it >= AB) {
                ok = mbar_wait(&acc_empty[buf], ((it / AB) - 1) & 1, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
            }
            const uint32_t d = tmem_base + (uint32_t)(buf * G::kDCols);
            // a tile of 64 rows takes the scale columns of its rows out of the unit's four (32 rows each)
            const uint32_t sub = BN < 128 ? (uint32_t)((w.n_tile * BN) & 64) >> 5 : 0u;
            for (int ku = K0(w); ku < K1(w); ++ku, set ^= 1, s + 1 == S ? (s = 0, par ^= 1) : ++s) {
                ok = mbar_wait(&full[s], par, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
                const uint64_t at = (uint64_t)(s * (G::kStage >> 4));
                const uint64_t at_a = FEW ? (uint64_t)((ku - K0(w)) * p.atoms * 64) : at, at_sa = FEW ? (uint64_t)((ku - K0(w)) * (G::kSc >> 4)) : at;
                const uint32_t sfa = tmem_base + (uint32_t)G::kSf0 + set * (uint32_t)G::kSfCols;
                const uint32_t sfw = sfa + (uint32_t)(G::kGroups * 4);
                copy_scales<1, G::kGroups>(sfa, desc_sa + at_sa, 4, sel);
#pragma unroll
                for (int b = 0; b < NB; ++b) copy_scales<1, G::kGroups>(sfw + 4 * b, desc_sw + at + b * G::kScStep, 4 * NB, sel);
                // two whole matrices are one MMA of N = 256 (their codes and their scale columns are adjacent), else one MMA each
                constexpr int MMAS = G::kWhole ? 1 : NB;
#pragma unroll
                for (int b = 0; b < MMAS; ++b)
                    mma_fp4_stage<1, FMT == QMM_MXFP4>(d + b * BN, desc_a + at_a, desc_w + at + b * G::kCodeStep, idesc_fp4(FMT == QMM_MXFP4, 128, G::kDCols / MMAS),
                                                       sfa, sfw + 4 * b + sub, 4 * NB, ku != K0(w), sel);
                mma_commit_sel(&empty[s], sel);
                __syncwarp();
            }
            if (ok) mma_commit_sel(&acc_full[buf], sel);
            __syncwarp();
        }
        if (!ok) *abort_flag = 1;
    } else if (warp >= EPI_WARP0) {
        // ================= epilogue: 32 rows x kCols columns of each matrix per warp
        constexpr int CW = G::kCols, C32 = CW / 32;
        const int quarter = warp & 3, part = (warp - EPI_WARP0) >> 2;
        const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(part * CW);
        bool ok = true;
        MxWork w;
        // every global write below comes after the previous kernel has completed (its readers of this buffer included)
        if (FEW) load_tokens();
        else if (!waited) pdl_wait();
        const float a_scale = p.a_scale ? __ldg(p.a_scale) : 1.0f;
        const TensorScale hs(GATEUP && p.h_scale ? __ldg(p.h_scale) : 1.0f);
        for (int it = 0; ok && get_work(it, w); ++it) {
            const int buf = it % AB;
            const ProductScale scale(a_scale, p.w_scale[0] ? __ldg(p.w_scale[0] + w.expert) : 1.0f);
            const ProductScale scale1(a_scale, GATEUP && p.w_scale[1] ? __ldg(p.w_scale[1] + w.expert) : 1.0f);
            const float alpha = scale.second;
            ok = mbar_wait(&acc_full[buf], (it / AB) & 1, abort_flag);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok && !SPLIT) break;                                         // (split: the epilogue's warps meet below, whatever became of the wait)
            tc_fence_after_sync();
            const int r = quarter * 32 + lane;                                // token row of the tile
            const bool warp_has_rows = (!SPLIT || ok) && quarter * 32 < w.rows;
            uint32_t v[NB * C32][32];
            if (warp_has_rows) {
#pragma unroll
                for (int c = 0; c < NB * C32; ++c)
                    tmem_ld_32x32b_x32(lanes + (uint32_t)(buf * G::kDCols + (c / C32) * BN + (c % C32) * 32), v[c]);
                tmem_wait_ld();
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[buf]);                      // the accumulators may be overwritten
            if (!SPLIT && !warp_has_rows) continue;
            const int n0 = w.n_tile * BN + part * CW;
            if constexpr (!SPLIT) {
#pragma unroll
                for (int c = 0; c < NB * C32; ++c) (GATEUP && c ? scale1 : scale).apply_first(v[c]);
            }
            if constexpr (GATEUP) {
                const int hku = (p.N + kUnitK - 1) / kUnitK;                  // k units of the output operand
                uint8_t* row_units = reinterpret_cast<uint8_t*>(p.y) + (int64_t)w.m_unit * hku * G::kUnit;
                // 32 features from k (a multiple of 32): codes, and the scale byte(s) of their block(s)
                auto put = [&](int k, const uint4& codes, uint32_t sc) {
                    uint8_t* unit = row_units + (int64_t)(k / kUnitK) * G::kUnit;
                    const uint32_t c = (uint32_t)(k % kUnitK) >> 5;
                    *reinterpret_cast<uint4*>(unit + chunk_offset(r, c)) = codes;
                    if (FMT == QMM_MXFP4) unit[scale_offset(r, c >> 2) + (c & 3)] = (uint8_t)sc;
                    else *reinterpret_cast<uint16_t*>(unit + scale_offset(r, c >> 1) + 2 * (c & 1)) = (uint16_t)sc;
                };
                const int left = p.N - n0;
                float h[32];
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    const float2 x = silu_mul2(make_float2(__uint_as_float(v[0][i]), __uint_as_float(v[0][i + 1])),
                                               make_float2(__uint_as_float(v[1][i]), __uint_as_float(v[1][i + 1])), alpha, scale1.second);
                    h[i] = x.x, h[i + 1] = x.y;
                }
                if (left < 32) {                                              // features past N are zeros of the operand's padding
#pragma unroll
                    for (int i = 0; i < 32; ++i) h[i] = i < left ? h[i] : 0.0f;
                }
                uint32_t sc;
                const uint4 codes = quantize32<FMT>(h, hs, sc);
                if (r < w.rows) {
                    put(n0, codes, sc);
                    if (w.n_tile == p.n_tiles - 1 && part == G::kParts - 1)
                        for (int k = p.n_tiles * BN; k < hku * kUnitK; k += 32) put(k, make_uint4(0, 0, 0, 0), 0);    // the rest of the last unit
                }
            } else if constexpr (SPLIT) {
                // Partial sums to memory; the block that finds the others' there already adds them in the order of K (same bits on every
                // call), all its epilogue warps sharing the tile, and stores.  Nobody waits for another block.
                const int tile = (int)blockIdx.x / p.splits, span = (min(p.M, 128) + 31) / 32 * 32 * BN;     // span: a tile's partial sums
                float* slots = p.partial + (int64_t)tile * p.splits * span;
                if (ok && r < w.rows) {
                    float* o = slots + ((int)blockIdx.x % p.splits) * span + r * BN + part * CW;
#pragma unroll
                    for (int c = 0; c < C32; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) st_global_256(o + 32 * c + 8 * i, &v[c][8 * i]);
                }
                __threadfence();
                bool last = false;
                const int e0 = (int)threadIdx.x - EPI_WARP0 * 32;
                if (epilogue_all<32 * G::kEpiWarps>(ok) && e0 == 0) {
                    __threadfence();
                    int* word = p.counters + (tile >> 1);                     // (at most eight blocks a tile: no carry into the other half)
                    const int shift = 16 * (tile & 1);
                    last = ((unsigned)atomicAdd(word, 1 << shift) >> shift & 0xFFFFu) == (unsigned)(p.splits - 1);
                    if (last) atomicSub(word, p.splits << shift);
                }
                if (!epilogue_any<32 * G::kEpiWarps>(last)) break;
                __threadfence();
                T* y = reinterpret_cast<T*>(p.y) + (int64_t)w.row0 * p.ldy + w.n_tile * BN;
                for (int e = 4 * e0; e < w.rows * BN; e += 128 * G::kEpiWarps) {       // four columns of a row: every split's in flight at once
                    float4 v4[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (q < p.splits) v4[q] = __ldcg(reinterpret_cast<const float4*>(slots + q * span + e));
                    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (q < p.splits) {
                            sum[0] += v4[q].x;
                            sum[1] += v4[q].y;
                            sum[2] += v4[q].z;
                            sum[3] += v4[q].w;
                        }
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[k] *= scale.first;
                    const int c = e % BN, left = p.N - w.n_tile * BN - c;
                    T* o = y + (e / BN) * p.ldy + c;
                    if (sizeof(T) == 2 && p.vec >= 16 && left >= 4) {
                        if constexpr (sizeof(T) == 2)
                            *reinterpret_cast<uint2*>(o) = make_uint2(Dt<T>::down2(alpha * sum[0], alpha * sum[1]), Dt<T>::down2(alpha * sum[2], alpha * sum[3]));
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (k < left) o[k] = Dt<T>::down(alpha * sum[k]);
                    }
                }
            } else {
                if (p.vec < 16) {
                    uint32_t* staging = reinterpret_cast<uint32_t*>(smem_raw + G::kSmem - G::kStaging + (warp - EPI_WARP0) * kRowStaging);
#pragma unroll
                    for (int c = 0; c < C32; ++c)
                        store_rows_any(staging, reinterpret_cast<T*>(p.y) + (int64_t)(w.row0 + quarter * 32) * p.ldy, p.ldy, v[c], alpha, lane,
                                       min(32, w.rows - quarter * 32), n0 + 32 * c, p.N, p.vec);
                } else if (r < w.rows) {
                    T* o = reinterpret_cast<T*>(p.y) + (int64_t)(w.row0 + r) * p.ldy + n0;
#pragma unroll
                    for (int c = 0; c < C32; ++c) {
                        float f[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = alpha * __uint_as_float(v[c][i]);
                        store32<T>(o + 32 * c, f, p.N - n0 - 32 * c, p.vec);
                    }
                }
            }
        }
        if (!ok) *abort_flag = 1;
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
// Bound by the tensor pipe, and that by the power limit: NVFP4 8192 x 8192 x 8192 199 us (5.5 PFLOP/s, the pipe 74 % busy) after a pause, 226 to 234
// back to back, 158 on constant data.
template <int FMT> struct MxPairGeom {
    static constexpr int kSc = scale_bytes(FMT);
    static constexpr int kA = 0, kB = unit_bytes(FMT), kSb = kB + kCodeBytes;              // A unit | B codes | scales of both B units
    static constexpr int kStage = kSb + 2 * kSc;
    static constexpr int kStaging = 8 * kRowStaging;                                       // at the end, for rows that 16-byte stores cannot reach
    static constexpr int kSmem = 227 * 1024;
    static constexpr int stages(bool staging)
    {
        const int fit = (kSmem - 2048 - (staging ? kStaging : 0)) / kStage;
        return fit < 6 ? fit : 6;
    }
    static constexpr int kGroups = kUnitK / FMT / 4;
    static constexpr int kSf0 = 256, kSfCols = kGroups * 12;
    static constexpr int kThreads = 12 * 32;
    static_assert(kSf0 + 2 * kSfCols <= 512 && stages(true) >= 4, "tensor memory or shared memory over-subscribed");
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
    constexpr int UNIT = unit_bytes(FMT);
    const int S = p.stages;                                                   // ring depth, at most 6

    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);                       // [S] loads of both blocks -> MMA (first block)
    uint64_t* empty = full + 6;                                               // [S] MMA -> loads
    uint64_t* acc_full = empty + 6;                                           // MMA -> epilogue
    uint64_t* acc_empty = acc_full + 1;                                       // epilogues of both blocks -> MMA (first block)
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t smem0 = smem_u32(smem) + 1024;                             // the ring
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
            int g = 0, s = 0, round = 0, early = 0;
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
                for (int ku = 0; ku < p.KU; ++ku, ++g, s + 1 == S ? (s = 0, ++round) : ++s) {
                    if (round > 0) ok = mbar_wait(&empty[s], (round - 1) & 1, abort_flag);
                    if (!ok) break;
                    if (g >= early) load_w(s, mt, nt, ku);
                    if (a < a_units) tma_load_2d_pair(smem0 + s * G::kStage, &maps.a, 0, (a * p.KU + ku) * ROWS, full0 + 8 * s);
                }
            }
            // the MMA's last arrivals, which come from the first block to both, before the block's shared memory is released
            for (int q = max(0, g - S); ok && q < g; ++q) ok = mbar_wait(&empty[q % S], (q / S) & 1, abort_flag);
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
        int s = 0, it = 0;
        uint32_t par = 0, set = 0;                                            // parity of the ring's round; set of scale columns
        for (int t = first; ok && t < total; t += pairs, ++it) {
            if (it > 0) {
                ok = mbar_wait(acc_empty, (it - 1) & 1, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
            }
            for (int ku = 0; ku < p.KU; ++ku, set ^= 1, s + 1 == S ? (s = 0, par ^= 1) : ++s) {
                ok = mbar_wait(&full[s], par, abort_flag);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
                const uint64_t at = (uint64_t)(s * (G::kStage >> 4));
                const uint32_t sfa = tmem_base + (uint32_t)G::kSf0 + set * (uint32_t)G::kSfCols;
                const uint32_t sfb = sfa + (uint32_t)(G::kGroups * 4);
                copy_scales<2, G::kGroups>(sfa, desc_sa + at, 4, sel);
                copy_scales<2, G::kGroups>(sfb, desc_sb + at, 8, sel);
                copy_scales<2, G::kGroups>(sfb + 4, desc_sb + at + (G::kSc >> 4), 8, sel);
                mma_fp4_stage<2, FMT == QMM_MXFP4>(tmem_base, desc_a + at, desc_b + at, idesc_fp4(FMT == QMM_MXFP4, 256, 256), sfa, sfb, 8, ku != 0, sel);
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
        const ProductScale scale(p.a_scale ? __ldg(p.a_scale) : 1.0f, p.w_scale[0] ? __ldg(p.w_scale[0]) : 1.0f);
        const float alpha = scale.second;
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
#pragma unroll
            for (int c = 0; c < 4; ++c) scale.apply_first(v[c]);
            int mt, nt;
            pair_tile(t, m_tiles, n_tiles, mt, nt);
            const int row = 256 * mt + 128 * (int)rank + quarter * 32 + lane;
            const int n0 = 256 * nt + 128 * half;
            if (p.vec < 16) {
                uint32_t* staging = reinterpret_cast<uint32_t*>(smem_raw + G::kSmem - G::kStaging + (warp - 4) * kRowStaging);
                const int row0 = row - lane;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    store_rows_any(staging, reinterpret_cast<T*>(p.y) + (int64_t)row0 * p.ldy, p.ldy, v[c], alpha, lane, min(32, p.M - row0), n0 + 32 * c, p.N, p.vec);
            } else if (row < p.M) {
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

template <int FMT, int BN, bool GATEUP, typename T, int FORM, bool SPLIT = false>
static qmm_status launch_t(const MxGemmParams& p, int64_t tiles, cudaStream_t st)
{
    auto kern = mx_gemm_kernel<FMT, BN, GATEUP, T, FORM, SPLIT>;
    using G = MxGeom<FMT, BN, GATEUP, FORM>;
    static std::atomic<uint64_t> configured{0};                               // devices that have the attribute
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) dev = 0;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0;
    if (!(configured.load(std::memory_order_relaxed) & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmem);
        if (e != cudaSuccess) return check_cuda(e, "microscaled product shared memory size");
        configured.fetch_or(bit, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles < kNumSMs ? tiles : kNumSMs));
    cfg.blockDim = dim3(G::kThreads);
    cfg.dynamicSmemBytes = G::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, p), "microscaled product launch");
}

// Widest access (bytes) that every row's start allows.
template <typename T> static int row_vec(const void* y, int64_t ldy)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(y) | (uintptr_t)(ldy * (int64_t)sizeof(T));
    return a % 32 == 0 ? 32 : a % 16 == 0 ? 16 : a % 4 == 0 ? 4 : 2;
}

// Few rows: shared memory that M token rows take over KU units.
static int few_resident(int fmt, int64_t M, int KU) { return KU * ((int)((M + 7) / 8) * 1024 + scale_bytes(fmt)); }

// Blocks that share a tile's K, where the tiles leave most SMs idle: 2 to 8, of at least four units of K each.  A unit is 0.3 us of a block's
// time; meeting costs about 2 us, and adding up 1 us more for 8 rows (every block's sums are written and read once).  So a share has to save
// 12 units, and half a unit more for every row past 16.  Shared / whole, MXFP4, N = 2048: one token, K = 4096 5.2 / 6.1 us, 8192 5.8 / 9.8, 16384
// 7.3 / 20.7; 16 tokens 6.9 / 8.0, 7.7 / 12.2; 64 tokens 10.6 / 8.4, 13.6 / 12.5, 15.1 / 20.7; 128 tokens, 16384 21.5 / 22.0; and two blocks a
// tile, N = 8192: one token, K = 4096 7.0 / 6.6, 8192 10.2 / 10.7.
static int mx_splits(int64_t M, int64_t N, int KU)
{
    const int64_t most = kNumSMs / ((N + 127) / 128), by_k = KU / 4;
    int64_t s = most < by_k ? most : by_k;
    if (s > 8) s = 8;
    if (M > 128 || s < 2 || g_knobs.mx_no_split) return 1;
    return KU - KU / s >= 12 + (M > 16 ? (M - 16) / 2 : 0) ? (int)s : 1;
}

// Workspace of a product behind the status word: counters (zero between calls) at kMxCounters, partial sums at kMxHeader.
size_t mx_gemm_partial_bytes(int64_t M, int64_t N, int64_t K)
{
    const int splits = mx_splits(M, N, (int)k_units(K));
    return splits > 1 ? (size_t)((N + 127) / 128 * splits) * ((M + 31) / 32 * 32) * 128 * sizeof(float) : 0;
}

// The most of it that any product of up to M rows takes (more rows may share less): what a size query answers, so that a workspace serves smaller batches too.
size_t mx_gemm_partial_bytes_up_to(int64_t M, int64_t N, int64_t K)
{
    size_t most = 0;
    for (int64_t m = 1; m <= M && m <= 128; ++m) {
        const size_t bytes = mx_gemm_partial_bytes(m, N, K);
        if (bytes > most) most = bytes;
    }
    return most;
}

template <int FMT, typename T, int FORM> static qmm_status launch_tiles(MxGemmParams p, int64_t row_tiles, cudaStream_t st)
{
    using G = MxGeom<FMT, 128, false, FORM>;
    p.vec = row_vec<T>(p.y, p.ldy);
    const int64_t tiles = row_tiles * p.n_tiles;
    p.splits = 1;
    if (FORM != kMxGrouped) {
        p.splits = mx_splits(p.M, p.N, p.KU);
        p.counters = p.status + kMxCounters / 4;
        p.partial = reinterpret_cast<float*>(reinterpret_cast<char*>(p.status) + kMxHeader);
    }
    const int room = G::kRoom - (FORM == kMxFew ? few_resident(FMT, p.M, (p.KU + p.splits - 1) / p.splits) : 0) - (p.vec < 16 && p.splits == 1 ? G::kStaging : 0);
    p.stages = room / G::kStage < 10 ? room / G::kStage : 10;
    if constexpr (FORM != kMxGrouped)
        if (p.splits > 1) return launch_t<FMT, 128, false, T, FORM, true>(p, tiles * p.splits, st);
    return launch_t<FMT, 128, false, T, FORM>(p, tiles, st);
}

// Gate/up: tiles of 64 + 64 weight rows spread a decode step better over the SMs, tiles of 128 + 128 move fewer token rows: 128 experts of
// 768 x 2048, 8 per token, 64 / 128: 4 tokens 14.3 / 16.2 us, 1024 tokens 40.8 / 45.3, 2048 tokens (128 rows an expert) 55.0 / 52.3.
template <int FMT> static qmm_status launch_gate_up(MxGemmParams p, int64_t pairs, int64_t row_tiles, cudaStream_t st)
{
    const int bn = g_knobs.mx_tile ? g_knobs.mx_tile : pairs >= 96LL * p.E ? 128 : 64;
    p.n_tiles = (p.N + bn - 1) / bn;
    if (bn == 128) {
        p.stages = MxGeom<FMT, 128, true, kMxGrouped>::kStages;
        return launch_t<FMT, 128, true, __half, kMxGrouped>(p, row_tiles * p.n_tiles, st);
    }
    p.stages = MxGeom<FMT, 64, true, kMxGrouped>::kStages;
    return launch_t<FMT, 64, true, __half, kMxGrouped>(p, row_tiles * p.n_tiles, st);
}

qmm_status make_unit_map(CUtensorMap* map, const void* packed, int64_t rows128, int box_rows);

template <int FMT, typename T> static qmm_status launch_pair_t(MxGemmParams p, int tiles, cudaStream_t st)
{
    p.vec = row_vec<T>(p.y, p.ldy);
    p.stages = MxPairGeom<FMT>::stages(p.vec < 16);
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

// Whether 256 x 256 tiles on pairs of SMs beat 128 x 128 tiles on single ones: estimated ns of each, rounds of tiles times (k units, with the
// hand-over; at least the time to store a tile) and a constant.  Measured (us, pairs / singles): 2048 x 8192 x 8192 49 / 58, x 2048 17.7 / 19.7,
// x 768 13.5 / 12.8; 1024 x 2048 x 8192 15.2 / 11.9; 2048 x 2048 x 8192 17.0 / 19.6, x 2048 9.2 / 8.1.
static bool pairs_pay(const MxGemmParams& p, int64_t pair_tiles)
{
    if (g_knobs.mx_pair) return g_knobs.mx_pair == 1;
    auto most = [](int64_t a, int64_t b) { return a > b ? a : b; };
    const int64_t singles = (int64_t)p.n_tiles * ((p.M + 127) / 128);
    const int64_t rounds2 = (pair_tiles + kNumSMs / 2 - 1) / (kNumSMs / 2), rounds1 = (singles + kNumSMs - 1) / kNumSMs;
    return 4600 + rounds2 * most(1900, 300 * p.KU + 1100) < 2000 + rounds1 * most(1250, 240 * p.KU + 600);
}

template <int FMT, typename T> static qmm_status dense_t(MxGemmParams p, cudaStream_t st)
{
    const int pair_tiles = ((p.n_tiles + 1) / 2) * ((p.M + 255) / 256);
    // (the pair form's row coordinates are 32-bit: operands below 2^31 rows of 128 bytes)
    const bool fits = ((int64_t)p.n_tiles + (p.M + 127) / 128) * p.KU * (unit_bytes(FMT) / 128) < (1LL << 31);
    if (p.M > 128 && pairs_pay(p, pair_tiles) && fits) return launch_pair_t<FMT, T>(p, pair_tiles, st);
    return launch_tiles<FMT, T, kMxDense>(p, (p.M + 127) / 128, st);
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

// Whether the product of a few rows takes them as they come (else they are quantised by a launch of their own).  Every block quantises all of them:
// up to 16 rows of 2048 that costs 1.4 us and saves a launch (one token, 2048 x 2048: 8.8 -> 4.1 us), 8 rows of 8192 would cost 3 to 5 us (where
// blocks share K, each takes its part only).  They may take 112 KB, half of the shared memory.
bool mx_few_fits(int fmt, int64_t M, int64_t N, int64_t K)
{
    const int KU = (int)k_units(K), splits = mx_splits(M, N, KU);
    return M <= 16 && M * K <= 32768 * splits && few_resident(fmt, M, (KU + splits - 1) / splits) <= 112 * 1024 && !g_knobs.mx_no_few;
}

template <int FMT, typename T> static qmm_status few_t(MxGemmParams p, cudaStream_t st)
{
    const int x_vec = row_vec<T>(p.x, p.M > 1 ? p.ldx : 0);
    p.x_vec = x_vec < 16 ? 0 : x_vec;
    p.atoms = (p.M + 7) / 8;
    return launch_tiles<FMT, T, kMxFew>(p, 1, st);
}

qmm_status launch_mx_few(int fmt, int dtype, const void* x, int64_t ldx, int64_t M, const void* w, int64_t N, int64_t K, const float* x_scale,
                         const float* w_scale, void* y, int64_t ldy, int* status, cudaStream_t st)
{
    MxGemmParams p = {};
    p.x = x;
    p.ldx = ldx;
    p.K = K;
    p.w[0] = (const uint8_t*)w;
    p.M = (int)M;
    p.N = (int)N;
    p.KU = (int)k_units(K);
    p.n_tiles = (int)((N + 127) / 128);
    p.a_scale = x_scale;
    p.w_scale[0] = w_scale;
    p.y = y;
    p.ldy = ldy;
    p.status = status;
    if (fmt == QMM_MXFP4)
        return dtype == QMM_F16 ? few_t<QMM_MXFP4, __half>(p, st) : dtype == QMM_BF16 ? few_t<QMM_MXFP4, __nv_bfloat16>(p, st) : few_t<QMM_MXFP4, float>(p, st);
    return dtype == QMM_F16 ? few_t<QMM_NVFP4, __half>(p, st) : dtype == QMM_BF16 ? few_t<QMM_NVFP4, __nv_bfloat16>(p, st) : few_t<QMM_NVFP4, float>(p, st);
}

// Most row units that P pairs over E experts can take.
int64_t mx_max_row_units(int64_t pairs, int E)
{
    const int64_t used = pairs < E ? pairs : E;
    return (pairs - used) / 128 + used;
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
    const int64_t row_tiles = mx_max_row_units(pairs, E);
    if (fmt == QMM_MXFP4) return launch_gate_up<QMM_MXFP4>(p, pairs, row_tiles, st);
    return launch_gate_up<QMM_NVFP4>(p, pairs, row_tiles, st);
}

template <int FMT, typename T> static qmm_status grouped_t(MxGemmParams p, int64_t row_tiles, cudaStream_t st)
{
    return launch_tiles<FMT, T, kMxGrouped>(p, row_tiles, st);
}

qmm_status launch_mx_experts_gemm(int fmt, const void* a, int64_t pairs, int E, const int* offsets, const int* units, const void* w, int64_t N,
                                  int64_t K, const float* a_scale, const float* w_scale, int dtype, void* y, int64_t ldy, bool list_ready, int* status,
                                  cudaStream_t st)
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
    p.list_ready = list_ready;
    p.a_scale = a_scale;
    p.w_scale[0] = w_scale;
    p.y = y;
    p.ldy = ldy;
    p.status = status;
    const int64_t row_tiles = mx_max_row_units(pairs, E);
    if (fmt == QMM_MXFP4)
        return dtype == QMM_F16 ? grouped_t<QMM_MXFP4, __half>(p, row_tiles, st) : dtype == QMM_BF16 ? grouped_t<QMM_MXFP4, __nv_bfloat16>(p, row_tiles, st) : grouped_t<QMM_MXFP4, float>(p, row_tiles, st);
    return dtype == QMM_F16 ? grouped_t<QMM_NVFP4, __half>(p, row_tiles, st) : dtype == QMM_BF16 ? grouped_t<QMM_NVFP4, __nv_bfloat16>(p, row_tiles, st) : grouped_t<QMM_NVFP4, float>(p, row_tiles, st);
}

}  // namespace qmm
