// qmm_layer_api.cu -- C ABI of what stands around the products in a layer: the router, the norm with 8-bit rows, and the low-rank adapters.
// The rules of the other entry points: everything is checked on the host before anything is enqueued, nothing allocates, errors go
// through the thread-local buffer.
#include "qmm_checks.cuh"
#include "qmm_lora.cuh"

#include <math.h>

namespace qmm {

qmm_status launch_expert_route(int dtype, const void* logits, int64_t ld, int T, int E, int topk, int sigmoid, const float* bias, int groups, int top_groups,
                               int group_top, int renorm, float scale, int* idx, float* w, cudaStream_t st);
qmm_status launch_expert_route_grad(int dtype, const float* dw, const void* logits, int64_t ld, const int* idx, int T, int E, int topk, int sigmoid, int renorm,
                                    float scale, void* dlogits, int64_t ldo, cudaStream_t st);
qmm_status launch_rms_norm(int dtype, const void* x, int64_t ldx, const void* res, int64_t ldr, const void* w, float eps, int64_t rows, int K, void* h, int64_t ldh,
                           void* y, int64_t ldy, int row8, void* codes, int64_t ldc, float* scales, int norm, cudaStream_t st);
size_t rms_norm_grad_workspace_bytes(int64_t rows, int K);
qmm_status launch_rms_norm_grad(int dtype, const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* w, float eps, int64_t rows, int K, const void* dh,
                                int64_t lddh, void* dx, int64_t lddx, float* dw, void* ws, cudaStream_t st);
qmm_status launch_rows8_dequantize(int row8, const void* codes, int64_t ldc, const float* scales, int64_t rows, int K, int dtype, void* out, int64_t ldo, cudaStream_t st);

qmm_status launch_lora_f16(const lora::LoraP& p, int r, bool x8, bool back, bool vx, bool vy, cudaStream_t st);
qmm_status launch_lora_bf16(const lora::LoraP& p, int r, bool x8, bool back, bool vx, bool vy, cudaStream_t st);
qmm_status launch_lora_wgrad_f16(const lora::WgradP& b, const lora::WgradP& a, int r, bool vb, bool va, cudaStream_t st);
qmm_status launch_lora_wgrad_f16_rows8(const lora::WgradP& b, const lora::WgradP& a, int r, bool vb, bool va, cudaStream_t st);
qmm_status launch_lora_wgrad_bf16(const lora::WgradP& b, const lora::WgradP& a, int r, bool vb, bool va, cudaStream_t st);
qmm_status launch_lora_wgrad_bf16_rows8(const lora::WgradP& b, const lora::WgradP& a, int r, bool vb, bool va, cudaStream_t st);
qmm_status launch_lora_join(int r, const int* units, int n, const lora::WgradParts& g0, const lora::WgradParts& g1, cudaStream_t st);
size_t expert_sort_workspace_bytes(int64_t P, int E);
qmm_status launch_expert_sort(const int* idx, int64_t P, int E, int* order, int* place, int* offsets, int* units, void* ws, cudaStream_t st);

static qmm_status check_route(const char* who, int32_t T, int32_t topk, int32_t E, int scores, float scale)
{
    QMM_TRY(check_pairs(who, T, topk, E));
    if (topk > E) return fail(QMM_ERR_INVALID_ARG, "%s: topk=%d of E=%d experts", who, topk, E);
    if (scores != QMM_SOFTMAX && scores != QMM_SIGMOID) return fail(QMM_ERR_INVALID_ARG, "%s: unknown scores %d (expected 0 or 1)", who, scores);
    if (!isfinite(scale)) return fail(QMM_ERR_INVALID_ARG, "%s: scale is not finite", who);
    return QMM_OK;
}

constexpr int64_t kMaxNormK = 32768;

static qmm_status check_norm(const char* who, int64_t rows, int64_t K, int dtype)
{
    if (!dtype_ok(dtype)) return fail(QMM_ERR_INVALID_ARG, "%s: unknown data type %d (expected 0, 1 or 2)", who, dtype);
    if (rows < 0 || K <= 0) return fail(QMM_ERR_INVALID_ARG, "%s: rows=%lld is negative or K=%lld not positive", who, (long long)rows, (long long)K);
    if (rows > (1 << 24) || K > kMaxNormK) return fail(QMM_ERR_UNSUPPORTED, "%s: %lld rows > 2^24 or K=%lld > %lld", who, (long long)rows, (long long)K, (long long)kMaxNormK);
    return QMM_OK;
}
static qmm_status check_eps(const char* who, float eps)
{
    return eps > 0.0f && isfinite(eps) ? QMM_OK : fail(QMM_ERR_INVALID_ARG, "%s: eps must be positive and finite", who);
}
static qmm_status check_weight(const char* who, int dtype, const void* w)
{
    return aligned(w, (size_t)dtype_size(dtype)) ? QMM_OK : fail(QMM_ERR_ALIGNMENT, "%s: weight is not aligned to its element type", who);
}
static qmm_status check_rows8(const char* who, int fmt, const void* codes, int64_t ldc, const float* scales, int64_t K)
{
    if (fmt != QMM_ROW_E4M3 && fmt != QMM_ROW_INT8) return fail(QMM_ERR_INVALID_ARG, "%s: unknown 8-bit format %d (expected 0 or 1)", who, fmt);
    if (!codes || !scales) return fail(QMM_ERR_INVALID_ARG, "%s: codes or scales is null", who);
    if (ldc < K) return fail(QMM_ERR_SHAPE, "%s: row pitch %lld of codes is below its width %lld", who, (long long)ldc, (long long)K);
    if (ldc > (1LL << 40)) return fail(QMM_ERR_UNSUPPORTED, "%s: row pitch %lld of codes > 2^40", who, (long long)ldc);
    if (!aligned(scales, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: scales must be 4-byte aligned", who);
    return QMM_OK;
}

// Workspace of the adapters: a plan of the rows by adapter, where the caller brings none, and s or ds.
struct LoraLayout {
    size_t order, place, offsets, units, sort, s, part, total;
};
static LoraLayout lora_layout(int64_t T, int n, int r)
{
    auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    LoraLayout l;
    l.order = 0;
    l.place = up(l.order + (size_t)T * 4);
    l.offsets = up(l.place + (size_t)T * 4);
    l.units = up(l.offsets + (size_t)(n + 1) * 4);
    l.sort = up(l.units + (size_t)(n + 1) * 4);
    l.s = up(l.sort + expert_sort_workspace_bytes(T, n));
    l.part = up(l.s + (size_t)T * r * 4);
    l.total = l.part + (T > lora::kSmallRows ? (size_t)lora::wgrad_blocks(r) * 2 * 128 * r * 4 : 0);         // sums of adapters that two blocks of a weight gradient share
    return l;
}

static qmm_status check_lora_sizes(const char* who, int32_t T, int32_t n, int32_t r)
{
    QMM_TRY(check_pairs(who, T, 1, n));
    if (r != 8 && r != 16 && r != 32 && r != 64 && r != 128) return fail(QMM_ERR_UNSUPPORTED, "%s: rank r=%d (8, 16, 32, 64 or 128; pad with zeros)", who, r);
    return QMM_OK;
}

// What forward and backward have in common.
static qmm_status check_lora(const char* who, const qmm_lora_args* a)
{
    if (!a) return fail(QMM_ERR_INVALID_ARG, "%s: args is null", who);
    QMM_TRY(check_lora_sizes(who, a->T, a->n, a->r));
    if (a->dtype != QMM_F16 && a->dtype != QMM_BF16) return fail(QMM_ERR_INVALID_ARG, "%s: data type %d (expected 0 or 1)", who, a->dtype);
    if (a->K <= 0 || a->N <= 0) return fail(QMM_ERR_INVALID_ARG, "%s: K=%lld and N=%lld must be positive", who, (long long)a->K, (long long)a->N);
    if (a->K > (1 << 20) || a->N > (1 << 20)) return fail(QMM_ERR_UNSUPPORTED, "%s: K=%lld or N=%lld > 2^20", who, (long long)a->K, (long long)a->N);
    if (a->T == 0) return QMM_OK;
    if (!a->idx || !a->A || !a->B) return fail(QMM_ERR_INVALID_ARG, "%s: idx, A or B is null", who);
    if (!aligned(a->idx, 4) || !aligned(a->scale, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: idx and scale must be 4-byte aligned", who);
    if (!aligned(a->A, 2) || !aligned(a->B, 2)) return fail(QMM_ERR_ALIGNMENT, "%s: A and B must be aligned to their element type", who);
    if ((!a->order) != (!a->offsets) || (!a->order) != (!a->units)) return fail(QMM_ERR_INVALID_ARG, "%s: order, offsets and units come together", who);
    if (!aligned(a->order, 4) || !aligned(a->offsets, 4) || !aligned(a->units, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: index arrays must be 4-byte aligned", who);
    if (!aligned(a->S, 16)) return fail(QMM_ERR_ALIGNMENT, "%s: S must be 16-byte aligned", who);
    return QMM_OK;
}
static qmm_status check_lora_x(const char* who, const qmm_lora_args* a)
{
    if (a->x_scale) return check_rows8(who, a->x_format, a->X, a->ldx, a->x_scale, a->K);
    return check_rows(who, "X", a->dtype, a->X, a->ldx, a->K);
}

static uintptr_t pitch_bits(const void* p, int64_t ld, int size) { return p ? reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size) : 0; }

// Lowest bits of the addresses and row pitches of the first product's rows and weights, of the second's (y0), and of its outputs with their width.
struct LoraBits {
    uintptr_t x, w1, y0, w2, y;
    bool vx() const { return (x | w1) % 16 == 0; }
    bool vy() const { return (y0 | w2 | y) % 16 == 0; }
    int words() const { return (x % 4 == 0) | (w1 % 4 == 0) << 1 | (y0 % 4 == 0) << 2 | (w2 % 4 == 0) << 3; }
};

// The rows by adapter: the caller's plan, or one made in the workspace.
static qmm_status lora_plan(const qmm_lora_args* a, const LoraLayout& l, char* ws, const int** order, const int** offsets, const int** units, cudaStream_t st)
{
    if (a->order) {
        *order = a->order, *offsets = a->offsets, *units = a->units;
        return QMM_OK;
    }
    *order = (int*)(ws + l.order), *offsets = (int*)(ws + l.offsets), *units = (int*)(ws + l.units);
    return launch_expert_sort(a->idx, a->T, a->n, (int*)(ws + l.order), (int*)(ws + l.place), (int*)(ws + l.offsets), (int*)(ws + l.units), ws + l.sort, st);
}

}  // namespace qmm

using namespace qmm;

extern "C" {

qmm_status qmm_expert_route(qmm_dtype dtype, const void* logits, int64_t ld, int32_t T, int32_t E, int32_t topk, qmm_scores scores, const float* bias, int32_t groups,
                            int32_t top_groups, int32_t group_top, int32_t renormalize, float scale, int32_t* idx, float* weights, void* stream)
{
    const char* who = "qmm_expert_route";
    QMM_TRY(check_route(who, T, topk, E, scores, scale));
    if (groups < 1 || groups > 32 || E % groups) return fail(QMM_ERR_INVALID_ARG, "%s: %d groups of E=%d experts (1 to 32 that divide E)", who, groups, E);
    if (top_groups < 1 || top_groups > groups) return fail(QMM_ERR_INVALID_ARG, "%s: top_groups=%d of %d groups", who, top_groups, groups);
    if (group_top != 1 && group_top != 2) return fail(QMM_ERR_INVALID_ARG, "%s: group_top=%d (expected 1 or 2)", who, group_top);
    if (T == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "logits", dtype, logits, ld, E));
    if (!idx || !weights) return fail(QMM_ERR_INVALID_ARG, "%s: idx or weights is null", who);
    if (!aligned(idx, 4) || !aligned(weights, 4) || !aligned(bias, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: idx, weights and bias must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_expert_route(dtype, logits, ld, T, E, topk, scores == QMM_SIGMOID, bias, groups, top_groups, group_top, renormalize != 0, scale, idx, weights,
                               (cudaStream_t)stream);
}

qmm_status qmm_expert_route_grad(qmm_dtype dtype, const float* dweights, const void* logits, int64_t ld, const int32_t* idx, int32_t T, int32_t E, int32_t topk,
                                 qmm_scores scores, int32_t renormalize, float scale, void* dlogits, int64_t ldd, void* stream)
{
    const char* who = "qmm_expert_route_grad";
    QMM_TRY(check_route(who, T, topk, E, scores, scale));
    if (T == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "logits", dtype, logits, ld, E));
    QMM_TRY(check_rows(who, "dlogits", dtype, dlogits, ldd, E));
    if (!idx || !dweights) return fail(QMM_ERR_INVALID_ARG, "%s: idx or dweights is null", who);
    if (!aligned(idx, 4) || !aligned(dweights, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: idx and dweights must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_expert_route_grad(dtype, dweights, logits, ld, idx, T, E, topk, scores == QMM_SIGMOID, renormalize != 0, scale, dlogits, ldd, (cudaStream_t)stream);
}

qmm_status qmm_rms_norm(qmm_dtype dtype, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight, float eps, int64_t rows, int64_t K,
                        void* h, int64_t ldh, void* y, int64_t ldy, qmm_row_format fmt, void* codes, int64_t ldc, float* scales, void* stream)
{
    const char* who = "qmm_rms_norm";
    QMM_TRY(check_norm(who, rows, K, dtype));
    QMM_TRY(check_eps(who, eps));
    if (rows == 0) return QMM_OK;
    if (!y && !codes) return fail(QMM_ERR_INVALID_ARG, "%s: neither y nor codes is given", who);
    QMM_TRY(check_rows(who, "x", dtype, x, ldx, K));
    if (residual) QMM_TRY(check_rows(who, "residual", dtype, residual, ldr, K));
    if (h) QMM_TRY(check_rows(who, "h", dtype, h, ldh, K));
    if (y) QMM_TRY(check_rows(who, "y", dtype, y, ldy, K));
    if (codes) QMM_TRY(check_rows8(who, fmt, codes, ldc, scales, K));
    QMM_TRY(check_weight(who, dtype, weight));
    QMM_TRY(check_device(who));
    return launch_rms_norm(dtype, x, ldx, residual, ldr, weight, eps, rows, (int)K, h, ldh, y, ldy, fmt == QMM_ROW_INT8, codes, ldc, scales, 1, (cudaStream_t)stream);
}

size_t qmm_rms_norm_grad_workspace_bytes(int64_t rows, int64_t K)
{
    if (check_norm("qmm_rms_norm_grad_workspace_bytes", rows, K, QMM_F32) != QMM_OK) return 0;
    return rms_norm_grad_workspace_bytes(rows, (int)K);
}

qmm_status qmm_rms_norm_grad(qmm_dtype dtype, const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* weight, float eps, int64_t rows, int64_t K,
                             const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dweight, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "qmm_rms_norm_grad";
    QMM_TRY(check_norm(who, rows, K, dtype));
    QMM_TRY(check_eps(who, eps));
    if (!dx && !dweight) return fail(QMM_ERR_INVALID_ARG, "%s: neither dx nor dweight is wanted", who);
    if (!aligned(dweight, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: dweight must be 4-byte aligned", who);
    if (rows > 0) {
        QMM_TRY(check_rows(who, "dy", dtype, dy, lddy, K));
        QMM_TRY(check_rows(who, "h", dtype, h, ldh, K));
        if (dh) QMM_TRY(check_rows(who, "dh", dtype, dh, lddh, K));
        if (dx) QMM_TRY(check_rows(who, "dx", dtype, dx, lddx, K));
        QMM_TRY(check_weight(who, dtype, weight));
        if (dweight) QMM_TRY(check_ws(who, ws, ws_bytes, rms_norm_grad_workspace_bytes(rows, (int)K), 16));
    } else if (!dweight) {
        return QMM_OK;
    }
    QMM_TRY(check_device(who));
    if (rows == 0) return check_cuda(cudaMemsetAsync(dweight, 0, (size_t)K * 4, (cudaStream_t)stream), who);
    return launch_rms_norm_grad(dtype, dy, lddy, h, ldh, weight, eps, rows, (int)K, dh, lddh, dx, lddx, dweight, ws, (cudaStream_t)stream);
}

qmm_status qmm_rows_quantize(qmm_dtype dtype, const void* x, int64_t ldx, int64_t rows, int64_t K, qmm_row_format fmt, void* codes, int64_t ldc, float* scales,
                              void* stream)
{
    const char* who = "qmm_rows_quantize";
    QMM_TRY(check_norm(who, rows, K, dtype));
    if (rows == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "x", dtype, x, ldx, K));
    QMM_TRY(check_rows8(who, fmt, codes, ldc, scales, K));
    QMM_TRY(check_device(who));
    return launch_rms_norm(dtype, x, ldx, nullptr, 0, nullptr, 1.0f, rows, (int)K, nullptr, 0, nullptr, 0, fmt == QMM_ROW_INT8, codes, ldc, scales, 0,
                           (cudaStream_t)stream);
}

qmm_status qmm_rows_dequantize(qmm_row_format fmt, const void* codes, int64_t ldc, const float* scales, int64_t rows, int64_t K, qmm_dtype dtype, void* out, int64_t ldo,
                                void* stream)
{
    const char* who = "qmm_rows_dequantize";
    QMM_TRY(check_norm(who, rows, K, dtype));
    if (rows == 0) return QMM_OK;
    QMM_TRY(check_rows8(who, fmt, codes, ldc, scales, K));
    QMM_TRY(check_rows(who, "out", dtype, out, ldo, K));
    QMM_TRY(check_device(who));
    return launch_rows8_dequantize(fmt == QMM_ROW_INT8, codes, ldc, scales, rows, (int)K, dtype, out, ldo, (cudaStream_t)stream);
}

size_t qmm_lora_workspace_bytes(int32_t T, int32_t n, int32_t r)
{
    if (check_lora_sizes("qmm_lora_workspace_bytes", T, n, r) != QMM_OK) return 0;
    return lora_layout(T, n, r).total;
}

qmm_status qmm_lora(const qmm_lora_args* a, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "qmm_lora";
    QMM_TRY(check_lora(who, a));
    if (a->T == 0) return QMM_OK;
    QMM_TRY(check_lora_x(who, a));
    if (a->Y0) QMM_TRY(check_rows(who, "Y0", a->dtype, a->Y0, a->ldy0, a->N));
    QMM_TRY(check_rows(who, "Y", a->dtype, a->Y, a->ldy, a->N));
    const LoraLayout l = lora_layout(a->T, a->n, a->r);
    const bool small = a->T <= lora::kSmallRows;
    if (!small && (!a->S || !a->order)) QMM_TRY(check_ws(who, ws, ws_bytes, l.total, 256));
    QMM_TRY(check_device(who));
    const cudaStream_t st = (cudaStream_t)stream;
    const int *order = nullptr, *offsets = nullptr, *units = nullptr;
    if (!small) QMM_TRY(lora_plan(a, l, (char*)ws, &order, &offsets, &units, st));
    const bool x8 = a->x_scale != nullptr, same = a->Y0 == a->Y && a->ldy0 == a->ldy;
    const LoraBits b = {pitch_bits(a->X, a->ldx, x8 ? 1 : 2), pitch_bits(a->A, a->K, 2), pitch_bits(a->Y0, a->ldy0, 2), pitch_bits(a->B, a->r, 2),
                        pitch_bits(a->Y, a->ldy, 2) | (uintptr_t)(a->N * 2)};
    const lora::LoraP p = {a->X, a->ldx, a->x_scale, a->x_format == QMM_ROW_INT8, a->idx, order, offsets, units, a->T, a->n, (int)a->K, (int)a->N, a->A, a->B, a->scale,
                           a->Y0, a->ldy0, a->Y, a->ldy, a->S ? a->S : small ? nullptr : (float*)((char*)ws + l.s), 0, !same, b.words()};
    return a->dtype == QMM_F16 ? launch_lora_f16(p, a->r, x8, false, b.vx(), b.vy(), st) : launch_lora_bf16(p, a->r, x8, false, b.vx(), b.vy(), st);
}

qmm_status qmm_lora_grad(const qmm_lora_args* a, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "qmm_lora_grad";
    QMM_TRY(check_lora(who, a));
    if (!a->dX && !a->dA && !a->dB) return fail(QMM_ERR_INVALID_ARG, "%s: none of dX, dA and dB is wanted", who);
    if (!aligned(a->dA, 16) || !aligned(a->dB, 16)) return fail(QMM_ERR_ALIGNMENT, "%s: dA and dB must be 16-byte aligned", who);
    const LoraLayout l = lora_layout(a->T, a->n, a->r);
    if (a->T > 0) {
        QMM_TRY(check_rows(who, "dY", a->dtype, a->dY, a->lddy, a->N));
        if (a->dA) QMM_TRY(check_lora_x(who, a));
        if (a->dB && !a->S) return fail(QMM_ERR_INVALID_ARG, "%s: dB needs S of the forward pass", who);
        if (a->dX) QMM_TRY(check_rows(who, "dX", a->dtype, a->dX, a->lddx, a->K));
        if (a->dX && a->dX0) QMM_TRY(check_rows(who, "dX0", a->dtype, a->dX0, a->lddx0, a->K));
        QMM_TRY(check_ws(who, ws, ws_bytes, l.total, 256));
    }
    QMM_TRY(check_device(who));
    const cudaStream_t st = (cudaStream_t)stream;
    if (a->T == 0) {
        const size_t n = (size_t)a->n * a->r * 4;
        if (a->dA) QMM_TRY(check_cuda(cudaMemsetAsync(a->dA, 0, n * (size_t)a->K, st), who));
        if (a->dB) QMM_TRY(check_cuda(cudaMemsetAsync(a->dB, 0, n * (size_t)a->N, st), who));
        return QMM_OK;
    }
    const int *order = nullptr, *offsets = nullptr, *units = nullptr;
    const bool small = a->T <= lora::kSmallRows, half = a->dtype == QMM_F16;
    if (!small || a->dA || a->dB) QMM_TRY(lora_plan(a, l, (char*)ws, &order, &offsets, &units, st));
    float* ds = (float*)((char*)ws + l.s);
    if (a->dX || a->dA) {
        const bool same = a->dX0 == a->dX && a->lddx0 == a->lddx;
        const LoraBits b = {pitch_bits(a->dY, a->lddy, 2), pitch_bits(a->B, a->r, 2), pitch_bits(a->dX0, a->lddx0, 2), pitch_bits(a->A, a->K, 2),
                            pitch_bits(a->dX, a->lddx, 2) | (uintptr_t)(a->K * 2)};
        const bool vx = b.vx() && a->N % 8 == 0;
        const lora::LoraP p = {a->dY, a->lddy, nullptr, 0, a->idx, order, offsets, units, a->T, a->n, (int)a->N, (int)a->K, a->B, a->A, a->scale, a->dX0, a->lddx0,
                               a->dX, a->lddx, ds, 1, a->dX && !same, b.words()};
        QMM_TRY(half ? launch_lora_f16(p, a->r, false, true, vx, b.vy(), st) : launch_lora_bf16(p, a->r, false, true, vx, b.vy(), st));
    }
    const int blocks = lora::wgrad_blocks(a->r);
    const int of_b = a->dB ? lora::wgrad_share(blocks, a->T, a->N, half, a->dA ? a->K : 0, half && !a->x_scale) : 0;
    const int of_a = a->dA ? lora::wgrad_share(blocks - of_b, a->T, a->K, half && !a->x_scale, 0, false) : 0;
    float* const part_b = small ? nullptr : (float*)((char*)ws + l.part);
    float* const part_a = small ? nullptr : part_b + (size_t)of_b * 2 * 128 * a->r;
    if (!a->dA && !a->dB) return QMM_OK;
    const bool x8 = a->dA && a->x_scale;
    const uintptr_t bits_b = a->dB ? pitch_bits(a->dY, a->lddy, 2) : 0, bits_a = a->dA ? pitch_bits(a->X, a->ldx, x8 ? 1 : 2) : 0;
    const lora::WgradP pb = {a->dY, a->lddy, nullptr, 0, a->S, a->scale, order, offsets, units, a->T, a->n, (int)a->N, a->dB, part_b, of_b, bits_b % 4 == 0};
    const lora::WgradP pa = {a->X, a->ldx, a->x_scale, a->x_format == QMM_ROW_INT8, ds, nullptr, order, offsets, units, a->T, a->n, (int)a->K, a->dA, part_a, of_a, bits_a % 4 == 0};
    const bool vb = !a->dB || (bits_b | (uintptr_t)(a->N * 2)) % 16 == 0, va = !a->dA || (bits_a | (uintptr_t)(a->K * 2)) % 16 == 0;
    if (half) QMM_TRY(x8 ? launch_lora_wgrad_f16_rows8(pb, pa, a->r, vb, va, st) : launch_lora_wgrad_f16(pb, pa, a->r, vb, va, st));
    else QMM_TRY(x8 ? launch_lora_wgrad_bf16_rows8(pb, pa, a->r, vb, va, st) : launch_lora_wgrad_bf16(pb, pa, a->r, vb, va, st));
    if (small) return QMM_OK;
    const lora::WgradParts gb = {part_b, a->dB, (int)a->N, of_b, 1}, ga = {part_a, a->dA, (int)a->K, of_a, 0};
    return launch_lora_join(a->r, units, a->n, of_b ? gb : ga, of_b ? ga : gb, st);
}

}  // extern "C"
