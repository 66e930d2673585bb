// qmm_mx_api.cu -- C ABI of the microscaled 4-bit operators and of the expert sort: argument checks and dispatch.
// The same rules as in qmm_api.cu: everything is checked on the host before anything is enqueued, nothing
// allocates, errors go through the thread-local buffer.
#include "qmm_mx.cuh"

namespace qmm {

using namespace mx;

qmm_status launch_mx_pack(int fmt, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t K, void* packed, cudaStream_t st);
qmm_status launch_mx_quantize(int fmt, int dtype, const void* x, int64_t ldx, int64_t rows, int64_t K, const float* ts, void* packed, bool early,
                              cudaStream_t st);
qmm_status launch_mx_quantize_experts(int fmt, int dtype, const void* x, int64_t ldx, int T, int topk, int E, int64_t K, const int* idx, const int* place,
                                      const int* offsets, const int* units, const float* ts, void* packed, bool early, cudaStream_t st);
qmm_status launch_mx_dequantize(int fmt, int dtype, const void* packed, int64_t rows, int64_t K, const float* ts, void* out, int64_t ldo, cudaStream_t st);
qmm_status launch_mx_gemm(int fmt, const void* a, int64_t M, const void* w, int64_t N, int64_t K, const float* a_scale, const float* w_scale, int dtype, void* y,
                          int64_t ldy, int* status, cudaStream_t st);
bool mx_few_fits(int fmt, int64_t M, int64_t N, int64_t K);
size_t mx_gemm_partial_bytes(int64_t M, int64_t N, int64_t K);
size_t mx_gemm_partial_bytes_up_to(int64_t M, int64_t N, int64_t K);
qmm_status launch_mx_few(int fmt, int dtype, const void* x, int64_t ldx, int64_t M, const void* w, int64_t N, int64_t K, const float* x_scale,
                         const float* w_scale, void* y, int64_t ldy, int* status, cudaStream_t st);
int64_t mx_max_row_units(int64_t pairs, int E);
qmm_status launch_mx_experts_gate_up(int fmt, const void* a, int64_t pairs, int E, const int* offsets, const int* units, const void* w_gate, const void* w_up,
                                     int64_t N, int64_t K, const float* a_scale, const float* gate_scale, const float* up_scale, const float* h_scale, void* h,
                                     int* status, cudaStream_t st);
qmm_status launch_mx_experts_gemm(int fmt, const void* a, int64_t pairs, int E, const int* offsets, const int* units, const void* w, int64_t N, int64_t K,
                                  const float* a_scale, const float* w_scale, int dtype, void* y, int64_t ldy, bool list_ready, int* status, cudaStream_t st);
size_t expert_sort_workspace_bytes(int64_t P, int E);
qmm_status launch_expert_sort(const int* idx, int64_t P, int E, int* order, int* place, int* offsets, int* units, void* ws, cudaStream_t st);
bool expert_sort_quantize_fits(int64_t P, int topk, int64_t K);
qmm_status launch_expert_sort_quantize(int fmt, int dtype, const int* idx, int64_t P, int topk, int E, int* order, int* place, int* offsets, int* units,
                                       const void* x, int64_t ldx, int64_t K, const float* ts, void* packed, cudaStream_t st);
qmm_status launch_expert_gather(int dtype, const void* x, int64_t ldx, int T, int topk, int64_t H, const int* order, const int* place, const float* weights,
                                void* xs, int64_t ldxs, cudaStream_t st);
qmm_status launch_expert_combine(int rows_dtype, int dtype, const void* ys, int64_t ldys, int T, int topk, int64_t H, const int* place, const float* weights, void* y,
                                 int64_t ldy, cudaStream_t st);
qmm_status launch_expert_combine_grad(int dtype, const void* dy, int64_t lddy, const void* ys, int64_t ldys, int T, int topk, int64_t H, const int* order,
                                      const int* place, const float* weights, void* dys, int64_t lddys, float* dw, cudaStream_t st);

constexpr size_t kMxStatusBytes = 256;

static bool mx_fmt_ok(int fmt) { return fmt == QMM_MXFP4 || fmt == QMM_NVFP4; }
static bool dtype_ok(int dt) { return dt == QMM_F16 || dt == QMM_BF16 || dt == QMM_F32; }
static int dtype_size(int dt) { return dt == QMM_F32 ? 4 : 2; }

static qmm_status check_mx(const char* who, int fmt, int64_t rows, int64_t K)
{
    if (!mx_fmt_ok(fmt)) return fail(QMM_ERR_INVALID_ARG, "%s: unknown microscaled format %d (expected 32 or 16)", who, fmt);
    if (rows < 0 || K <= 0) return fail(QMM_ERR_INVALID_ARG, "%s: rows=%lld is negative or K=%lld not positive", who, (long long)rows, (long long)K);
    if (rows > (1 << 24) || K > (1 << 20)) return fail(QMM_ERR_UNSUPPORTED, "%s: %lld rows > 2^24 or K=%lld > 2^20", who, (long long)rows, (long long)K);
    return QMM_OK;
}

// A matrix of plain elements: type, row pitch, element alignment.
static qmm_status check_rows(const char* who, const char* name, int dtype, const void* p, int64_t ld, int64_t width)
{
    if (!dtype_ok(dtype)) return fail(QMM_ERR_INVALID_ARG, "%s: unknown data type %d (expected 0, 1 or 2)", who, dtype);
    if (!p) return fail(QMM_ERR_INVALID_ARG, "%s: %s is null", who, name);
    if (ld < width) return fail(QMM_ERR_SHAPE, "%s: row pitch %lld of %s is below its width %lld", who, (long long)ld, name, (long long)width);
    if (ld > (1LL << 40)) return fail(QMM_ERR_UNSUPPORTED, "%s: row pitch %lld of %s > 2^40", who, (long long)ld, name);
    if (!aligned(p, (size_t)dtype_size(dtype))) return fail(QMM_ERR_ALIGNMENT, "%s: %s is not aligned to its element type", who, name);
    return QMM_OK;
}

static qmm_status check_packed(const char* who, const char* name, const void* p)
{
    if (!p) return fail(QMM_ERR_INVALID_ARG, "%s: %s is null", who, name);
    if (!aligned(p, 16)) return fail(QMM_ERR_ALIGNMENT, "%s: %s must be 16-byte aligned", who, name);
    return QMM_OK;
}

static qmm_status check_scale(const char* who, int fmt, const float* s)
{
    if (s && fmt == QMM_MXFP4) return fail(QMM_ERR_INVALID_ARG, "%s: MXFP4 takes no tensor scale", who);
    if (!aligned(s, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: a tensor scale must be 4-byte aligned", who);
    return QMM_OK;
}

static qmm_status check_ws(const char* who, const void* ws, size_t given, size_t need, size_t align)
{
    if (!ws || given < need) return fail(QMM_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws ? given : (size_t)0);
    if (!aligned(ws, align)) return fail(QMM_ERR_ALIGNMENT, "%s: workspace must be %zu-byte aligned", who, align);
    return QMM_OK;
}

static qmm_status check_pairs(const char* who, int32_t T, int32_t topk, int32_t E)
{
    if (T < 0 || topk <= 0 || E <= 0) return fail(QMM_ERR_INVALID_ARG, "%s: T=%d topk=%d E=%d out of range", who, T, topk, E);
    if (E > 1024 || topk > 32) return fail(QMM_ERR_UNSUPPORTED, "%s: E=%d > 1024 or topk=%d > 32", who, E, topk);
    if ((int64_t)T * topk > (1 << 22)) return fail(QMM_ERR_UNSUPPORTED, "%s: T*topk=%lld > 2^22", who, (long long)T * topk);
    return QMM_OK;
}

// Operands of a dense product: M rows against N >= 1 weight rows.
static qmm_status check_product(const char* who, int fmt, int64_t M, int64_t N, int64_t K)
{
    const qmm_status s = check_mx(who, fmt, M, K);
    if (s != QMM_OK) return s;
    if (N == 0) return fail(QMM_ERR_INVALID_ARG, "%s: N must be positive", who);
    return check_mx(who, fmt, N, K);
}

static size_t mx_bytes(int fmt, int64_t row_units, int64_t K) { return (size_t)row_units * (size_t)k_units(K) * (size_t)unit_bytes(fmt); }

#define QMM_TRY(call)                    \
    do {                                 \
        const qmm_status s_ = (call);    \
        if (s_ != QMM_OK) return s_;     \
    } while (0)

// Type of the experts' rows on their way to the weighted sum.  Rounding them to the output's 16 bits halves their traffic and adds half an ulp to each term of the
// sum; which one it is is the caller's choice (128 experts x 768 x 2048, 8 per token, fp16: 2048 tokens 121 us, 153 with fp32 rows; 4 tokens 31.1, 31.4).
static int rows_dtype(const qmm_mx_moe_args* a) { return a->rows_f32 ? QMM_F32 : a->dtype; }

// Workspace of qmm_mx_moe.
struct MxMoeLayout {
    size_t order, place, offsets, units, sort, sort_bytes, xq, h, d, total;
};
static MxMoeLayout mx_moe_layout(const qmm_mx_moe_args* a)
{
    MxMoeLayout l;
    const size_t P = (size_t)a->T * a->topk;
    const int64_t row_units = mx_max_row_units((int64_t)P, a->E);
    size_t o = kMxStatusBytes;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += (bytes + 255) / 256 * 256;
        return at;
    };
    l.order = take(P * 4);
    l.place = take(P * 4);
    l.offsets = take((size_t)(a->E + 1) * 4);
    l.units = take((size_t)(a->E + 1) * 4);
    l.sort_bytes = expert_sort_workspace_bytes((int64_t)P, a->E);
    l.sort = take(l.sort_bytes);
    l.xq = take(mx_bytes(a->fmt, row_units, a->H));
    l.h = take(mx_bytes(a->fmt, row_units, a->I));
    l.d = take(P * (size_t)a->H * dtype_size(rows_dtype(a)));
    l.total = o;
    return l;
}

static qmm_status check_mx_moe(const char* who, const qmm_mx_moe_args* a)
{
    if (!a) return fail(QMM_ERR_INVALID_ARG, "%s: null args", who);
    QMM_TRY(check_pairs(who, a->T, a->topk, a->E));
    QMM_TRY(check_mx(who, a->fmt, a->I, a->H));
    QMM_TRY(check_mx(who, a->fmt, a->H, a->I));
    if (!dtype_ok(a->dtype)) return fail(QMM_ERR_INVALID_ARG, "%s: unknown data type %d (expected 0, 1 or 2)", who, a->dtype);
    if (a->rows_f32 != 0 && a->rows_f32 != 1) return fail(QMM_ERR_INVALID_ARG, "%s: rows_f32=%d (expected 0 or 1)", who, a->rows_f32);
    return QMM_OK;
}

}  // namespace qmm

using namespace qmm;

extern "C" {

size_t qmm_mx_bytes(qmm_mx_format fmt, int64_t rows, int64_t K)
{
    if (check_mx("qmm_mx_bytes", fmt, rows, K) != QMM_OK) return 0;
    return mx_bytes(fmt, (rows + 127) / 128, K);
}

qmm_status qmm_mx_pack(qmm_mx_format fmt, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t K, void* packed, void* stream)
{
    QMM_TRY(check_mx("qmm_mx_pack", fmt, rows, K));
    if (rows == 0) return QMM_OK;
    if (!codes || !scales) return fail(QMM_ERR_INVALID_ARG, "qmm_mx_pack: null pointer");
    QMM_TRY(check_packed("qmm_mx_pack", "packed", packed));
    QMM_TRY(check_device("qmm_mx_pack"));
    return launch_mx_pack(fmt, codes, scales, rows, K, packed, (cudaStream_t)stream);
}

qmm_status qmm_mx_quantize(qmm_mx_format fmt, qmm_dtype dtype, const void* x, int64_t ldx, int64_t rows, int64_t K, const float* tensor_scale, void* packed,
                           void* stream)
{
    QMM_TRY(check_mx("qmm_mx_quantize", fmt, rows, K));
    QMM_TRY(check_scale("qmm_mx_quantize", fmt, tensor_scale));
    if (rows == 0) return QMM_OK;
    QMM_TRY(check_rows("qmm_mx_quantize", "x", dtype, x, ldx, K));
    QMM_TRY(check_packed("qmm_mx_quantize", "packed", packed));
    QMM_TRY(check_device("qmm_mx_quantize"));
    return launch_mx_quantize(fmt, dtype, x, ldx, rows, K, tensor_scale, packed, false, (cudaStream_t)stream);
}

qmm_status qmm_mx_dequantize(qmm_mx_format fmt, const void* packed, int64_t rows, int64_t K, const float* tensor_scale, qmm_dtype dtype, void* out, int64_t ldo,
                             void* stream)
{
    QMM_TRY(check_mx("qmm_mx_dequantize", fmt, rows, K));
    QMM_TRY(check_scale("qmm_mx_dequantize", fmt, tensor_scale));
    if (rows == 0) return QMM_OK;
    QMM_TRY(check_rows("qmm_mx_dequantize", "out", dtype, out, ldo, K));
    QMM_TRY(check_packed("qmm_mx_dequantize", "packed", packed));
    QMM_TRY(check_device("qmm_mx_dequantize"));
    return launch_mx_dequantize(fmt, dtype, packed, rows, K, tensor_scale, out, ldo, (cudaStream_t)stream);
}

size_t qmm_mx_gemm_workspace_bytes(qmm_mx_format fmt, int64_t M, int64_t N, int64_t K)
{
    if (check_product("qmm_mx_gemm_workspace_bytes", fmt, M, N, K) != QMM_OK) return 0;
    return kMxHeader + mx_gemm_partial_bytes_up_to(M, N, K);
}

qmm_status qmm_mx_gemm(qmm_mx_format fmt, const void* a, int64_t M, const void* w, int64_t N, int64_t K, const float* a_scale, const float* w_scale, qmm_dtype dtype,
                       void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "qmm_mx_gemm";
    QMM_TRY(check_product(who, fmt, M, N, K));
    QMM_TRY(check_scale(who, fmt, a_scale));
    QMM_TRY(check_scale(who, fmt, w_scale));
    if (M == 0) return QMM_OK;
    QMM_TRY(check_packed(who, "a", a));
    QMM_TRY(check_packed(who, "w", w));
    QMM_TRY(check_rows(who, "Y", dtype, Y, ldy, N));
    QMM_TRY(check_ws(who, ws, ws_bytes, kMxHeader + mx_gemm_partial_bytes(M, N, K), 256));
    QMM_TRY(check_device(who));
    return launch_mx_gemm(fmt, a, M, w, N, K, a_scale, w_scale, dtype, Y, ldy, (int*)ws, (cudaStream_t)stream);
}

size_t qmm_mx_linear_workspace_bytes(qmm_mx_format fmt, int64_t M, int64_t N, int64_t K)
{
    if (check_product("qmm_mx_linear_workspace_bytes", fmt, M, N, K) != QMM_OK) return 0;
    return kMxHeader + mx_gemm_partial_bytes_up_to(M, N, K) + mx_bytes(fmt, (M + 127) / 128, K);
}

qmm_status qmm_mx_linear(qmm_mx_format fmt, qmm_dtype dtype, const void* X, int64_t ldx, int64_t M, const void* w, int64_t N, int64_t K, const float* x_scale,
                         const float* w_scale, void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "qmm_mx_linear";
    QMM_TRY(check_product(who, fmt, M, N, K));
    QMM_TRY(check_scale(who, fmt, x_scale));
    QMM_TRY(check_scale(who, fmt, w_scale));
    if (M == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "X", dtype, X, ldx, K));
    QMM_TRY(check_packed(who, "w", w));
    QMM_TRY(check_rows(who, "Y", dtype, Y, ldy, N));
    const size_t before_a = kMxHeader + mx_gemm_partial_bytes(M, N, K);        // status word, counters, partial sums; then the quantised rows
    const bool few = mx_few_fits(fmt, M, N, K);
    QMM_TRY(check_ws(who, ws, ws_bytes, before_a + (few ? 0 : mx_bytes(fmt, (M + 127) / 128, K)), 256));
    QMM_TRY(check_device(who));
    if (few) return launch_mx_few(fmt, dtype, X, ldx, M, w, N, K, x_scale, w_scale, Y, ldy, (int*)ws, (cudaStream_t)stream);
    void* a = (char*)ws + before_a;
    QMM_TRY(launch_mx_quantize(fmt, dtype, X, ldx, M, K, x_scale, a, true, (cudaStream_t)stream));
    return launch_mx_gemm(fmt, a, M, w, N, K, x_scale, w_scale, dtype, Y, ldy, (int*)ws, (cudaStream_t)stream);
}

size_t qmm_expert_sort_workspace_bytes(int32_t T, int32_t topk, int32_t E)
{
    if (check_pairs("qmm_expert_sort_workspace_bytes", T, topk, E) != QMM_OK) return 0;
    return expert_sort_workspace_bytes((int64_t)T * topk, E);
}

qmm_status qmm_expert_sort(const int32_t* idx, int32_t T, int32_t topk, int32_t E, int32_t* order, int32_t* place, int32_t* offsets, int32_t* units, void* ws,
                           size_t ws_bytes, void* stream)
{
    const char* who = "qmm_expert_sort";
    QMM_TRY(check_pairs(who, T, topk, E));
    if (!offsets || !units || (T > 0 && (!idx || !order || !place))) return fail(QMM_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned(idx, 4) || !aligned(order, 4) || !aligned(place, 4) || !aligned(offsets, 4) || !aligned(units, 4))
        return fail(QMM_ERR_ALIGNMENT, "%s: index arrays must be 4-byte aligned", who);
    const size_t need = expert_sort_workspace_bytes((int64_t)T * topk, E);
    if (need > 0) QMM_TRY(check_ws(who, ws, ws_bytes, need, 4));
    QMM_TRY(check_device(who));
    return launch_expert_sort(idx, (int64_t)T * topk, E, order, place, offsets, units, ws, (cudaStream_t)stream);
}

qmm_status qmm_expert_gather(qmm_dtype dtype, const void* x, int64_t ldx, int32_t T, int32_t topk, int64_t H, const int32_t* order, const int32_t* place,
                             const float* weights, void* xs, int64_t ldxs, void* stream)
{
    const char* who = "qmm_expert_gather";
    QMM_TRY(check_pairs(who, T, topk, 1));
    if (H <= 0 || H > (1 << 24)) return fail(QMM_ERR_INVALID_ARG, "%s: H=%lld outside [1, 2^24]", who, (long long)H);
    if (T == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "x", dtype, x, ldx, H));
    QMM_TRY(check_rows(who, "xs", dtype, xs, ldxs, H));
    if (!order || !place) return fail(QMM_ERR_INVALID_ARG, "%s: order or place is null", who);
    if (!aligned(order, 4) || !aligned(place, 4) || !aligned(weights, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: order, place and weights must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_expert_gather(dtype, x, ldx, T, topk, H, order, place, weights, xs, ldxs, (cudaStream_t)stream);
}

qmm_status qmm_expert_combine(qmm_dtype dtype, const void* ys, int64_t ldys, int32_t T, int32_t topk, int64_t H, const int32_t* place, const float* weights, void* y,
                              int64_t ldy, void* stream)
{
    const char* who = "qmm_expert_combine";
    QMM_TRY(check_pairs(who, T, topk, 1));
    if (H <= 0 || H > (1 << 24)) return fail(QMM_ERR_INVALID_ARG, "%s: H=%lld outside [1, 2^24]", who, (long long)H);
    if (T == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "ys", dtype, ys, ldys, H));
    QMM_TRY(check_rows(who, "y", dtype, y, ldy, H));
    if (!place) return fail(QMM_ERR_INVALID_ARG, "%s: place is null", who);
    if (!aligned(place, 4) || !aligned(weights, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: place and weights must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_expert_combine(dtype, dtype, ys, ldys, T, topk, H, place, weights, y, ldy, (cudaStream_t)stream);
}

qmm_status qmm_expert_combine_grad(qmm_dtype dtype, const void* dy, int64_t lddy, const void* ys, int64_t ldys, int32_t T, int32_t topk, int64_t H,
                                   const int32_t* order, const int32_t* place, const float* weights, void* dys, int64_t lddys, float* dw, void* stream)
{
    const char* who = "qmm_expert_combine_grad";
    QMM_TRY(check_pairs(who, T, topk, 1));
    if (H <= 0 || H > (1 << 24)) return fail(QMM_ERR_INVALID_ARG, "%s: H=%lld outside [1, 2^24]", who, (long long)H);
    if (T == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "dy", dtype, dy, lddy, H));
    QMM_TRY(check_rows(who, "ys", dtype, ys, ldys, H));
    QMM_TRY(check_rows(who, "dys", dtype, dys, lddys, H));
    if (!order || !place || !weights || !dw) return fail(QMM_ERR_INVALID_ARG, "%s: order, place, weights or dw is null", who);
    if (!aligned(order, 4) || !aligned(place, 4) || !aligned(weights, 4) || !aligned(dw, 4))
        return fail(QMM_ERR_ALIGNMENT, "%s: order, place, weights and dw must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_expert_combine_grad(dtype, dy, lddy, ys, ldys, T, topk, H, order, place, weights, dys, lddys, dw, (cudaStream_t)stream);
}

size_t qmm_mx_experts_bytes(qmm_mx_format fmt, int32_t T, int32_t topk, int32_t E, int64_t K)
{
    if (check_mx("qmm_mx_experts_bytes", fmt, T, K) != QMM_OK || check_pairs("qmm_mx_experts_bytes", T, topk, E) != QMM_OK) return 0;
    return mx_bytes(fmt, mx_max_row_units((int64_t)T * topk, E), K);
}

qmm_status qmm_mx_quantize_experts(qmm_mx_format fmt, qmm_dtype dtype, const void* x, int64_t ldx, int32_t T, int32_t topk, int32_t E, int64_t K,
                                   const int32_t* idx, const int32_t* place, const int32_t* offsets, const int32_t* units, const float* tensor_scale,
                                   void* packed, void* stream)
{
    const char* who = "qmm_mx_quantize_experts";
    QMM_TRY(check_pairs(who, T, topk, E));
    QMM_TRY(check_mx(who, fmt, T, K));
    QMM_TRY(check_scale(who, fmt, tensor_scale));
    if (T == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "x", dtype, x, ldx, K));
    QMM_TRY(check_packed(who, "packed", packed));
    if (!idx || !place || !offsets || !units) return fail(QMM_ERR_INVALID_ARG, "%s: idx, place, offsets or units is null", who);
    if (!aligned(idx, 4) || !aligned(place, 4) || !aligned(offsets, 4) || !aligned(units, 4))
        return fail(QMM_ERR_ALIGNMENT, "%s: index arrays must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_mx_quantize_experts(fmt, dtype, x, ldx, T, topk, E, K, idx, place, offsets, units, tensor_scale, packed, false, (cudaStream_t)stream);
}

qmm_status qmm_mx_experts_gate_up(qmm_mx_format fmt, const void* a, int32_t T, int32_t topk, int32_t E, const int32_t* offsets, const int32_t* units,
                                  const void* w_gate, const void* w_up, int64_t N, int64_t K, const float* a_scale, const float* gate_scale,
                                  const float* up_scale, const float* h_scale, void* h, int32_t* status, void* stream)
{
    const char* who = "qmm_mx_experts_gate_up";
    QMM_TRY(check_pairs(who, T, topk, E));
    QMM_TRY(check_mx(who, fmt, N, K));
    if (N == 0) return fail(QMM_ERR_INVALID_ARG, "%s: N must be positive", who);
    for (const float* s : {a_scale, gate_scale, up_scale, h_scale}) QMM_TRY(check_scale(who, fmt, s));
    if (T == 0) return QMM_OK;
    QMM_TRY(check_packed(who, "a", a));
    QMM_TRY(check_packed(who, "w_gate", w_gate));
    QMM_TRY(check_packed(who, "w_up", w_up));
    QMM_TRY(check_packed(who, "h", h));
    if (!offsets || !units) return fail(QMM_ERR_INVALID_ARG, "%s: offsets or units is null", who);
    if (!aligned(offsets, 4) || !aligned(units, 4) || !aligned(status, 4))
        return fail(QMM_ERR_ALIGNMENT, "%s: offsets, units and status must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_mx_experts_gate_up(fmt, a, (int64_t)T * topk, E, offsets, units, w_gate, w_up, N, K, a_scale, gate_scale, up_scale, h_scale, h, status,
                                     (cudaStream_t)stream);
}

qmm_status qmm_mx_experts_gemm(qmm_mx_format fmt, const void* a, int32_t T, int32_t topk, int32_t E, const int32_t* offsets, const int32_t* units, const void* w,
                               int64_t N, int64_t K, const float* a_scale, const float* w_scale, qmm_dtype dtype, void* Y, int64_t ldy, int32_t* status,
                               void* stream)
{
    const char* who = "qmm_mx_experts_gemm";
    QMM_TRY(check_pairs(who, T, topk, E));
    QMM_TRY(check_mx(who, fmt, N, K));
    if (N == 0) return fail(QMM_ERR_INVALID_ARG, "%s: N must be positive", who);
    QMM_TRY(check_scale(who, fmt, a_scale));
    QMM_TRY(check_scale(who, fmt, w_scale));
    if (T == 0) return QMM_OK;
    QMM_TRY(check_packed(who, "a", a));
    QMM_TRY(check_packed(who, "w", w));
    QMM_TRY(check_rows(who, "Y", dtype, Y, ldy, N));
    if (!offsets || !units) return fail(QMM_ERR_INVALID_ARG, "%s: offsets or units is null", who);
    if (!aligned(offsets, 4) || !aligned(units, 4) || !aligned(status, 4))
        return fail(QMM_ERR_ALIGNMENT, "%s: offsets, units and status must be 4-byte aligned", who);
    QMM_TRY(check_device(who));
    return launch_mx_experts_gemm(fmt, a, (int64_t)T * topk, E, offsets, units, w, N, K, a_scale, w_scale, dtype, Y, ldy, false, status, (cudaStream_t)stream);
}

size_t qmm_mx_moe_workspace_bytes(const qmm_mx_moe_args* args)
{
    if (check_mx_moe("qmm_mx_moe_workspace_bytes", args) != QMM_OK) return 0;
    return mx_moe_layout(args).total;
}

qmm_status qmm_mx_moe(const qmm_mx_moe_args* a, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "qmm_mx_moe";
    QMM_TRY(check_mx_moe(who, a));
    for (const float* s : {a->x_scale, a->h_scale, a->gate_scale, a->up_scale, a->down_scale}) QMM_TRY(check_scale(who, a->fmt, s));
    if (a->T == 0) return QMM_OK;
    QMM_TRY(check_rows(who, "X", a->dtype, a->X, a->ldx, a->H));
    QMM_TRY(check_rows(who, "out", a->dtype, a->out, a->ldo, a->H));
    if (!a->idx || !a->weights) return fail(QMM_ERR_INVALID_ARG, "%s: idx or weights is null", who);
    if (!aligned(a->idx, 4) || !aligned(a->weights, 4)) return fail(QMM_ERR_ALIGNMENT, "%s: idx and weights must be 4-byte aligned", who);
    QMM_TRY(check_packed(who, "w_gate", a->w_gate));
    QMM_TRY(check_packed(who, "w_up", a->w_up));
    QMM_TRY(check_packed(who, "w_down", a->w_down));
    const MxMoeLayout l = mx_moe_layout(a);
    QMM_TRY(check_ws(who, ws, ws_bytes, l.total, 256));
    QMM_TRY(check_device(who));
    const cudaStream_t st = (cudaStream_t)stream;
    char* base = (char*)ws;
    int *order = (int*)(base + l.order), *place = (int*)(base + l.place), *offsets = (int*)(base + l.offsets), *units = (int*)(base + l.units);
    const int64_t P = (int64_t)a->T * a->topk;
    if (expert_sort_quantize_fits(P, a->topk, a->H)) {
        QMM_TRY(launch_expert_sort_quantize(a->fmt, a->dtype, a->idx, P, a->topk, a->E, order, place, offsets, units, a->X, a->ldx, a->H, a->x_scale, base + l.xq, st));
    } else {
        QMM_TRY(launch_expert_sort(a->idx, P, a->E, order, place, offsets, units, base + l.sort, st));
        QMM_TRY(launch_mx_quantize_experts(a->fmt, a->dtype, a->X, a->ldx, a->T, a->topk, a->E, a->H, a->idx, place, offsets, units, a->x_scale, base + l.xq, true,
                                           st));
    }
    QMM_TRY(launch_mx_experts_gate_up(a->fmt, base + l.xq, P, a->E, offsets, units, a->w_gate, a->w_up, a->I, a->H, a->x_scale, a->gate_scale, a->up_scale,
                                      a->h_scale, base + l.h, (int*)ws, st));
    QMM_TRY(launch_mx_experts_gemm(a->fmt, base + l.h, P, a->E, offsets, units, a->w_down, a->H, a->I, a->h_scale, a->down_scale, rows_dtype(a), base + l.d, a->H,
                                   true, (int*)ws, st));                                 // gate/up waited for the sort before it let this one go
    return launch_expert_combine(rows_dtype(a), a->dtype, base + l.d, a->H, a->T, a->topk, a->H, place, a->weights, a->out, a->ldo, st);
}

}  // extern "C"
