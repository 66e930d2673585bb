// qmm_checks.cuh -- argument checks shared by the C entry points of the microscaled operators, the expert moves, the router, the
// norm and the adapters.  Everything is checked on the host before anything is enqueued; messages go to the thread-local buffer.
#pragma once

#include "qmm_common.cuh"

namespace qmm {

static inline bool dtype_ok(int dt) { return dt == QMM_F16 || dt == QMM_BF16 || dt == QMM_F32; }
static inline int dtype_size(int dt) { return dt == QMM_F32 ? 4 : 2; }

// A matrix of plain elements: type, row pitch, element alignment.
static inline qmm_status check_rows(const char* who, const char* name, int dtype, const void* p, int64_t ld, int64_t width)
{
    if (!dtype_ok(dtype)) return fail(QMM_ERR_INVALID_ARG, "%s: unknown data type %d (expected 0, 1 or 2)", who, dtype);
    if (!p) return fail(QMM_ERR_INVALID_ARG, "%s: %s is null", who, name);
    if (ld < width) return fail(QMM_ERR_SHAPE, "%s: row pitch %lld of %s is below its width %lld", who, (long long)ld, name, (long long)width);
    if (ld > (1LL << 40)) return fail(QMM_ERR_UNSUPPORTED, "%s: row pitch %lld of %s > 2^40", who, (long long)ld, name);
    if (!aligned(p, (size_t)dtype_size(dtype))) return fail(QMM_ERR_ALIGNMENT, "%s: %s is not aligned to its element type", who, name);
    return QMM_OK;
}

static inline qmm_status check_ws(const char* who, const void* ws, size_t given, size_t need, size_t align)
{
    if (!ws || given < need) return fail(QMM_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws ? given : (size_t)0);
    if (!aligned(ws, align)) return fail(QMM_ERR_ALIGNMENT, "%s: workspace must be %zu-byte aligned", who, align);
    return QMM_OK;
}

static inline qmm_status check_pairs(const char* who, int32_t T, int32_t topk, int32_t E)
{
    if (T < 0 || topk <= 0 || E <= 0) return fail(QMM_ERR_INVALID_ARG, "%s: T=%d topk=%d E=%d out of range", who, T, topk, E);
    if (E > 1024 || topk > 32) return fail(QMM_ERR_UNSUPPORTED, "%s: E=%d > 1024 or topk=%d > 32", who, E, topk);
    if ((int64_t)T * topk > (1 << 22)) return fail(QMM_ERR_UNSUPPORTED, "%s: T*topk=%lld > 2^22", who, (long long)T * topk);
    return QMM_OK;
}

#define QMM_TRY(call)                    \
    do {                                 \
        const qmm_status s_ = (call);    \
        if (s_ != QMM_OK) return s_;     \
    } while (0)

}  // namespace qmm
