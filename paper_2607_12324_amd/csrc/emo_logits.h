// What the calls on logits share: operands, their checks, reductions.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "emo_internal.h"

namespace {

// ------------------------------------------------------------------------------ operands

// A checked operand.  Row r of a call reads row r % rows; data NULL: absent.
struct Mat {
    const char *data;
    int64_t row_stride, col_stride;   // elements
    uint32_t rows;
    int32_t cols;
    int32_t dtype;
};

template <typename T>
__device__ __forceinline__ const T *row_of(const Mat &m, uint32_t r) {
    return reinterpret_cast<const T *>(m.data) + static_cast<int64_t>(r % m.rows) * m.row_stride;
}

__device__ __forceinline__ float row_value(const Mat &m, uint32_t r, float absent) {
    return m.data ? *row_of<float>(m, r) : absent;
}

// Id k of a row as an index below vocab, or -1.
__device__ __forceinline__ int32_t load_id(const Mat &m, uint32_t row, int32_t k, int32_t vocab) {
    const int64_t at = static_cast<int64_t>(row) * m.row_stride + k * m.col_stride;
    int64_t id;
    if (m.dtype == EMO_U8) id = reinterpret_cast<const uint8_t *>(m.data)[at];
    else if (m.dtype == EMO_I32) id = reinterpret_cast<const int32_t *>(m.data)[at];
    else id = reinterpret_cast<const int64_t *>(m.data)[at];
    return id >= 0 && id < vocab ? static_cast<int32_t>(id) : -1;
}

__device__ __forceinline__ float load_float(const Mat &m, uint32_t row, int32_t k) {
    const int64_t at = static_cast<int64_t>(row) * m.row_stride + k * m.col_stride;
    if (m.dtype == EMO_F32) return reinterpret_cast<const float *>(m.data)[at];
    if (m.dtype == EMO_F16) return static_cast<float>(reinterpret_cast<const _Float16 *>(m.data)[at]);
    return static_cast<float>(reinterpret_cast<const __bf16 *>(m.data)[at]);
}

__device__ __forceinline__ bool allowed(const uint32_t *mask, int32_t v) {
    return !mask || (mask[v >> 5] >> (v & 31)) & 1u;
}

constexpr int kThreads = 256;

// ------------------------------------------------------------------------------ host

emo_status fail(emo_status s, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return emo::report(s, buf);
}

emo_status launched(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(EMO_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
    return emo::report(EMO_OK, "");
}

constexpr int64_t kMaxRows = int64_t(1) << 31;
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxBlocks = int64_t(1) << 20;    // workgroups of a launch: kernels go on by strides

constexpr unsigned bit(int dtype) { return 1u << dtype; }
constexpr unsigned kFloats = bit(EMO_F32) | bit(EMO_F16) | bit(EMO_BF16);
constexpr unsigned kIndices = bit(EMO_U8) | bit(EMO_I32) | bit(EMO_I64);

int64_t size_of(int32_t dtype) {
    switch (dtype) {
        case EMO_U8: return 1;
        case EMO_F16: case EMO_BF16: return 2;
        case EMO_I64: return 8;
        default: return 4;
    }
}

// Checks the operands of one call against its sizes, and their memory against each other.
struct Checker {
    int64_t rows;
    emo_status status = EMO_OK;

    struct Range {
        const char *name;
        uintptr_t begin, end;
        bool output;
        const emo_tensor *t;
    } ranges[16];
    int n = 0;

    void bad(emo_status s) {
        if (status == EMO_OK) status = s;
    }

    // An operand (absent when t is NULL) of `cols` columns (-1: any).  Outputs have all rows.
    Mat take(const char *name, const emo_tensor *t, unsigned types, int64_t cols, bool dense, bool output) {
        Mat m = {};
        if (!t || status != EMO_OK) return m;
        if (t->dtype < EMO_F32 || t->dtype > EMO_I64 || !(types & bit(t->dtype)))
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s has a type that this call does not take (%d)", name, (int)t->dtype)), m;
        if (cols >= 0 && t->cols != cols)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s has %lld columns, needs %lld", name, (long long)t->cols, (long long)cols)), m;
        if (t->cols < 0 || t->cols >= kMaxRows || t->rows < 0 || t->rows >= kMaxRows)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s is %lld x %lld: outside [0, 2^31)", name, (long long)t->rows, (long long)t->cols)), m;
        if (rows == 0) return m;
        if (output ? t->rows != rows : t->rows < 1 || rows % t->rows != 0)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, output ? "%s has %lld rows, needs %lld" : "%s has %lld rows, which do not divide the call's %lld",
                            name, (long long)t->rows, (long long)rows)), m;
        if (t->row_stride < 0 || t->col_stride < 0 || t->row_stride > kMaxStride || t->col_stride > kMaxStride)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s has strides outside [0, 2^40]", name)), m;
        if (dense && t->cols > 1 && t->col_stride != 1)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s needs columns next to each other (col_stride 1)", name)), m;
        if (output && t->rows > 1 && t->row_stride < t->cols)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "rows of %s overlap", name)), m;
        m.rows = static_cast<uint32_t>(t->rows);
        m.cols = static_cast<int32_t>(t->cols);
        m.row_stride = t->row_stride;
        m.col_stride = t->col_stride;
        m.dtype = t->dtype;
        if (t->cols == 0) return m;
        if (!t->data) return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s has no data", name)), m;
        const int64_t size = size_of(t->dtype);
        const uintptr_t p = reinterpret_cast<uintptr_t>(t->data);
        if (p % size) return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s is not aligned to its elements", name)), m;
        const __int128 last = static_cast<__int128>(t->rows - 1) * t->row_stride + static_cast<__int128>(t->cols - 1) * t->col_stride;
        if (last >= (static_cast<__int128>(1) << 48))
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s spans more than an address space", name)), m;
        m.data = static_cast<const char *>(t->data);
        if (n < 16) ranges[n++] = {name, p, p + static_cast<uintptr_t>((static_cast<int64_t>(last) + 1) * size), output, t};
        return m;
    }

    void workspace(const void *p, int64_t have, int64_t need) {
        if (status != EMO_OK || need == 0) return;
        if (!p || have < need)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "workspace of %lld bytes, needs %lld", (long long)(p ? have : 0), (long long)need));
        const uintptr_t b = reinterpret_cast<uintptr_t>(p);
        if (b % 16) return bad(fail(EMO_ERR_INVALID_ARGUMENT, "workspace is not 16-byte aligned"));
        if (n < 16) ranges[n++] = {"workspace", b, b + static_cast<uintptr_t>(need), true, nullptr};
    }

    // Outputs lie apart from everything else; `twin` may be the very memory of `of`.
    emo_status apart(const emo_tensor *twin, const emo_tensor *of) {
        if (status != EMO_OK) return status;
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j) {
                if (i == j || !ranges[i].output || ranges[i].begin >= ranges[j].end || ranges[j].begin >= ranges[i].end) continue;
                const emo_tensor *x = ranges[i].t, *y = ranges[j].t;
                if (twin && x && y && ((x == twin && y == of) || (x == of && y == twin)) && x->data == y->data && x->dtype == y->dtype &&
                    x->rows == y->rows && x->cols == y->cols && (x->rows == 1 || x->row_stride == y->row_stride))
                    continue;
                return status = fail(EMO_ERR_INVALID_ARGUMENT, "%s overlaps %s", ranges[i].name, ranges[j].name);
            }
        return EMO_OK;
    }
};

emo_status check_sizes(int64_t rows, int64_t vocab) {
    if (rows < 0 || rows >= kMaxRows) return fail(EMO_ERR_INVALID_ARGUMENT, "rows %lld outside [0, 2^31)", (long long)rows);
    if (vocab < 1 || vocab >= kMaxRows) return fail(EMO_ERR_INVALID_ARGUMENT, "vocab %lld outside [1, 2^31)", (long long)vocab);
    return EMO_OK;
}

emo_status check_written(const emo_tensor *out, const emo_tensor *logits, const char *name) {
    if (out && out->dtype != logits->dtype && out->dtype != EMO_F32)
        return fail(EMO_ERR_INVALID_ARGUMENT, "%s must have the logits' type or fp32", name);
    return EMO_OK;
}

unsigned row_blocks(int64_t rows) { return static_cast<unsigned>(rows < kMaxBlocks ? rows : kMaxBlocks); }

// Calls f.template run<T, O>() for the logits' type T and the written type O (T or float).
template <typename F>
void by_types(int32_t in, int32_t out, const F &f) {
    if (in == EMO_F32) f.template run<float, float>();
    else if (in == EMO_F16 && out == EMO_F32) f.template run<_Float16, float>();
    else if (in == EMO_F16) f.template run<_Float16, _Float16>();
    else if (out == EMO_F32) f.template run<__bf16, float>();
    else f.template run<__bf16, __bf16>();
}

emo_status workspace_bytes_of(int64_t (*of)(int64_t, int64_t), int64_t rows, int64_t vocab, int64_t *bytes) {
    if (!bytes) return fail(EMO_ERR_INVALID_ARGUMENT, "bytes is NULL");
    const emo_status s = check_sizes(rows, vocab);
    if (s != EMO_OK) return s;
    *bytes = of(rows, vocab);
    return emo::report(EMO_OK, "");
}

}  // namespace
