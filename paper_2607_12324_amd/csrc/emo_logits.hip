// Proposing policies: logits adjusted and chosen from, and distillation of logits from a teacher's top
// entries (the calls of emo.h from emo_tensor on): argument checks and kernels.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "emo_internal.h"

// adjust's values are defined to the bit: no multiplication is fused into an addition
#pragma clang fp contract(off)

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

// ------------------------------------------------------------------------------ adjust

struct AdjustArgs {
    uint32_t rows;
    int32_t vocab;
    Mat logits, history, lengths, repetition, frequency, presence, bias, inv_temperature, mask, noise;
    char *out;
    int64_t out_stride;
    char *choice;
    int64_t choice_stride;
    int32_t choice_dtype;
};

constexpr int kThreads = 256;
constexpr int kTile = 4096;     // entries whose counts lie in LDS at once

struct Best {
    float value;
    int32_t at;
};

// The greater value, on equal values the lower index; {-inf, INT32_MAX} is no entry.
__device__ __forceinline__ Best better(Best a, Best b) {
    return b.value > a.value || (b.value == a.value && b.at < a.at) ? b : a;
}

__device__ __forceinline__ Best wave_best(Best b) {
    for (int off = 32; off > 0; off >>= 1) {
        Best o;
        o.value = __shfl_xor(b.value, off, 64);
        o.at = __shfl_xor(b.at, off, 64);
        b = better(b, o);
    }
    return b;
}

__device__ __forceinline__ void store_choice(const AdjustArgs &a, uint32_t r, Best b) {
    const int32_t c = b.value > -INFINITY ? b.at : -1;
    const int64_t at = static_cast<int64_t>(r) * a.choice_stride;
    if (a.choice_dtype == EMO_U8) reinterpret_cast<uint8_t *>(a.choice)[at] = static_cast<uint8_t>(c);
    else if (a.choice_dtype == EMO_I32) reinterpret_cast<int32_t *>(a.choice)[at] = c;
    else reinterpret_cast<int64_t *>(a.choice)[at] = c;
}

// A workgroup per row, tile after tile: the history's ids in the tile are counted in LDS (integer
// atomics: any order gives the same counts), then every entry goes through the formula once.
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads) adjust_row_kernel(AdjustArgs a) {
    __shared__ uint32_t s_count[kTile];
    __shared__ Best s_best[kThreads / 64];
    const int tid = threadIdx.x;
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *logits = row_of<T>(a.logits, r);
        const float *bias = a.bias.data ? row_of<float>(a.bias, r) : nullptr;
        const float *noise = a.noise.data ? row_of<float>(a.noise, r) : nullptr;
        const uint32_t *mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
        const uint32_t hrow = a.history.data ? r % a.history.rows : 0;
        int32_t L = a.history.data ? a.history.cols : 0;
        if (a.lengths.data) L = min(max(*row_of<int32_t>(a.lengths, r), 0), L);
        const float rep = row_value(a.repetition, r, 1.f);
        const float freq = row_value(a.frequency, r, 0.f);
        const float pres = row_value(a.presence, r, 0.f);
        const float inv_t = row_value(a.inv_temperature, r, 1.f);
        Best best = {-INFINITY, INT32_MAX};
        for (int64_t v0 = 0; v0 < a.vocab; v0 += kTile) {
            const int32_t n = static_cast<int32_t>(min(static_cast<int64_t>(kTile), a.vocab - v0));
            if (L > 0) {
                __syncthreads();
                for (int i = tid; i < n; i += kThreads) s_count[i] = 0;
                __syncthreads();
                for (int32_t i = tid; i < L; i += kThreads) {
                    const int64_t id = load_id(a.history, hrow, i, a.vocab) - v0;
                    if (id >= 0 && id < n) atomicAdd(&s_count[id], 1u);
                }
                __syncthreads();
            }
            for (int i = tid; i < n; i += kThreads) {
                const int32_t v = static_cast<int32_t>(v0 + i);
                float x = static_cast<float>(logits[v]);
                const uint32_t seen = L > 0 ? s_count[i] : 0;
                if (seen) {
                    if (a.repetition.data) x = x > 0.f ? x / rep : x * rep;
                    if (a.frequency.data) x = x - static_cast<float>(seen) * freq;
                    if (a.presence.data) x = x - pres;
                }
                if (bias) x = x + bias[v];
                if (a.inv_temperature.data) x = x * inv_t;
                if (!allowed(mask, v)) x = -INFINITY;
                if (a.out) reinterpret_cast<O *>(a.out)[static_cast<int64_t>(r) * a.out_stride + v] = static_cast<O>(x);
                const float y = noise ? x + noise[v] : x;
                if (y > best.value && x > -INFINITY) best = {y, v};
            }
        }
        if (a.choice) {
            best = wave_best(best);
            __syncthreads();
            if (tid % 64 == 0) s_best[tid / 64] = best;
            __syncthreads();
            if (tid == 0) {
                for (int w = 1; w < kThreads / 64; ++w) best = better(best, s_best[w]);
                store_choice(a, r, best);
            }
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------------------ distillation

struct DistillArgs {
    uint32_t rows;
    int32_t vocab;
    int32_t entries;        // K
    float inv_tau, tau;     // 1 / temperature, temperature
    float log2e_tau;        // log2(e) / temperature: exp(d / temperature) = 2^(d * log2e_tau)
    Mat logits, ids, teacher, mask, scale, stats;
    char *loss, *stats_out, *grad;
    int64_t loss_stride, stats_stride, grad_stride;
};

constexpr int kMaxEntries = 1024;

__device__ __forceinline__ float wave_sum(float x) {
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

__device__ __forceinline__ float wave_max(float x) {
    for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
    return x;
}

// Sum (or maximum) over the workgroup, to every thread; s_red has a slot per wave.
template <bool Max>
__device__ __forceinline__ float block_reduce(float x, float *s_red) {
    x = Max ? wave_max(x) : wave_sum(x);
    __syncthreads();
    if (threadIdx.x % 64 == 0) s_red[threadIdx.x / 64] = x;
    __syncthreads();
    x = s_red[0];
    for (int w = 1; w < kThreads / 64; ++w) x = Max ? fmaxf(x, s_red[w]) : x + s_red[w];
    return x;
}

// A workgroup per row.  Forward: the greatest logit, then the sum of exponentials below it.  The
// teacher's probabilities lie in LDS; the gradient goes tile after tile, each tile's probabilities
// gathered by entry in the list's order, so that equal ids add up in a fixed order.
template <typename T, typename O, bool Forward, bool Backward>
__global__ void __launch_bounds__(kThreads) distill_row_kernel(DistillArgs a) {
    __shared__ int32_t s_id[kMaxEntries];
    __shared__ float s_p[kMaxEntries];
    __shared__ float s_red[kThreads / 64];
    const int tid = threadIdx.x;
    const int K = a.entries;
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *logits = row_of<T>(a.logits, r);
        const uint32_t *mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
        float m = -INFINITY, s = 0.f;
        if (Forward) {
            for (int64_t v = tid; v < a.vocab; v += kThreads)
                if (allowed(mask, static_cast<int32_t>(v))) m = fmaxf(m, static_cast<float>(logits[v]));
            m = block_reduce<true>(m, s_red);
            const float ref = m == -INFINITY ? 0.f : m;
            for (int64_t v = tid; v < a.vocab; v += kThreads)
                if (allowed(mask, static_cast<int32_t>(v)))
                    s += exp2f((static_cast<float>(logits[v]) - ref) * a.log2e_tau);
            s = block_reduce<false>(s, s_red);
            if (a.stats_out && tid == 0) {
                float *st = reinterpret_cast<float *>(a.stats_out) + static_cast<int64_t>(r) * a.stats_stride;
                st[0] = m;
                st[1] = s;
            }
        } else {
            const float *st = row_of<float>(a.stats, r);
            m = st[0];
            s = st[1];
        }
        const uint32_t irow = K ? r % a.ids.rows : 0, trow = K ? r % a.teacher.rows : 0;
        float tm = -INFINITY;
        float any = 0.f;
        for (int k = tid; k < K; k += kThreads) {
            int32_t id = load_id(a.ids, irow, k, a.vocab);
            const float t = load_float(a.teacher, trow, k);
            if (id >= 0 && (t == -INFINITY || !allowed(mask, id))) id = -1;
            s_id[k] = id;
            s_p[k] = t;
            if (id >= 0) {
                tm = fmaxf(tm, t);
                any = 1.f;
            }
        }
        tm = block_reduce<true>(tm, s_red);
        const bool has = block_reduce<true>(any, s_red) > 0.f;
        float ts = 0.f;
        for (int k = tid; k < K; k += kThreads) {
            s_p[k] = s_id[k] >= 0 ? exp2f((s_p[k] - tm) * a.log2e_tau) : 0.f;
            ts += s_p[k];
        }
        ts = block_reduce<false>(ts, s_red);
        float loss = 0.f;
        for (int k = tid; k < K; k += kThreads) {
            if (s_id[k] < 0) continue;
            const float p = s_p[k] / ts;
            s_p[k] = p;
            if (Forward && p != 0.f) loss += p * (logf(s) - (static_cast<float>(logits[s_id[k]]) - m) * a.inv_tau);
        }
        if (Forward && a.loss) {
            loss = block_reduce<false>(loss, s_red);
            if (tid == 0)
                reinterpret_cast<float *>(a.loss)[static_cast<int64_t>(r) * a.loss_stride] = a.tau * a.tau * loss;
        }
        if (Backward) {
            __syncthreads();
            const float c = row_value(a.scale, r, 1.f) * a.tau;
            O *grad = reinterpret_cast<O *>(a.grad) + static_cast<int64_t>(r) * a.grad_stride;
            for (int64_t i = tid; i < a.vocab; i += kThreads) {
                const int32_t v = static_cast<int32_t>(i);
                float g = 0.f;
                if (has && allowed(mask, v)) {
                    float p = 0.f;
                    for (int k = 0; k < K; ++k) p += s_id[k] == v ? s_p[k] : 0.f;
                    g = c * (exp2f((static_cast<float>(logits[v]) - m) * a.log2e_tau) / s - p);
                }
                grad[v] = static_cast<O>(g);
            }
        }
        __syncthreads();
    }
}

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

struct AdjustLaunch {
    const AdjustArgs &a;
    hipStream_t st;
    template <typename T, typename O>
    void run() const {
        hipLaunchKernelGGL((adjust_row_kernel<T, O>), dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
    }
};

template <bool Forward, bool Backward>
struct DistillLaunch {
    const DistillArgs &a;
    hipStream_t st;
    template <typename T, typename O>
    void run() const {
        hipLaunchKernelGGL((distill_row_kernel<T, O, Forward, Backward>), dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
    }
};

// Workspace bytes of a call.
int64_t adjust_bytes(int64_t, int64_t) { return 0; }
int64_t distill_bytes(int64_t, int64_t) { return 0; }

emo_status workspace_bytes_of(int64_t (*of)(int64_t, int64_t), int64_t rows, int64_t vocab, int64_t *bytes) {
    if (!bytes) return fail(EMO_ERR_INVALID_ARGUMENT, "bytes is NULL");
    const emo_status s = check_sizes(rows, vocab);
    if (s != EMO_OK) return s;
    *bytes = of(rows, vocab);
    return emo::report(EMO_OK, "");
}

// The operands every distillation call has.
emo_status distill_operands(Checker &c, DistillArgs &a, int64_t rows, int64_t vocab, const emo_tensor *logits,
                            const emo_tensor *ids, const emo_tensor *teacher, float temperature, const emo_tensor *mask) {
    emo_status s = check_sizes(rows, vocab);
    if (s != EMO_OK) return s;
    if (!logits || !ids || !teacher) return fail(EMO_ERR_INVALID_ARGUMENT, "logits, ids or teacher is NULL");
    if (!(temperature > 0.f) || isinf(temperature)) return fail(EMO_ERR_INVALID_ARGUMENT, "temperature must be finite and > 0");
    if (ids->cols < 0 || ids->cols > kMaxEntries)
        return fail(EMO_ERR_INVALID_ARGUMENT, "ids has %lld columns, outside [0, %d]", (long long)ids->cols, kMaxEntries);
    a = {};
    a.rows = static_cast<uint32_t>(rows);
    a.vocab = static_cast<int32_t>(vocab);
    a.entries = static_cast<int32_t>(ids->cols);
    a.tau = temperature;
    a.inv_tau = static_cast<float>(1.0 / static_cast<double>(temperature));
    a.log2e_tau = static_cast<float>(1.4426950408889634 / static_cast<double>(temperature));
    a.logits = c.take("logits", logits, kFloats, vocab, true, false);
    if (c.status == EMO_OK && rows > 0 && logits->rows != rows)
        return fail(EMO_ERR_INVALID_ARGUMENT, "logits has %lld rows, needs %lld", (long long)logits->rows, (long long)rows);
    a.ids = c.take("ids", ids, kIndices, -1, false, false);
    a.teacher = c.take("teacher", teacher, kFloats, ids->cols, false, false);
    a.mask = c.take("mask", mask, bit(EMO_I32), (vocab + 31) / 32, true, false);
    return c.status;
}

}  // namespace

extern "C" {

emo_status emo_adjust_workspace(int64_t rows, int64_t vocab, int64_t *bytes) {
    return workspace_bytes_of(adjust_bytes, rows, vocab, bytes);
}

emo_status emo_adjust_logits(int64_t rows, int64_t vocab, const emo_tensor *logits, const emo_tensor *history,
                             const emo_tensor *lengths, const emo_tensor *repetition, const emo_tensor *frequency,
                             const emo_tensor *presence, const emo_tensor *bias, const emo_tensor *inv_temperature,
                             const emo_tensor *mask, const emo_tensor *noise, const emo_tensor *out,
                             const emo_tensor *choice, void *workspace, int64_t workspace_bytes, void *stream) {
    emo_status s = check_sizes(rows, vocab);
    if (s != EMO_OK) return s;
    if (!logits) return fail(EMO_ERR_INVALID_ARGUMENT, "logits is NULL");
    if (!history && (lengths || repetition || frequency || presence))
        return fail(EMO_ERR_INVALID_ARGUMENT, "lengths and penalties need a history");
    if (choice && choice->dtype == EMO_U8 && vocab > 255)
        return fail(EMO_ERR_INVALID_ARGUMENT, "a choice among %lld entries does not fit a byte (255 is none)", (long long)vocab);
    Checker c{rows};
    AdjustArgs a = {};
    a.rows = static_cast<uint32_t>(rows);
    a.vocab = static_cast<int32_t>(vocab);
    a.logits = c.take("logits", logits, kFloats, vocab, true, false);
    a.history = c.take("history", history, kIndices, -1, false, false);
    a.lengths = c.take("lengths", lengths, bit(EMO_I32), 1, false, false);
    a.repetition = c.take("repetition", repetition, bit(EMO_F32), 1, false, false);
    a.frequency = c.take("frequency", frequency, bit(EMO_F32), 1, false, false);
    a.presence = c.take("presence", presence, bit(EMO_F32), 1, false, false);
    a.bias = c.take("bias", bias, bit(EMO_F32), vocab, true, false);
    a.inv_temperature = c.take("inv_temperature", inv_temperature, bit(EMO_F32), 1, false, false);
    a.mask = c.take("mask", mask, bit(EMO_I32), (vocab + 31) / 32, true, false);
    a.noise = c.take("noise", noise, bit(EMO_F32), vocab, true, false);
    const Mat o = c.take("out", out, kFloats, vocab, true, true);
    const Mat ch = c.take("choice", choice, kIndices, 1, false, true);
    if (rows > 0 && choice) c.workspace(workspace, workspace_bytes, adjust_bytes(rows, vocab));
    s = c.apart(out, logits);
    if (s == EMO_OK) s = check_written(out, logits, "out");
    if (s != EMO_OK) return s;
    if (rows == 0 || (!out && !choice)) return emo::report(EMO_OK, "");
    if (!repetition && !frequency && !presence) a.history = Mat{};
    a.out = const_cast<char *>(o.data);
    a.out_stride = o.row_stride;
    a.choice = const_cast<char *>(ch.data);
    a.choice_stride = ch.row_stride;
    a.choice_dtype = ch.dtype;
    by_types(a.logits.dtype, out ? o.dtype : a.logits.dtype, AdjustLaunch{a, static_cast<hipStream_t>(stream)});
    return launched("emo_adjust_logits");
}

emo_status emo_distill_workspace(int64_t rows, int64_t vocab, int64_t *bytes) {
    return workspace_bytes_of(distill_bytes, rows, vocab, bytes);
}

emo_status emo_distill_forward(int64_t rows, int64_t vocab, const emo_tensor *logits, const emo_tensor *ids,
                               const emo_tensor *teacher, float temperature, const emo_tensor *mask,
                               const emo_tensor *loss, const emo_tensor *stats, void *workspace,
                               int64_t workspace_bytes, void *stream) {
    Checker c{rows};
    DistillArgs a;
    emo_status s = distill_operands(c, a, rows, vocab, logits, ids, teacher, temperature, mask);
    if (s != EMO_OK) return s;
    const Mat l = c.take("loss", loss, bit(EMO_F32), 1, false, true);
    const Mat st = c.take("stats", stats, bit(EMO_F32), 2, true, true);
    if (rows > 0) c.workspace(workspace, workspace_bytes, distill_bytes(rows, vocab));
    s = c.apart(nullptr, nullptr);
    if (s != EMO_OK) return s;
    if (rows == 0 || (!loss && !stats)) return emo::report(EMO_OK, "");
    a.loss = const_cast<char *>(l.data);
    a.loss_stride = l.row_stride;
    a.stats_out = const_cast<char *>(st.data);
    a.stats_stride = st.row_stride;
    by_types(a.logits.dtype, EMO_F32, DistillLaunch<true, false>{a, static_cast<hipStream_t>(stream)});
    return launched("emo_distill_forward");
}

emo_status emo_distill_backward(int64_t rows, int64_t vocab, const emo_tensor *logits, const emo_tensor *stats,
                                const emo_tensor *ids, const emo_tensor *teacher, float temperature,
                                const emo_tensor *scale, const emo_tensor *mask, const emo_tensor *gradient, void *stream) {
    Checker c{rows};
    DistillArgs a;
    emo_status s = distill_operands(c, a, rows, vocab, logits, ids, teacher, temperature, mask);
    if (s != EMO_OK) return s;
    if (!stats || !gradient) return fail(EMO_ERR_INVALID_ARGUMENT, "stats or gradient is NULL");
    a.stats = c.take("stats", stats, bit(EMO_F32), 2, true, false);
    if (c.status == EMO_OK && rows > 0 && stats->rows != rows)
        return fail(EMO_ERR_INVALID_ARGUMENT, "stats has %lld rows, needs %lld", (long long)stats->rows, (long long)rows);
    a.scale = c.take("scale", scale, bit(EMO_F32), 1, false, false);
    const Mat g = c.take("gradient", gradient, kFloats, vocab, true, true);
    s = c.apart(gradient, logits);
    if (s == EMO_OK) s = check_written(gradient, logits, "gradient");
    if (s != EMO_OK) return s;
    if (rows == 0) return emo::report(EMO_OK, "");
    a.grad = const_cast<char *>(g.data);
    a.grad_stride = g.row_stride;
    by_types(a.logits.dtype, g.dtype, DistillLaunch<false, true>{a, static_cast<hipStream_t>(stream)});
    return launched("emo_distill_backward");
}

emo_status emo_distill_step(int64_t rows, int64_t vocab, const emo_tensor *logits, const emo_tensor *ids,
                            const emo_tensor *teacher, float temperature, const emo_tensor *scale, const emo_tensor *mask,
                            const emo_tensor *loss, const emo_tensor *gradient, void *workspace, int64_t workspace_bytes,
                            void *stream) {
    Checker c{rows};
    DistillArgs a;
    emo_status s = distill_operands(c, a, rows, vocab, logits, ids, teacher, temperature, mask);
    if (s != EMO_OK) return s;
    if (!gradient) return fail(EMO_ERR_INVALID_ARGUMENT, "gradient is NULL");
    a.scale = c.take("scale", scale, bit(EMO_F32), 1, false, false);
    const Mat l = c.take("loss", loss, bit(EMO_F32), 1, false, true);
    const Mat g = c.take("gradient", gradient, kFloats, vocab, true, true);
    if (rows > 0) c.workspace(workspace, workspace_bytes, distill_bytes(rows, vocab));
    s = c.apart(gradient, logits);
    if (s == EMO_OK) s = check_written(gradient, logits, "gradient");
    if (s != EMO_OK) return s;
    if (rows == 0) return emo::report(EMO_OK, "");
    a.loss = const_cast<char *>(l.data);
    a.loss_stride = l.row_stride;
    a.grad = const_cast<char *>(g.data);
    a.grad_stride = g.row_stride;
    by_types(a.logits.dtype, g.dtype, DistillLaunch<true, true>{a, static_cast<hipStream_t>(stream)});
    return launched("emo_distill_step");
}

}  // extern "C"
