// Distillation of logits from a teacher's top entries (emo_distill_forward, _backward, _step).
#include "emo_logits.h"

namespace {

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
        const uint32_t irow = row_index(a.ids, r), trow = row_index(a.teacher, r);
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
int64_t distill_bytes(int64_t, int64_t) { return 0; }

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
