// Logits adjusted and chosen from (emo_adjust_logits).
#include "emo_logits.h"

// the values are defined to the bit: no multiplication is fused into an addition
#pragma clang fp contract(off)

namespace {

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

struct AdjustLaunch {
    const AdjustArgs &a;
    hipStream_t st;
    template <typename T, typename O>
    void run() const {
        hipLaunchKernelGGL((adjust_row_kernel<T, O>), dim3(row_blocks(a.rows)), dim3(kThreads), 0, st, a);
    }
};

// Workspace bytes of a call.
int64_t adjust_bytes(int64_t, int64_t) { return 0; }

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

}  // extern "C"
