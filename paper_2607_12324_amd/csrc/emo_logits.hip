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

// A workgroup's best entry, valid in thread 0.
template <int Threads>
__device__ __forceinline__ Best block_best(Best b) {
    b = wave_best(b);
    if constexpr (Threads > 64) {
        __shared__ Best s_best[Threads / 64];
        __syncthreads();
        if (threadIdx.x % 64 == 0) s_best[threadIdx.x / 64] = b;
        __syncthreads();
        for (int w = 0; w < Threads / 64; ++w) b = better(b, s_best[w]);
    }
    return b;
}

// What the steps need of a row.
struct RowRates {
    float repetition, frequency, presence, inv_temperature;
};

__device__ __forceinline__ RowRates rates_of(const AdjustArgs &a, uint32_t r) {
    return {row_value(a.repetition, r, 1.f), row_value(a.frequency, r, 0.f), row_value(a.presence, r, 0.f),
            row_value(a.inv_temperature, r, 1.f)};
}

// Adjusts N entries (x) that the history holds n times, and keeps the best for the choice.
template <int N>
__device__ __forceinline__ void adjust_entries(const AdjustArgs &a, const RowRates &rate, float (&x)[N], const uint32_t (&n)[N],
                                               bool penalties, const float (&bias)[N], const float (&noise)[N], uint32_t bits,
                                               int32_t v, Best &best) {
    if (penalties) {
        for (int j = 0; j < N; ++j) {
            if (n[j] == 0) continue;
            if (a.repetition.data) x[j] = x[j] > 0.f ? x[j] / rate.repetition : x[j] * rate.repetition;
            if (a.frequency.data) x[j] = x[j] - static_cast<float>(n[j]) * rate.frequency;
            if (a.presence.data) x[j] = x[j] - rate.presence;
        }
    }
    for (int j = 0; j < N; ++j) {
        if (a.bias.data) x[j] = x[j] + bias[j];
        if (a.inv_temperature.data) x[j] = x[j] * rate.inv_temperature;
        if (!(bits >> j & 1)) x[j] = -INFINITY;
        const float y = a.noise.data ? x[j] + noise[j] : x[j];
        if (y > best.value && x[j] > -INFINITY) best = {y, v + j};
    }
}

__device__ __forceinline__ int32_t live_history(const AdjustArgs &a, uint32_t r) {
    if (!a.history.data) return 0;
    const int32_t L = a.history.cols;
    return a.lengths.data ? min(max(*row_of<int32_t>(a.lengths, r), 0), L) : L;
}

constexpr int kPerThread = 32;      // entries a thread holds

// A workgroup per tile of Threads * 32 entries of a row.  Bound by memory: a thread's logits (64 or 128
// bytes) are all in flight before anything else; while they come, the history's ids in the tile are
// counted in LDS (4 bytes an entry; integer atomics: any order gives the same counts).  The choice of a
// row of several tiles goes through `parts`, one best entry a tile, and choose_kernel.
template <typename T, typename O, int Threads, bool History>
__global__ void __launch_bounds__(Threads) adjust_tile_kernel(AdjustArgs a, int32_t tiles, Best *parts) {
    constexpr int N = kChunk<T>, C = kPerThread / N, Tile = Threads * kPerThread;
    __shared__ alignas(16) uint32_t s_count[History ? Tile : 4];
    const int tid = threadIdx.x;
    const int64_t blocks = static_cast<int64_t>(a.rows) * tiles;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const uint32_t r = static_cast<uint32_t>(tiles == 1 ? b : b / tiles);
        const int64_t v0 = (b - static_cast<int64_t>(r) * tiles) * Tile;
        const T *logits = row_of<T>(a.logits, r);
        const float *bias = a.bias.data ? row_of<float>(a.bias, r) : nullptr;
        const float *noise = a.noise.data ? row_of<float>(a.noise, r) : nullptr;
        const uint32_t *mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
        u32x4 raw[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t v = v0 + (c * Threads + tid) * N;
            if (v < a.vocab) raw[c] = load_chunk(logits, v, a.vocab);
        }
        const RowRates rate = rates_of(a, r);
        const int32_t L = History ? live_history(a, r) : 0;
        if (History && L > 0) {
            const uint32_t hrow = row_index(a.history, r);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < Tile; i += 4 * Threads) *reinterpret_cast<u32x4 *>(&s_count[i + 4 * tid]) = u32x4{0, 0, 0, 0};
            __syncthreads();
            for (int32_t i = tid; i < L; i += Threads) {
                const int64_t id = load_id(a.history, hrow, i, a.vocab) - v0;
                if (id >= 0 && id < Tile) atomicAdd(&s_count[id], 1u);
            }
            __syncthreads();
        }
        Best best = {-INFINITY, INT32_MAX};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * Threads + tid) * N;
            const int64_t v = v0 + e;
            if (v >= a.vocab) break;
            float x[N], bs[N], ns[N];
            uint32_t n[N];
            if (bias) load_floats(bias, v, a.vocab, bs);
            if (noise) load_floats(noise, v, a.vocab, ns);
            const uint32_t bits = mask_bits<N>(mask, v);
            for (int j = 0; j < N; ++j) x[j] = entry<T>(raw[c], j);
            if (History && L > 0) {
                for (int j = 0; j < N; j += 4) {
                    const u32x4 q = *reinterpret_cast<const u32x4 *>(&s_count[e + j]);
                    for (int i = 0; i < 4; ++i) n[j + i] = q[i];
                }
            }
            adjust_entries(a, rate, x, n, History && L > 0, bs, ns, bits, static_cast<int32_t>(v), best);
            if (a.out) store_chunk(reinterpret_cast<O *>(a.out) + static_cast<int64_t>(r) * a.out_stride, v, a.vocab, x);
        }
        if (a.choice) {
            best = block_best<Threads>(best);
            if (tid == 0) {
                if (tiles == 1) store_choice(a, r, best);
                else parts[b] = best;
            }
        }
    }
}

// Rows of at most 64 entries: a group of 2^lg lanes per row, four entries a lane, so that a wave reads
// neighbouring rows in one piece; the choice is a reduction within the group.  The history (short: see
// small_rows) is compared entry by entry.
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads) adjust_group_kernel(AdjustArgs a, int lg) {
    const int lanes = 1 << lg;
    const int64_t total = static_cast<int64_t>(a.rows) << lg;
    for (int64_t b = static_cast<int64_t>(blockIdx.x) * kThreads; b < total; b += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t g = b + threadIdx.x;
        const bool live = g < total;
        const uint32_t r = static_cast<uint32_t>((live ? g : total - 1) >> lg);
        const int32_t v = (threadIdx.x & (lanes - 1)) * 4;
        Best best = {-INFINITY, INT32_MAX};
        if (live && v < a.vocab) {
            float x[4], bias[4], noise[4];
            uint32_t n[4] = {0, 0, 0, 0};
            if (a.noise.data) load_floats(row_of<float>(a.noise, r), v, a.vocab, noise);
            load_four(row_of<T>(a.logits, r), v, a.vocab, x);
            if (a.bias.data) load_floats(row_of<float>(a.bias, r), v, a.vocab, bias);
            const uint32_t bits = mask_bits<4>(a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr, v);
            const int32_t L = live_history(a, r);
            if (L > 0) {
                const uint32_t hrow = row_index(a.history, r);
                for (int32_t i = 0; i < L; ++i) {
                    const int32_t id = load_id(a.history, hrow, i, a.vocab) - v;
                    for (int j = 0; j < 4; ++j) n[j] += id == j;
                }
            }
            adjust_entries(a, rates_of(a, r), x, n, L > 0, bias, noise, bits, v, best);
            if (a.out) store_chunk(reinterpret_cast<O *>(a.out) + static_cast<int64_t>(r) * a.out_stride, v, a.vocab, x);
        }
        if (a.choice) {
            for (int off = lanes >> 1; off > 0; off >>= 1) {
                Best o;
                o.value = __shfl_xor(best.value, off, 64);
                o.at = __shfl_xor(best.at, off, 64);
                best = better(best, o);
            }
            if (live && v == 0) store_choice(a, r, best);
        }
    }
}

// The choice of rows of several tiles, a workgroup per row.
__global__ void __launch_bounds__(kThreads) choose_kernel(AdjustArgs a, int32_t tiles, const Best *parts) {
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        Best best = {-INFINITY, INT32_MAX};
        for (int32_t t = threadIdx.x; t < tiles; t += kThreads) best = better(best, parts[static_cast<int64_t>(r) * tiles + t]);
        best = block_best<kThreads>(best);
        if (threadIdx.x == 0) store_choice(a, r, best);
    }
}

// A row's tiles: of 8,192 entries for workgroups of 256 threads while that gives work to every compute
// unit (4 workgroups each), of 2,048 for single waves on shorter rows and for few rows.
// Rows that a group of lanes takes: of at most 64 entries, with a history of at most 64 ids (each is
// compared with every entry; longer ones are counted in LDS).
bool small_rows(const AdjustArgs &a) { return a.vocab <= 64 && (!a.history.data || a.history.cols <= 64); }

struct Tiling {
    int threads;
    int64_t tiles;
};

Tiling tiling(int64_t rows, int64_t vocab) {
    const int64_t wide = (vocab + 8191) / 8192;
    if (vocab > 2048 && rows * wide >= 1024) return {256, wide};
    return {64, (vocab + 2047) / 2048};
}

unsigned blocks_for(int64_t n) { return static_cast<unsigned>(n < kMaxBlocks ? n : kMaxBlocks); }

struct AdjustLaunch {
    const AdjustArgs &a;
    Best *parts;
    hipStream_t st;

    template <typename T, typename O, int Threads>
    void tiles(int32_t n) const {
        const dim3 grid(blocks_for(static_cast<int64_t>(a.rows) * n));
        if (a.history.data)
            hipLaunchKernelGGL((adjust_tile_kernel<T, O, Threads, true>), grid, dim3(Threads), 0, st, a, n, parts);
        else
            hipLaunchKernelGGL((adjust_tile_kernel<T, O, Threads, false>), grid, dim3(Threads), 0, st, a, n, parts);
        if (a.choice && n > 1) hipLaunchKernelGGL(choose_kernel, dim3(blocks_for(a.rows)), dim3(kThreads), 0, st, a, n, parts);
    }

    template <typename T, typename O>
    void run() const {
        if (small_rows(a)) {
            int lg = 0;
            while ((4 << lg) < a.vocab) ++lg;
            const int64_t blocks = ((static_cast<int64_t>(a.rows) << lg) + kThreads - 1) / kThreads;
            hipLaunchKernelGGL((adjust_group_kernel<T, O>), dim3(blocks_for(blocks)), dim3(kThreads), 0, st, a, lg);
            return;
        }
        const Tiling t = tiling(a.rows, a.vocab);
        if (t.threads == 64) tiles<T, O, 64>(static_cast<int32_t>(t.tiles));
        else tiles<T, O, 256>(static_cast<int32_t>(t.tiles));
    }
};

// Workspace bytes of a call: the best entry of every tile of rows of several.
int64_t adjust_bytes(int64_t rows, int64_t vocab) {
    const int64_t tiles = tiling(rows, vocab).tiles;
    return tiles > 1 ? rows * tiles * static_cast<int64_t>(sizeof(Best)) : 0;
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
    by_types(a.logits.dtype, out ? o.dtype : a.logits.dtype, AdjustLaunch{a, static_cast<Best *>(workspace), static_cast<hipStream_t>(stream)});
    return launched("emo_adjust_logits");
}

}  // extern "C"
