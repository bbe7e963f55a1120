// Logits adjusted and chosen from (emo_adjust_logits).
#include "emo_logits.h"

#include <type_traits>

// the values are defined to the bit: no multiplication is fused into an addition
#pragma clang fp contract(off)

namespace {

struct AdjustArgs {
    uint32_t rows;
    int32_t vocab;
    Mat logits, history, lengths, repetition, frequency, presence, bias, inv_temperature, mask, noise;
    char *out;
    int64_t out_stride;
    int32_t out_size;       // bytes of an entry
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

// The penalties on N entries that the history holds n times.
template <int N>
__device__ __forceinline__ void penalise(const AdjustArgs &a, const RowRates &rate, float (&x)[N], const uint32_t (&n)[N]) {
    for (int j = 0; j < N; ++j) {
        float p = x[j];
        if (a.repetition.data) p = p > 0.f ? p / rate.repetition : p * rate.repetition;
        if (a.frequency.data) p = p - static_cast<float>(n[j]) * rate.frequency;
        if (a.presence.data) p = p - rate.presence;
        x[j] = n[j] ? p : x[j];
    }
}

template <int N>
__device__ __forceinline__ void mask_entries(float (&x)[N], uint32_t bits) {
    if (bits != (1u << N) - 1)
        for (int j = 0; j < N; ++j) x[j] = bits >> j & 1 ? x[j] : -INFINITY;
}

__device__ __forceinline__ int32_t live_history(const AdjustArgs &a, uint32_t r) {
    if (!a.history.data) return 0;
    const int32_t L = a.history.cols;
    return a.lengths.data ? min(max(*row_of<int32_t>(a.lengths, r), 0), L) : L;
}

constexpr int kPerThread = 32;      // entries a thread holds

// A workgroup per tile of Threads * 32 entries of a row.  Bound by memory: a thread's logits (64 or 128
// bytes) are all in flight before anything else; while they come, the history's ids in the tile are
// counted in LDS (Count: 16 bits an entry while the history has fewer ids than that holds, which lets 8
// workgroups of 256 threads onto a compute unit; integer atomics: any order gives the same counts).  The
// choice of a row of several tiles goes through `parts`, one best entry a tile, and choose_kernel.
template <typename T, typename O, int Threads, typename Count>
__global__ void __launch_bounds__(Threads) adjust_tile_kernel(AdjustArgs a, int64_t first, int32_t tiles, Best *parts) {
    constexpr bool History = !std::is_void<Count>::value;
    constexpr int N = kChunk<T>, C = kPerThread / N, Tile = Threads * kPerThread;
    constexpr int PerWord = !History ? 1 : 4 / sizeof(typename std::conditional<History, Count, int>::type);
    __shared__ alignas(16) uint32_t s_count[History ? Tile / PerWord : 4];
    const int tid = threadIdx.x;
    const int64_t b = first + blockIdx.x;
    const uint32_t r = static_cast<uint32_t>(tiles == 1 ? b : b / tiles);
    const int64_t v0 = (b - static_cast<int64_t>(r) * tiles) * Tile;
    const T *logits = row_of<T>(a.logits, r);
    u32x4 raw[C];
    uint32_t bits[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t v = v0 + (c * Threads + tid) * N;
        if (v < a.vocab) raw[c] = load_chunk(logits, v, a.vocab);
    }
    const int32_t L = History ? live_history(a, r) : 0;
    const RowRates rate = rates_of(a, r);
    const uint32_t *mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t v = v0 + (c * Threads + tid) * N;
        if (v < a.vocab) bits[c] = mask_bits<N>(mask, v, a.vocab);
    }
    if (History && L > 0) {
        const uint32_t hrow = row_index(a.history, r);
#pragma unroll
        for (int i = 0; i < Tile / PerWord; i += 4 * Threads) *reinterpret_cast<u32x4 *>(&s_count[i + 4 * tid]) = u32x4{0, 0, 0, 0};
        __syncthreads();
        for (int32_t i = tid; i < L; i += Threads) {
            const int64_t id = load_id(a.history, hrow, i, a.vocab) - v0;
            if (id >= 0 && id < Tile) atomicAdd(&s_count[id / PerWord], 1u << id % PerWord * 16);
        }
        __syncthreads();
    }
    const float *bias = a.bias.data ? row_of<float>(a.bias, r) : nullptr;
    const float *noise = a.noise.data ? row_of<float>(a.noise, r) : nullptr;
    O *out = reinterpret_cast<O *>(a.out) + static_cast<int64_t>(r) * a.out_stride;
    Best best = {-INFINITY, INT32_MAX};
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = (c * Threads + tid) * N;
        const int64_t v = v0 + e;
        if (v < a.vocab) {
            float x[N], f[N];
            for (int j = 0; j < N; ++j) x[j] = entry<T>(raw[c], j);
            if (History && L > 0) {
                uint32_t n[N], any = 0;
                for (int j = 0; j < N; ++j) {
                    n[j] = PerWord == 1 ? s_count[e + j] : s_count[(e + j) / 2] >> j % 2 * 16 & 0xffffu;
                    any |= n[j];
                }
                if (any) penalise(a, rate, x, n);
            }
            if (bias) {
                load_floats(bias, v, a.vocab, f);
                for (int j = 0; j < N; ++j) x[j] = x[j] + f[j];
            }
            if (a.inv_temperature.data)
                for (int j = 0; j < N; ++j) x[j] = x[j] * rate.inv_temperature;
            mask_entries(x, bits[c]);
            if (a.out) store_chunk(out, v, a.vocab, x);
            if (a.choice) {
                if (noise) {
                    load_floats(noise, v, a.vocab, f);
                    for (int j = 0; j < N; ++j) x[j] = x[j] + f[j];
                }
                for (int j = 0; j < N; ++j)
                    if (x[j] > best.value) best = {x[j], static_cast<int32_t>(v) + j};
            }
        }
    }
    if (a.choice) {
        best = block_best<Threads>(best);
        if (tid == 0) {
            if (tiles == 1) store_choice(a, r, best);
            else parts[b] = best;
        }
    }
}

// The operands of adjust_group_kernel besides those of AdjustArgs: a row's address per group of lanes.
struct GroupArgs {
    int64_t total;              // rows << lg
    int32_t lg, vocab;
    Rows logits, bias, inv_temperature, mask, noise;
    char *out, *choice;
    uint32_t out_stride;        // bytes
    uint32_t choice_stride;
    int32_t choice_dtype;
};

// Rows of at most 64 entries: a group of 2^lg lanes per row, four entries a lane, so that a wave reads
// neighbouring rows in one piece, and U rows a lane, whose loads are in flight together.  The choice is
// the group's maximum, then the least index that has it.  The history (short: see small_rows) is compared
// entry by entry.
template <typename T, typename O, bool Penalties, int U>
__global__ void __launch_bounds__(kThreads) adjust_group_kernel(GroupArgs g, int64_t first, AdjustArgs a) {
    const int32_t v = (threadIdx.x & ((1 << g.lg) - 1)) * 4;
    const int64_t g0 = (first + blockIdx.x) * (kThreads * U) + threadIdx.x;
    const bool mine = v < g.vocab;
    uint32_t r[U];
    float x[U][4], f[U][4];
    uint32_t bits[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = g0 + u * kThreads;
        r[u] = static_cast<uint32_t>((i < g.total ? i : g.total - 1) >> g.lg);      // rows past the last: the last again
    }
    if (mine) {
#pragma unroll
        for (int u = 0; u < U; ++u) load_four(reinterpret_cast<const T *>(row_at(g.logits, r[u])), v, g.vocab, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            bits[u] = mask_bits<4>(g.mask.data ? reinterpret_cast<const uint32_t *>(row_at(g.mask, r[u])) : nullptr, v, g.vocab);
        if (Penalties) {
            for (int u = 0; u < U; ++u) {
                const int32_t L = live_history(a, r[u]);
                if (L == 0) continue;
                const uint32_t hrow = row_index(a.history, r[u]);
                uint32_t n[4] = {0, 0, 0, 0};
                for (int32_t i = 0; i < L; ++i) {
                    const int32_t id = load_id(a.history, hrow, i, g.vocab) - v;
                    for (int j = 0; j < 4; ++j) n[j] += id == j;
                }
                penalise(a, rates_of(a, r[u]), x[u], n);
            }
        }
        if (g.bias.data) {
#pragma unroll
            for (int u = 0; u < U; ++u) load_floats(reinterpret_cast<const float *>(row_at(g.bias, r[u])), v, g.vocab, f[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                for (int j = 0; j < 4; ++j) x[u][j] = x[u][j] + f[u][j];
        }
        if (g.inv_temperature.data) {
            float t[U];
#pragma unroll
            for (int u = 0; u < U; ++u) t[u] = *reinterpret_cast<const float *>(row_at(g.inv_temperature, r[u]));
#pragma unroll
            for (int u = 0; u < U; ++u)
                for (int j = 0; j < 4; ++j) x[u][j] = x[u][j] * t[u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) mask_entries(x[u], bits[u]);
        if (g.out) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (g0 + u * kThreads < g.total)
                    store_chunk(reinterpret_cast<O *>(g.out + static_cast<uint64_t>(r[u]) * g.out_stride), v, g.vocab, x[u]);
        }
    }
    if (!g.choice) return;
    if (mine && g.noise.data) {
#pragma unroll
        for (int u = 0; u < U; ++u) load_floats(reinterpret_cast<const float *>(row_at(g.noise, r[u])), v, g.vocab, f[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            for (int j = 0; j < 4; ++j) x[u][j] = x[u][j] + f[u][j];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float m = mine ? fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3])) : -INFINITY;
        m = group_max(m, g.lg);
        int32_t at = !mine ? INT32_MAX : x[u][0] == m ? v : x[u][1] == m ? v + 1 : x[u][2] == m ? v + 2 : x[u][3] == m ? v + 3 : INT32_MAX;
        at = group_min(at, g.lg);
        if (v == 0 && g0 + u * kThreads < g.total) {
            const int32_t c = m > -INFINITY ? at : -1;      // m is NaN where every entry is: none
            char *to = g.choice + static_cast<uint64_t>(r[u]) * g.choice_stride;
            if (g.choice_dtype == EMO_U8) *reinterpret_cast<uint8_t *>(to) = static_cast<uint8_t>(c);
            else if (g.choice_dtype == EMO_I32) *reinterpret_cast<int32_t *>(to) = c;
            else *reinterpret_cast<int64_t *>(to) = c;
        }
    }
}

// The choice of rows of several tiles, a workgroup per row.
__global__ void __launch_bounds__(kThreads) choose_kernel(AdjustArgs a, int64_t first, int32_t tiles, const Best *parts) {
    const uint32_t r = static_cast<uint32_t>(first + blockIdx.x);
    Best best = {-INFINITY, INT32_MAX};
    for (int32_t t = threadIdx.x; t < tiles; t += kThreads) best = better(best, parts[static_cast<int64_t>(r) * tiles + t]);
    best = block_best<kThreads>(best);
    if (threadIdx.x == 0) store_choice(a, r, best);
}

// Whether groups of lanes take the rows: of at most 64 entries, with a history of at most 64 ids (each is
// compared with every entry; longer ones are counted in LDS), strides below 4 GiB.
bool small_rows(const AdjustArgs &a, GroupArgs *g) {
    if (a.vocab > 64 || (a.history.data && a.history.cols > 64)) return false;
    const int64_t out_bytes = a.out_stride * a.out_size, choice_bytes = a.choice_stride * size_of(a.choice_dtype);
    if (out_bytes >= (int64_t(1) << 32) || choice_bytes >= (int64_t(1) << 32)) return false;
    *g = {};
    while ((4 << g->lg) < a.vocab) ++g->lg;
    g->total = static_cast<int64_t>(a.rows) << g->lg;
    g->vocab = a.vocab;
    g->out = a.out;
    g->out_stride = static_cast<uint32_t>(out_bytes);
    g->choice = a.choice;
    g->choice_stride = static_cast<uint32_t>(choice_bytes);
    g->choice_dtype = a.choice_dtype;
    return narrow(a.logits, &g->logits) && narrow(a.bias, &g->bias) && narrow(a.inv_temperature, &g->inv_temperature) &&
           narrow(a.mask, &g->mask) && narrow(a.noise, &g->noise);
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

struct AdjustLaunch {
    const AdjustArgs &a;
    Best *parts;
    hipStream_t st;

    template <typename T, typename O, int Threads>
    void tiles(int32_t n) const {
        in_launches(static_cast<int64_t>(a.rows) * n, [&](int64_t first, unsigned count) {
            if (!a.history.data)
                hipLaunchKernelGGL((adjust_tile_kernel<T, O, Threads, void>), dim3(count), dim3(Threads), 0, st, a, first, n, parts);
            else if (a.history.cols < 65536)
                hipLaunchKernelGGL((adjust_tile_kernel<T, O, Threads, uint16_t>), dim3(count), dim3(Threads), 0, st, a, first, n, parts);
            else
                hipLaunchKernelGGL((adjust_tile_kernel<T, O, Threads, uint32_t>), dim3(count), dim3(Threads), 0, st, a, first, n, parts);
        });
        if (a.choice && n > 1)
            in_launches(a.rows, [&](int64_t first, unsigned count) {
                hipLaunchKernelGGL(choose_kernel, dim3(count), dim3(kThreads), 0, st, a, first, n, parts);
            });
    }

    template <typename T, typename O>
    void run() const {
        GroupArgs g;
        if (small_rows(a, &g)) {
            constexpr int U = 4;
            in_launches((g.total + kThreads * U - 1) / (kThreads * U), [&](int64_t first, unsigned count) {
                if (a.history.data)
                    hipLaunchKernelGGL((adjust_group_kernel<T, O, true, U>), dim3(count), dim3(kThreads), 0, st, g, first, a);
                else
                    hipLaunchKernelGGL((adjust_group_kernel<T, O, false, U>), dim3(count), dim3(kThreads), 0, st, g, first, a);
            });
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
    a.out_size = static_cast<int32_t>(size_of(o.dtype));
    a.choice = const_cast<char *>(ch.data);
    a.choice_stride = ch.row_stride;
    a.choice_dtype = ch.dtype;
    by_types(a.logits.dtype, out ? o.dtype : a.logits.dtype, AdjustLaunch{a, static_cast<Best *>(workspace), static_cast<hipStream_t>(stream)});
    return launched("emo_adjust_logits");
}

}  // extern "C"
