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

// The penalties on an entry that the history holds n > 0 times.
__device__ __forceinline__ float penalise(const AdjustArgs &a, const RowRates &rate, float x, uint32_t n) {
    if (a.repetition.data) x = x > 0.f ? x / rate.repetition : x * rate.repetition;
    if (a.frequency.data) x = x - static_cast<float>(n) * rate.frequency;
    if (a.presence.data) x = x - rate.presence;
    return x;
}

// -infinity where the bit is 0: the bit as a word of ones or zeros selects between the two bit by bit.
template <int N>
__device__ __forceinline__ void mask_entries(float (&x)[N], uint32_t bits) {
    if (bits != (1u << N) - 1)
        for (int j = 0; j < N; ++j) {
            const uint32_t on = static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - j)) >> 31);
            x[j] = __uint_as_float((__float_as_uint(x[j]) & on) | (0xff800000u & ~on));
        }
}

__device__ __forceinline__ int32_t live_history(const AdjustArgs &a, uint32_t r) {
    if (!a.history.data) return 0;
    const int32_t L = a.history.cols;
    return a.lengths.data ? min(max(*row_of<int32_t>(a.lengths, r), 0), L) : L;
}

// What a tile's table holds of an entry: kUnseen plus its count, then the bits of the penalised logit.  kUnseen's
// bits are a NaN too, which a rate may hand on, so a NaN is kept as the usual one.
constexpr uint32_t kUnseen = 0xffffffffu;

__device__ __forceinline__ uint32_t seen_bits(float x) { return x != x ? 0x7fc00000u : __float_as_uint(x); }

constexpr int64_t kMaxHistory = int64_t(1) << 30;      // 32 bits hold a place beyond the last id that a thread asks for

// A workgroup per tile of Threads * PerThread entries of a row.  Bound by memory and, with a history, by what
// has to follow each other in a workgroup: so everything that needs nothing is loaded at once (logits, mask,
// bias, length, the first ids), and one more round trip fetches the logits of the ids in the tile.  The ids
// are counted in a table in LDS (a word an entry, kUnseen plus the count; integer atomics: any order gives
// the same counts), and whoever counts an id first puts the penalised logit in the count's place: penalties
// cost a few of the history's ids, not every entry (a division each where any lane of a wave has a seen
// entry, which is nearly always, took 320 of 700 instructions a chunk).  The choice of a row of several
// tiles goes through `parts`, one best entry a tile, and choose_kernel.  256 x 131,072 bf16 with 1,024 ids,
// bias and mask: 33 us, 4.2 TB/s of the 5.0 a copy reaches.
template <typename T, typename O, int Threads, int PerThread, bool History>
__global__ void __launch_bounds__(Threads) adjust_tile_kernel(AdjustArgs a, uint32_t first, Pieces pieces, Best *parts) {
    constexpr int N = kChunk<T>, C = PerThread / N, Tile = Threads * PerThread;
    __shared__ alignas(16) uint32_t s_seen[History ? Tile : 4];
    const int tid = threadIdx.x;
    const uint32_t local = piece_row(pieces, blockIdx.x), r = first + local, part = blockIdx.x - local * pieces.parts;
    const int32_t v0 = static_cast<int32_t>(part) * Tile;
    const int32_t n = min(Tile, a.vocab - v0);      // entries of this tile
    const int32_t whole = n / N * N, rest = whole + tid;
    const T *logits = row_of<T>(a.logits, r) + v0;
    u32x4 raw[C];
    uint32_t bytes[C];
    load_chunks<T, Threads, C>(logits, whole, raw);
    float x_rest = rest < n ? static_cast<float>(logits[rest]) : 0.f;
    const uint32_t *mask = a.mask.data ? row_of<uint32_t>(a.mask, r) + v0 / 32 : nullptr;
    if (mask) load_mask<T, Threads, C>(mask, whole, bytes);
    const float inv_t = row_value(a.inv_temperature, r, 1.f);
    const float *bias = a.bias.data ? row_of<float>(a.bias, r) + v0 : nullptr;
    const float *noise = a.noise.data && a.choice ? row_of<float>(a.noise, r) + v0 : nullptr;
    float add[C][N];
    if (bias) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = (c * Threads + tid) * N;
            if (e < whole) load_floats(bias, e, add[c]);
        }
    }
    int32_t L = 0;
    if (History) {
        constexpr int Held = Threads == 64 ? 8 : Threads == 1024 ? 2 : 4;     // ids a thread takes in the first round trip
        int32_t id[Held];
        float held[Held];
        const uint32_t hrow = row_index(a.history, r);
        load_ids<Threads, Held>(a.history, hrow, 0, id);
        L = live_history(a, r);
        const RowRates rate = rates_of(a, r);
#pragma unroll
        for (int i = 0; i < Tile; i += 4 * Threads)
            *reinterpret_cast<u32x4 *>(&s_seen[i + 4 * tid]) = u32x4{kUnseen, kUnseen, kUnseen, kUnseen};
        __syncthreads();
        if (L > 0) {
#pragma unroll
            for (int h = 0; h < Held; ++h) {
                id[h] = tid + h * Threads < L && id[h] >= v0 && id[h] - v0 < n ? id[h] - v0 : -1;
                if (id[h] >= 0) held[h] = static_cast<float>(logits[id[h]]);
            }
#pragma unroll
            for (int h = 0; h < Held; ++h)
                if (id[h] >= 0 && atomicAdd(&s_seen[id[h]], 1u) != kUnseen) id[h] = -1;    // another's
            uint64_t mine = 0;      // of the ids beyond those held, which this thread counted first
            for (int32_t from = Held * Threads, k = 0; from < L; from += Held * Threads, k += Held) {
                int32_t more[Held];
                load_ids<Threads, Held>(a.history, hrow, from, more);
#pragma unroll
                for (int h = 0; h < Held; ++h) {
                    const int32_t e = more[h] >= v0 ? more[h] - v0 : n;
                    if (from + tid + h * Threads < L && e < n && atomicAdd(&s_seen[e], 1u) == kUnseen && k < 64) mine |= uint64_t(1) << (k + h);
                }
            }
            __syncthreads();
            if (L <= (Held + 64) * Threads) {
#pragma unroll
                for (int h = 0; h < Held; ++h)
                    if (id[h] >= 0) s_seen[id[h]] = seen_bits(penalise(a, rate, held[h], s_seen[id[h]] + 1));
                for (; mine; mine &= mine - 1) {
                    const int32_t i = tid + (Held + __builtin_ctzll(mine)) * Threads;
                    const int32_t e = load_id(a.history, hrow, i, a.vocab) - v0;
                    s_seen[e] = seen_bits(penalise(a, rate, static_cast<float>(logits[e]), s_seen[e] + 1));
                }
            } else {
                for (int e = tid; e < n; e += Threads)
                    if (s_seen[e] != kUnseen)
                        s_seen[e] = seen_bits(penalise(a, rate, static_cast<float>(logits[e]), s_seen[e] + 1));
            }
            __syncthreads();
        }
    }
    O *out = reinterpret_cast<O *>(a.out) + static_cast<int64_t>(r) * a.out_stride + v0;
    Best best = {-INFINITY, INT32_MAX};
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = (c * Threads + tid) * N;
        if (e < whole) {
            float x[N], g[N];
            if (noise) load_floats(noise, e, g);
            for (int j = 0; j < N; ++j) x[j] = entry<T>(raw[c], j);
            if (History && L > 0) {
                for (int j = 0; j < N; ++j) {
                    const uint32_t seen = s_seen[e + j];
                    x[j] = seen != kUnseen ? __uint_as_float(seen) : x[j];
                }
            }
            if (bias)
                for (int j = 0; j < N; ++j) x[j] = x[j] + add[c][j];
            if (a.inv_temperature.data)
                for (int j = 0; j < N; ++j) x[j] = x[j] * inv_t;
            if (mask) mask_entries(x, chunk_bits<T>(bytes[c]));
            if (a.out) store_chunk<true>(out, e, x);
            if (noise)
                for (int j = 0; j < N; ++j) x[j] = x[j] + g[j];
            if (a.choice)
                for (int j = 0; j < N; ++j)
                    if (x[j] > best.value) best = {x[j], e + j};
        }
    }
    if (rest < n) {
        if (History && L > 0 && s_seen[rest] != kUnseen) x_rest = __uint_as_float(s_seen[rest]);
        if (bias) x_rest = x_rest + bias[rest];
        if (a.inv_temperature.data) x_rest = x_rest * inv_t;
        if (!allowed(mask, rest)) x_rest = -INFINITY;
        if (a.out) out[rest] = static_cast<O>(x_rest);
        if (noise) x_rest = x_rest + noise[rest];
        if (x_rest > best.value) best = {x_rest, rest};
    }
    if (a.choice) {
        best = block_best<Threads>(best);
        if (tid == 0) {
            if (best.at != INT32_MAX) best.at += v0;
            if (pieces.parts == 1) store_choice(a, r, best);
            else parts[static_cast<int64_t>(r) * pieces.parts + part] = best;
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
// neighbouring rows in one piece, and U rows a lane, whose loads are in flight together (2^21 rows of 16 with
// noise: 30 us, 4.5 TB/s; bound by latency: waves wait 60 % of their time, vector instructions take 20 us of
// it).  The choice is the group's maximum, then the least index that has it.  The history (short: see small_rows) is compared
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
                const RowRates rate = rates_of(a, r[u]);
                for (int j = 0; j < 4; ++j) x[u][j] = n[j] ? penalise(a, rate, x[u][j], n[j]) : x[u][j];
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
        for (int u = 0; u < U; ++u) load_floats_once(reinterpret_cast<const float *>(row_at(g.noise, r[u])), v, g.vocab, f[u]);
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
template <int Threads>
__global__ void __launch_bounds__(Threads) choose_kernel(AdjustArgs a, int64_t first, int32_t tiles, const Best *parts) {
    const uint32_t r = static_cast<uint32_t>(first + blockIdx.x);
    Best best = {-INFINITY, INT32_MAX};
    for (int32_t t = threadIdx.x; t < tiles; t += Threads) best = better(best, parts[static_cast<int64_t>(r) * tiles + t]);
    best = block_best<Threads>(best);
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

// A row's tiles: one of 2,048 entries by a wave; longer rows of 4,096 by 256 threads (2 x 2^20 entries: 5.7 us,
// tiles of 2,048 by single waves 7.7).  A tile looks through its row's whole history, so a long one wants more
// threads and fewer tiles: past 512 ids a row of a wave's goes to 256 threads (12 rows of 650 with 6,707 ids: 11.5 us,
// 22 by a wave), past 2,048 every row but those below to 512 threads with tiles of 8,192 (12 rows of 650: 9.1; 300 rows of 7,000 with
// 4,000 ids: 10, 18 by 256 threads; 1,000 x 32,000 bf16 with up to 4,096 ids: 48 against 60, with 8,192 ids 66
// against 86; 333 x 100,003 fp16: 56 against 57, 69 against 75; one row of 2^20 13 against 16; the other way only where
// many rows fill little of a tile: 1,112 rows of 992 with 7,467 ids 18, 16 by 256 threads).
constexpr int kWaveTile = 2048, kTile = 4096, kLongTile = 8192;
constexpr int kShortHistory = 512, kLongHistory = 2048;      // a wave takes 512 ids at once

// A choice from rows of up to 16,384 entries by 512 threads, or few of up to 32,768 by 1,024: a workgroup per row
// needs neither the second launch nor a workspace (one row of 32,768: 10.5 us of the calling thread's time
// against 16; 300 rows of 8,305: 7.3 us against 12; 3,000 rows of 5,000 with 200 ids 29 against 25).
constexpr int kRowTile = 32768;

constexpr int kMiddleTile = 16384;

bool whole_rows(int64_t rows, int64_t vocab) { return vocab > kTile && (vocab <= kMiddleTile || (vocab <= kRowTile && rows <= 256)); }

int64_t tiles_of(int64_t vocab, int tile) { return (vocab + tile - 1) / tile; }

struct AdjustLaunch {
    const AdjustArgs &a;
    Best *parts;
    hipStream_t st;

    template <typename T, typename O, int Threads, int PerThread>
    void tiles() const {
        const int32_t n = static_cast<int32_t>(tiles_of(a.vocab, Threads * PerThread));
        in_pieces(a.rows, n, [&](uint32_t first, unsigned count, const Pieces &pieces) {
            if (a.history.data)
                hipLaunchKernelGGL((adjust_tile_kernel<T, O, Threads, PerThread, true>), dim3(count), dim3(Threads), 0, st, a, first, pieces, parts);
            else
                hipLaunchKernelGGL((adjust_tile_kernel<T, O, Threads, PerThread, false>), dim3(count), dim3(Threads), 0, st, a, first, pieces, parts);
        });
        if (a.choice && n > 1)
            in_launches(a.rows, [&](int64_t first, unsigned count) {
                if (n <= 256) hipLaunchKernelGGL((choose_kernel<64>), dim3(count), dim3(64), 0, st, a, first, n, parts);
                else hipLaunchKernelGGL((choose_kernel<256>), dim3(count), dim3(256), 0, st, a, first, n, parts);
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
        const int32_t ids = a.history.data ? a.history.cols : 0;
        if (a.vocab <= kWaveTile && ids <= kShortHistory) tiles<T, O, 64, 32>();
        else if (ids > kLongHistory && a.vocab <= kLongTile) tiles<T, O, 512, 16>();
        else if (a.choice && whole_rows(a.rows, a.vocab) && a.vocab <= kMiddleTile) tiles<T, O, 512, 32>();
        else if (a.choice && whole_rows(a.rows, a.vocab)) tiles<T, O, 1024, 32>();
        else if (ids > kLongHistory) tiles<T, O, 512, 16>();
        else tiles<T, O, 256, 16>();
    }
};

// Workspace bytes of a call: the best entry of every tile of rows of several (with the smaller tiles).
int64_t adjust_bytes(int64_t rows, int64_t vocab) {
    return vocab <= kTile || whole_rows(rows, vocab) ? 0 : rows * tiles_of(vocab, kTile) * static_cast<int64_t>(sizeof(Best));
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
    if (history && history->cols > kMaxHistory)
        return fail(EMO_ERR_INVALID_ARGUMENT, "history has %lld columns, outside [0, 2^30]", (long long)history->cols);
    if (choice && choice->dtype == EMO_U8 && vocab > 255)
        return fail(EMO_ERR_INVALID_ARGUMENT, "a choice among %lld entries does not fit a byte (255 is none)", (long long)vocab);
    Checker c{rows};
    AdjustArgs a = {};
    a.rows = static_cast<uint32_t>(rows);
    a.vocab = static_cast<int32_t>(vocab);
    a.logits = c.take("logits", logits, kFloats, vocab, true, false);
    const int of = c.last;
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
    const int twin = c.last;
    const Mat ch = c.take("choice", choice, kIndices, 1, false, true);
    if (rows > 0 && choice) c.workspace(workspace, workspace_bytes, adjust_bytes(rows, vocab));
    s = c.apart(twin, of);
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
