// Distillation of logits from a teacher's top entries (emo_distill_forward, _backward, _step).
#include "emo_logits.h"

#include <algorithm>

namespace {

struct DistillArgs {
    uint32_t rows;
    int32_t vocab;
    int32_t entries;        // K
    float tau;              // temperature
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

// Sum (or maximum) over the workgroup, to every thread, in a fixed order; s_red has a slot per wave.
template <int Threads, bool Max>
__device__ __forceinline__ float block_reduce(float x, float *s_red) {
    x = Max ? wave_max(x) : wave_sum(x);
    if constexpr (Threads > 64) {
        __syncthreads();
        if (threadIdx.x % 64 == 0) s_red[threadIdx.x / 64] = x;
        __syncthreads();
        x = s_red[0];
        for (int w = 1; w < Threads / 64; ++w) x = Max ? fmaxf(x, s_red[w]) : x + s_red[w];
    }
    return x;
}

// The hardware's 2^x: within a unit in the last place, 0 below 2^-126.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's teacher in LDS, K places each: the entry's id (-1: does not count), its probability, the logit at
// the id, and the probability summed over equal ids.
struct Teacher {
    int32_t *id;
    float *p, *x, *sum;
};
// Floats of LDS that it takes.
__host__ __device__ constexpr int teacher_floats(int K) { return (K + 3) / 4 * 4 * 4; }

__device__ __forceinline__ Teacher teacher_in(float4 *lds, int K) {
    const int places = (K + 3) / 4 * 4;
    float *f = reinterpret_cast<float *>(lds);
    return {reinterpret_cast<int32_t *>(lds), f + places, f + 2 * places, f + 3 * places};
}

// Loads a row's teacher and makes its probabilities, by one wave (the others stream meanwhile): ids outside
// [lo, hi) count for the probabilities, but their logits are not read.  True if any entry counts.
template <typename T>
__device__ __forceinline__ bool load_teacher(const DistillArgs &a, uint32_t r, const T *logits, const uint32_t *mask, int64_t lo,
                                             int64_t hi, const Teacher &t) {
    const int K = a.entries, lane = threadIdx.x % 64;
    const uint32_t irow = row_index(a.ids, r), trow = row_index(a.teacher, r);
    float tm = -INFINITY;
    constexpr int Held = 2;     // 128 entries a round trip
    for (int from = 0; from < K; from += 64 * Held) {
        int32_t id[Held];
        float v[Held], x[Held];
        uint32_t open[Held];
        load_ids<64, Held>(a.ids, irow, from, id);
        load_values<64, Held>(a.teacher, trow, from, v);
#pragma unroll
        for (int h = 0; h < Held; ++h) {
            const bool counts = id[h] >= 0 && id[h] < a.vocab;
            open[h] = counts ? 1u : 0u;
            if (counts && mask) open[h] = mask[id[h] >> 5] >> (id[h] & 31);
            if (id[h] >= lo && id[h] < hi) x[h] = static_cast<float>(logits[id[h]]);
        }
#pragma unroll
        for (int h = 0; h < Held; ++h) {
            const int k = from + h * 64 + lane;
            if (k >= K) continue;
            if (v[h] == -INFINITY || !(open[h] & 1u)) id[h] = -1;
            t.id[k] = id[h];
            t.p[k] = v[h];
            t.x[k] = x[h];
            if (id[h] >= 0) tm = fmaxf(tm, fmaxf(v[h], -3.4028235e38f));      // a NaN that counts is no -infinity
        }
    }
    for (int k = K + lane; k < (K + 3) / 4 * 4; k += 64) t.id[k] = -1;
    tm = wave_max(tm);
    float total = 0.f;
    for (int k = lane; k < K; k += 64) {
        const float e = t.id[k] >= 0 ? exp2_fast((t.p[k] - tm) * a.log2e_tau) : 0.f;
        t.p[k] = e;
        total += e;
    }
    total = wave_sum(total);
    for (int k = lane; k < K; k += 64) t.p[k] = t.p[k] / total;
    return tm > -INFINITY;
}

// The probabilities of equal ids in [lo, hi) summed in the list's order: sum[k] at the first entry of an id,
// -1 at its others.  K comparisons an entry, four a step, by as many threads as there are entries.
template <int Threads>
__device__ __forceinline__ void sum_equal_ids(const Teacher &t, int K, int64_t lo, int64_t hi) {
    for (int k = threadIdx.x; k < K; k += Threads) {
        const int32_t id = t.id[k];
        if (id < 0 || id < lo || id >= hi) {
            t.sum[k] = -1.f;
            continue;
        }
        float sum = 0.f;
        bool first = true;
        for (int i = 0; i < K; i += 4) {
            const int4 other = *reinterpret_cast<const int4 *>(t.id + i);
            const float4 p = *reinterpret_cast<const float4 *>(t.p + i);
            sum += other.x == id ? p.x : 0.f;
            sum += other.y == id ? p.y : 0.f;
            sum += other.z == id ? p.z : 0.f;
            sum += other.w == id ? p.w : 0.f;
            first = first && !((other.x == id && i < k) || (other.y == id && i + 1 < k) || (other.z == id && i + 2 < k));
            first = first && !(other.w == id && i + 3 < k);
        }
        t.sum[k] = first ? sum : -1.f;
    }
}

// A row's probabilities by entry, for the rows a wave takes: a table in LDS of `n` floats and tags to share it
// out.  64 entries of the list at a time; of those with equal ids (or equal tags) the lowest lane adds to the
// table, then the next: the list's order, at as many turns as an id stands among the 64.  (Comparing all ids
// bounded rows of few entries and long lists: 5,985 rows of 86 with 128 entries took 24 us.)
constexpr int kTags = 256;

// Whether a wave's row has the table: clearing and reading it has to be worth the comparisons (64 entries of the
// list: even at rows of 1,000; at 2,000 the table costs 1.5 us more).
__host__ __device__ constexpr bool by_table(int threads, int vocab, int K) { return threads == 64 && vocab <= 16 * K; }

__device__ __forceinline__ void gather_probabilities(const Teacher &t, int K, int n, volatile float *table, volatile uint32_t *tags) {
    const int lane = threadIdx.x % 64;
    for (int i = lane; i < n; i += 64) table[i] = 0.f;
    for (int i = lane; i < kTags; i += 64) tags[i] = ~0u;
    for (int from = 0; from < K; from += 64) {
        const int32_t id = from + lane < K ? t.id[from + lane] : -1;
        const float p = id >= 0 ? t.p[from + lane] : 0.f;
        volatile uint32_t *tag = tags + (id & (kTags - 1));
        bool pending = id >= 0;
        while (__any(pending)) {
            if (pending) {
                atomicMin(const_cast<uint32_t *>(tag), static_cast<uint32_t>(lane));
                if (*tag == static_cast<uint32_t>(lane)) {
                    table[id] = table[id] + p;
                    *tag = ~0u;
                    pending = false;
                }
            }
        }
    }
}

// The loss, by one wave: the entries' distances below the row's logarithm of sums, in units of the logits, so that
// one of the lowest value's size is no infinity below a temperature of 1.
__device__ __forceinline__ float teacher_loss(const DistillArgs &a, const Teacher &t, float m, float s) {
    const float log_s = logf(s) * a.tau;
    float loss = 0.f;
    for (int k = threadIdx.x % 64; k < a.entries; k += 64)
        if (t.id[k] >= 0 && t.p[k] != 0.f) loss += t.p[k] * (log_s - (t.x[k] - m));
    return wave_sum(loss) * a.tau;
}

__device__ __forceinline__ void store_stats(const DistillArgs &a, uint32_t r, float m, float s) {
    float *st = reinterpret_cast<float *>(a.stats_out) + static_cast<int64_t>(r) * a.stats_stride;
    st[0] = m;
    st[1] = s;
}

__device__ __forceinline__ void store_loss(const DistillArgs &a, uint32_t r, float loss) {
    reinterpret_cast<float *>(a.loss)[static_cast<int64_t>(r) * a.loss_stride] = loss;
}

// The statistics of one thread's entries so far: the greatest and the sum of exponentials below it.
struct Running {
    float m = -INFINITY, s = 0.f;
};

// Where exponents are measured from: the maximum, or 0 if there is none.
__device__ __forceinline__ float origin(float m) { return m == -INFINITY ? 0.f : m; }

// The compiler forgets what it knows of the chunks: else it keeps every entry as a float from one pass over
// them to the next, twice the registers of 2-byte types (and spills those of long rows), to save the
// conversion (a shift).
template <int C>
__device__ __forceinline__ void anew(u32x4 (&raw)[C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) asm volatile("" : "+v"(raw[c]));
}

// Adds the entries of C chunks and one more: one maximum and one change of origin for all of them.  A chunk's
// exponentials are summed by themselves, then the chunks, then these sums: a row's additions follow each other by
// these few steps, where one running sum rounded each entry at the size of all before (131,072 equal entries by
// 256 threads: 6e-6 of s, now 2e-7).
template <typename T, int C>
__device__ __forceinline__ void add_entries(Running &run, u32x4 (&raw)[C], float x, float log2e_tau) {
    constexpr int N = kChunk<T>;
    float m = fmaxf(run.m, x);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        for (int j = 0; j < N; ++j) m = fmaxf(m, entry<T>(raw[c], j));
        __builtin_amdgcn_sched_barrier(0);      // a chunk at a time: see anew
    }
    anew(raw);
    const float o = origin(m);
    const float before = run.s * exp2_fast((run.m - o) * log2e_tau);
    float s = exp2_fast((x - o) * log2e_tau);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float sum = exp2_fast((entry<T>(raw[c], 0) - o) * log2e_tau);
        for (int j = 1; j < N; ++j) sum += exp2_fast((entry<T>(raw[c], j) - o) * log2e_tau);
        s += sum;
        __builtin_amdgcn_sched_barrier(0);
    }
    anew(raw);
    s += before;
    asm volatile("" : "+v"(s));     // summed here, not where it is read: the exponents of all entries would live until then
    run = {m, s};
}

// The workgroup's statistics, to every thread.
template <int Threads>
__device__ __forceinline__ Running block_stats(const Running &run, float log2e_tau, float *s_red) {
    const float m = block_reduce<Threads, true>(run.m, s_red);
    const float s = block_reduce<Threads, false>(run.s * exp2_fast((run.m - origin(m)) * log2e_tau), s_red);
    return {m, s};
}

// What a workgroup holds of a row: n entries from v0 on, those of whole chunks 16 bytes a lane, the rest (fewer
// than a chunk) an entry a lane.  Masked entries are -infinity.  Once: a hint that the logits are not read again.  The
// forward pass has it (2,048 x 131,072 bf16: 92 us against 103 without; 1,024 x 50,021 fp32 42 against 46; rows that the
// caches hold from call to call lose: 4,096 x 8,000 bf16 22 against 19), the backward pass has not (183 us against 190
// with it; 88 against 83; 32 against 36).
template <typename T, int Threads, int C, bool Once>
struct Piece {
    static constexpr bool Early = C <= 8;       // longer rows have no registers to hold the mask's bytes meanwhile: LDS does
    u32x4 raw[C];
    uint32_t bytes[C];
    float x;            // this lane's entry of the rest, or -infinity

    __device__ __forceinline__ void load(const T *logits, const uint32_t *mask, int32_t n) {
        const int32_t whole = n / kChunk<T> * kChunk<T>, e = whole + static_cast<int32_t>(threadIdx.x);
        load_chunks<T, Threads, C, Once>(logits, whole, raw);
        x = -INFINITY;
        if (e < n && allowed(mask, e)) x = static_cast<float>(logits[e]);
        if (Early && mask) load_mask<T, Threads, C>(mask, whole, bytes);
    }

    // `n` as in load; `staged`: the mask's words in LDS, where the bytes were not loaded.
    __device__ __forceinline__ void apply(const uint32_t *mask, const uint32_t *staged, int32_t n) {
        if (!mask) return;
        if (!Early) load_mask<T, Threads, C>(staged, n / kChunk<T> * kChunk<T>, bytes);
#pragma unroll
        for (int c = 0; c < C; ++c) mask_chunk<T>(raw[c], chunk_bits<T>(bytes[c]));
    }
};

// Forward: a workgroup per part of a row (`span` entries, a multiple of what it holds at once).  Bound by
// memory: the next Threads * 32 entries are loaded while these are added (2,048 x 131,072 bf16: 92 us, 5.9 TB/s,
// what a sum over 1 GiB reaches; 4,000 rows 162 us, 6.5 TB/s).  A row of one part is finished here,
// others leave their statistics to finish_kernel.
template <typename T, int Threads>
__global__ void __launch_bounds__(Threads) forward_kernel(DistillArgs a, uint32_t first, Pieces pieces, int32_t span, float2 *partial) {
    constexpr int C = 32 / kChunk<T>, Step = Threads * 32;
    extern __shared__ float4 lds[];
    __shared__ float s_red[Threads / 64];
    const int tid = threadIdx.x;
    const uint32_t local = piece_row(pieces, blockIdx.x), r = first + local, part = blockIdx.x - local * pieces.parts;
    const int32_t v0 = static_cast<int32_t>(part) * span;
    const int32_t n = min(span, a.vocab - v0);
    const T *row = row_of<T>(a.logits, r);
    const T *logits = row + v0;
    const uint32_t *row_mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
    const uint32_t *mask = row_mask ? row_mask + v0 / 32 : nullptr;
    Piece<T, Threads, C, true> now, next;
    next.load(logits, mask, min(n, Step));
    const Teacher t = teacher_in(lds, a.entries);
    bool has = false;
    if (pieces.parts == 1 && a.loss && tid < 64) has = load_teacher(a, r, row, row_mask, 0, a.vocab, t);
    Running run;
    for (int32_t at = 0; at < n; at += Step) {
        now = next;
        if (n - at > Step) next.load(logits + at + Step, mask ? mask + (at + Step) / 32 : nullptr, min(n - at - Step, Step));
        now.apply(mask, nullptr, min(n - at, Step));
        add_entries<T, C>(run, now.raw, now.x, a.log2e_tau);
    }
    run = block_stats<Threads>(run, a.log2e_tau, s_red);
    if (pieces.parts > 1) {
        if (tid == 0) partial[static_cast<int64_t>(r) * pieces.parts + part] = {run.m, run.s};
        return;
    }
    if (a.stats_out && tid == 0) store_stats(a, r, run.m, run.s);
    if (a.loss && tid < 64) {
        const float loss = has ? teacher_loss(a, t, run.m, run.s) : 0.f;
        if (tid == 0) store_loss(a, r, loss);
    }
}

// The statistics of a row's parts joined, and its loss: a wave per row.
template <typename T>
__global__ void __launch_bounds__(64) finish_kernel(DistillArgs a, int64_t first, int32_t parts, const float2 *partial) {
    extern __shared__ float4 lds[];
    const uint32_t r = static_cast<uint32_t>(first + blockIdx.x);
    const Teacher t = teacher_in(lds, a.entries);
    const uint32_t *mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
    Running run;
    for (int32_t i = threadIdx.x; i < parts; i += 64) {
        const float2 p = partial[static_cast<int64_t>(r) * parts + i];
        const float m = fmaxf(run.m, p.x), o = origin(m);
        run = {m, run.s * exp2_fast((run.m - o) * a.log2e_tau) + p.y * exp2_fast((p.x - o) * a.log2e_tau)};
    }
    run = block_stats<64>(run, a.log2e_tau, nullptr);
    if (a.stats_out && threadIdx.x == 0) store_stats(a, r, run.m, run.s);
    if (a.loss) {
        const bool has = load_teacher(a, r, row_of<T>(a.logits, r), mask, 0, a.vocab, t);
        const float loss = has ? teacher_loss(a, t, run.m, run.s) : 0.f;
        if (threadIdx.x == 0) store_loss(a, r, loss);
    }
}

// Writes the gradient of a workgroup's piece (n entries from v0 of the row on).  A wave's row may have the teacher's
// probabilities by entry in `table`; others are written over at the teacher's entries (`sum`).
// rate = scale * temperature.
template <typename T, typename O, int Threads, int C, bool Once>
__device__ __forceinline__ void write_gradient(const DistillArgs &a, const Piece<T, Threads, C, Once> &piece, const uint32_t *mask, O *grad,
                                               int32_t v0, int32_t n, bool has, float m, float s, float rate, const Teacher &t,
                                               const volatile float *table) {
    constexpr int N = kChunk<T>;
    const int tid = threadIdx.x;
    const int32_t whole = n / N * N;
    // a masked entry's exponential is 0; its product with a share that is no number has to be 0 too
    const float share = rate / s;
    const bool odd = mask && !(fabsf(share) < INFINITY);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int32_t e = (c * Threads + tid) * N;
        if (e < whole) {
            float g[N];
            for (int j = 0; j < N; ++j) g[j] = has ? share * exp2_fast((entry<T>(piece.raw[c], j) - m) * a.log2e_tau) : 0.f;
            if (Threads == 64 && table && has)
                for (int j = 0; j < N; ++j) g[j] = g[j] - rate * table[e + j];
            if (odd)
                for (int j = 0; j < N; ++j) g[j] = allowed(mask, e + j) ? g[j] : 0.f;
            store_chunk<true>(grad, e, g);
        }
    }
    if (whole + tid < n) {
        float g = share * exp2_fast((piece.x - m) * a.log2e_tau);
        if (Threads == 64 && table && has) g = g - rate * table[whole + tid];
        grad[whole + tid] = static_cast<O>(has && allowed(mask, whole + tid) ? g : 0.f);
    }
    if ((Threads == 64 && table) || !has) return;
    __syncthreads();        // the entries' own values are in memory before the teacher's go over them
    for (int k = tid; k < a.entries; k += Threads)
        if (!(t.sum[k] < 0.f))
            grad[t.id[k] - v0] = static_cast<O>(rate * (exp2_fast((t.x[k] - m) * a.log2e_tau) / s - t.sum[k]));
}

// Backward: a workgroup per tile of a row (2,048 x 131,072 bf16: 183 us, 5.9 TB/s; bound by memory).
template <typename T, typename O, int Threads>
__global__ void __launch_bounds__(Threads) backward_kernel(DistillArgs a, uint32_t first, Pieces pieces) {
    constexpr int C = 32 / kChunk<T>, Tile = Threads * 32;
    extern __shared__ float4 lds[];
    __shared__ int s_has;
    const int tid = threadIdx.x;
    const uint32_t local = piece_row(pieces, blockIdx.x), r = first + local;
    const int32_t v0 = static_cast<int32_t>(blockIdx.x - local * pieces.parts) * Tile;
    const int32_t n = min(Tile, a.vocab - v0);
    const T *row = row_of<T>(a.logits, r);
    const uint32_t *row_mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
    const uint32_t *mask = row_mask ? row_mask + v0 / 32 : nullptr;
    Piece<T, Threads, C, false> piece;
    piece.load(row + v0, mask, n);
    const Teacher t = teacher_in(lds, a.entries);
    const int64_t hi = static_cast<int64_t>(v0) + n;
    if (tid < 64) {
        const bool has = load_teacher(a, r, row, row_mask, v0, hi, t);
        if (tid == 0) s_has = has;
    }
    const float *st = row_of<float>(a.stats, r);
    const float m = st[0], s = st[1];
    const float rate = row_value(a.scale, r, 1.f) * a.tau;
    piece.apply(mask, nullptr, n);
    __syncthreads();
    float *table = reinterpret_cast<float *>(lds) + teacher_floats(a.entries);
    const bool tabled = by_table(Threads, a.vocab, a.entries);
    if (tabled) gather_probabilities(t, a.entries, n, table, reinterpret_cast<uint32_t *>(table) + n);
    else sum_equal_ids<Threads>(t, a.entries, v0, hi);
    O *grad = reinterpret_cast<O *>(a.grad) + static_cast<int64_t>(r) * a.grad_stride + v0;
    write_gradient(a, piece, mask, grad, v0, n, s_has != 0, m, s, rate, t, tabled ? table : nullptr);
}

// Loss and gradient of rows that fit a workgroup's registers: read once, written once (8,192 x 32,768 bf16:
// 197 us, 5.5 TB/s; the forward and the backward kernel one after the other take half as long again).
template <typename T, typename O, int Threads, int PerThread>
__global__ void __launch_bounds__(Threads) step_kernel(DistillArgs a, int64_t first) {
    constexpr int C = PerThread / kChunk<T>;
    extern __shared__ float4 lds[];
    __shared__ float s_red[Threads / 64];
    __shared__ int s_has;
    const int tid = threadIdx.x;
    const uint32_t r = static_cast<uint32_t>(first + blockIdx.x);
    const T *logits = row_of<T>(a.logits, r);
    const uint32_t *mask = a.mask.data ? row_of<uint32_t>(a.mask, r) : nullptr;
    // The teacher first, by one wave: loads return in order, so behind the row's it would wait for all of them.
    // The other waves' rows are on their way meanwhile, and still while equal ids are summed.
    const Teacher t = teacher_in(lds, a.entries);
    if (tid < 64) {
        const bool has = load_teacher(a, r, logits, mask, 0, a.vocab, t);
        if (tid == 0) s_has = has;
        asm volatile("" ::: "memory");
    }
    using Held = Piece<T, Threads, C, true>;
    Held piece;
    constexpr int Words = Held::Early ? 1 : PerThread / 32;
    __shared__ uint32_t s_mask[Held::Early ? 1 : Words * Threads];
    const int32_t all_words = (a.vocab + 31) / 32;
    if (!Held::Early && mask) {
        uint32_t words[Words];
#pragma unroll
        for (int i = 0; i < Words; ++i)
            if (tid + i * Threads < all_words) words[i] = mask[tid + i * Threads];
        piece.load(logits, mask, a.vocab);
#pragma unroll
        for (int i = 0; i < Words; ++i)
            if (tid + i * Threads < all_words) s_mask[tid + i * Threads] = words[i];
    } else {
        piece.load(logits, mask, a.vocab);
    }
    const float rate = row_value(a.scale, r, 1.f) * a.tau;
    __syncthreads();
    float *table = reinterpret_cast<float *>(lds) + teacher_floats(a.entries);
    const bool tabled = by_table(Threads, a.vocab, a.entries);
    if (tabled) gather_probabilities(t, a.entries, a.vocab, table, reinterpret_cast<uint32_t *>(table) + a.vocab);
    else sum_equal_ids<Threads>(t, a.entries, 0, a.vocab);
    piece.apply(mask, s_mask, a.vocab);
    Running run;
    add_entries<T, C>(run, piece.raw, piece.x, a.log2e_tau);
    run = block_stats<Threads>(run, a.log2e_tau, s_red);
    const bool has = s_has != 0;
    if (a.loss && tid < 64) {
        const float loss = has ? teacher_loss(a, t, run.m, run.s) : 0.f;
        if (tid == 0) store_loss(a, r, loss);
    }
    anew(piece.raw);
    O *grad = reinterpret_cast<O *>(a.grad) + static_cast<int64_t>(r) * a.grad_stride;
    write_gradient(a, piece, mask, grad, 0, a.vocab, has, run.m, run.s, rate, t, tabled ? table : nullptr);
}

// Rows of at most 64 entries: 64 rows a workgroup, in two phases.  The teacher's: a lane per row and a wave per
// slice of the list, so that level bytes [K][rows] come 64 to a load; each lane adds its slice's weights to
// its row's table in LDS in the list's order (no two lanes share a table: a fixed order without comparing
// all ids with each other; reads and stores four at a time, as LDS's own float additions took 0.3 us each).  The student's: a group of 2^lg
// lanes per row, four entries a lane.
struct SmallArgs {
    int32_t lg, vocab, entries;
    uint32_t rows;
    float tau, log2e_tau;
    uint32_t id_step, teacher_step;     // bytes from one entry to the next
    Rows logits, ids, teacher, mask, scale, stats;     // from a 32-byte border on: loaded 8 words at once (a step of 65,536 x 16 0.2 us less)
    int32_t id_type, teacher_type;
    char *loss, *stats_out, *grad;
    uint32_t loss_stride, stats_stride, grad_stride;    // bytes
};

constexpr int kSmallRows = 64;

// Loads entries k to k + Batch of a row's list, those from k1 on repeating the last: get(i, address) for each, in
// flight together, at a scalar address plus the row's 32-bit offset.  The scalar part is opaque, or the
// compiler adds the row's offset first and multiplies in vector registers, at a quarter of their rate.
template <int Batch, typename F>
__device__ __forceinline__ void small_entries(const char *list, uint32_t row, uint32_t step, int k, int k1, const F &get) {
    const char *p = list + static_cast<uint64_t>(static_cast<uint32_t>(k)) * step;
#pragma unroll
    for (int i = 0; i < Batch; ++i) {
        const uint64_t here = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(here));
        const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(here >> 32));
        p = reinterpret_cast<const char *>(static_cast<uint64_t>(hi) << 32 | lo);
        get(i, p + row);
        p += k + i + 1 < k1 ? step : 0;
    }
}

// An id that is no index is 2^31 - 1 or more.  The type is looked at once: a branch an entry would wait for each.
template <int Batch>
__device__ __forceinline__ void small_ids(const char *ids, uint32_t row, uint32_t step, int32_t type, int k, int k1, uint32_t (&id)[Batch]) {
    if (type == EMO_U8) {
        small_entries<Batch>(ids, row, step, k, k1, [&](int i, const char *p) { id[i] = *reinterpret_cast<const uint8_t *>(p); });
    } else if (type == EMO_I32) {
        small_entries<Batch>(ids, row, step, k, k1, [&](int i, const char *p) { id[i] = *reinterpret_cast<const uint32_t *>(p); });
    } else {
        uint64_t wide[Batch];
        small_entries<Batch>(ids, row, step, k, k1, [&](int i, const char *p) { wide[i] = *reinterpret_cast<const uint64_t *>(p); });
#pragma unroll
        for (int i = 0; i < Batch; ++i) id[i] = static_cast<uint32_t>(wide[i] < 0x7fffffffu ? wide[i] : 0x7fffffffu);
    }
}

template <int Batch>
__device__ __forceinline__ void small_floats(const char *from, uint32_t row, uint32_t step, int32_t type, int k, int k1, float (&t)[Batch]) {
    if (type == EMO_F32) {
        small_entries<Batch>(from, row, step, k, k1, [&](int i, const char *p) { t[i] = *reinterpret_cast<const float *>(p); });
    } else {
        uint16_t half[Batch];
        small_entries<Batch>(from, row, step, k, k1, [&](int i, const char *p) { half[i] = *reinterpret_cast<const uint16_t *>(p); });
#pragma unroll
        for (int i = 0; i < Batch; ++i)
            t[i] = type == EMO_F16 ? static_cast<float>(__builtin_bit_cast(_Float16, half[i])) : __uint_as_float(static_cast<uint32_t>(half[i]) << 16);
    }
}

template <typename T, typename O, int Slices, int Most, bool Forward, bool Backward>
__global__ void __launch_bounds__(kThreads) small_kernel(SmallArgs a, int64_t first) {
    constexpr int Width = Most + 1, Batch = 16;     // a table's rows start in different banks
    constexpr int Turns = Most / 16;                // rows that a group of lanes takes
    __shared__ alignas(16) float s_table[Slices * kSmallRows * Width];
    __shared__ float s_max[Slices][kSmallRows], s_sum[Slices][kSmallRows];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const uint32_t r0 = static_cast<uint32_t>((first + blockIdx.x) * kSmallRows);
    const uint32_t rows = min(a.rows - r0, static_cast<uint32_t>(kSmallRows));
    const bool teaching = (Backward || a.loss) && a.entries > 0;

    // the student's loads are in flight over the teacher's phase
    const int v = (tid & ((1 << a.lg) - 1)) * 4;
    const bool mine = v < a.vocab;
    float x[Turns][4], m[Turns], s[Turns], rate[Turns];
    uint32_t bits[Turns];
#pragma unroll
    for (int u = 0; u < Turns; ++u) {
        const uint32_t local = u * (kThreads >> a.lg) + (tid >> a.lg);
        const uint32_t r = r0 + min(local, rows - 1);       // rows past the last: the last again
        for (int j = 0; j < 4; ++j) x[u][j] = -INFINITY;
        bits[u] = 0;
        if (mine) {
            load_four(reinterpret_cast<const T *>(row_at(a.logits, r)), v, a.vocab, x[u]);
            bits[u] = mask_bits<4>(a.mask.data ? reinterpret_cast<const uint32_t *>(row_at(a.mask, r)) : nullptr, v, a.vocab);
        }
        if (Backward) rate[u] = a.scale.data ? *reinterpret_cast<const float *>(row_at(a.scale, r)) : 1.f;
        if (!Forward) {
            m[u] = reinterpret_cast<const float *>(row_at(a.stats, r))[0];
            s[u] = reinterpret_cast<const float *>(row_at(a.stats, r))[1];
        }
    }

    if (teaching) {
        const bool slice = wave < Slices;       // the barriers stand outside the branches
        const uint32_t r = r0 + min(static_cast<uint32_t>(lane), rows - 1);
        const int span = (a.entries + Slices - 1) / Slices, k0 = wave * span, k1 = slice ? min(a.entries, k0 + span) : 0;
        const uint32_t id_row = row_index32(a.ids, r) * a.ids.stride, teacher_row = row_index32(a.teacher, r) * a.teacher.stride;
        using Open = typename std::conditional<Most <= 32, uint32_t, uint64_t>::type;
        Open open = ~Open(0);       // the ids that count
        if (a.mask.data) {
            const uint32_t *words = reinterpret_cast<const uint32_t *>(row_at(a.mask, r));
            open = words[0];
            if (Most > 32 && a.vocab > 32) open |= static_cast<Open>(static_cast<uint64_t>(words[1]) << 32);
        }
        if (a.vocab < static_cast<int>(8 * sizeof(Open))) open &= (Open(1) << a.vocab) - 1;
        uint32_t id[Batch];
        float t[Batch];     // -infinity where the entry does not count; its id then is the place behind the table's row
        const auto load = [&](int k) {
            small_ids<Batch>(a.ids.data, id_row, a.id_step, a.id_type, k, k1, id);
            small_floats<Batch>(a.teacher.data, teacher_row, a.teacher_step, a.teacher_type, k, k1, t);
#pragma unroll
            for (int i = 0; i < Batch; ++i) {
                const bool counts = id[i] < 8 * sizeof(Open) && k + i < k1 && (open >> (id[i] % (8 * sizeof(Open))) & 1);
                t[i] = counts ? t[i] : -INFINITY;
                id[i] = counts ? id[i] : Most;
            }
        };
        for (int i = tid * 4; i < Slices * kSmallRows * Width; i += kThreads * 4)
            *reinterpret_cast<float4 *>(s_table + i) = make_float4(0.f, 0.f, 0.f, 0.f);
        float top = -INFINITY;
        bool nan = false;
        for (int k = k0; k < k1; k += Batch) {
            load(k);
#pragma unroll
            for (int i = 0; i < Batch; ++i) {
                top = fmaxf(top, t[i]);
                nan = nan || t[i] != t[i];
            }
        }
        if (slice) s_max[wave][lane] = nan ? INFINITY : top;     // where every exponential comes out as NaN
        __syncthreads();
#pragma unroll
        for (int q = 0; q < Slices; ++q) top = fmaxf(top, s_max[q][lane]);
        top = origin(top);
        float total = 0.f;
        float *table = s_table + (wave % Slices * kSmallRows + lane) * Width;
        for (int k = k0; k < k1; k += Batch) {
            if (span > Batch) load(k);      // a slice of one batch is still there
#pragma unroll
            for (int i = 0; i < Batch; i += 4) {
                // four entries at once: the later of equal ids adds to the earlier's sum, and is stored after it
                float w[4], sum[4];
                for (int j = 0; j < 4; ++j) {
                    w[j] = exp2_fast((t[i + j] - top) * a.log2e_tau);
                    total += w[j];
                    sum[j] = table[id[i + j]];
                }
                for (int j = 0; j < 4; ++j) {
                    for (int b = 0; b < j; ++b) sum[j] = id[i + j] == id[i + b] ? sum[b] : sum[j];
                    sum[j] += w[j];
                }
                for (int j = 0; j < 4; ++j) table[id[i + j]] = sum[j];
            }
        }
        if (slice) s_sum[wave][lane] = total;
        __syncthreads();
    }

#pragma unroll
    for (int u = 0; u < Turns; ++u) {
        const uint32_t local = u * (kThreads >> a.lg) + (tid >> a.lg);
        if (local >= rows) break;       // whole groups
        const uint32_t r = r0 + local;
        for (int j = 0; j < 4; ++j) x[u][j] = bits[u] >> j & 1 ? x[u][j] : -INFINITY;
        float p[4] = {0.f, 0.f, 0.f, 0.f};
        bool has = false;
        if (teaching) {
            float total = 0.f;
#pragma unroll
            for (int q = 0; q < Slices; ++q) {
                total += s_sum[q][local];
                has = has || s_max[q][local] > -INFINITY;
            }
            if (mine && has) {
                const float share = __builtin_amdgcn_rcpf(total);
                for (int j = 0; j < 4; ++j) {
                    if (v + j >= a.vocab) continue;
#pragma unroll
                    for (int q = 0; q < Slices; ++q) p[j] += s_table[(q * kSmallRows + local) * Width + v + j];
                    p[j] = p[j] * share;
                }
            }
        }
        if (Forward) {
            m[u] = group_max(fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3])), a.lg);
            if (!(m[u] > -INFINITY)) m[u] = -INFINITY;      // a row of NaN alone
        }
        float e[4];
        for (int j = 0; j < 4; ++j) e[j] = exp2_fast((x[u][j] - origin(m[u])) * a.log2e_tau);
        if (Forward) s[u] = group_sum((e[0] + e[1]) + (e[2] + e[3]), a.lg);
        if (Forward && a.stats_out && v == 0) {
            float *to = reinterpret_cast<float *>(a.stats_out + static_cast<uint64_t>(r) * a.stats_stride);
            to[0] = m[u];
            to[1] = s[u];
        }
        if (Forward && a.loss) {
            const float log_s = 0.69314718f * __builtin_amdgcn_logf(s[u]) * a.tau;     // the hardware's log2, within a unit or so
            float loss = 0.f;
            for (int j = 0; j < 4; ++j)
                if (p[j] != 0.f) loss += p[j] * (log_s - (x[u][j] - m[u]));      // in the logits' units: see teacher_loss
            loss = group_sum(loss, a.lg) * a.tau;
            if (v == 0) *reinterpret_cast<float *>(a.loss + static_cast<uint64_t>(r) * a.loss_stride) = has ? loss : 0.f;
        }
        if (Backward && mine) {
            // a row without an entry above -infinity has no distribution
            const float share = m[u] > -INFINITY || m[u] != m[u] ? __builtin_amdgcn_rcpf(s[u]) : NAN;
            for (int j = 0; j < 4; ++j) {
                const float q = e[j] * share;
                x[u][j] = has && (bits[u] >> j & 1) ? rate[u] * a.tau * (q - p[j]) : 0.f;
            }
            store_chunk(reinterpret_cast<O *>(a.grad + static_cast<uint64_t>(r) * a.grad_stride), v, a.vocab, x[u]);
        }
    }
}

// ------------------------------------------------------------------------------ launches

// The parts of a row of the forward pass: of whole 8,192 entries, as many as bring 2,048 workgroups (8 a
// compute unit) while a row has that many.  More rows than that fill the card unsplit: split up to 4,096 workgroups,
// 2,049 rows of 131,072 bf16 took 94 us against 92, 3,000 131 against 124, 3,000 rows of 32,768 42 against 36.
struct Parts {
    int32_t parts, span;
};

Parts forward_parts(int64_t rows, int64_t vocab) {
    if (vocab <= 2048) return {1, 2048};
    const int64_t most = (vocab + 8191) / 8192;
    const int64_t want = rows >= 2048 ? 1 : std::min<int64_t>(most, (2048 + rows - 1) / std::max<int64_t>(rows, 1));
    const int64_t span = std::min<int64_t>((most + want - 1) / want * 8192, INT32_MAX / 8192 * 8192);
    return {static_cast<int32_t>((vocab + span - 1) / span), static_cast<int32_t>(span)};
}

// Rows that step_kernel takes: up to 131,072 entries of 2 bytes or 65,536 of 4 (half a compute unit's
// registers); others go by the forward and the backward kernels, and so do few of the widest, which leave
// most of the card idle (16 x 130,000 bf16: 15 us in three launches, 19 in one; 128 rows: 32 against 24).
constexpr int64_t kResident = 65536;

bool resident(int64_t rows, int64_t vocab, int32_t dtype) {
    return vocab <= kResident || (vocab <= 2 * kResident && dtype != EMO_F32 && rows > 32);
}

int64_t partial_bytes(int64_t rows, int64_t vocab) {
    const Parts p = forward_parts(rows, vocab);
    return p.parts > 1 ? rows * p.parts * static_cast<int64_t>(sizeof(float2)) : 0;
}

// Workspace bytes of a call: the statistics of the rows' parts, and those of the rows of a step in two passes.
int64_t distill_bytes(int64_t rows, int64_t vocab) {
    return partial_bytes(rows, vocab) + (vocab > kResident ? rows * static_cast<int64_t>(sizeof(float2)) : 0);
}

// Bytes from an operand's first row to its last.
int64_t extent(const Mat &m) { return m.rows > 1 ? static_cast<int64_t>(m.rows - 1) * m.row_stride * size_of(m.dtype) : 0; }

// Whether small_kernel takes the rows: of at most 64 entries, strides and the lists' extents below 4 GiB.
bool small_rows(const DistillArgs &a, int32_t grad_size, SmallArgs *s) {
    constexpr int64_t most = int64_t(1) << 32;
    const int64_t id_step = a.ids.col_stride * size_of(a.ids.dtype), teacher_step = a.teacher.col_stride * size_of(a.teacher.dtype);
    if (a.vocab > 64 || a.loss_stride * 4 >= most || a.stats_stride * 4 >= most || a.grad_stride * grad_size >= most || id_step >= most ||
        teacher_step >= most || extent(a.ids) >= most || extent(a.teacher) >= most)
        return false;
    *s = {};
    while ((4 << s->lg) < a.vocab) ++s->lg;
    s->vocab = a.vocab;
    s->entries = a.entries;
    s->rows = a.rows;
    s->tau = a.tau;
    s->log2e_tau = a.log2e_tau;
    s->id_step = static_cast<uint32_t>(id_step);
    s->teacher_step = static_cast<uint32_t>(teacher_step);
    s->id_type = a.ids.dtype;
    s->teacher_type = a.teacher.dtype;
    s->loss = a.loss;
    s->stats_out = a.stats_out;
    s->grad = a.grad;
    s->loss_stride = static_cast<uint32_t>(a.loss_stride * 4);
    s->stats_stride = static_cast<uint32_t>(a.stats_stride * 4);
    s->grad_stride = static_cast<uint32_t>(a.grad_stride * grad_size);
    return narrow(a.logits, &s->logits) && narrow(a.ids, &s->ids) && narrow(a.teacher, &s->teacher) && narrow(a.mask, &s->mask) &&
           narrow(a.scale, &s->scale) && narrow(a.stats, &s->stats);
}

// Tables of 4 slices of the list, or of 2 for rows of more than 32 entries (34 KB either way: four
// workgroups a compute unit).
template <typename T, typename O, bool Forward, bool Backward>
void launch_small(const SmallArgs &s, hipStream_t st) {
    in_launches((static_cast<int64_t>(s.rows) + kSmallRows - 1) / kSmallRows, [&](int64_t first, unsigned count) {
        if (s.vocab <= 16)
            hipLaunchKernelGGL((small_kernel<T, O, 4, 16, Forward, Backward>), dim3(count), dim3(kThreads), 0, st, s, first);
        else if (s.vocab <= 32)
            hipLaunchKernelGGL((small_kernel<T, O, 4, 32, Forward, Backward>), dim3(count), dim3(kThreads), 0, st, s, first);
        else
            hipLaunchKernelGGL((small_kernel<T, O, 2, 64, Forward, Backward>), dim3(count), dim3(kThreads), 0, st, s, first);
    });
}

unsigned teacher_lds(const DistillArgs &a) { return static_cast<unsigned>(teacher_floats(a.entries) * sizeof(float)); }

// With a wave's table of probabilities and its tags.
unsigned gradient_lds(const DistillArgs &a, int threads) {
    return teacher_lds(a) + (by_table(threads, a.vocab, a.entries) ? static_cast<unsigned>((a.vocab + kTags) * sizeof(float)) : 0u);
}

struct ForwardLaunch {
    const DistillArgs &a;
    float2 *partial;
    hipStream_t st;

    template <typename T, typename>
    void run() const {
        SmallArgs small;
        if (small_rows(a, 4, &small)) return launch_small<T, float, true, false>(small, st);
        const Parts p = forward_parts(a.rows, a.vocab);
        in_pieces(a.rows, p.parts, [&](uint32_t first, unsigned count, const Pieces &pieces) {
            if (a.vocab <= 2048)
                hipLaunchKernelGGL((forward_kernel<T, 64>), dim3(count), dim3(64), teacher_lds(a), st, a, first, pieces, p.span, partial);
            else
                hipLaunchKernelGGL((forward_kernel<T, 256>), dim3(count), dim3(256), teacher_lds(a), st, a, first, pieces, p.span, partial);
        });
        if (p.parts > 1)
            in_launches(a.rows, [&](int64_t first, unsigned count) {
                hipLaunchKernelGGL((finish_kernel<T>), dim3(count), dim3(64), teacher_lds(a), st, a, first, p.parts, partial);
            });
    }
};

struct BackwardLaunch {
    const DistillArgs &a;
    hipStream_t st;

    template <typename T, typename O, int Threads>
    void tiles() const {
        const int64_t tiles = (static_cast<int64_t>(a.vocab) + Threads * 32 - 1) / (Threads * 32);
        in_pieces(a.rows, tiles, [&](uint32_t first, unsigned count, const Pieces &pieces) {
            hipLaunchKernelGGL((backward_kernel<T, O, Threads>), dim3(count), dim3(Threads), gradient_lds(a, Threads), st, a, first, pieces);
        });
    }

    template <typename T, typename O>
    void run() const {
        SmallArgs small;
        if (small_rows(a, sizeof(O), &small)) return launch_small<T, O, false, true>(small, st);
        if (a.vocab <= 2048) tiles<T, O, 64>();
        else tiles<T, O, 256>();
    }
};

struct StepLaunch {
    const DistillArgs &a;
    hipStream_t st;

    // Whether there are more rows than the card holds workgroups of that many threads (2,048 threads a compute
    // unit; from twice as many for 4-byte types, whose 64 entries a lane take twice the registers, so that
    // fewer waves stay).  Then half the threads with 64 entries each: a row takes about as long, its latencies
    // above all, and more rows are on their way (3,000 x 9,333 bf16: 38 us against 47; 300 rows: 12.2 against 11.8; 3,000 x 9,333 fp32:
    // 54 against 61, 1,500 rows 33 against 31).
    template <typename T>
    bool more_than_held(int threads) const {
        return static_cast<int64_t>(a.rows) * threads > int64_t(256) * 2048 * (sizeof(T) == 4 ? 2 : 1);
    }

    template <typename T, typename O, int Threads, int PerThread>
    void rows() const {
        in_launches(a.rows, [&](int64_t first, unsigned count) {
            hipLaunchKernelGGL((step_kernel<T, O, Threads, PerThread>), dim3(count), dim3(Threads), gradient_lds(a, Threads), st, a, first);
        });
    }

    template <typename T, typename O>
    void run() const {
        SmallArgs small;
        if (small_rows(a, sizeof(O), &small)) return launch_small<T, O, true, true>(small, st);
        if (a.vocab <= 2048) rows<T, O, 64, 32>();
        else if (a.vocab <= 4096) more_than_held<T>(128) ? rows<T, O, 64, 64>() : rows<T, O, 128, 32>();
        else if (a.vocab <= 8192) more_than_held<T>(256) ? rows<T, O, 128, 64>() : rows<T, O, 256, 32>();
        else if (a.vocab <= 16384) more_than_held<T>(512) ? rows<T, O, 256, 64>() : rows<T, O, 512, 32>();
        else if (a.vocab <= 32768) rows<T, O, 512, 64>();
        else if constexpr (sizeof(T) == 4) rows<T, O, 1024, 64>();
        else if (a.vocab <= 65536) rows<T, O, 512, 128>();
        else rows<T, O, 1024, 128>();
    }
};

// The operands every distillation call has; the logits' range is the first.
constexpr int kLogitsRange = 0;

emo_status distill_operands(Checker &c, DistillArgs &a, int64_t rows, int64_t vocab, const emo_tensor *logits,
                            const emo_tensor *ids, const emo_tensor *teacher, float temperature, const emo_tensor *mask) {
    emo_status s = check_sizes(rows, vocab);
    if (s != EMO_OK) return s;
    if (!logits || !ids || !teacher) return fail(EMO_ERR_INVALID_ARGUMENT, "logits, ids or teacher is NULL");
    // its square and log2(e) divided by it are fp32 numbers with room
    if (!(temperature >= 0x1p-60f && temperature <= 0x1p60f))
        return fail(EMO_ERR_INVALID_ARGUMENT, "temperature must be in [2^-60, 2^60]");
    if (ids->cols < 0 || ids->cols > kMaxEntries)
        return fail(EMO_ERR_INVALID_ARGUMENT, "ids has %lld columns, outside [0, %d]", (long long)ids->cols, kMaxEntries);
    a = {};
    a.rows = static_cast<uint32_t>(rows);
    a.vocab = static_cast<int32_t>(vocab);
    a.entries = static_cast<int32_t>(ids->cols);
    a.tau = temperature;
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
    s = c.apart(-1, -1);
    if (s != EMO_OK) return s;
    if (rows == 0 || (!loss && !stats)) return emo::report(EMO_OK, "");
    a.loss = const_cast<char *>(l.data);
    a.loss_stride = l.row_stride;
    a.stats_out = const_cast<char *>(st.data);
    a.stats_stride = st.row_stride;
    by_types(a.logits.dtype, EMO_F32, ForwardLaunch{a, static_cast<float2 *>(workspace), static_cast<hipStream_t>(stream)});
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
    const int twin = c.last;
    s = c.apart(twin, kLogitsRange);
    if (s == EMO_OK) s = check_written(gradient, logits, "gradient");
    if (s != EMO_OK) return s;
    if (rows == 0) return emo::report(EMO_OK, "");
    a.grad = const_cast<char *>(g.data);
    a.grad_stride = g.row_stride;
    by_types(a.logits.dtype, g.dtype, BackwardLaunch{a, static_cast<hipStream_t>(stream)});
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
    const int twin = c.last;
    if (rows > 0) c.workspace(workspace, workspace_bytes, distill_bytes(rows, vocab));
    s = c.apart(twin, kLogitsRange);
    if (s == EMO_OK) s = check_written(gradient, logits, "gradient");
    if (s != EMO_OK) return s;
    if (rows == 0) return emo::report(EMO_OK, "");
    a.loss = const_cast<char *>(l.data);
    a.loss_stride = l.row_stride;
    a.grad = const_cast<char *>(g.data);
    a.grad_stride = g.row_stride;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (resident(rows, vocab, a.logits.dtype)) {
        by_types(a.logits.dtype, g.dtype, StepLaunch{a, st});
        return launched("emo_distill_step");
    }
    // the rows' statistics behind those of their parts
    char *kept = static_cast<char *>(workspace) + partial_bytes(rows, vocab);
    a.stats_out = kept;
    a.stats_stride = 2;
    by_types(a.logits.dtype, EMO_F32, ForwardLaunch{a, static_cast<float2 *>(workspace), st});
    a.stats = {};
    a.stats.data = kept;
    a.stats.row_stride = 2;
    a.stats.rows = a.rows;
    a.stats.dtype = EMO_F32;
    by_types(a.logits.dtype, g.dtype, BackwardLaunch{a, st});
    return launched("emo_distill_step");
}

}  // extern "C"
