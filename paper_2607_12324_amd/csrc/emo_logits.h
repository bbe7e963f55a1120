// What the calls on logits share: operands, their checks, reductions.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <numeric>
#include <type_traits>

#include "emo_internal.h"

namespace {

// ------------------------------------------------------------------------------ operands

// A checked operand.  Row r of a call reads row r % rows; data NULL: absent.
struct Mat {
    const char *data;
    int64_t row_stride, col_stride;   // elements
    uint32_t rows;
    uint32_t magic, shift;            // r / rows = mulhi(r, magic) >> shift; magic 0: see row_index
    int32_t cols;
    int32_t dtype;
};

// The operand's row that row r < 2^31 of the call reads.  With magic 0 that is r itself: the operand has
// all rows, or one with a row stride of 0.  A remainder by the compiler's division takes about 20
// instructions an operand, which bounded rows of a few entries.
__device__ __forceinline__ uint32_t row_index(const Mat &m, uint32_t r) {
    if (m.magic == 0) return r;
    return r - (__umulhi(r, m.magic) >> m.shift) * m.rows;
}

template <typename T>
__device__ __forceinline__ const T *row_of(const Mat &m, uint32_t r) {
    return reinterpret_cast<const T *>(m.data) + static_cast<int64_t>(row_index(m, r)) * m.row_stride;
}

// An operand with a row per group of lanes: its row's address is one 32-bit multiplication and addition
// (the stride in bytes below 2^32), and a kernel holds six scalar registers of it.
struct Rows {
    const char *data;
    uint32_t stride, rows, magic, shift;
};

__device__ __forceinline__ uint32_t row_index32(const Rows &m, uint32_t r) {
    return m.magic ? r - (__umulhi(r, m.magic) >> m.shift) * m.rows : r;
}

__device__ __forceinline__ const char *row_at(const Rows &m, uint32_t r) {
    return m.data + static_cast<uint64_t>(row_index32(m, r)) * m.stride;
}

// The workgroups of rows of `parts` pieces: workgroup b < 2^31 of a launch takes piece b % parts of the
// launch's row b / parts (divided as in row_index: the compiler's 64-bit division is 100 scalar
// instructions a workgroup).
struct Pieces {
    uint32_t parts, magic, shift;
};

__device__ __forceinline__ uint32_t piece_row(const Pieces &p, uint32_t b) { return p.magic ? __umulhi(b, p.magic) >> p.shift : b; }

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

// Ids `from` to from + Held * Threads of a row, as they stand, all in flight together (ids of 64 bits that do not
// fit 32 as -1; the last one again from `cols` on): the type is looked at once, a branch an id would wait for
// each.
template <int Threads, int Held>
__device__ __forceinline__ void load_ids(const Mat &m, uint32_t row, int32_t from, int32_t (&id)[Held]) {
    const int64_t base = static_cast<int64_t>(row) * m.row_stride;
    const int32_t first = from + static_cast<int32_t>(threadIdx.x % Threads);
    const auto at = [&](int h) { return base + static_cast<int64_t>(min(first + h * Threads, m.cols - 1)) * m.col_stride; };
    if (m.dtype == EMO_U8) {
#pragma unroll
        for (int h = 0; h < Held; ++h) id[h] = reinterpret_cast<const uint8_t *>(m.data)[at(h)];
    } else if (m.dtype == EMO_I32) {
#pragma unroll
        for (int h = 0; h < Held; ++h) id[h] = reinterpret_cast<const int32_t *>(m.data)[at(h)];
    } else {
        int64_t wide[Held];
#pragma unroll
        for (int h = 0; h < Held; ++h) wide[h] = reinterpret_cast<const int64_t *>(m.data)[at(h)];
#pragma unroll
        for (int h = 0; h < Held; ++h) id[h] = wide[h] == static_cast<int32_t>(wide[h]) ? static_cast<int32_t>(wide[h]) : -1;
    }
}

// Values of a row likewise.
template <int Threads, int Held>
__device__ __forceinline__ void load_values(const Mat &m, uint32_t row, int32_t from, float (&v)[Held]) {
    const int64_t base = static_cast<int64_t>(row) * m.row_stride;
    const int32_t first = from + static_cast<int32_t>(threadIdx.x % Threads);
    const auto at = [&](int h) { return base + static_cast<int64_t>(min(first + h * Threads, m.cols - 1)) * m.col_stride; };
    if (m.dtype == EMO_F32) {
#pragma unroll
        for (int h = 0; h < Held; ++h) v[h] = reinterpret_cast<const float *>(m.data)[at(h)];
    } else {
        uint16_t half[Held];
#pragma unroll
        for (int h = 0; h < Held; ++h) half[h] = reinterpret_cast<const uint16_t *>(m.data)[at(h)];
#pragma unroll
        for (int h = 0; h < Held; ++h)
            v[h] = m.dtype == EMO_F16 ? static_cast<float>(__builtin_bit_cast(_Float16, half[h])) : __uint_as_float(static_cast<uint32_t>(half[h]) << 16);
    }
}

// Entries of a row that a lane holds at once: 16 bytes of logits, loaded at any alignment of the type (rows
// of an odd count start anywhere; the hardware takes 16-byte accesses at such addresses).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2), may_alias));
template <typename T>
constexpr int kChunk = 16 / sizeof(T);

template <typename T>
__device__ __forceinline__ float entry(u32x4 raw, int j);
template <>
__device__ __forceinline__ float entry<float>(u32x4 raw, int j) { return __uint_as_float(raw[j]); }
template <>
__device__ __forceinline__ float entry<_Float16>(u32x4 raw, int j) {
    return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(raw[j >> 1] >> (j & 1) * 16)));
}
template <>
__device__ __forceinline__ float entry<__bf16>(u32x4 raw, int j) {
    return __uint_as_float(j & 1 ? raw[j >> 1] & 0xffff0000u : raw[j >> 1] << 16);
}

template <typename T>
__device__ __forceinline__ uint32_t bits_of(float x) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(x);
    else return __builtin_bit_cast(uint16_t, static_cast<T>(x));
}

// Two floats as two 16-bit values of a word, each rounded to nearest even.
template <typename T>
__device__ __forceinline__ uint32_t pack_two(float lo, float hi) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef T t2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), t2));
}

// Entry v of a row, or of a tile of a wide one, below 2^30: addressed as a scalar base and 32 bits of bytes.
template <typename P>
__device__ __forceinline__ P *at_entry(P *row, int32_t v) {
    using B = typename std::conditional<std::is_const<P>::value, const char, char>::type;
    return reinterpret_cast<P *>(reinterpret_cast<B *>(row) + static_cast<uint32_t>(v) * static_cast<uint32_t>(sizeof(P)));
}

// The whole chunk at entry v of a row; Once: a hint to the caches that it is not read again.
template <typename T, bool Once = false>
__device__ __forceinline__ u32x4 load_chunk(const T *row, int32_t v) {
    const u32x4_any *p = reinterpret_cast<const u32x4_any *>(at_entry(row, v));
    if constexpr (Once) return __builtin_nontemporal_load(p);
    else return *p;
}

// The chunks of a workgroup's thread among `whole` entries (a multiple of the chunk): chunk c is at entry
// (c * Threads + thread) * kChunk; those behind are -infinity.  No load waits for another: what a row has
// beyond whole chunks is taken by a lane an entry, apart from this (a guard per entry here costs a wait
// per chunk and, where a row fills the registers, spills).
template <typename T, int Threads, int C, bool Once = false>
__device__ __forceinline__ void load_chunks(const T *row, int32_t whole, u32x4 (&raw)[C]) {
    const uint32_t none = sizeof(T) == 4 ? 0xff800000u : bits_of<T>(-INFINITY) * 0x10001u;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int32_t e = (c * Threads + static_cast<int32_t>(threadIdx.x)) * kChunk<T>;
        raw[c] = u32x4{none, none, none, none};
        if (e < whole) raw[c] = load_chunk<T, Once>(row, e);
    }
}

// The mask's bits of those chunks, a byte each: chunk_bits takes the chunk's own.
template <typename T, int Threads, int C>
__device__ __forceinline__ void load_mask(const uint32_t *mask, int32_t whole, uint32_t (&bytes)[C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int32_t e = (c * Threads + static_cast<int32_t>(threadIdx.x)) * kChunk<T>;
        bytes[c] = 0xff;
        if (e < whole) bytes[c] = reinterpret_cast<const uint8_t *>(mask)[static_cast<uint32_t>(e) >> 3];
    }
}

template <typename T>
__device__ __forceinline__ uint32_t chunk_bits(uint32_t byte) {
    return kChunk<T> == 8 ? byte : byte >> (threadIdx.x & 1) * 4 & 0xfu;
}

// Four entries at v of a row of V, as floats (-infinity from V on).
template <typename T>
__device__ __forceinline__ void load_four(const T *row, int32_t v, int32_t V, float (&x)[4]) {
    if constexpr (sizeof(T) == 4) {
        u32x4 raw;
        if (v + 4 <= V) {
            raw = load_chunk(row, v);
        } else {
            for (int w = 0; w < 4; ++w) raw[w] = v + w < V ? reinterpret_cast<const uint32_t *>(row)[v + w] : 0xff800000u;
        }
        for (int j = 0; j < 4; ++j) x[j] = entry<T>(raw, j);
    } else {
        u32x4 raw = {0, 0, 0, 0};
        if (v + 4 <= V) {
            const auto two = *reinterpret_cast<const u32x2_any *>(row + v);
            raw[0] = two[0];
            raw[1] = two[1];
        } else {
            const uint16_t *p = reinterpret_cast<const uint16_t *>(row);
            const uint32_t none = bits_of<T>(-INFINITY);
            for (int w = 0; w < 2; ++w)
                raw[w] = (v + 2 * w < V ? p[v + 2 * w] : none) | (v + 2 * w + 1 < V ? p[v + 2 * w + 1] : none) << 16;
        }
        for (int j = 0; j < 4; ++j) x[j] = entry<T>(raw, j);
    }
}

// The floats of a whole chunk.
template <int N>
__device__ __forceinline__ void load_floats(const float *row, int32_t v, float (&f)[N]) {
    for (int i = 0; i < N; i += 4) {
        const u32x4 raw = *reinterpret_cast<const u32x4_any *>(at_entry(row, v) + i);
        for (int j = 0; j < 4; ++j) f[i + j] = __uint_as_float(raw[j]);
    }
}

// N floats at entry v of a row of V (zeros from V on).
template <int N>
__device__ __forceinline__ void load_floats(const float *row, int32_t v, int32_t V, float (&f)[N]) {
    if (v + N <= V) {
        load_floats(row, v, f);
    } else {
        for (int j = 0; j < N; ++j) f[j] = v + j < V ? row[v + j] : 0.f;
    }
}

// The same of floats that nothing reads again: they pass the caches, which keep what is.  (Noise of 2^21 rows
// of 16: 29 to 33 us against 34.)
template <int N>
__device__ __forceinline__ void load_floats_once(const float *row, int32_t v, int32_t V, float (&f)[N]) {
    if (v + N <= V) {
        for (int i = 0; i < N; i += 4) {
            const u32x4 raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any *>(at_entry(row, v) + i));
            for (int j = 0; j < 4; ++j) f[i + j] = __uint_as_float(raw[j]);
        }
    } else {
        load_floats(row, v, V, f);
    }
}

// Wide rows are written as a stream, which the caches pass on: kept, they drive out what other workgroups still
// read (256 x 131,072 bf16 adjusted: 33 us against 40; 517 x 50,021 fp32, a step: 65 against 70).
// (Two functions: a template's parameter would be the type without its alignment of 2.)
template <bool Stream>
__device__ __forceinline__ void store_words(u32x4_any *to, u32x4 raw) {
    if constexpr (Stream) __builtin_nontemporal_store(raw, to);
    else *to = raw;
}
template <bool Stream>
__device__ __forceinline__ void store_words(u32x2_any *to, u32x2 raw) {
    if constexpr (Stream) __builtin_nontemporal_store(raw, to);
    else *to = raw;
}

// A whole chunk of N values at entry v, each rounded once to the row's type.
template <bool Stream, typename O, int N>
__device__ __forceinline__ void store_chunk(O *row, int32_t v, const float (&f)[N]) {
    if constexpr (sizeof(O) == 4) {
        for (int i = 0; i < N; i += 4) {
            u32x4 raw;
            for (int j = 0; j < 4; ++j) raw[j] = __float_as_uint(f[i + j]);
            store_words<Stream>(reinterpret_cast<u32x4_any *>(at_entry(row, v) + i), raw);
        }
    } else if constexpr (N == 4) {
        const u32x2 raw = {pack_two<O>(f[0], f[1]), pack_two<O>(f[2], f[3])};
        store_words<Stream>(reinterpret_cast<u32x2_any *>(at_entry(row, v)), raw);
    } else {
        u32x4 raw;
        for (int w = 0; w < 4; ++w) raw[w] = pack_two<O>(f[2 * w], f[2 * w + 1]);
        store_words<Stream>(reinterpret_cast<u32x4_any *>(at_entry(row, v)), raw);
    }
}

// N values at entry v of a row of V.
template <typename O, int N>
__device__ __forceinline__ void store_chunk(O *row, int32_t v, int32_t V, const float (&f)[N]) {
    if (v + N <= V) {
        store_chunk<false>(row, v, f);
    } else {
        for (int j = 0; j < N; ++j)
            if (v + j < V) row[v + j] = static_cast<O>(f[j]);
    }
}

// The mask's bits of the N entries from v on, a multiple of N (N 4 or 8), of a row of V: a row's words are
// read by the byte.  Entries from V on are not allowed.
template <int N>
__device__ __forceinline__ uint32_t mask_bits(const uint32_t *mask, int32_t v, int32_t V) {
    const uint32_t all = v + N <= V ? (1u << N) - 1 : (1u << (V - v)) - 1;     // v < V
    if (!mask) return all;
    return (reinterpret_cast<const uint8_t *>(mask)[static_cast<uint32_t>(v) >> 3] >> (v & 7)) & all;
}

// Puts -infinity where a chunk's bit is 0.
template <typename T>
__device__ __forceinline__ void mask_chunk(u32x4 &raw, uint32_t bits) {
    constexpr int N = kChunk<T>;
    if (bits == (1u << N) - 1) return;
    const auto ones = [&](int j) { return static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - j)) >> 31); };
    const uint32_t none = sizeof(T) == 4 ? 0xff800000u : bits_of<T>(-INFINITY) * 0x10001u;
    for (int w = 0; w < 4; ++w) {
        const uint32_t on = N == 4 ? ones(w) : (ones(2 * w) & 0xffffu) | (ones(2 * w + 1) << 16);
        raw[w] = (raw[w] & on) | (none & ~on);
    }
}

// Reductions over groups of 2^lg neighbouring lanes, lg <= 4, to every lane: exchanges within rows of 16
// lanes are operand modifiers (DPP), where a shuffle goes through LDS.
template <int Control>
__device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_update_dpp(x, x, Control, 0xf, 0xf, false); }
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;

template <typename F>
__device__ __forceinline__ int group_reduce(int x, int lg, const F &f) {
    if (lg > 0) x = f(x, dpp<kSwap1>(x));
    if (lg > 1) x = f(x, dpp<kSwap2>(x));
    if (lg > 2) x = f(x, dpp<kMirror8>(x));      // the quads are uniform by now: a mirror exchanges them
    if (lg > 3) x = f(x, dpp<kMirror16>(x));
    return x;
}
__device__ __forceinline__ float group_max(float x, int lg) {
    return __int_as_float(group_reduce(__float_as_int(x), lg, [](int a, int b) { return __float_as_int(fmaxf(__int_as_float(a), __int_as_float(b))); }));
}
__device__ __forceinline__ float group_sum(float x, int lg) {
    return __int_as_float(group_reduce(__float_as_int(x), lg, [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}
__device__ __forceinline__ int group_min(int x, int lg) {
    return group_reduce(x, lg, [](int a, int b) { return min(a, b); });
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
constexpr int64_t kMaxBlocks = int64_t(1) << 21;    // workgroups of a launch (below 2^32 threads): more go into further launches

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

// For 2 <= n < 2^31 and s the least with n <= 2^s: r * (2^(31 + s) / n + 1) >> (31 + s) is r / n for r < 2^31.
void magic_of(int64_t n, uint32_t *magic, uint32_t *shift) {
    int s = 1;
    while ((int64_t(1) << s) < n) ++s;
    *magic = static_cast<uint32_t>((static_cast<unsigned __int128>(1) << (31 + s)) / static_cast<uint64_t>(n) + 1);
    *shift = static_cast<uint32_t>(s - 1);
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
        int64_t size;                   // bytes of an element (a workspace is one)
        int64_t stride[2], width[2];    // bytes from a row to the next and of a row, and those of the columns (strides of one: 0)
    } ranges[16];
    int n = 0;
    int last = -1;      // the range of the operand taken last, -1 if it has none

    void bad(emo_status s) {
        if (status == EMO_OK) status = s;
    }

    // An operand (absent when t is NULL) of `cols` columns (-1: any).  Outputs have all rows.
    Mat take(const char *name, const emo_tensor *t, unsigned types, int64_t cols, bool dense, bool output) {
        Mat m = {};
        last = -1;
        if (!t || status != EMO_OK) return m;
        if (t->dtype < EMO_F32 || t->dtype > EMO_I64 || !(types & bit(t->dtype)))
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s has a type that this call does not take (%d)", name, (int)t->dtype)), m;
        if (t->reserved != 0) return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s has a reserved field that is not 0", name)), m;
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
        if (t->rows == 1) {
            m.row_stride = 0;
        } else if (t->rows != rows) {
            magic_of(t->rows, &m.magic, &m.shift);
        }
        if (t->cols == 0) return m;
        if (!t->data) return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s has no data", name)), m;
        const int64_t size = size_of(t->dtype);
        const uintptr_t p = reinterpret_cast<uintptr_t>(t->data);
        if (p % size) return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s is not aligned to its elements", name)), m;
        const __int128 end = static_cast<__int128>(t->rows - 1) * t->row_stride + static_cast<__int128>(t->cols - 1) * t->col_stride;
        if (end >= (static_cast<__int128>(1) << 48))
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "%s spans more than an address space", name)), m;
        m.data = static_cast<const char *>(t->data);
        if (n < 16) {
            last = n;
            Range &g = ranges[n++];
            g = {name, p, p + static_cast<uintptr_t>((static_cast<int64_t>(end) + 1) * size), output, t, size,
                 {t->rows > 1 ? t->row_stride * size : 0, t->cols > 1 ? t->col_stride * size : 0}, {}};
            g.width[0] = (t->cols - 1) * g.stride[1] + size;
            g.width[1] = (t->rows - 1) * g.stride[0] + size;
        }
        return m;
    }

    void workspace(const void *p, int64_t have, int64_t need) {
        if (status != EMO_OK || need == 0) return;
        if (!p || have < need)
            return bad(fail(EMO_ERR_INVALID_ARGUMENT, "workspace of %lld bytes, needs %lld", (long long)(p ? have : 0), (long long)need));
        const uintptr_t b = reinterpret_cast<uintptr_t>(p);
        if (b % 16) return bad(fail(EMO_ERR_INVALID_ARGUMENT, "workspace is not 16-byte aligned"));
        if (n < 16) ranges[n++] = {"workspace", b, b + static_cast<uintptr_t>(need), true, nullptr, need, {0, 0}, {need, need}};
    }

    // Whether two ranges that meet share no byte.  Every row (or column) of either begins a multiple of `unit` behind its
    // first, so that what they take of each `unit` bytes is one interval; it is checked that the two intervals are apart.
    // So are columns of one buffer and parts of its rows; with `unit` from all strides, elements by turns.
    static bool between(const Range &x, const Range &y) {
        const uint64_t ahead = x.begin <= y.begin ? y.begin - x.begin : x.begin - y.begin;
        const auto apart_in = [&](int64_t unit, int64_t x_width, int64_t y_width) {
            if (unit == 0) return false;
            const int64_t rest = static_cast<int64_t>(ahead % static_cast<uint64_t>(unit));
            const int64_t from_x = x.begin <= y.begin || rest == 0 ? rest : unit - rest;      // to the next interval of y
            return x_width <= from_x && y_width <= unit - from_x;
        };
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j)
                if (apart_in(std::gcd(x.stride[i], y.stride[j]), x.width[i], y.width[j])) return true;
        return apart_in(std::gcd(std::gcd(x.stride[0], x.stride[1]), std::gcd(y.stride[0], y.stride[1])), x.size, y.size);
    }

    // Outputs lie apart from everything else; the output of range `twin` may be the very memory of range `of`
    // (-1: none may).  The ranges name the operands: records do not, since one can describe several.
    emo_status apart(int twin, int of) {
        if (status != EMO_OK) return status;
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j) {
                if (i == j || !ranges[i].output || ranges[i].begin >= ranges[j].end || ranges[j].begin >= ranges[i].end) continue;
                const emo_tensor *x = ranges[i].t, *y = ranges[j].t;
                if (i == twin && j == of && x->data == y->data && x->dtype == y->dtype && x->rows == y->rows && x->cols == y->cols &&
                    (x->rows == 1 || x->row_stride == y->row_stride))
                    continue;
                if (between(ranges[i], ranges[j])) continue;
                return status = fail(EMO_ERR_INVALID_ARGUMENT, "%s overlaps %s", ranges[i].name, ranges[j].name);
            }
        return EMO_OK;
    }
};

// The operand for row_at; false if its stride does not fit.
bool narrow(const Mat &m, Rows *out) {
    const int64_t bytes = m.row_stride * size_of(m.dtype);
    if (m.data && bytes >= (int64_t(1) << 32)) return false;
    *out = {m.data, static_cast<uint32_t>(bytes), m.rows, m.magic, m.shift};
    return true;
}

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

// Launches `blocks` workgroups, launch(first block, count) for each kMaxBlocks of them.
template <typename F>
void in_launches(int64_t blocks, const F &launch) {
    for (int64_t b = 0; b < blocks; b += kMaxBlocks)
        launch(b, static_cast<unsigned>(blocks - b < kMaxBlocks ? blocks - b : kMaxBlocks));
}

// Launches the workgroups of rows of `parts` pieces, launch(first row, count, pieces) for as many rows as fit.
template <typename F>
void in_pieces(int64_t rows, int64_t parts, const F &launch) {
    Pieces p = {static_cast<uint32_t>(parts), 0, 0};
    if (parts > 1) magic_of(parts, &p.magic, &p.shift);
    const int64_t most = parts < kMaxBlocks ? kMaxBlocks / parts : 1;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = rows - r < most ? rows - r : most;
        launch(static_cast<uint32_t>(r), static_cast<unsigned>(n * parts), p);
    }
}

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
