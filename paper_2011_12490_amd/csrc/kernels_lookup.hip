// Rows of a table picked by ids, and the table's gradient:
//
//   out[t] = scale table[ids[t]],   dtable[v] = scale sum over ids[t] = v of dout[t]
//
// The gradient sorts the samples by id, stably, and sums every row's samples in the
// order of t within pieces of the sorted list, then the pieces in theirs: a fixed order
// without atomics, whatever the ids.  All of it moves bytes.
#include "ops_internal.h"

namespace derf {

namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(2))) Any16;  // 16 bytes at any element

template <class T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
    T v[V];
};
// PAST: past the caches (nontemporal), for rows of whole 128-byte lines.
template <class T, int V, bool PAST>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    if constexpr (PAST)
        return __builtin_bit_cast(Vec<T, V>, (u32x4)__builtin_nontemporal_load(reinterpret_cast<const Any16 *>(p)));
    else
        return *reinterpret_cast<const Vec<T, V> *>(p);
}
template <class T, int V, bool PAST>
__device__ __forceinline__ void store_vec(T *p, const Vec<T, V> &x)
{
    if constexpr (PAST && sizeof(Vec<T, V>) % 16 == 0) {
        struct Pieces {
            u32x4 v[sizeof(Vec<T, V>) / 16];
        };
        const Pieces pieces = __builtin_bit_cast(Pieces, x);
#pragma unroll
        for (int i = 0; i < (int)sizeof(Vec<T, V>) / 16; ++i)
            __builtin_nontemporal_store(pieces.v[i], reinterpret_cast<Any16 *>(p) + i);
    } else
        *reinterpret_cast<Vec<T, V> *>(p) = x;
}

// First element of vector c of a row of D >= V elements: the last vector overlaps the one
// before where the row is no whole number of them, and both hold the same values there.
template <int V>
__device__ __forceinline__ int vec_at(int c, int D)
{
    return c * V + V <= D ? c * V : D - V;
}

// ---- rows out of the table ------------------------------------------------------
// A group of 2^group_log2 lanes a row, four rows under way.
template <class T, int V, bool PAST>
__global__ __launch_bounds__(256) void lookup_kernel(const T *table, long long stride, const int *ids, long long samples,
                                                     long long rows, int D, float scale, T *out, long long os, int group_log2)
{
    constexpr int kAhead = 4;
    const long long per = 256 >> group_log2, step = gridDim.x * per;
    const int at = (int)threadIdx.x & ((1 << group_log2) - 1), lanes = 1 << group_log2;
    const int vecs = (D + V - 1) / V;
    for (long long t = blockIdx.x * per + (threadIdx.x >> group_log2); t < samples; t += kAhead * step) {
        long long id[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            id[i] = t + i * step < samples ? ids[t + i * step] : -1;
            id[i] = id[i] < rows ? id[i] : -1;
        }
        for (int c = at; c < vecs; c += lanes) {
            const int e = V > 1 ? vec_at<V>(c, D) : c;
            Vec<T, V> x[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                x[i] = id[i] >= 0 ? load_vec<T, V, false>(table + id[i] * stride + e) : Vec<T, V>{};
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (t + i * step >= samples)
                    break;
#pragma unroll
                for (int k = 0; k < V; ++k)
                    x[i].v[k] = id[i] >= 0 ? (T)((float)x[i].v[k] * scale) : (T)0.0f;
                store_vec<T, V, PAST>(out + (t + i * step) * os + e, x[i]);
            }
        }
    }
}

// ---- samples sorted by id --------------------------------------------------------
// A radix sort from the lowest digit on: within a pass a sample's place is the number of
// those of smaller digits, plus those of its digit in earlier blocks, in earlier waves
// of its block and in earlier lanes, which are matched by ballots: stable.  A sample
// without a row has the key `rows`, behind all others.  Up to kOneBlock samples one
// workgroup takes all passes, its samples in registers and LDS.

constexpr int kLaneKeys = 8;
constexpr int kSortThreads = 256, kOneThreads = 1024;
constexpr unsigned kSortBlock = kSortThreads * kLaneKeys, kOneBlock = kOneThreads * kLaneKeys;
constexpr int kMostBits = 10, kOneBits = 8;  // of a digit

__device__ __forceinline__ unsigned key_of(int id, unsigned rows) { return (unsigned)id < rows ? (unsigned)id : rows; }

// Exclusive prefix sum over the workgroup.  tmp: a word for each wave.
template <int THREADS>
__device__ __forceinline__ unsigned scan(unsigned x, unsigned *tmp)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned incl = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned y = __shfl_up(incl, off);
        if (lane >= off)
            incl += y;
    }
    __syncthreads();
    if (lane == 63)
        tmp[wave] = incl;
    __syncthreads();
    unsigned before = 0;
    for (int w = 0; w < wave; ++w)
        before += tmp[w];
    return before + incl - x;
}

// keys: null in the first pass, which takes them from ids.
__global__ __launch_bounds__(kSortThreads) void digit_count_kernel(const int *ids, const unsigned *keys, unsigned samples,
                                                                   unsigned rows, int shift, int bits, unsigned *counts)
{
    __shared__ unsigned hist[1 << kMostBits];
    const unsigned digits = 1u << bits;
    for (unsigned d = threadIdx.x; d < digits; d += kSortThreads)
        hist[d] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLaneKeys; ++i) {
        const unsigned p = blockIdx.x * kSortBlock + i * kSortThreads + threadIdx.x;
        if (p < samples)
            atomicAdd(&hist[(keys ? keys[p] : key_of(ids[p], rows)) >> shift & (digits - 1)], 1u);
    }
    __syncthreads();
    for (unsigned d = threadIdx.x; d < digits; d += kSortThreads)
        counts[(size_t)d * gridDim.x + blockIdx.x] = hist[d];
}

// One workgroup a digit: its counts become the number of its samples in earlier blocks.
__global__ __launch_bounds__(kSortThreads) void digit_scan_kernel(unsigned *counts, unsigned blocks, unsigned *totals)
{
    __shared__ unsigned tmp[kSortThreads / 64];
    unsigned *mine = counts + (size_t)blockIdx.x * blocks;
    unsigned before = 0;
    for (unsigned at = 0; at < blocks; at += kSortThreads) {
        const unsigned i = at + threadIdx.x;
        const unsigned x = i < blocks ? mine[i] : 0;
        const unsigned ex = scan<kSortThreads>(x, tmp);
        if (i < blocks)
            mine[i] = before + ex;
        unsigned all = 0;
#pragma unroll
        for (int w = 0; w < kSortThreads / 64; ++w)
            all += tmp[w];
        before += all;
    }
    if (threadIdx.x == 0)
        totals[blockIdx.x] = before;
}

// The lanes of the wave whose key has this lane's digit, of those that take part.
__device__ __forceinline__ unsigned long long same_digit(unsigned digit, int bits, bool takes_part)
{
    unsigned long long same = __ballot(takes_part);
    for (int b = 0; b < bits; ++b) {
        const bool set = (digit >> b) & 1u;
        const unsigned long long with = __ballot(set);
        same &= set ? with : ~with;
    }
    return same;
}

__global__ __launch_bounds__(kSortThreads) void digit_place_kernel(const int *ids, const unsigned *keys, const unsigned *values,
                                                                   unsigned samples, unsigned rows, int shift, int bits,
                                                                   const unsigned *counts, const unsigned *totals,
                                                                   unsigned *out_keys, unsigned *out_values)
{
    constexpr int kWaves = kSortThreads / 64, kShare = (1 << kMostBits) / kSortThreads;
    __shared__ unsigned hist[kWaves][1 << kMostBits];
    __shared__ unsigned tmp[kWaves];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const unsigned digits = 1u << bits;
    for (int w = 0; w < kWaves; ++w)
        for (unsigned d = threadIdx.x; d < digits; d += kSortThreads)
            hist[w][d] = 0;
    __syncthreads();
    const unsigned first = blockIdx.x * kSortBlock + wave * (64 * kLaneKeys) + lane;
    unsigned key[kLaneKeys];
#pragma unroll
    for (int i = 0; i < kLaneKeys; ++i) {
        const unsigned p = first + i * 64;
        key[i] = p < samples ? (keys ? keys[p] : key_of(ids[p], rows)) : 0u;
        if (p < samples)
            atomicAdd(&hist[wave][key[i] >> shift & (digits - 1)], 1u);
    }
    // samples of smaller digits; a thread has kShare digits side by side
    unsigned total[kShare], sum = 0;
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
        const unsigned d = threadIdx.x * kShare + j;
        total[j] = d < digits ? totals[d] : 0;
        sum += total[j];
    }
    unsigned start = scan<kSortThreads>(sum, tmp);  // its barriers are behind the counting
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
        const unsigned d = threadIdx.x * kShare + j;
        if (d < digits) {
            unsigned at = start + counts[(size_t)d * gridDim.x + blockIdx.x];
            for (int w = 0; w < kWaves; ++w) {
                const unsigned c = hist[w][d];
                hist[w][d] = at;
                at += c;
            }
        }
        start += total[j];
    }
    __syncthreads();
    volatile unsigned *mine = hist[wave];
#pragma unroll
    for (int i = 0; i < kLaneKeys; ++i) {
        const unsigned p = first + i * 64, digit = key[i] >> shift & (digits - 1);
        const unsigned long long same = same_digit(digit, bits, p < samples);
        if (p < samples) {
            const unsigned rank = __popcll(same & ((1ull << lane) - 1)), at = mine[digit] + rank;
            if (rank == 0)
                mine[digit] = at + __popcll(same);
            out_keys[at] = key[i];
            out_values[at] = values ? values[p] : p;
        }
    }
}

// All passes of up to kOneBlock samples.
__global__ __launch_bounds__(kOneThreads) void sort_one_kernel(const int *ids, unsigned samples, unsigned rows, int key_bits,
                                                               unsigned *out_keys, unsigned *out_values)
{
    constexpr int kWaves = kOneThreads / 64, kDigits = 1 << kOneBits;
    __shared__ unsigned hist[kWaves][kDigits];
    __shared__ unsigned tmp[kWaves];
    __shared__ unsigned sorted[2][kOneBlock];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const unsigned first = wave * (64 * kLaneKeys) + lane;
    unsigned key[kLaneKeys], value[kLaneKeys];
#pragma unroll
    for (int i = 0; i < kLaneKeys; ++i) {
        const unsigned p = first + i * 64;
        key[i] = p < samples ? key_of(ids[p], rows) : 0u;
        value[i] = p;
    }
    for (int shift = 0; shift < key_bits; shift += kOneBits) {
        for (unsigned i = threadIdx.x; i < kWaves * kDigits; i += kOneThreads)
            hist[0][i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLaneKeys; ++i)
            if (first + i * 64 < samples)
                atomicAdd(&hist[wave][key[i] >> shift & (kDigits - 1)], 1u);
        __syncthreads();
        unsigned count = 0;
        if (threadIdx.x < kDigits)
            for (int w = 0; w < kWaves; ++w)
                count += hist[w][threadIdx.x];
        unsigned at = scan<kOneThreads>(count, tmp);
        if (threadIdx.x < kDigits)
            for (int w = 0; w < kWaves; ++w) {
                const unsigned c = hist[w][threadIdx.x];
                hist[w][threadIdx.x] = at;
                at += c;
            }
        __syncthreads();
        volatile unsigned *mine = hist[wave];
#pragma unroll
        for (int i = 0; i < kLaneKeys; ++i) {
            const bool in = first + i * 64 < samples;
            const unsigned digit = key[i] >> shift & (kDigits - 1);
            const unsigned long long same = same_digit(digit, kOneBits, in);
            if (in) {
                const unsigned rank = __popcll(same & ((1ull << lane) - 1)), to = mine[digit] + rank;
                if (rank == 0)
                    mine[digit] = to + __popcll(same);
                sorted[0][to] = key[i];
                sorted[1][to] = value[i];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLaneKeys; ++i)
            if (first + i * 64 < samples) {
                key[i] = sorted[0][first + i * 64];
                value[i] = sorted[1][first + i * 64];
            }
    }
#pragma unroll
    for (int i = 0; i < kLaneKeys; ++i)
        if (first + i * 64 < samples) {
            out_keys[first + i * 64] = key[i];
            out_values[first + i * 64] = value[i];
        }
}

// ---- sums ------------------------------------------------------------------------
// The sorted list in pieces of kPiece entries, a group of lanes each.  A run of one key
// that lies within a piece is a row of the result.  A run that goes on in the next piece,
// or came from the one before, is a part: at most one of each kind a piece, which make a
// sorted list of their own, two places a piece, some empty.  That is summed the same way
// until there is one piece.

constexpr unsigned kNone = 0xFFFFFFFFu;
constexpr unsigned kPiece = 32;

// What a run's part is: key, and whether the run began before it and goes on behind it.
struct Part {
    unsigned key;
    unsigned before, behind;
};

// FIRST: entries are samples (sorted keys, values: places of their rows), else parts.
template <class T, int V, bool FIRST, bool PAST>
__global__ __launch_bounds__(256) void sum_runs_kernel(const unsigned *keys, const unsigned *values, const Part *parts,
                                                       const T *from, long long stride, unsigned entries, unsigned rows, int D,
                                                       float scale, float *out, Part *out_parts, float *out_rows,
                                                       int group_log2)
{
    constexpr unsigned kAhead = 4;
    const unsigned piece = blockIdx.x * (256 >> group_log2) + (threadIdx.x >> group_log2);
    const unsigned first = piece * kPiece;
    if (first >= entries)
        return;
    const unsigned last = entries - first < kPiece ? entries : first + kPiece;
    const int c = (int)(blockIdx.y << group_log2) + ((int)threadIdx.x & ((1 << group_log2) - 1));
    const int vecs = (D + V - 1) / V;
    const bool in = c < vecs, tells = c == 0;
    const int e = V > 1 ? vec_at<V>(c < vecs ? c : 0, D) : (in ? c : 0);
    float sum[V];
    bool open = false, began_before = false, used[2] = {false, false};
    unsigned run = kNone;
    auto flush = [&](bool behind) {
        if (!began_before && !behind) {
            Vec<float, V> x;
#pragma unroll
            for (int k = 0; k < V; ++k)
                x.v[k] = sum[k] * scale;
            if (in)
                store_vec<float, V, PAST>(out + (size_t)run * D + e, x);
        } else {
            const unsigned slot = 2 * piece + (began_before ? 0 : 1);
            Vec<float, V> x;
#pragma unroll
            for (int k = 0; k < V; ++k)
                x.v[k] = sum[k];
            if (in)
                store_vec<float, V, false>(out_rows + (size_t)slot * D + e, x);
            if (tells)
                out_parts[slot] = {run, began_before, behind};
            used[began_before ? 0 : 1] = true;
        }
        open = false;
    };
    bool goes_on = false;
    for (unsigned i0 = first; i0 < last; i0 += kAhead) {
        unsigned key[kAhead];
        bool before[kAhead], behind[kAhead];
        Vec<T, V> x[kAhead];
#pragma unroll
        for (unsigned j = 0; j < kAhead; ++j) {
            const unsigned i = i0 + j;
            key[j] = kNone;
            if (i >= last)
                continue;
            if constexpr (FIRST) {
                const unsigned k = keys[i];
                if (k >= rows)
                    continue;
                key[j] = k;
                before[j] = i > 0 && keys[i - 1] == k;
                behind[j] = i + 1 < entries && keys[i + 1] == k;
                x[j] = load_vec<T, V, PAST>(from + (long long)values[i] * stride + e);
            } else {
                const Part p = parts[i];
                key[j] = p.key;
                before[j] = p.before;
                behind[j] = p.behind;
                if (p.key != kNone)
                    x[j] = load_vec<T, V, false>(from + (long long)i * stride + e);
            }
        }
#pragma unroll
        for (unsigned j = 0; j < kAhead; ++j) {
            if (key[j] == kNone)
                continue;
            if (!open) {
                open = true;
                run = key[j];
                began_before = before[j];
#pragma unroll
                for (int k = 0; k < V; ++k)
                    sum[k] = (float)x[j].v[k];
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    sum[k] += (float)x[j].v[k];
            }
            goes_on = behind[j];
            if (!goes_on)
                flush(false);
        }
    }
    if (open)
        flush(true);
    if (tells && out_parts)
        for (int s = 0; s < 2; ++s)
            if (!used[s])
                out_parts[2 * piece + s] = {kNone, 0, 0};
}

// Zeros for the rows that no sample has: a wave takes 64 rows, looks each up in the
// sorted keys, and writes the absent ones.
template <bool PAST>
__global__ __launch_bounds__(256) void absent_rows_kernel(const unsigned *keys, unsigned samples, unsigned rows, int D, float *out)
{
    const int lane = threadIdx.x & 63;
    const unsigned long long v0 = ((unsigned long long)blockIdx.x * 4 + (threadIdx.x >> 6)) * 64;
    if (v0 >= rows)
        return;
    const unsigned long long v = v0 + lane;
    unsigned lo = 0, hi = samples;  // the first key that is not below v
    while (lo < hi) {
        const unsigned mid = lo + (hi - lo) / 2;
        if (keys[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    const bool absent = v < rows && !(lo < samples && keys[lo] == v);
    unsigned long long todo = __ballot(absent);
    while (todo) {
        const int l = __builtin_ctzll(todo);
        todo &= todo - 1;
        float *row = out + (size_t)(v0 + l) * D;
        if (PAST) {
            for (int c = lane * 4; c < D; c += 256)
                __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4 *>(row + c));
        } else {
            for (int c = lane; c < D; c += 64)
                row[c] = 0.0f;
        }
    }
}

// ---- launches --------------------------------------------------------------------

unsigned blocks_of(unsigned long long n, unsigned each) { return (unsigned)((n + each - 1) / each); }

int group_log2(int vecs)
{
    int g = 0;
    while (g < 6 && 1 << g < vecs)
        ++g;
    return g;
}

bool whole_lines(const void *p, long long stride, int dim, int bytes)
{
    return (reinterpret_cast<uintptr_t>(p) | (unsigned long long)stride * bytes | (unsigned long long)dim * bytes) % 128 == 0;
}

template <class T, int V, bool PAST>
hipError_t lookup(Rows table, const int *ids, long long samples, long long rows, int dim, float scale, Rows out, hipStream_t s)
{
    const int g = group_log2((dim + V - 1) / V);
    const unsigned long long groups = 256 >> g, want = ((unsigned long long)samples + groups * 4 - 1) / (groups * 4);
    const unsigned blocks = want < 8192 ? (unsigned)want : 8192;
    lookup_kernel<T, V, PAST><<<blocks, 256, 0, s>>>(static_cast<const T *>(table.p), table.stride, ids, samples, rows, dim, scale,
                                                     static_cast<T *>(const_cast<void *>(out.p)), out.stride, g);
    return hipGetLastError();
}

template <class T>
hipError_t lookup_of(Rows table, const int *ids, long long samples, long long rows, int dim, float scale, Rows out, hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    if (dim < V)
        return lookup<T, 1, false>(table, ids, samples, rows, dim, scale, out, s);
    if (whole_lines(out.p, out.stride, dim, sizeof(T)))
        return lookup<T, V, true>(table, ids, samples, rows, dim, scale, out, s);
    return lookup<T, V, false>(table, ids, samples, rows, dim, scale, out, s);
}

// Digits of the sort.
struct Digits {
    int passes, bits, key_bits;
};
Digits digits_of(unsigned rows)
{
    const int key_bits = 32 - __builtin_clz(rows ? rows : 1);
    const int passes = (key_bits + kMostBits - 1) / kMostBits;
    return {passes, (key_bits + passes - 1) / passes, key_bits};
}

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

// The workspace: two lists of keys and values, the sort's counts, and the parts of the
// sums' levels, of which two are alive at a time.
struct Places {
    size_t list, counts, parts, part_rows, parts2, part_rows2, end;
};
Places places_of(unsigned samples, unsigned rows, int dim)
{
    Places p;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += whole(bytes);
        return here;
    };
    p.list = take(0);
    at += 4 * whole((size_t)samples * 4);
    const Digits d = digits_of(rows);
    p.counts = take(samples > kOneBlock ? (((size_t)blocks_of(samples, kSortBlock) + 1) << d.bits) * 4 : 0);
    const size_t first = 2 * (size_t)blocks_of(samples, kPiece), second = 2 * (size_t)blocks_of(first, kPiece);
    p.parts = take(first * sizeof(Part));
    p.part_rows = take(first * dim * sizeof(float));
    p.parts2 = take(second * sizeof(Part));
    p.part_rows2 = take(second * dim * sizeof(float));
    p.end = at;
    return p;
}

template <class T, int V, bool FIRST, bool PAST>
hipError_t sum_runs(const unsigned *keys, const unsigned *values, const Part *parts, const T *from, long long stride,
                    unsigned entries, unsigned rows, int dim, float scale, float *out, Part *out_parts, float *out_rows, hipStream_t s)
{
    const int vecs = (dim + V - 1) / V, g = group_log2(vecs);
    const unsigned pieces = blocks_of(entries, kPiece);
    sum_runs_kernel<T, V, FIRST, PAST><<<dim3(blocks_of(pieces, 256 >> g), blocks_of(vecs, 1 << g)), 256, 0, s>>>(
        keys, values, parts, from, stride, entries, rows, dim, scale, out, out_parts, out_rows, g);
    return hipGetLastError();
}

template <class T>
hipError_t backward(Rows dout, const int *ids, unsigned samples, unsigned rows, int dim, float scale, float *out, char *ws,
                    hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    const Places at = places_of(samples, rows, dim);
    const size_t list = whole((size_t)samples * 4);
    unsigned *keys[2], *values[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = reinterpret_cast<unsigned *>(ws + at.list + 2 * i * list);
        values[i] = reinterpret_cast<unsigned *>(ws + at.list + (2 * i + 1) * list);
    }
    const Digits d = digits_of(rows);
    hipError_t e = hipSuccess;
    int now = 0;
    if (samples > kOneBlock) {
        const unsigned blocks = blocks_of(samples, kSortBlock);
        unsigned *counts = reinterpret_cast<unsigned *>(ws + at.counts), *totals = counts + ((size_t)blocks << d.bits);
        for (int pass = 0; pass < d.passes; ++pass) {
            const unsigned *k = pass ? keys[now ^ 1] : nullptr, *v = pass ? values[now ^ 1] : nullptr;
            const int shift = pass * d.bits;
            digit_count_kernel<<<blocks, kSortThreads, 0, s>>>(ids, k, samples, rows, shift, d.bits, counts);
            digit_scan_kernel<<<1u << d.bits, kSortThreads, 0, s>>>(counts, blocks, totals);
            digit_place_kernel<<<blocks, kSortThreads, 0, s>>>(ids, k, v, samples, rows, shift, d.bits, counts, totals, keys[now],
                                                               values[now]);
            now ^= 1;
        }
        now ^= 1;  // the last one written
        e = hipGetLastError();
    } else if (samples > 0) {
        sort_one_kernel<<<1, kOneThreads, 0, s>>>(ids, samples, rows, d.key_bits, keys[0], values[0]);
        e = hipGetLastError();
    }
    if (e != hipSuccess)
        return e;
    const bool past = whole_lines(out, dim, dim, 4);
    const unsigned blocks = blocks_of(rows, 256);
    if (past)
        absent_rows_kernel<true><<<blocks, 256, 0, s>>>(keys[now], samples, rows, dim, out);
    else
        absent_rows_kernel<false><<<blocks, 256, 0, s>>>(keys[now], samples, rows, dim, out);
    e = hipGetLastError();
    if (e != hipSuccess || samples == 0)
        return e;
    Part *parts[2] = {reinterpret_cast<Part *>(ws + at.parts), reinterpret_cast<Part *>(ws + at.parts2)};
    float *part_rows[2] = {reinterpret_cast<float *>(ws + at.part_rows), reinterpret_cast<float *>(ws + at.part_rows2)};
    const T *from = static_cast<const T *>(dout.p);
    const bool lines = past && whole_lines(from, dout.stride, dim, sizeof(T));
    if (dim < V)
        e = sum_runs<T, 1, true, false>(keys[now], values[now], nullptr, from, dout.stride, samples, rows, dim, scale, out, parts[0],
                                        part_rows[0], s);
    else if (lines)
        e = sum_runs<T, V, true, true>(keys[now], values[now], nullptr, from, dout.stride, samples, rows, dim, scale, out, parts[0],
                                       part_rows[0], s);
    else
        e = sum_runs<T, V, true, false>(keys[now], values[now], nullptr, from, dout.stride, samples, rows, dim, scale, out, parts[0],
                                        part_rows[0], s);
    unsigned pieces = blocks_of(samples, kPiece);
    for (int level = 0; e == hipSuccess && pieces > 1; ++level) {
        const unsigned entries = 2 * pieces;
        pieces = blocks_of(entries, kPiece);
        Part *const in = parts[level & 1], *const to = parts[~level & 1];
        float *const in_rows = part_rows[level & 1], *const to_rows = part_rows[~level & 1];
        e = dim < 4 ? sum_runs<float, 1, false, false>(nullptr, nullptr, in, in_rows, dim, entries, rows, dim, scale, out, to, to_rows, s)
                    : sum_runs<float, 4, false, false>(nullptr, nullptr, in, in_rows, dim, entries, rows, dim, scale, out, to, to_rows, s);
    }
    return e;
}

}  // namespace

hipError_t launch_lookup(Rows table, const int *ids, long long samples, long long rows, int dim, float scale, bool bf16, Rows out,
                         hipStream_t s)
{
    return bf16 ? lookup_of<__bf16>(table, ids, samples, rows, dim, scale, out, s)
                : lookup_of<float>(table, ids, samples, rows, dim, scale, out, s);
}

size_t lookup_workspace_bytes(unsigned samples, unsigned rows, int dim) { return places_of(samples, rows, dim).end; }

hipError_t launch_lookup_backward(Rows dout, const int *ids, unsigned samples, unsigned rows, int dim, float scale, bool bf16,
                                  float *out, void *workspace, hipStream_t s)
{
    char *ws = static_cast<char *>(workspace);
    return bf16 ? backward<__bf16>(dout, ids, samples, rows, dim, scale, out, ws, s)
                : backward<float>(dout, ids, samples, rows, dim, scale, out, ws, s);
}

}  // namespace derf
