// Rows of a table picked by ids, and the table's gradient:
//
//   out[t] = scale table[ids[t]],   dtable[v] = scale sum over ids[t] = v of dout[t]
//
// The gradient sorts the samples by id, stably, and sums every row's samples in the
// order of t within pieces of the sorted list, then the pieces in theirs: a fixed order
// without atomics, whatever the ids.  All of it moves bytes.
#include "ops_internal.h"

#include <type_traits>

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
// A group of 2^group_log2 lanes a row, four rows under way.  Bound by its bytes: 524,288 rows
// of 512 bf16 values out of 200,000 in 154 us, 537 MB written and 257 read (5.2 TB/s).
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
// workgroup takes all passes, its samples in registers and LDS (the gradient's us so and in
// launches, rows of 48: 2,000 samples of 500 rows 21, 23; 8,192 of 500 22, 23; of 100,000 33, 38).
// Bound by a launch's waits: 524,288 samples of 200,000 rows take two passes of 21 us; one
// workgroup has 8,192 samples in 11 us (66 % of its waves' cycles waiting), the sums behind it 12.
// Ids in runs of 128, as the samples of rays have them, and drawn: 262,144 of 1,000 rows of 48 33, 36
// us; a million of 30 rows of 16 48, 55; but 8,192 of 500 of 48 28, 22: a wave's counts meet in one
// place.

constexpr int kOneKeys = 8;
constexpr int kSortThreads = 256, kOneThreads = 1024;
constexpr unsigned kOneBlock = kOneThreads * kOneKeys;
constexpr int kMostBits = 10;  // of a digit

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

// KEYS: of a lane.  keys: null in the first pass, which takes them from ids.
template <int KEYS>
__global__ __launch_bounds__(kSortThreads) void digit_count_kernel(const int *ids, const unsigned *keys, unsigned samples,
                                                                   unsigned rows, int shift, int bits, unsigned *counts)
{
    __shared__ unsigned hist[1 << kMostBits];
    const unsigned digits = 1u << bits;
    for (unsigned d = threadIdx.x; d < digits; d += kSortThreads)
        hist[d] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
        const unsigned p = blockIdx.x * (kSortThreads * KEYS) + i * kSortThreads + threadIdx.x;
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

template <int KEYS>
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
    const unsigned first = blockIdx.x * (kSortThreads * KEYS) + wave * (64 * KEYS) + lane;
    // all loads before anything waits: a thread has kShare digits side by side
    unsigned key[KEYS], value[KEYS], total[kShare], before[kShare], sum = 0;
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
        const unsigned p = first + i * 64;
        key[i] = p < samples ? (keys ? keys[p] : (unsigned)ids[p]) : 0u;
        value[i] = p < samples && values ? values[p] : p;
    }
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
        const unsigned d = threadIdx.x * kShare + j;
        total[j] = d < digits ? totals[d] : 0;
        before[j] = d < digits ? counts[(size_t)d * gridDim.x + blockIdx.x] : 0;
    }
    for (int w = 0; w < kWaves; ++w)
        for (unsigned d = threadIdx.x; d < digits; d += kSortThreads)
            hist[w][d] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
        if (!keys)
            key[i] = key_of((int)key[i], rows);
        if (first + i * 64 < samples)
            atomicAdd(&hist[wave][key[i] >> shift & (digits - 1)], 1u);
    }
#pragma unroll
    for (int j = 0; j < kShare; ++j)
        sum += total[j];
    unsigned start = scan<kSortThreads>(sum, tmp);  // samples of smaller digits; its barriers are behind the counting
#pragma unroll
    for (int j = 0; j < kShare; ++j) {
        const unsigned d = threadIdx.x * kShare + j;
        if (d < digits) {
            unsigned at = start + before[j];
#pragma unroll
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
    for (int i = 0; i < KEYS; ++i) {
        const unsigned p = first + i * 64, digit = key[i] >> shift & (digits - 1);
        const unsigned long long same = same_digit(digit, bits, p < samples);
        if (p < samples) {
            const unsigned rank = __popcll(same & ((1ull << lane) - 1)), at = mine[digit] + rank;
            if (rank == 0)
                mine[digit] = at + __popcll(same);
            out_keys[at] = key[i];
            out_values[at] = value[i];
        }
    }
}

// Up to kRanked samples: a sample's place is the number of samples with smaller keys, or the
// same one and before it, counted for 256 samples a workgroup against all of them in LDS, a
// quarter of them by each of four threads.  Half as many where the digits are one pass.  The
// gradient's us so and by digits, rows of 48: 500 samples of 500 rows 18.5, 20.5; 1,000 of 500 23,
// 21, of 100,000 25, 29.
constexpr unsigned kRanked = 1024;
__global__ __launch_bounds__(1024) void rank_kernel(const int *ids, unsigned samples, unsigned rows, unsigned *out_keys,
                                                    unsigned *out_values)
{
    __shared__ u32x4 keys[kRanked / 4];
    __shared__ unsigned parts[3][256];
    unsigned *const key_of_sample = reinterpret_cast<unsigned *>(keys);
    const unsigned fours = (samples + 255) / 256 * 64, own = blockIdx.x * 64;
    if (threadIdx.x < fours * 4)
        key_of_sample[threadIdx.x] = threadIdx.x < samples ? key_of(ids[threadIdx.x], rows) : 0xFFFFFFFFu;  // behind all
    __syncthreads();
    const unsigned t = threadIdx.x & 255, quarter = threadIdx.x >> 8, i = own * 4 + t, mine = key_of_sample[i];
    const unsigned from = quarter * (fours / 4), to = from + fours / 4;
    unsigned place = 0;
    auto between = [&](unsigned a, unsigned b, auto &&counts) {
        a = a > from ? a : from;
        b = b < to ? b : to;
#pragma unroll 8
        for (unsigned j = a; j < b; ++j) {
            const u32x4 k = keys[j];
#pragma unroll
            for (unsigned e = 0; e < 4; ++e)
                place += counts(k[e], j * 4 + e);
        }
    };
    between(0, own, [&](unsigned k, unsigned) { return (unsigned)(k <= mine); });
    between(own, own + 64, [&](unsigned k, unsigned at) { return (unsigned)(k < mine) | ((unsigned)(k == mine) & (unsigned)(at < i)); });
    between(own + 64, fours, [&](unsigned k, unsigned) { return (unsigned)(k < mine); });
    if (quarter)
        parts[quarter - 1][t] = place;
    __syncthreads();
    if (quarter == 0 && i < samples) {
        place += parts[0][t] + parts[1][t] + parts[2][t];
        out_keys[place] = mine;
        out_values[place] = i;
    }
}

static_assert(kOneThreads == 1 << kMostBits, "a thread a digit");
// All passes of up to kOneBlock samples.
__global__ __launch_bounds__(kOneThreads) void sort_one_kernel(const int *ids, unsigned samples, unsigned rows, int key_bits, int bits,
                                                               unsigned *out_keys, unsigned *out_values)
{
    constexpr int kWaves = kOneThreads / 64;
    __shared__ unsigned hist[kWaves][1 << kMostBits];
    __shared__ unsigned tmp[kWaves];
    __shared__ unsigned sorted[2][kOneBlock];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const unsigned digits = 1u << bits;
    const unsigned first = wave * (64 * kOneKeys) + lane;
    unsigned key[kOneKeys], value[kOneKeys];
#pragma unroll
    for (int i = 0; i < kOneKeys; ++i) {
        const unsigned p = first + i * 64;
        key[i] = p < samples ? key_of(ids[p], rows) : 0u;
        value[i] = p;
    }
    for (int shift = 0; shift < key_bits; shift += bits) {
        for (int w = 0; w < kWaves; ++w)
            if (threadIdx.x < digits)
                hist[w][threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kOneKeys; ++i)
            if (first + i * 64 < samples)
                atomicAdd(&hist[wave][key[i] >> shift & (digits - 1)], 1u);
        __syncthreads();
        unsigned count = 0;
        if (threadIdx.x < digits)
            for (int w = 0; w < kWaves; ++w)
                count += hist[w][threadIdx.x];
        unsigned at = scan<kOneThreads>(count, tmp);
        if (threadIdx.x < digits)
            for (int w = 0; w < kWaves; ++w) {
                const unsigned c = hist[w][threadIdx.x];
                hist[w][threadIdx.x] = at;
                at += c;
            }
        __syncthreads();
        volatile unsigned *mine = hist[wave];
#pragma unroll
        for (int i = 0; i < kOneKeys; ++i) {
            const bool in = first + i * 64 < samples;
            const unsigned digit = key[i] >> shift & (digits - 1);
            const unsigned long long same = same_digit(digit, bits, in);
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
        for (int i = 0; i < kOneKeys; ++i)
            if (first + i * 64 < samples) {
                key[i] = sorted[0][first + i * 64];
                value[i] = sorted[1][first + i * 64];
            }
    }
#pragma unroll
    for (int i = 0; i < kOneKeys; ++i)
        if (first + i * 64 < samples) {
            out_keys[first + i * 64] = key[i];
            out_values[first + i * 64] = value[i];
        }
}

// ---- sums ------------------------------------------------------------------------
// The sorted list in pieces of kPiece entries, a group of lanes each.  A run of one key
// that lies within a piece is a row of the result.  Of a run that goes on in the next
// piece its beginning is kept as the piece's trail, and what came from the piece before as
// its lead; where a run began, its trail and the leads behind are joined.  Bound by its
// bytes: 524,288 samples of 512 bf16 values into 200,000 rows, 947 MB, in 194 us (4.9 TB/s).

constexpr unsigned kNone = 0xFFFFFFFFu;
constexpr unsigned kPiece = 32;
constexpr int kLeastLanes = 2;  // log2 of a group's: the entries of a workgroup's pieces lie in LDS

// Of a piece: the key of its trail, or kNone, and whether its lead goes on behind it.
struct Ends {
    unsigned trail, lead_goes_on;
};

// Zeros for the rows that no sample has: a wave takes rows_each of up to 64, looks each up in
// the sorted keys, and writes the absent ones.
template <bool PAST>
__device__ __forceinline__ void absent_rows(unsigned block, const unsigned *keys, unsigned samples, unsigned rows, int D, float *out,
                                            int rows_each)
{
    const int lane = threadIdx.x & 63;
    const unsigned long long v0 = ((unsigned long long)block * 4 + (threadIdx.x >> 6)) * rows_each;
    if (v0 >= rows)
        return;
    const unsigned long long v = lane < rows_each ? v0 + lane : rows;
    unsigned lo = 0, hi = v < rows ? samples : 0;  // the first key that is not below v
    while (lo < hi) {
        const unsigned mid = lo + (hi - lo) / 2;
        if (keys[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    const bool absent = v < rows && !(lo < samples && keys[lo] == v);
    unsigned long long todo = __ballot(absent);
    if (D <= 64) {  // short rows: all of them side by side
        float *first = out + (size_t)v0 * D;
        if (D % 4 == 0) {
            const int vecs = D / 4;
            for (int i = lane; i < rows_each * vecs; i += 64)
                if (todo >> (i / vecs) & 1)
                    *reinterpret_cast<Any16 *>(first + i * 4) = u32x4{0, 0, 0, 0};
        } else {
            for (int i = lane; i < rows_each * D; i += 64)
                if (todo >> (i / D) & 1)
                    first[i] = 0.0f;
        }
        return;
    }
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

template <int V>
__device__ __forceinline__ void add(float (&sum)[V], const Vec<float, V> &x)
{
#pragma unroll
    for (int k = 0; k < V; ++k)
        sum[k] += x.v[k];
}
template <int V, bool PAST>
__device__ __forceinline__ void write_sum(float *to, const float (&sum)[V], float scale)
{
    Vec<float, V> x;
#pragma unroll
    for (int k = 0; k < V; ++k)
        x.v[k] = sum[k] * scale;
    store_vec<float, V, PAST>(to, x);
}

// The first sum_blocks workgroups of a column of them sum; those behind write the absent
// rows.
template <class T, int V, bool PAST>
__global__ __launch_bounds__(256) void sum_kernel(const unsigned *keys, const unsigned *values, const T *from, long long stride,
                                                  unsigned samples, unsigned rows, int D, float scale, float *out, Ends *ends,
                                                  float *leads, float *trails, int group_log2, unsigned sum_blocks, int rows_each)
{
    constexpr int kAhead = 8;
    constexpr unsigned kMostEntries = (256u >> kLeastLanes) * kPiece;
    __shared__ unsigned key_of_entry[kMostEntries + 2];  // one before and one behind
    __shared__ unsigned row_of_entry[kMostEntries];
    if (blockIdx.x >= sum_blocks) {
        if (blockIdx.y == 0)
            absent_rows<PAST>(blockIdx.x - sum_blocks, keys, samples, rows, D, out, rows_each);
        return;
    }
    const unsigned entries = (256u >> group_log2) * kPiece, first = blockIdx.x * entries;
    for (unsigned i = threadIdx.x; i < entries + 2; i += 256) {
        const unsigned at = first + i - 1;  // in front of the first: beyond any list
        key_of_entry[i] = at < samples ? keys[at] : kNone;
        if (i < entries && first + i < samples)
            row_of_entry[i] = values[first + i];
    }
    __syncthreads();
    const unsigned group = threadIdx.x >> group_log2, piece = blockIdx.x * (256u >> group_log2) + group;
    const unsigned *key = key_of_entry + group * kPiece + 1, *row = row_of_entry + group * kPiece;
    if (first + group * kPiece >= samples)
        return;
    const int c = (int)(blockIdx.y << group_log2) + ((int)threadIdx.x & ((1 << group_log2) - 1));
    const int vecs = (D + V - 1) / V;
    const bool in = c < vecs;
    const int e = V > 1 ? vec_at<V>(in ? c : 0, D) : (in ? c : 0);
    Ends mine = {kNone, 0};
    float sum[V];
    bool led = key[-1] == key[0];  // the run came from the piece before
    for (unsigned i0 = 0; i0 < kPiece; i0 += kAhead) {
        if (key[i0] >= rows)
            break;
        Vec<T, V> x[kAhead];
#pragma unroll
        for (unsigned j = 0; j < kAhead; ++j)
            if (key[i0 + j] < rows)
                x[j] = load_vec<T, V, PAST>(from + (long long)row[i0 + j] * stride + e);
#pragma unroll
        for (unsigned j = 0; j < kAhead; ++j) {
            const unsigned i = i0 + j, k = key[i];
            if (k >= rows)
                continue;
            if (i == 0 || key[(int)i - 1] != k)
#pragma unroll
                for (int n = 0; n < V; ++n)
                    sum[n] = (float)x[j].v[n];
            else
#pragma unroll
                for (int n = 0; n < V; ++n)
                    sum[n] += (float)x[j].v[n];
            const bool goes_on = key[i + 1] == k;
            if (goes_on && i + 1 < kPiece)
                continue;
            if (led) {
                mine.lead_goes_on = goes_on;
                if (in)
                    write_sum<V, false>(leads + (size_t)piece * D + e, sum, 1.0f);
                led = false;
            } else if (goes_on) {
                mine.trail = k;
                if (in)
                    write_sum<V, false>(trails + (size_t)piece * D + e, sum, 1.0f);
            } else if (in) {
                write_sum<V, PAST>(out + (size_t)k * D + e, sum, scale);
            }
        }
    }
    if (c == 0)
        ends[piece] = mine;
}

// A wave takes a piece, and the run that began in it and goes on: alone where it ends within
// 64 more pieces, else the whole workgroup.  2^row_log2 lanes have a row, or 64 of its vectors,
// and the lanes that are left share the run's parts.  262,144 samples of 1,000 rows of 48 6 us,
// a million of 3 rows of 8 19.
template <int V>
__global__ __launch_bounds__(256) void join_kernel(const unsigned *keys, unsigned samples, const Ends *ends, const float *leads,
                                                   const float *trails, unsigned pieces, int D, float scale, float *out,
                                                   int row_log2)
{
    constexpr int kAhead = 8;
    __shared__ unsigned char long_runs[4];
    __shared__ float sums[3][64][V];
    const unsigned of_row = 1u << row_log2, subs = 64u >> row_log2;
    const unsigned wave = threadIdx.x >> 6, lane = threadIdx.x & 63, sub = lane >> row_log2, first = blockIdx.x * 4;
    const int c = (int)(blockIdx.y * of_row + (lane & (of_row - 1))), vecs = (D + V - 1) / V;
    const bool in = c < vecs;
    const int e = V > 1 ? vec_at<V>(in ? c : 0, D) : (in ? c : 0);
    // parts 0, 1, ...: the trail of a piece, the lead of the next, and so on; those from `from`
    // on, `step` apart, below `parts`
    auto sum_of = [&](unsigned piece, unsigned from, unsigned step, unsigned parts, float(&sum)[V]) {
        for (unsigned i0 = from; i0 < parts; i0 += kAhead * step) {
            Vec<float, V> x[kAhead];
#pragma unroll
            for (unsigned j = 0; j < kAhead; ++j) {
                const unsigned i = i0 + j * step;
                if (i < parts)
                    x[j] = load_vec<float, V, false>((i ? leads + (size_t)(piece + i) * D : trails + (size_t)piece * D) + e);
            }
#pragma unroll
            for (unsigned j = 0; j < kAhead; ++j)
                if (i0 + j * step < parts)
                    add<V>(sum, x[j]);
        }
    };
    auto join_subs = [&](float(&sum)[V]) {
        for (unsigned off = of_row; off < 64; off <<= 1)
#pragma unroll
            for (int k = 0; k < V; ++k)
                sum[k] += __shfl_xor(sum[k], off);
    };
    const unsigned piece = first + wave;
    const unsigned key = piece < pieces ? ends[piece].trail : kNone;
    const bool ends_here = key != kNone && (piece + 1 + lane >= pieces || !ends[piece + 1 + lane].lead_goes_on);
    const unsigned long long all = __ballot(ends_here);
    if (all) {
        float sum[V] = {};
        sum_of(piece, sub, subs, (unsigned)__builtin_ctzll(all) + 2, sum);
        join_subs(sum);
        if (in && sub == 0)
            write_sum<V, false>(out + (size_t)key * D + e, sum, scale);
    }
    if (lane == 0)
        long_runs[wave] = key != kNone && !all;
    __syncthreads();
    for (unsigned w = 0; w < 4; ++w) {
        if (!long_runs[w])
            continue;
        const unsigned from = first + w;
        // its last sample: keys[lo] is its key, keys[hi] is not
        const unsigned run = ends[from].trail;
        unsigned lo = (from + 1) * kPiece, hi = samples;
        while (hi - lo > 1) {
            const unsigned step = (hi - lo + 255) / 256, at = (threadIdx.x + 1) * step;
            const unsigned below = __syncthreads_count(at < hi - lo && keys[lo + at] == run);
            lo += below * step;
            hi = hi - lo < step ? hi : lo + step;
        }
        float sum[V] = {};
        sum_of(from, wave * subs + sub, 4 * subs, lo / kPiece - from + 1, sum);
        join_subs(sum);
        if (wave)
#pragma unroll
            for (int k = 0; k < V; ++k)
                sums[wave - 1][lane][k] = sum[k];
        __syncthreads();
        if (wave == 0) {
            for (unsigned i = 0; i < 3; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    sum[k] += sums[i][lane][k];
            if (in && sub == 0)
                write_sum<V, false>(out + (size_t)run * D + e, sum, scale);
        }
        __syncthreads();
    }
}

// Few samples in one launch: a workgroup takes some rows and columns, notes the samples that
// are its rows', in order, and sums them row by row, a group of lanes each, kAhead entries of
// its list at a time; rows without a sample, and workgroups, are told apart before.  Bound by a
// launch's waits, and with many samples of a row by the pieces' loads, one after the other: 64
// samples of 500 rows of 48 values 3.7 us, 256 samples of one of them 29 (bf16 56; sorted 14 and
// 17); or by the bytes of a large table: 13 samples of 992,618 rows of 65 33 us, 258 MB.
constexpr unsigned kFewSamples = 256;
template <class T, int V>
__global__ __launch_bounds__(256) void few_kernel(const int *ids, const T *from, long long stride, unsigned samples, unsigned rows, int D,
                                                  float scale, float *out, int group_log2, unsigned rows_each)
{
    constexpr unsigned kAhead = 16;
    static_assert(kFewSamples % kAhead == 0, "whole pieces of the list");
    __shared__ unsigned of_wave[4];
    __shared__ __attribute__((aligned(16))) unsigned row_of[kFewSamples], sample_of[kFewSamples];
    __shared__ unsigned met[32];  // a bit for each row, by its number's lowest ten
    if (threadIdx.x < 32)
        met[threadIdx.x] = 0;
    const unsigned v0 = blockIdx.x * rows_each, here = rows - v0 < rows_each ? rows - v0 : rows_each;
    const int id = threadIdx.x < samples ? ids[threadIdx.x] : -1;
    const bool mine = (unsigned)id >= v0 && (unsigned)id - v0 < here;
    const unsigned long long ballot = __ballot(mine);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0)
        of_wave[wave] = __popcll(ballot);
    __syncthreads();
    unsigned at = __popcll(ballot & ((1ull << lane) - 1)), count = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < wave)
            at += of_wave[w];
        count += of_wave[w];
    }
    if (count == 0) {  // zeros side by side, shared by the workgroups of these rows
        float *first = out + (size_t)v0 * D;
        const size_t all = (size_t)here * D;
        for (size_t i = blockIdx.y * 256u + threadIdx.x; i < all / 4; i += gridDim.y * 256u)
            *reinterpret_cast<Any16 *>(first + i * 4) = u32x4{0, 0, 0, 0};
        if (blockIdx.y == 0 && threadIdx.x < all % 4)
            first[all / 4 * 4 + threadIdx.x] = 0.0f;
        return;
    }
    if (threadIdx.x >= count)
        row_of[threadIdx.x] = kNone;
    if (mine) {
        row_of[at] = (unsigned)id - v0;
        sample_of[at] = threadIdx.x;
        atomicOr(&met[row_of[at] >> 5 & 31], 1u << (row_of[at] & 31));
    }
    __syncthreads();
    const unsigned groups = 256u >> group_log2, lanes = 1u << group_log2;
    const int c = (int)(blockIdx.y * lanes + (threadIdx.x & (lanes - 1)));
    if (c >= (D + V - 1) / V)
        return;
    const int e = V > 1 ? vec_at<V>(c, D) : c;
    for (unsigned v = threadIdx.x >> group_log2; v < here; v += groups) {
        float sum[V] = {};
        const unsigned end = met[v >> 5 & 31] >> (v & 31) & 1 ? count : 0;  // most rows have no sample
        for (unsigned i = 0; i < end; i += kAhead) {
            Vec<T, V> x[kAhead];
#pragma unroll
            for (unsigned j = 0; j < kAhead; ++j)
                if (row_of[i + j] == v)
                    x[j] = load_vec<T, V, false>(from + (long long)sample_of[i + j] * stride + e);
#pragma unroll
            for (unsigned j = 0; j < kAhead; ++j)
                if (row_of[i + j] == v)
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        sum[k] += (float)x[j].v[k];
        }
        write_sum<V, false>(out + (size_t)(v0 + v) * D + e, sum, scale);
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
    // Whole lines past the caches where these would not hold the result (256 MB) for the operator
    // that reads it.  us past them and through them, and so with a concatenation behind: bf16
    // rows of 512 of 20,000, 65,536 samples (67 MB) 20, 21 and 72, 53; 131,072 38, 40 and 138,
    // 112; 262,144 73, 76 and 290, 305; 524,288 146, 158 and 568, 589; float32 rows of 64 of 1,000,
    // 524,288 samples (134 MB) 27, 23 and 152, 145; rows of 512, 131,072 samples 76, 78 and 208, 220.
    if (whole_lines(out.p, out.stride, dim, sizeof(T)) && (unsigned long long)samples * dim * sizeof(T) >= (256ull << 20))
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

// Whether few samples go in one launch: while those of a workgroup's rows, as many as ids
// spread evenly bring, are no more than 96.  us so and sorted, float32 (and bf16), 256 samples: of
// 2 rows of 48 29, 13 (55, 17), of 9 of 48 24, 14 (51, 18), of 9 of 256 12, 14 (27, 17), of 50 of
// 48 10, 15 (20, 19), of 500 of 8 8, 17 (16, 19), of 500 of 1,024 4, 17 (4, 20); 128: of 2 of 48
// 16, 13 (29, 17), of 50 of 48 6, 15 (13, 19); 64 of 2 of 48 9, 14 (15, 17).
bool is_few(unsigned samples, unsigned rows, int dim)
{
    const unsigned each = 256u >> group_log2((dim + 3) / 4);  // bf16's workgroups have twice as many
    return samples <= kFewSamples && (unsigned long long)samples * (each < rows ? each : rows) <= 96ull * rows;
}

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Samples of a block of the sort: 1,024, or 2,048 where there are blocks for all of the chip.
// The gradient's us with 1,024 and 2,048: 15,000 samples of 23 rows 29, 31; 70,000 of 8,612
// 41, 46; 262,144 of 1,000 40, 41; 524,288 of 200,000 340, 333; 1,000,000 of 500,000 159, 154.
unsigned sort_block(unsigned samples) { return samples < 256u * 8 * kSortThreads ? 4 * kSortThreads : 8 * kSortThreads; }

// The workspace: two lists of keys and values, the sort's counts, and the pieces' parts.
struct Places {
    size_t list, counts, ends, leads, trails, end;
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
    if (is_few(samples, rows, dim)) {
        p.counts = p.ends = p.leads = p.trails = p.end = 0;
        return p;
    }
    at += 4 * whole((size_t)samples * 4);
    const Digits d = digits_of(rows);
    p.counts = take(samples > kOneBlock ? (((size_t)blocks_of(samples, sort_block(samples)) + 1) << d.bits) * 4 : 0);
    const size_t pieces = blocks_of(samples, kPiece);
    p.ends = take(pieces * sizeof(Ends));
    p.leads = take(pieces * dim * sizeof(float));
    p.trails = take(pieces * dim * sizeof(float));
    p.end = at;
    return p;
}

template <class T, int V>
hipError_t few(Rows dout, const int *ids, unsigned samples, unsigned rows, int dim, float scale, float *out, hipStream_t s)
{
    const int vecs = (dim + V - 1) / V, g = group_log2(vecs);
    // rows of a workgroup: one for each group, and more where there are too many workgroups
    unsigned each = 256u >> g;
    if (blocks_of(rows, each) > 4096)
        each = blocks_of(rows, 4096);
    few_kernel<T, V><<<dim3(blocks_of(rows, each), blocks_of(vecs, 1 << g)), 256, 0, s>>>(
        ids, static_cast<const T *>(dout.p), dout.stride, samples, rows, dim, scale, out, g, each);
    return hipGetLastError();
}

template <class T, int V, bool PAST>
hipError_t sums(const unsigned *keys, const unsigned *values, Rows dout, unsigned samples, unsigned rows, int dim, float scale, float *out,
                Ends *ends, float *leads, float *trails, hipStream_t s)
{
    const int vecs = (dim + V - 1) / V, least = group_log2(vecs), g = least < kLeastLanes ? kLeastLanes : least;
    const unsigned pieces = blocks_of(samples, kPiece), blocks = blocks_of(pieces, 256 >> g);
    int rows_each = 64;  // of a wave that writes absent rows, fewer where there are few waves
    while (rows_each > 4 && rows / rows_each < 2048)
        rows_each /= 2;
    sum_kernel<T, V, PAST><<<dim3(blocks + blocks_of(rows, 4 * rows_each), blocks_of(vecs, 1 << g)), 256, 0, s>>>(
        keys, values, static_cast<const T *>(dout.p), dout.stride, samples, rows, dim, scale, out, ends, leads, trails, g, blocks,
        rows_each);
    return hipGetLastError();
}

template <int V>
hipError_t join(const unsigned *keys, unsigned samples, const Ends *ends, const float *leads, const float *trails, unsigned pieces,
                int dim, float scale, float *out, hipStream_t s)
{
    const int vecs = (dim + V - 1) / V, g = group_log2(vecs);
    join_kernel<V><<<dim3(blocks_of(pieces, 4), blocks_of(vecs, 1 << g)), 256, 0, s>>>(keys, samples, ends, leads, trails, pieces, dim, scale,
                                                                                               out, g);
    return hipGetLastError();
}

template <class T>
hipError_t backward(Rows dout, const int *ids, unsigned samples, unsigned rows, int dim, float scale, float *out, char *ws,
                    hipStream_t s)
{
    constexpr int V = 16 / sizeof(T);
    if (is_few(samples, rows, dim))
        return dim < V ? few<T, 1>(dout, ids, samples, rows, dim, scale, out, s) : few<T, V>(dout, ids, samples, rows, dim, scale, out, s);
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
        const unsigned blocks = blocks_of(samples, sort_block(samples));
        unsigned *counts = reinterpret_cast<unsigned *>(ws + at.counts), *totals = counts + ((size_t)blocks << d.bits);
        for (int pass = 0; pass < d.passes; ++pass) {
            const unsigned *k = pass ? keys[now ^ 1] : nullptr, *v = pass ? values[now ^ 1] : nullptr;
            const int shift = pass * d.bits;
            auto launch = [&](auto keys_each) {
                constexpr int KEYS = decltype(keys_each)::value;
                digit_count_kernel<KEYS><<<blocks, kSortThreads, 0, s>>>(ids, k, samples, rows, shift, d.bits, counts);
                digit_scan_kernel<<<1u << d.bits, kSortThreads, 0, s>>>(counts, blocks, totals);
                digit_place_kernel<KEYS><<<blocks, kSortThreads, 0, s>>>(ids, k, v, samples, rows, shift, d.bits, counts, totals,
                                                                         keys[now], values[now]);
            };
            if (sort_block(samples) == 4 * kSortThreads)
                launch(std::integral_constant<int, 4>{});
            else
                launch(std::integral_constant<int, 8>{});
            now ^= 1;
        }
        now ^= 1;  // the last one written
        e = hipGetLastError();
    } else {
        if (samples <= kRanked && (samples <= kRanked / 2 || d.passes > 1))
            rank_kernel<<<blocks_of(samples, 256), 1024, 0, s>>>(ids, samples, rows, keys[0], values[0]);
        else
            sort_one_kernel<<<1, kOneThreads, 0, s>>>(ids, samples, rows, d.key_bits, d.bits, keys[0], values[0]);
        e = hipGetLastError();
    }
    if (e != hipSuccess)
        return e;
    Ends *ends = reinterpret_cast<Ends *>(ws + at.ends);
    float *leads = reinterpret_cast<float *>(ws + at.leads), *trails = reinterpret_cast<float *>(ws + at.trails);
    const unsigned *k = keys[now], *v = values[now];
    // Past the caches where they would not hold it all (256 MB).  us with and without: bf16
    // 131,072 samples of 50,000 rows of 512 (237 MB) 81, 68; 262,144 of 100,000 (473 MB) 145, 150;
    // 524,288 of 200,000 (946 MB) 250, 268; float32 65,536 of 20,000 (175 MB) 60, 55; 131,072 of
    // 50,000 (371 MB) 101, 109.
    const bool past = ((size_t)samples * sizeof(T) + (size_t)rows * 4) * dim > (256u << 20);
    if (dim < V)
        e = sums<T, 1, false>(k, v, dout, samples, rows, dim, scale, out, ends, leads, trails, s);
    else if (past && whole_lines(out, dim, dim, 4) && whole_lines(dout.p, dout.stride, dim, sizeof(T)))
        e = sums<T, V, true>(k, v, dout, samples, rows, dim, scale, out, ends, leads, trails, s);
    else
        e = sums<T, V, false>(k, v, dout, samples, rows, dim, scale, out, ends, leads, trails, s);
    const unsigned pieces = blocks_of(samples, kPiece);
    if (e != hipSuccess || pieces == 1)
        return e;
    return dim < 4 ? join<1>(k, samples, ends, leads, trails, pieces, dim, scale, out, s)
                   : join<4>(k, samples, ends, leads, trails, pieces, dim, scale, out, s);
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
