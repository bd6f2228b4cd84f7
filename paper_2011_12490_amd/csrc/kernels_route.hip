// Samples to their heads and back: the stable sort of (sample, slot) pairs by
// head, rows into that order, and their weighted sums back with the gradients.
// All of it moves bytes; nothing here computes much.
#include "ops_internal.h"

#include <type_traits>

namespace derf {

namespace {

// ---- the sort ---------------------------------------------------------------
// A counting sort: a pair's key is its head, or num_heads where it has none,
// and its row is the number of pairs of smaller keys, plus those of its key in
// earlier blocks, in earlier waves of its block, and in earlier lanes.  Pairs are
// matched with those of a wave's other lanes, not by atomics in an order of their
// own, so the sort is stable.  524,288 pairs of 64 heads: 6, 5 and 9 us in three
// launches, latency of each.  Up to 8,192 pairs one workgroup does all in 4.5 to 9 us;
// with more, 9,000 pairs, of 4 to 256 heads, it takes 14 to 23 us, three launches 10 to 13.

constexpr int kLanePairs = 8;  // pairs of a lane
constexpr int kSortThreads = 256;
constexpr int kOneThreads = 1024;  // the form with a single workgroup
constexpr unsigned kSortBlock = kSortThreads * kLanePairs;
constexpr unsigned kOneBlock = kOneThreads * kLanePairs;
constexpr int kMaxKeys = 257;

__device__ __forceinline__ unsigned key_of(int head, unsigned num_heads)
{
    return (unsigned)head < num_heads ? (unsigned)head : num_heads;
}

// Exclusive prefix sum over the workgroup's first 256 threads; *total: the sum.
// Every thread of the workgroup calls it.  tmp: 4 words of LDS.
__device__ __forceinline__ unsigned scan256(unsigned x, unsigned *tmp, unsigned *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned incl = x;
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned y = __shfl_up(incl, off);
        if (lane >= off)
            incl += y;
    }
    if (lane == 63 && wave < 4)
        tmp[wave] = incl;
    __syncthreads();
    unsigned before = 0, all = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < wave)
            before += tmp[w];
        all += tmp[w];
    }
    __syncthreads();
    *total = all;
    return before + incl - x;
}

__global__ __launch_bounds__(kSortThreads) void route_count_kernel(const int *heads, unsigned pairs,
                                                                   unsigned num_heads,
                                                                   unsigned *counts)
{
    __shared__ unsigned hist[kMaxKeys];
    for (unsigned b = threadIdx.x; b <= num_heads; b += kSortThreads)
        hist[b] = 0;
    __syncthreads();
    for (int i = 0; i < kLanePairs; ++i) {
        const unsigned p = blockIdx.x * kSortBlock + i * kSortThreads + threadIdx.x;
        if (p < pairs)
            atomicAdd(&hist[key_of(heads[p], num_heads)], 1u);
    }
    __syncthreads();
    for (unsigned b = threadIdx.x; b <= num_heads; b += kSortThreads)
        counts[(size_t)b * gridDim.x + blockIdx.x] = hist[b];
}

// One workgroup a key: its counts become the number of its pairs in earlier blocks.
__global__ __launch_bounds__(kSortThreads) void route_scan_kernel(unsigned *counts, unsigned blocks,
                                                                  unsigned *totals)
{
    __shared__ unsigned tmp[4];
    unsigned *mine = counts + (size_t)blockIdx.x * blocks;
    unsigned before = 0;
    for (unsigned at = 0; at < blocks; at += kSortThreads) {
        const unsigned i = at + threadIdx.x;
        const unsigned x = i < blocks ? mine[i] : 0;
        unsigned total;
        const unsigned ex = scan256(x, tmp, &total);
        if (i < blocks)
            mine[i] = before + ex;
        before += total;
    }
    if (threadIdx.x == 0)
        totals[blockIdx.x] = before;
}

// ONE: a single workgroup that counts by itself (counts, totals unused).
template <int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void route_place_kernel(const int *heads, unsigned pairs,
                                                              unsigned num_heads,
                                                              const unsigned *counts,
                                                              const unsigned *totals, int *offsets,
                                                              int *pair, int *row)
{
    constexpr int kWaves = THREADS / 64;
    __shared__ unsigned hist[kWaves][kMaxKeys];
    __shared__ unsigned tmp[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (unsigned i = threadIdx.x; i < kWaves * kMaxKeys; i += THREADS)
        hist[0][i] = 0;
    __syncthreads();
    const unsigned first =
        blockIdx.x * (THREADS * kLanePairs) + wave * (64 * kLanePairs) + lane;
    unsigned key[kLanePairs];
#pragma unroll
    for (int i = 0; i < kLanePairs; ++i) {
        const unsigned p = first + i * 64;
        key[i] = p < pairs ? key_of(heads[p], num_heads) : 0u;
        if (p < pairs)
            atomicAdd(&hist[wave][key[i]], 1u);
    }
    __syncthreads();
    // rows in front of each head's first pair of this block
    const unsigned k = threadIdx.x;
    unsigned count = 0, headed;
    if (k < num_heads) {
        if (ONE)
            for (int w = 0; w < kWaves; ++w)
                count += hist[w][k];
        else
            count = totals[k];
    }
    unsigned start = scan256(count, tmp, &headed);
    if (blockIdx.x == 0) {
        if (k < num_heads)
            offsets[k] = (int)start;
        if (k == 0)
            offsets[num_heads] = (int)headed;
    }
    auto spread = [&](unsigned b, unsigned at) {
        if (!ONE)
            at += counts[(size_t)b * gridDim.x + blockIdx.x];
        for (int w = 0; w < kWaves; ++w) {
            const unsigned c = hist[w][b];
            hist[w][b] = at;
            at += c;
        }
    };
    if (k < num_heads)
        spread(k, start);
    if (k == 0)
        spread(num_heads, headed);
    __syncthreads();
    const int bits = 32 - __builtin_clz(num_heads);
    volatile unsigned *mine = hist[wave];
#pragma unroll
    for (int i = 0; i < kLanePairs; ++i) {
        const unsigned p = first + i * 64;
        unsigned long long same = __ballot(p < pairs);
        for (int b = 0; b < bits; ++b) {
            const bool set = (key[i] >> b) & 1u;
            const unsigned long long with = __ballot(set);
            same &= set ? with : ~with;
        }
        if (p < pairs) {
            const unsigned rank = __popcll(same & ((1ull << lane) - 1));
            const unsigned at = mine[key[i]] + rank;
            if (rank == 0)
                mine[key[i]] = at + __popcll(same);
            pair[at] = (int)p;
            row[p] = key[i] < num_heads ? (int)at : -1 - (int)at;
        }
    }
}

// ---- rows ---------------------------------------------------------------------
// A row is handled in vectors of V elements by a group of G lanes.  A row of
// D >= V elements that is no whole number of vectors ends with a vector that
// overlaps the one before; D < V goes element by element (V = 1).

constexpr int kRowThreads = 256;

template <class T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
    T v[V];
};
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(2))) Any16;  // 16 bytes at any element

// ONCE: what is read once, or written and not read again before much else is,
// goes past the caches (nontemporal).  For rows of whole 128-byte lines: there
// 524,288 rows of 1,024 bf16 are written in the order of heads in 215 us, 432 with
// ordinary stores, and summed back in 222, 264 with ordinary loads; 262,144 rows
// of 63 float, whose lines are shared, take 31 and 21 us so, 29 and 19 without.
template <class T, int V, bool ONCE = false>
__device__ __forceinline__ Vec<T, V> load_vec(const T *p)
{
    if constexpr (ONCE)
        return __builtin_bit_cast(Vec<T, V>, (u32x4)__builtin_nontemporal_load(reinterpret_cast<const Any16 *>(p)));
    else
        return *reinterpret_cast<const Vec<T, V> *>(p);
}
template <class T, int V, bool ONCE>
__device__ __forceinline__ void store_vec(T *p, const Vec<T, V> &x)
{
    if constexpr (ONCE)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), reinterpret_cast<Any16 *>(p));
    else
        *reinterpret_cast<Vec<T, V> *>(p) = x;
}

// First element of vector c of a row of D elements.
template <int V>
__device__ __forceinline__ int vec_at(int c, int D)
{
    return c * V + V <= D ? c * V : D - V;
}

// The group's first item and the distance to its next; the lane's place within
// the group and the group's lanes.
struct Lane {
    long long item, stride;
    int at, step;
};
__device__ __forceinline__ Lane lane_of(int group_log2)
{
    const int per = kRowThreads >> group_log2;
    return {(long long)blockIdx.x * per + (threadIdx.x >> group_log2), (long long)gridDim.x * per,
            (int)threadIdx.x & ((1 << group_log2) - 1), 1 << group_log2};
}

// The place of a pair's row, and whether it has a head.
__device__ __forceinline__ unsigned place_of(int row) { return row < 0 ? (unsigned)(-1 - row) : (unsigned)row; }

// Vectors of a row that a lane has under way at once.
constexpr int kAhead = 4;

// A row is read once and written top_k times, whole rows one after another.
// 131,072 rows of 1,024 bf16 to 524,288: 224 us, 5.4 TB/s of memory traffic.
template <class T, int V, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void dispatch_kernel(const T *x, long long xs,
                                                               const int *row, long long tokens,
                                                               int top_k, int D, T *out,
                                                               long long os, int group_log2)
{
    const Lane l = lane_of(group_log2);
    const Vec<T, V> zero = {};
    const int vecs = (D + V - 1) / V;
    for (long long t = l.item; t < tokens; t += l.stride) {
        const T *xr = x + t * xs;
        const int *rr = row + t * top_k;
        for (int c0 = l.at; c0 < vecs; c0 += kAhead * l.step) {
            Vec<T, V> v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (c0 + i * l.step < vecs)
                    v[i] = load_vec<T, V>(xr + vec_at<V>(c0 + i * l.step, D));
            for (int j = 0; j < top_k; ++j) {
                const int r = rr[j];
                T *to = out + (long long)place_of(r) * os;
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (c0 + i * l.step < vecs)
                        store_vec<T, V, ONCE>(to + vec_at<V>(c0 + i * l.step, D), r < 0 ? zero : v[i]);
            }
        }
    }
}

// Vectors of four of a sample's rows are read at once; the sum goes in the
// order of j.  524,288 rows of 1,024 bf16 to 131,072: 213 us, 1.34 GB at 6.3 TB/s,
// a third of it from the caches; 131,072 of 2,048 with weights to 16,384: 143 us.
template <class T, int V, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void combine_kernel(const T *rows, long long rs,
                                                              const float *weights, const int *row,
                                                              long long tokens, int top_k, int D,
                                                              T *out, long long os, int group_log2)
{
    constexpr int kRows = 4, kVecs = ONCE ? 2 : 1;  // short rows leave the second idle
    const Lane l = lane_of(group_log2);
    const int vecs = (D + V - 1) / V;
    for (long long t = l.item; t < tokens; t += l.stride) {
        const int *rr = row + t * top_k;
        const float *wr = weights ? weights + t * top_k : nullptr;
        for (int c0 = l.at; c0 < vecs; c0 += kVecs * l.step) {
            int e[kVecs];
            float sum[kVecs][V];
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                e[k] = c0 + k * l.step < vecs ? vec_at<V>(c0 + k * l.step, D) : -1;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    sum[k][i] = 0.0f;
            }
            for (int j0 = 0; j0 < top_k; j0 += kRows) {
                int r[kRows];
                float w[kRows];
                Vec<T, V> v[kRows][kVecs];
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    r[j] = j0 + j < top_k ? rr[j0 + j] : -1;
                    w[j] = r[j] >= 0 && wr ? wr[j0 + j] : 1.0f;
                }
#pragma unroll
                for (int j = 0; j < kRows; ++j)
                    if (r[j] >= 0)
#pragma unroll
                        for (int k = 0; k < kVecs; ++k)
                            if (k == 0 || e[k] >= 0)
                                v[j][k] = load_vec<T, V, ONCE>(rows + (long long)r[j] * rs + e[k]);
#pragma unroll
                for (int j = 0; j < kRows; ++j)
                    if (r[j] >= 0)
#pragma unroll
                        for (int k = 0; k < kVecs; ++k)
#pragma unroll
                            for (int i = 0; i < V; ++i)
                                sum[k][i] = fmaf(w[j], (float)v[j][k].v[i], sum[k][i]);
            }
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                Vec<T, V> y;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    y.v[i] = (T)sum[k][i];
                if (k == 0 || e[k] >= 0)
                    store_vec<T, V, ONCE>(out + t * os + e[k], y);
            }
        }
    }
}

// A group of lanes takes one pair: one reading of its row for its weight's gradient,
// dweight[t][j] = <rows[r], dy[t]>, and of dy[t], which its siblings share through the
// caches, for drows[r] = w dy[t].  131,072 rows of 2,048 bf16: 219 us, 5.2 TB/s.
template <class T, int V, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void combine_backward_kernel(
    const T *dout, long long ds, const T *rows, long long rs, const float *weights, const int *row,
    long long pairs, int top_k, int D, T *drows, long long os, float *dweights, int group_log2)
{
    const Lane l = lane_of(group_log2);
    const int vecs = (D + V - 1) / V;
    // the lanes of a wave leave together: they exchange their sums
    const long long from = l.item - (threadIdx.x & 63) / l.step;
    for (long long off = 0; from + off < pairs; off += l.stride) {
        const long long p = l.item + off;
        float dot = 0.0f;
        if (p < pairs) {
            const int r = row[p];
            const long long place = place_of(r);
            const T *dr = dout + p / top_k * ds;
            const T *xr = rows + place * rs;
            const float w = r < 0 ? 0.0f : weights ? weights[p] : 1.0f;
            for (int c = l.at; c < vecs; c += l.step) {
                const int e = vec_at<V>(c, D);
                Vec<T, V> y = {};
                if (r >= 0) {
                    const Vec<T, V> d = load_vec<T, V>(dr + e);
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        y.v[i] = (T)(w * (float)d.v[i]);
                    if (dweights) {
                        const Vec<T, V> v = load_vec<T, V, ONCE>(xr + e);
                        const int skip = c * V - e;  // elements that the vector before has too
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            if (i >= skip)
                                dot = fmaf((float)d.v[i], (float)v.v[i], dot);
                    }
                }
                store_vec<T, V, ONCE>(drows + place * os + e, y);
            }
        }
        if (dweights) {
            for (int o = l.step >> 1; o > 0; o >>= 1)
                dot += __shfl_xor(dot, o);
            if (p < pairs && l.at == 0)
                dweights[p] = dot;
        }
    }
}

// Lanes of a group: the power of two, at most a wave, that covers the row's vectors.
int group_log2_of(int vecs)
{
    int g = 0;
    while (g < 6 && (1 << g) < vecs)
        ++g;
    return g;
}

unsigned groups_grid(long long items, int group_log2)
{
    const long long per = kRowThreads >> group_log2;
    const long long blocks = (items + per - 1) / per;
    return (unsigned)(blocks < (1 << 22) ? blocks : 1 << 22);
}

// Whole 128-byte lines.
bool whole_lines(const Rows &r, int D, int size)
{
    return D * size % 128 == 0 && r.stride * size % 128 == 0 && reinterpret_cast<uintptr_t>(r.p) % 128 == 0;
}

// Calls f(T{}, V, ONCE) with the rows' type, the vector length for rows of D and
// whether they are whole lines.
template <class F>
hipError_t with_rows(bool bf16, int D, bool lines, F f)
{
    using Yes = std::true_type;
    using No = std::false_type;
    if (bf16)
        lines ? f(__bf16{}, std::integral_constant<int, 8>{}, Yes{})
        : D >= 8 ? f(__bf16{}, std::integral_constant<int, 8>{}, No{})
                 : f(__bf16{}, std::integral_constant<int, 1>{}, No{});
    else
        lines ? f(float{}, std::integral_constant<int, 4>{}, Yes{})
        : D >= 4 ? f(float{}, std::integral_constant<int, 4>{}, No{})
                 : f(float{}, std::integral_constant<int, 1>{}, No{});
    return hipGetLastError();
}

}  // namespace

size_t route_workspace_bytes(unsigned pairs, int num_heads)
{
    if (pairs <= kOneBlock)
        return 0;
    const size_t blocks = (pairs + (size_t)kSortBlock - 1) / kSortBlock;
    return (blocks + 1) * (num_heads + 1) * sizeof(unsigned);
}

hipError_t launch_route(const int *heads, unsigned pairs, int num_heads, int *offsets, int *pair,
                        int *row, unsigned *workspace, hipStream_t s)
{
    if (pairs <= kOneBlock) {
        route_place_kernel<kOneThreads, true><<<1, kOneThreads, 0, s>>>(
            heads, pairs, num_heads, nullptr, nullptr, offsets, pair, row);
        return hipGetLastError();
    }
    const unsigned blocks = (unsigned)((pairs + (size_t)kSortBlock - 1) / kSortBlock);
    unsigned *totals = workspace, *counts = workspace + num_heads + 1;
    route_count_kernel<<<blocks, kSortThreads, 0, s>>>(heads, pairs, num_heads, counts);
    route_scan_kernel<<<num_heads + 1, kSortThreads, 0, s>>>(counts, blocks, totals);
    route_place_kernel<kSortThreads, false><<<blocks, kSortThreads, 0, s>>>(
        heads, pairs, num_heads, counts, totals, offsets, pair, row);
    return hipGetLastError();
}

hipError_t launch_dispatch(Rows x, const int *row, long long tokens, int top_k, int dim, bool bf16,
                           Rows out, hipStream_t s)
{
    const int size = bf16 ? 2 : 4;
    const bool lines = whole_lines(out, dim, size);
    return with_rows(bf16, dim, lines, [&](auto t, auto v, auto once) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        constexpr bool ONCE = decltype(once)::value;
        const int g = group_log2_of((dim + V - 1) / V);
        dispatch_kernel<T, V, ONCE><<<groups_grid(tokens, g), kRowThreads, 0, s>>>(
            static_cast<const T *>(x.p), x.stride, row, tokens, top_k, dim,
            static_cast<T *>(const_cast<void *>(out.p)), out.stride, g);
    });
}

hipError_t launch_combine(Rows rows, const float *weights, const int *row, long long tokens,
                          int top_k, int dim, bool bf16, Rows out, hipStream_t s)
{
    const int size = bf16 ? 2 : 4;
    const bool lines = whole_lines(rows, dim, size) && whole_lines(out, dim, size);
    return with_rows(bf16, dim, lines, [&](auto t, auto v, auto once) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        constexpr bool ONCE = decltype(once)::value;
        const int g = group_log2_of((dim + V - 1) / V);
        combine_kernel<T, V, ONCE><<<groups_grid(tokens, g), kRowThreads, 0, s>>>(
            static_cast<const T *>(rows.p), rows.stride, weights, row, tokens, top_k, dim,
            static_cast<T *>(const_cast<void *>(out.p)), out.stride, g);
    });
}

hipError_t launch_combine_backward(Rows dout, Rows rows, const float *weights, const int *row,
                                   long long tokens, int top_k, int dim, bool bf16, Rows drows,
                                   float *dweights, hipStream_t s)
{
    const int size = bf16 ? 2 : 4;
    const bool lines = whole_lines(drows, dim, size) && (!dweights || whole_lines(rows, dim, size));
    return with_rows(bf16, dim, lines, [&](auto t, auto v, auto once) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        constexpr bool ONCE = decltype(once)::value;
        const int g = group_log2_of((dim + V - 1) / V);
        combine_backward_kernel<T, V, ONCE><<<groups_grid(tokens * top_k, g), kRowThreads, 0, s>>>(
            static_cast<const T *>(dout.p), dout.stride, static_cast<const T *>(rows.p),
            rows.stride, weights, row, tokens * top_k, top_k, dim,
            static_cast<T *>(const_cast<void *>(drows.p)), drows.stride, dweights, g);
    });
}

}  // namespace derf
