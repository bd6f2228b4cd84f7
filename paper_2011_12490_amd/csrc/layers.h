// The heads' layers' kernels and the choice among them, for the units that launch them:
// rows (the layer, and its rows' gradient), weights, both in one launch, both in one
// pass.  The products are those of kernels_linear.hip's first lines.
#pragma once
#include "product.h"

#include <type_traits>

namespace derf {

namespace {

// A tile of the result: rows [t.first, t.last), columns from n0 on.
template <class C>
__device__ __forceinline__ void write_rows(const RowTile &t, int n0, int width, const f32x4 (&acc)[C::FP][C::FQ],
                                           const float *bias, bool relu, char *results,
                                           typename C::T *y, long long ys)
{
    using T = typename C::T;
    constexpr int V = Type<T>::kVec;
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wp = (wave % C::WP) * C::FP * 16, wq = (wave / C::WP) * C::FQ * 16;
    char *mine = results + wave * 16 * kResultRow<C>;
    const bool past = C::FP * 16 * sizeof(T) >= 128 && past_caches(y, ys, width);  // a wave's are lines too
#pragma unroll
    for (int j = 0; j < C::FQ; ++j) {
#pragma unroll
        for (int i = 0; i < C::FP; ++i) {
            const int e = i * 16 + (lane >> 4) * 4;
            f32x4 v = acc[i][j];
            if (bias)
                v += *reinterpret_cast<const f32x4 *>(bias + wp + e);
            if (relu)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[k] = v[k] < 0.0f ? 0.0f : v[k];
            if constexpr (sizeof(T) == 4) {
                const unsigned row = t.first + wq + j * 16 + (lane & 15);
                const int n = n0 + wp + e;
                if (row < t.last && n < width)
                    write_piece(y + (row * ys + n), __builtin_bit_cast(u32x4, v), width - n, T{});
            } else {
                store_values(mine + (lane & 15) * kResultRow<C> + e * sizeof(T), v, T{});
            }
        }
        if constexpr (sizeof(T) == 4)
            continue;
        __builtin_amdgcn_wave_barrier();
        constexpr int kPieces = C::FP * 16 / V;  // of a row
#pragma unroll
        for (int i = 0; i < (16 * kPieces + 63) / 64; ++i) {
            const int r = (i * 64 + lane) / kPieces, c = (i * 64 + lane) % kPieces * V;
            if (16 * kPieces % 64 && r >= 16)
                continue;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(mine + r * kResultRow<C> + c * sizeof(T));
            const unsigned row = t.first + wq + j * 16 + r;
            const int n = n0 + wp + c;
            if (row >= t.last || n >= width)
                continue;
            write_result(y + (row * ys + n), v, width - n, past);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- gated layers: their result ---------------------------------------------------

// Of act(g), and for the gradient its slope.  The hardware's exponential and reciprocal: a
// unit in the last place of float each, and the exponent's rounding, 2^-24 |g| of the value.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float logistic(float g) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-g)); }
// The normal distribution's share below g, and bell = exp(-g^2 / 2).  For x >= 0
// erfc(x) exp(x^2) / 2 is t P(t) with t = 1 / (1 + 0.45 x), P of degree 9 fitted to least
// relative error over t in (0, 1] (3.2e-8; 6 x 2^-24 with float32's roundings): a third of
// the instructions of erfcf.  A layer of 63 to 128 on 98,301 rows of float32: 60 us, 66 with
// erfcf.
__device__ __forceinline__ float below(float g, float &bell)
{
    constexpr float kP[10] = {0.126942664f, 0.126941577f, 0.114135817f, 0.0876260847f, 0.0599751174f,
                              -0.0111786677f, 0.0711999312f, -0.150290668f, 0.095343627f, -0.0206954815f};
    bell = exp_of(-0.5f * g * g);
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.318198052f, 1.0f));
    float v = kP[9];
#pragma unroll
    for (int k = 8; k >= 0; --k)
        v = fmaf(v, t, kP[k]);
    v *= t * bell;
    return g < 0.0f ? v : 1.0f - v;
}
// v = act(g) u for N vectors; the activation is chosen once for all, so that their
// instructions interleave.
template <int N>
__device__ __forceinline__ void activate(const f32x4 (&g)[N], const f32x4 (&u)[N], int act, f32x4 (&v)[N])
{
    if (act == DERF_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 4 * N; ++i)
            v[i / 4][i % 4] = g[i / 4][i % 4] < 0.0f ? 0.0f : g[i / 4][i % 4];
    } else if (act == DERF_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) {
            float bell;
            v[i / 4][i % 4] = g[i / 4][i % 4] * below(g[i / 4][i % 4], bell);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4 * N; ++i)
            v[i / 4][i % 4] = logistic(g[i / 4][i % 4]);
        if (act == DERF_ACT_SILU)
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] *= g[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] *= u[i];
}

// Of 16 rows: gates in the even results of acc, ups in the odd ones.  y = act(gate) up,
// and, where `pre` is wanted, both as they are, the ups `width` columns behind the gates.
template <class T, int PAIRS, bool STAGE = sizeof(T) == 2>
__device__ __forceinline__ void write_gated(const f32x4 (&acc)[2 * PAIRS], const float *gate_bias, const float *up_bias, int act,
                                            char *mine, unsigned row0, unsigned last, int n0, int width, T *y, long long ys,
                                            T *pre, long long pres)
{
    f32x4 g[PAIRS], u[PAIRS], v[PAIRS];
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) {
        const int e = i * 16 + (threadIdx.x & 63) / 16 * 4;
        g[i] = acc[2 * i];
        u[i] = acc[2 * i + 1];
        if (gate_bias) {
            g[i] += *reinterpret_cast<const f32x4 *>(gate_bias + e);
            u[i] += *reinterpret_cast<const f32x4 *>(up_bias + e);
        }
    }
    activate<PAIRS>(g, u, act, v);
    write_16_rows<T, PAIRS * 16, STAGE>(v, mine, row0, last, n0, width, y, ys);
    if (pre) {
        write_16_rows<T, PAIRS * 16, STAGE>(g, mine, row0, last, n0, width, pre, pres);
        write_16_rows<T, PAIRS * 16, STAGE>(u, mine, row0, last, n0, width, pre + width, pres);
    }
}

// A tile of a gated layer's result: rows [t.first, t.last), columns from n0 on.
// bias: TP values, the gates' first.
template <class C>
__device__ __forceinline__ void write_pairs(const RowTile &t, int n0, int width, const f32x4 (&acc)[C::FP][C::FQ],
                                            const float *bias, int act, char *results, typename C::T *y, long long ys,
                                            typename C::T *pre, long long pres)
{
    using T = typename C::T;
    constexpr int PAIRS = C::FP / 2;
    const int wave = uniform(threadIdx.x >> 6);
    const int wp = (wave % C::WP) * PAIRS * 16, wq = (wave / C::WP) * C::FQ * 16;
    char *mine = results + wave * 16 * kPieceRow<T, PAIRS * 16>;
#pragma unroll
    for (int j = 0; j < C::FQ; ++j) {
        f32x4 column[C::FP];
#pragma unroll
        for (int i = 0; i < C::FP; ++i)
            column[i] = acc[i][j];
        write_gated<T, PAIRS>(column, bias ? bias + wp : nullptr, bias ? bias + C::kCols + wp : nullptr, act, mine,
                              t.first + wq + j * 16, t.last, n0 + wp, width, y, ys, pre, pres);
    }
}

// ---- rows: the layer, and its rows' gradient --------------------------------------

// P: the weights (width columns of the result), Q: rows.  Where operands go to LDS by
// themselves a workgroup goes on from tile to tile with its loads two steps ahead;
// tiles that share rows or weights run on one XCD.  2,048 to 4,096 on 32,768 rows of
// bf16: 493 us, 1,115 TFLOP/s; what depth adds runs at 1,430, the rest is a tile's
// start and its results' stores.  1,024 to 4,096 on 26 rows of 16 heads, the weights'
// reading: 18 us.  act: a ReLU or none, or (kPair, a gated layer) a derf_activation; pre:
// kPair's gates and ups, or null.
template <class C>
__global__ __launch_bounds__(C::kThreads, 2) void rows_kernel(
    Problem p, Matrix<typename C::T> w, Matrix<typename C::T> x, const float *bias, int act,
    typename C::T *y, long long ys, typename C::T *pre, long long pres, int width, int depth, unsigned from)
{
    constexpr int kBiases = C::kAsync ? 4 : 1;  // of the tiles under way
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    __shared__ __attribute__((aligned(16))) char results[C::kAsync ? kResultBytes<C> : 16];
    __shared__ __attribute__((aligned(16))) float biases[kBiases][C::TP];
    __shared__ unsigned before[kMaxHeads + 1];
    static_assert(C::kAsync || kJoinBytes<C> + kResultBytes<C> <= C::kLds, "parts and results take the stages' place");
    count_tiles(p, C::TQ, before);
    const unsigned headed = uniform(before[p.heads]), headless = bound(p, p.heads);
    const unsigned tail = (unsigned)(((unsigned long long)(p.rows - headless) + C::TQ - 1) / C::TQ);
    const unsigned row_tiles = headed + tail, col_tiles = (width + C::kCols - 1) / C::kCols;
    const unsigned all = row_tiles * col_tiles, end = runs_end(all);
    const size_t head_size = (size_t)p.fan_in * p.fan_out * (C::kPair ? 2 : 1);
    // what workgroup number b does: false if nothing
    auto tile_at = [&](unsigned b, RowTile &t, int &n0) {
        const unsigned at = by_xcd(b, all);
        if (at >= all)
            return false;
        const Place2 where = in_groups(at, row_tiles, col_tiles);
        n0 = (int)where.b * C::kCols;
        if (where.a < headed) {
            t = head_tile(p, before, where.a, C::TQ);
        } else {
            t.first = headless + (where.a - headed) * C::TQ;
            t.last = p.rows - t.first > (unsigned)C::TQ ? t.first + C::TQ : p.rows;
            t.head = p.heads;
        }
        return true;
    };
    auto sources = [&](const RowTile &t, int n0, typename C::P::Source &ps, typename C::Q::Source &qs) {
        ps = {w, (unsigned)n0, C::kPair ? (unsigned)width : 0u};
        ps.m.p += t.head * head_size;
        qs = {x, 0};
        qs.m.p += t.first * x.stride;
        qs.m.mask += t.first * x.mask_stride;
        qs.m.rows = t.last - t.first;
    };
    RowTile t;
    int n0;
    if constexpr (C::kAsync) {
        unsigned ahead = blockIdx.x, loaded = 0, done = 0;
        auto next_tile = [&](Pipe<C> &pipe) {
            RowTile u;
            int m0;
            for (; ahead < end; ahead += gridDim.x) {
                if (!tile_at(ahead, u, m0) || u.head >= p.heads)
                    continue;
                ahead += gridDim.x;
                // its biases too: the first waves bring 64 each
                if (bias && threadIdx.x < C::TP) {
                    const unsigned wave = uniform(threadIdx.x >> 6), half = wave * 64 / C::kCols;  // kPair: of the ups
                    const Window b = window(bias + ((size_t)u.head * (C::kPair ? 2 : 1) + half) * width, width, 1, width, 0, m0);
                    read4_to_lds(b, (threadIdx.x % C::kCols) * 4, lds_byte(reinterpret_cast<const char *>(biases[loaded & 3])) + wave * 256);
                }
                ++loaded;
                typename C::P::Source ps;
                typename C::Q::Source qs;
                sources(u, m0, ps, qs);
                pipe.load_tile(ps, qs, depth);
                return;
            }
            pipe.load_nothing();
        };
        Pipe<C> pipe;
        pipe.start(lds, next_tile);
        for (unsigned b = blockIdx.x; b < end; b += gridDim.x) {
            if (!tile_at(b, t, n0))
                continue;
            f32x4 acc[C::FP][C::FQ] = {};
            const bool has = t.head < p.heads;
            if (has)
#pragma unroll 1
                for (int k = 0; k < depth; k += C::kDepth)
                    pipe.step(acc, next_tile, [](auto &) {});
            if constexpr (C::kPair)
                write_pairs<C>(t, n0, width, acc, has && bias ? biases[done & 3] : nullptr, act, results, y, ys, pre, pres);
            else
                write_rows<C>(t, n0, width, acc, has && bias ? biases[done & 3] : nullptr, has && act, results, y, ys);
            done += has;
        }
        arrived<0>();
    } else {
        if (!tile_at(from + blockIdx.x, t, n0))
            return;
        f32x4 acc[C::FP][C::FQ] = {};
        const bool has = t.head < p.heads;
        if (has) {
            if (bias && threadIdx.x < C::TP) {
                const int n = n0 + (int)threadIdx.x % C::kCols, half = (int)threadIdx.x / C::kCols;  // kPair: of the ups
                biases[0][threadIdx.x] =
                    n < width ? bias[((size_t)t.head * (C::kPair ? 2 : 1) + half) * width + n] : 0.0f;
            }
            typename C::P::Source ps;
            typename C::Q::Source qs;
            sources(t, n0, ps, qs);
            tile_product<C>(ps, qs, depth, lds, acc, [](auto &) {});
        }
        if constexpr (C::kTeams > 1)
            if (!join_teams<C>(lds, acc))
                return;
        if constexpr (C::kPair)
            write_pairs<C>(t, n0, width, acc, has && bias ? biases[0] : nullptr, act, lds + kJoinBytes<C>, y, ys, pre, pres);
        else
            write_rows<C>(t, n0, width, acc, has && bias ? biases[0] : nullptr, has && act, lds + kJoinBytes<C>, y, ys);
    }
}

// ---- weights ----------------------------------------------------------------------

// The sums over rows of a tile of dz: a thread's are over every (threads /
// kPerRow)-th row of its columns, V of them.
template <class C>
struct RowSums {
    using T = typename C::T;
    static constexpr int V = Type<T>::kVec, kRowsOfThreads = C::kThreads / C::Q::kPerRow;
    static constexpr int kBytes = kRowsOfThreads * (C::TQ + 1) * (int)sizeof(float);
    bool on;
    float v[V];
    __device__ __forceinline__ void begin(bool on_)
    {
        on = on_;
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] = 0.0f;
    }
    __device__ __forceinline__ void add(const typename C::Q::S &share)
    {
        if (!on)
            return;
#pragma unroll
        for (int i = 0; i < C::Q::kShare; ++i) {
            union {
                u32x4 v;
                T e[V];
            } piece = {share.x[i]};
#pragma unroll
            for (int k = 0; k < V; ++k)
                v[k] += (float)piece.e[k];
        }
    }
    // to[m] for m0 + m < O; lds: kBytes
    __device__ __forceinline__ void write(float *to, int m0, int O, char *lds) const
    {
        if (!on)
            return;
        float(*part)[C::TQ + 1] = reinterpret_cast<float(*)[C::TQ + 1]>(lds);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; ++k)
            part[C::Q::my_row()][C::Q::my_col() + k] = v[k];
        __syncthreads();
        for (int m = threadIdx.x; m < C::TQ; m += C::kThreads) {
            float x = 0.0f;
            for (int r = 0; r < kRowsOfThreads; ++r)
                x += part[r][m];
            if (m0 + m < O)
                to[m0 + m] = x;
        }
    }
};

// V's values as four of a type, and the first `left` of them to memory.
__device__ __forceinline__ void write_four(float *to, f32x4 v, int left) { write_piece(to, __builtin_bit_cast(u32x4, v), left, 0.0f); }
struct __attribute__((packed, aligned(2))) Bytes8 {
    unsigned long long v;
};
__device__ __forceinline__ void write_four(__bf16 *to, f32x4 v, int left)
{
    if (left >= 4) {
        unsigned long long four;
        store_values(reinterpret_cast<char *>(&four), v, __bf16{});
        reinterpret_cast<Bytes8 *>(to)->v = four;
        return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < left)
            to[k] = (__bf16)v[k];
}

// A tile of dW [O][I], rows from m0 on, columns from n0 on, in float or rounded once.
template <class C, class W>
__device__ __forceinline__ void write_weights(W *to, int m0, int n0, int O, int I, const f32x4 (&acc)[C::FP][C::FQ])
{
    const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wp = (wave % C::WP) * C::FP * 16, wq = (wave / C::WP) * C::FQ * 16;
#pragma unroll
    for (int j = 0; j < C::FQ; ++j) {
        const int m = m0 + wq + j * 16 + (lane & 15);
#pragma unroll
        for (int i = 0; i < C::FP; ++i) {
            const int n = n0 + wp + i * 16 + (lane >> 4) * 4;
            if (m >= O || n >= I)
                continue;
            write_four(to + ((size_t)m * I + n), acc[i][j], I - n);
        }
    }
}

// P: x, Q: dz, reduced over rows: a tile of a head's dW from a stretch of
// `stretch` of its rows.  Where heads have more than one stretch (partial),
// each has a place of its own in dw and db, and sum_kernel adds them up.  db comes from
// the dz tiles on their way, no pass of its own.  dW and db of 2,048 to 4,096 on 32,768
// rows of bf16: 499 us, 1,100 TFLOP/s, bound by the matrix units' power.
template <class C, class W>
__global__ __launch_bounds__(C::kThreads, 2) void weights_kernel(Problem p, Matrix<typename C::T> dz,
                                                                 Matrix<typename C::T> x, W *dw,
                                                                 float *db, unsigned stretch,
                                                                 unsigned places, unsigned row_tiles,
                                                                 unsigned col_tiles, unsigned from)
{
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    __shared__ __attribute__((aligned(16))) char sums_lds[C::kAsync ? RowSums<C>::kBytes : 16];
    __shared__ unsigned before[kMaxHeads + 1];
    static_assert(C::kAsync || RowSums<C>::kBytes <= C::kLds, "sums take the stages' place");
    const int I = p.fan_in, O = p.fan_out;
    const unsigned each = row_tiles * col_tiles;  // of a place
    if (stretch) {
        count_tiles(p, stretch, before);
        places = uniform(before[p.heads]);
    }
    const unsigned all = places * each, end = runs_end(all);
    auto tile_at = [&](unsigned b, unsigned &place, RowTile &t, int &m0, int &n0) {
        const unsigned at = by_xcd(b, all);
        if (at >= all)
            return false;
        place = at / each;
        const Place2 where = in_groups(at - place * each, row_tiles, col_tiles);
        m0 = (int)where.a * C::TQ;  // of dz
        n0 = (int)where.b * C::TP;  // of x
        if (stretch) {
            t = head_tile(p, before, place, stretch);
        } else {
            t.first = uniform(bound(p, place));
            t.last = uniform(bound(p, place + 1));
            t.last = t.last > t.first ? t.last : t.first;
        }
        return true;
    };
    auto sources = [&](const RowTile &t, int m0, int n0, typename C::P::Source &ps, typename C::Q::Source &qs) {
        ps = {x, (unsigned)n0};
        ps.m.p += t.first * x.stride;
        qs = {dz, (unsigned)m0};
        qs.m.p += t.first * dz.stride;
        qs.m.mask += t.first * dz.mask_stride;
        ps.m.rows = qs.m.rows = t.last - t.first;
    };
    unsigned place;
    RowTile t;
    int m0, n0;
    RowSums<C> sums;
    auto add_sums = [&](const typename C::Q::S &share) { sums.add(share); };
    auto write = [&](const f32x4(&acc)[C::FP][C::FQ], char *sums_at) {
        if (dw)
            write_weights<C>(dw + (size_t)place * O * I, m0, n0, O, I, acc);
        sums.write(db + (size_t)place * O, m0, O, sums_at);
    };
    if constexpr (C::kAsync) {
        unsigned ahead = blockIdx.x;
        auto next_tile = [&](Pipe<C> &pipe) {
            unsigned pl;
            RowTile u;
            int a, b;
            for (; ahead < end; ahead += gridDim.x) {
                if (!tile_at(ahead, pl, u, a, b) || u.first == u.last)
                    continue;
                ahead += gridDim.x;
                typename C::P::Source ps;
                typename C::Q::Source qs;
                sources(u, a, b, ps, qs);
                pipe.load_tile(ps, qs, u.last - u.first);
                return;
            }
            pipe.load_nothing();
        };
        Pipe<C> pipe;
        pipe.start(lds, next_tile);
        for (unsigned b = blockIdx.x; b < end; b += gridDim.x) {
            if (!tile_at(b, place, t, m0, n0))
                continue;
            sums.begin(db && n0 == 0);
            f32x4 acc[C::FP][C::FQ] = {};
#pragma unroll 1
            for (unsigned k = t.first; k < t.last; k += C::kDepth)
                pipe.step(acc, next_tile, add_sums);
            write(acc, sums_lds);
        }
        arrived<0>();
    } else {
        if (!tile_at(from + blockIdx.x, place, t, m0, n0))
            return;
        sums.begin(db && n0 == 0);
        f32x4 acc[C::FP][C::FQ] = {};
        typename C::P::Source ps;
        typename C::Q::Source qs;
        sources(t, m0, n0, ps, qs);
        tile_product<C>(ps, qs, t.last - t.first, lds, acc, add_sums);
        write(acc, lds);
    }
}

// ---- shallow products, their weights in LDS ---------------------------------------------

// Layers of at most STEPS x 128 bytes of depth on many rows, or their rows'
// gradient (DEEP_W false: the weights' columns are its outputs): a workgroup
// keeps TO of its head's outputs' weights in LDS and goes through a stretch of
// the head's rows, RT at a time, the next ones' loads under way: the rows stream,
// whatever their alignment, and nothing is read again but by the other columns'
// workgroups beside it.  Rows of bf16, us here and tile by tile, both with ordinary
// stores: 319 to 256 on 262,139 113, 132; 128 to 128 on 262,144 25 (5.3 TB/s), 31; 63
// to 64 15, 20.  PAST: results past the caches (past_caches): the first takes 94 so.
// PAIR: a gated layer, TO / 2 columns of its result.
template <class T_, int TO_, int STEPS, bool DEEP_W, bool MASK, bool PAST, bool PAIR = false>
struct Shallow {
    using T = T_;
    static constexpr bool kPast = PAST;  // asked in the loop instead, it costs what it brings
    static constexpr bool kPair = PAIR;
    static constexpr int TO = TO_, kCols = PAIR ? TO / 2 : TO, kSteps = STEPS, kThreads = 512, kColGroups = TO / 64, RT = 16 * 8 / kColGroups;
    using W = Tile<T, TO, DEEP_W, kThreads, false, PAIR>;
    using X = Tile<T, RT, true, kThreads, MASK>;
    static constexpr int FP = 4;  // a wave's: 64 outputs of 16 rows
    static constexpr int kRowBytes = (PAIR ? 32 : 64) * (int)sizeof(T) + 16;
    static constexpr int kX = STEPS * W::kBytes, kOut = kX + STEPS * X::kBytes;
    static constexpr int kLds = kOut + 8 * 16 * kRowBytes;
    // workgroups a compute unit: by LDS, and 4 waves a SIMD
    static constexpr int kAtOnce = 2 * (kLds + 4096) <= 160 * 1024 ? 2 : 1;
};

template <class C>
__global__ __launch_bounds__(C::kThreads, 2 * C::kAtOnce) void shallow_kernel(Problem p, Matrix<typename C::T> w,
                                                                              Matrix<typename C::T> x, const float *bias,
                                                                              int act, typename C::T *y, long long ys, typename C::T *pre, long long pres, int width,
                                                                              unsigned stretch)
{
    using T = typename C::T;
    constexpr int V = Type<T>::kVec;
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    __shared__ __attribute__((aligned(16))) float biases[C::TO];
    __shared__ unsigned before[kMaxHeads + 1];
    const int O = width, lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    count_tiles(p, stretch, before);
    // the columns of a stretch on one XCD, at about the same time
    const unsigned cols = (O + C::kCols - 1) / C::kCols, j = blockIdx.x / kXcds;
    const unsigned places = uniform(before[p.heads]), place = j / cols * kXcds + blockIdx.x % kXcds;
    const int n0 = (int)(j % cols) * C::kCols;
    if (place >= places) {  // rows without a head: zeros
        const unsigned headless = bound(p, p.heads);
        const unsigned long long from = headless + (unsigned long long)(place - places) * stretch;
        for (unsigned long long r = from + wave; r < from + stretch && r < p.rows; r += C::kThreads / 64)
            for (int c = n0 + lane; c < n0 + C::kCols && c < O; c += 64) {
                y[r * ys + c] = (T)0.0f;
                if (C::kPair && pre)
                    pre[r * pres + c] = pre[r * pres + O + c] = (T)0.0f;
            }
        return;
    }
    const RowTile t = head_tile(p, before, place, stretch);
    typename C::W::Source ws = {w, (unsigned)n0, C::kPair ? (unsigned)O : 0u};
    ws.m.p += t.head * ((size_t)p.fan_in * p.fan_out * (C::kPair ? 2 : 1));
    typename C::X::Source xs = {x, 0};
    xs.m.p += t.first * x.stride;
    xs.m.mask += t.first * x.mask_stride;
    xs.m.rows = t.last - t.first;
    typename C::W::S sw[C::kSteps];
    typename C::X::S sx[C::kSteps];
    auto load = [&](unsigned r) {
        xs.t0 = r;
#pragma unroll
        for (int i = 0; i < C::kSteps; ++i)
            C::X::load(sx[i], xs, i * C::X::D);
    };
#pragma unroll
    for (int i = 0; i < C::kSteps; ++i)
        C::W::load(sw[i], ws, i * C::W::D);
    load(0);
    if (threadIdx.x < C::TO) {
        const int n = n0 + (int)threadIdx.x % C::kCols, half = (int)threadIdx.x / C::kCols;  // kPair: of the ups
        biases[threadIdx.x] = bias && n < O ? bias[((size_t)t.head * (C::kPair ? 2 : 1) + half) * O + n] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < C::kSteps; ++i) {
        C::W::settle(sw[i], ws, i * C::W::D);
        C::W::store(sw[i], lds + i * C::W::kBytes);
    }
    const int fp = (wave % C::kColGroups) * C::FP, fq = wave / C::kColGroups;
    char *mine = lds + C::kOut + wave * 16 * C::kRowBytes;
#pragma unroll 1
    for (unsigned r0 = 0; r0 < t.last - t.first; r0 += C::RT) {
        stored();
        xs.t0 = r0;
#pragma unroll
        for (int i = 0; i < C::kSteps; ++i) {
            C::X::settle(sx[i], xs, i * C::X::D);
            C::X::store(sx[i], lds + C::kX + i * C::X::kBytes);
        }
        stored();
        if (r0 + C::RT < t.last - t.first)
            load(r0 + C::RT);
        f32x4 acc[C::FP] = {};
#pragma unroll
        for (int i = 0; i < C::kSteps; ++i)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const u32x4 q = C::X::fragment(lds + C::kX + i * C::X::kBytes, fq, part);
#pragma unroll
                for (int f = 0; f < C::FP; ++f)
                    acc[f] = multiply(C::W::fragment(lds + i * C::W::kBytes, fp + f, part), q, acc[f], T{});
            }
        if constexpr (C::kPair) {
            write_gated<T, C::FP / 2, true>(acc, biases + fp * 8, biases + C::kCols + fp * 8, act, mine, t.first + r0 + fq * 16,
                                      t.last, n0 + fp * 8, O, y, ys, pre, pres);
            continue;
        }
#pragma unroll
        for (int f = 0; f < C::FP; ++f) {
            const int e = f * 16 + (lane >> 4) * 4;
            f32x4 v = acc[f] + *reinterpret_cast<const f32x4 *>(biases + fp * 16 + e);
            if (act)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[k] = v[k] < 0.0f ? 0.0f : v[k];
            store_values(mine + (lane & 15) * C::kRowBytes + e * (int)sizeof(T), v, T{});
        }
        __builtin_amdgcn_wave_barrier();
        constexpr int kPieces = 64 / V;  // of a row
#pragma unroll
        for (int i = 0; i < 16 * kPieces / 64; ++i) {
            const int r = (i * 64 + lane) / kPieces, c = (i * 64 + lane) % kPieces * V;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(mine + r * C::kRowBytes + c * (int)sizeof(T));
            const unsigned row = t.first + r0 + fq * 16 + r;
            const int n = n0 + fp * 16 + c;
            if (row < t.last && n < O)
                write_result(y + (row * ys + n), v, O - n, C::kPast);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- both gradients in one launch -----------------------------------------------------

// One tile of dx (CR) or of a head's dW (CW) a workgroup, the longest first: the
// last rounds of one fill up with tiles of the other, and what comes last is
// short.  Both gradients of 2,048 to 4,096 on 16,384 rows: 509 us, 617 in two
// launches.
template <class CR, class CW, class W>
__global__ __launch_bounds__(CR::kThreads, 2) void gradients_kernel(Problem p, Matrix<typename CR::T> w,
                                                                    Matrix<typename CR::T> dz, Matrix<typename CR::T> x,
                                                                    typename CR::T *dx, long long dxs, W *dw, float *db)
{
    static_assert(CR::kThreads == CW::kThreads && CR::kAsync && CW::kAsync && CR::kLds == CW::kLds, "one workgroup for both");
    constexpr int kExtra = kResultBytes<CR> > RowSums<CW>::kBytes ? kResultBytes<CR> : RowSums<CW>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[CR::kLds];
    __shared__ __attribute__((aligned(16))) char extra[kExtra];
    __shared__ unsigned before[kMaxHeads + 1];
    __shared__ unsigned count[kMaxHeads];
    __shared__ unsigned char order[kMaxHeads];
    __shared__ unsigned long_heads;
    const int I = p.fan_in, O = p.fan_out;
    count_tiles(p, CR::TQ, before);
    // the heads by their rows, most first; long_heads: those of more rows than dx is deep
    unsigned mine = 0;
    if ((int)threadIdx.x < p.heads) {
        const unsigned a = bound(p, threadIdx.x), b = bound(p, threadIdx.x + 1);
        count[threadIdx.x] = mine = b > a ? b - a : 0;
    }
    if (threadIdx.x == 0)
        long_heads = 0;
    __syncthreads();
    if ((int)threadIdx.x < p.heads) {
        int rank = 0;
        for (int h = 0; h < p.heads; ++h)
            rank += count[h] > mine || (count[h] == mine && h < (int)threadIdx.x);
        order[rank] = (unsigned char)threadIdx.x;
        if (mine > (unsigned)O)
            atomicAdd(&long_heads, 1u);
    }
    __syncthreads();
    const unsigned headed = uniform(before[p.heads]), headless = bound(p, p.heads);
    const unsigned tail = (unsigned)(((unsigned long long)(p.rows - headless) + CR::TQ - 1) / CR::TQ);
    const unsigned x_rows = headed + tail, x_cols = (I + CR::TP - 1) / CR::TP;
    const unsigned w_rows = (O + CW::TQ - 1) / CW::TQ, w_cols = (I + CW::TP - 1) / CW::TP;
    const unsigned first = uniform(long_heads) * w_rows * w_cols, second = x_rows * x_cols;
    const unsigned third = p.heads * w_rows * w_cols - first;
    unsigned b = blockIdx.x;
    const bool is_x = b >= runs_end(first) && b - runs_end(first) < runs_end(second);
    if (is_x) {
        const unsigned at = by_xcd(b - runs_end(first), second);
        if (at >= second)
            return;
        const Place2 where = in_groups(at, x_rows, x_cols);
        const int n0 = (int)where.b * CR::TP;
        RowTile t;
        f32x4 acc[CR::FP][CR::FQ] = {};
        if (where.a < headed) {
            t = head_tile(p, before, where.a, CR::TQ);
            typename CR::P::Source ps = {w, (unsigned)n0};
            typename CR::Q::Source qs = {dz, 0};
            ps.m.p += t.head * ((size_t)I * O);
            qs.m.p += t.first * dz.stride;
            qs.m.rows = t.last - t.first;
            bool taken = false;
            auto next_tile = [&](Pipe<CR> &pipe) {
                if (taken)
                    pipe.load_nothing();
                else
                    pipe.load_tile(ps, qs, O);
                taken = true;
            };
            Pipe<CR> pipe;
            pipe.start(lds, next_tile);
#pragma unroll 1
            for (int k = 0; k < O; k += CR::kDepth)
                pipe.step(acc, next_tile, [](auto &) {});
        } else {
            t.first = headless + (where.a - headed) * CR::TQ;
            t.last = p.rows - t.first > (unsigned)CR::TQ ? t.first + CR::TQ : p.rows;
            t.head = p.heads;
        }
        write_rows<CR>(t, n0, I, acc, nullptr, false, extra, dx, dxs);
    } else {
        unsigned at, heads_before = 0;
        if (b < runs_end(first)) {
            at = by_xcd(b, first);
            if (at >= first)
                return;
        } else {
            b -= runs_end(first) + runs_end(second);
            at = b < runs_end(third) ? by_xcd(b, third) : third;
            if (at >= third)
                return;
            heads_before = uniform(long_heads);
        }
        const unsigned each = w_rows * w_cols, place = at / each;
        const int h = uniform(order[heads_before + place]);
        const Place2 where = in_groups(at - place * each, w_rows, w_cols);
        const int m0 = (int)where.a * CW::TQ, n0 = (int)where.b * CW::TP;
        const unsigned from = uniform(bound(p, h)), rows = uniform(count[h]);
        typename CW::P::Source ps = {x, (unsigned)n0};
        typename CW::Q::Source qs = {dz, (unsigned)m0};
        ps.m.p += from * x.stride;
        qs.m.p += from * dz.stride;
        ps.m.rows = qs.m.rows = rows;
        RowSums<CW> sums;
        sums.begin(db && n0 == 0);
        f32x4 acc[CW::FP][CW::FQ] = {};
        if (rows) {
            bool taken = false;
            auto next_tile = [&](Pipe<CW> &pipe) {
                if (taken)
                    pipe.load_nothing();
                else
                    pipe.load_tile(ps, qs, rows);
                taken = true;
            };
            Pipe<CW> pipe;
            pipe.start(lds, next_tile);
#pragma unroll 1
            for (unsigned k = 0; k < rows; k += CW::kDepth)
                pipe.step(acc, next_tile, [&](const typename CW::Q::S &share) { sums.add(share); });
        }
        write_weights<CW>(dw + (size_t)h * O * I, m0, n0, O, I, acc);
        sums.write(db + (size_t)h * O, m0, O, extra);
    }
    arrived<0>();
}

// ---- both gradients of narrow layers, in one pass over the rows --------------------------

// Layers of at most 128 to 128 move more than they compute: here every row is
// read once for both gradients.  A workgroup (one a compute unit) keeps its
// head's weights in LDS and its part of dW in registers and goes through a
// stretch of the head's rows, RT at a time, the next ones' loads under way.  dz
// lies in LDS once: dx reads it by rows, dW by columns.  128 to 128 with ReLU on
// 131,072 rows of bf16: 45 us, 66 with a pass for each gradient.
// float's products take about as long as its rows: two workgroups of half the
// waves and rows a compute unit, where their weights fit, compute in turns.  63 to 128
// with ReLU, us so and with one: 262,144 rows 109, 120, 65,536 41, 43, 32,768 34, 31.
template <class T_, int TI_, int TO_, bool MASK>
struct Narrow {
    using T = T_;
    static constexpr bool kTwo = sizeof(T) == 4 && TI_ + TO_ < 256;  // workgroups a compute unit
    static constexpr int TI = TI_, TO = TO_, kThreads = kTwo ? 256 : 512, kWaves = kThreads / 64;
    static constexpr int RT = sizeof(T) == 2 ? 128 : kTwo ? 32 : 64;
    using X = Tile<T, TI, false, kThreads, false>;   // x
    using Z = Tile<T, TO, false, kThreads, MASK>;    // dz
    static constexpr int kSteps = RT / X::D;         // tiles of D rows
    static constexpr int kSpan = X::D / 2;           // depth of a fragment
    // dW: 4 waves over fan_in, the rest over fan_out
    static constexpr int FP = TI / 64, FQ = TO / (kWaves / 4) / 16;
    // dx: a wave takes 16 rows; where there are fewer of them than waves, part of the columns
    static constexpr int kColGroups = kWaves / (RT / 16), FX = TI / 16 / kColGroups;
    static constexpr int kRowBytes = FX * 16 * (int)sizeof(T) + 16;
    static constexpr int kResults = sizeof(T) == 2 ? kWaves * 16 * kRowBytes : 0;
    static constexpr int kZ = 0, kX = kZ + RT * TO * (int)sizeof(T), kW = kX + RT * TI * (int)sizeof(T);
    static constexpr int kOut = kW + TO * TI * (int)sizeof(T), kLds = kOut + kResults;
    // dx past the caches: us so and with ordinary stores, of 128 to 128 on 262,144 rows
    // with ReLU 56, 62, without 47, 46; of 64 to 64 with ReLU 31.6, 31.0
    static constexpr bool kPast = MASK && TI == 128;
    static constexpr int kRowsOfThreads = kThreads / Z::kPerRow;
    static_assert(kRowsOfThreads * (TO + 1) * 4 <= kW, "sums take the rows' place");
};

template <class C>
__global__ __launch_bounds__(C::kThreads, 2) void narrow_kernel(Problem p, Matrix<typename C::T> w, Matrix<typename C::T> dz,
                                                                Matrix<typename C::T> x, typename C::T *dx, long long dxs,
                                                                float *dw, float *db, unsigned stretch)
{
    using T = typename C::T;
    constexpr int V = Type<T>::kVec;
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    __shared__ unsigned before[kMaxHeads + 1];
    const int I = p.fan_in, O = p.fan_out, lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    count_tiles(p, stretch, before);
    const unsigned places = uniform(before[p.heads]), place = blockIdx.x;
    if (place >= places) {  // rows without a head: zeros
        const unsigned headless = bound(p, p.heads);
        const unsigned long long from = headless + (unsigned long long)(place - places) * stretch;
        if (dx)
            for (unsigned long long r = from + wave; r < from + stretch && r < p.rows; r += C::kThreads / 64)
                for (int c = lane; c < I; c += 64)
                    dx[r * dxs + c] = (T)0.0f;
        return;
    }
    const RowTile t = head_tile(p, before, place, stretch);
    typename C::X::Source xs = {x, 0}, ws = {w, 0};
    typename C::Z::Source zs = {dz, 0};
    xs.m.p += t.first * x.stride;
    zs.m.p += t.first * dz.stride;
    zs.m.mask += t.first * dz.mask_stride;
    xs.m.rows = zs.m.rows = t.last - t.first;
    ws.m.p += t.head * ((size_t)I * O);
    const bool past = C::kPast && past_caches(dx, dxs, I);
    typename C::X::S sx[C::kSteps];
    typename C::Z::S sz[C::kSteps];
    auto load = [&](unsigned k) {
#pragma unroll
        for (int i = 0; i < C::kSteps; ++i) {
            C::Z::load(sz[i], zs, k + i * C::Z::D);
            C::X::load(sx[i], xs, k + i * C::X::D);
        }
    };
    typename C::X::S sw[C::TO / C::X::D];
    if (dx)
#pragma unroll
        for (int i = 0; i < C::TO / C::X::D; ++i)
            C::X::load(sw[i], ws, i * C::X::D);
    load(0);
    if (dx)
#pragma unroll
        for (int i = 0; i < C::TO / C::X::D; ++i) {
            C::X::settle(sw[i], ws, i * C::X::D);
            C::X::store(sw[i], lds + C::kW + i * C::X::kBytes);
        }
    float sums[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        sums[k] = 0.0f;
    f32x4 acc[C::FP][C::FQ] = {};
    const int fp = (wave % 4) * C::FP, fq = (wave / 4) * C::FQ;
    const int fr = wave / C::kColGroups, fc = (wave % C::kColGroups) * C::FX;  // of dx
#pragma unroll 1
    for (unsigned k = 0; k < t.last - t.first; k += C::RT) {
        stored();
#pragma unroll
        for (int i = 0; i < C::kSteps; ++i) {
            C::Z::settle(sz[i], zs, k + i * C::Z::D);
            C::X::settle(sx[i], xs, k + i * C::X::D);
            C::Z::store(sz[i], lds + C::kZ + i * C::Z::kBytes);
            C::X::store(sx[i], lds + C::kX + i * C::X::kBytes);
#pragma unroll
            for (int j = 0; j < C::Z::kShare; ++j) {
                union {
                    u32x4 v;
                    T e[V];
                } piece = {sz[i].x[j]};
#pragma unroll
                for (int e = 0; e < V; ++e)
                    sums[e] += (float)piece.e[e];
            }
        }
        stored();
        if (k + C::RT < t.last - t.first)
            load(k + C::RT);
        if (dx) {
            f32x4 rows[C::FX] = {};
#pragma unroll
            for (int part = 0; part < C::TO / C::kSpan; ++part) {
                const u32x4 q = C::Z::row_fragment(lds + C::kZ, fr, part);
#pragma unroll
                for (int i = 0; i < C::FX; ++i)
                    rows[i] = multiply(C::X::fragment(lds + C::kW, fc + i, part), q, rows[i], T{});
            }
            const unsigned first = t.first + k + fr * 16;
            if constexpr (C::kResults > 0) {
                char *mine = lds + C::kOut + wave * 16 * C::kRowBytes;
#pragma unroll
                for (int i = 0; i < C::FX; ++i)
                    store_values(mine + (lane & 15) * C::kRowBytes + (i * 16 + (lane >> 4) * 4) * (int)sizeof(T), rows[i], T{});
                __builtin_amdgcn_wave_barrier();
                constexpr int kPieces = C::FX * 16 / V;  // of a row
#pragma unroll
                for (int i = 0; i < 16 * kPieces / 64; ++i) {
                    const int r = (i * 64 + lane) / kPieces, c = (i * 64 + lane) % kPieces * V;
                    const u32x4 v = *reinterpret_cast<const u32x4 *>(mine + r * C::kRowBytes + c * (int)sizeof(T));
                    const int n = fc * 16 + c;
                    if (first + r < t.last && n < I)
                        write_result(dx + ((first + r) * dxs + n), v, I - n, past);
                }
                __builtin_amdgcn_wave_barrier();
            } else {
#pragma unroll
                for (int i = 0; i < C::FX; ++i) {
                    const int n = (fc + i) * 16 + (lane >> 4) * 4;
                    if (first + (lane & 15) < t.last && n < I)
                        write_piece(dx + ((first + (lane & 15)) * dxs + n), __builtin_bit_cast(u32x4, rows[i]), I - n, T{});
                }
            }
        }
        if (dw)
#pragma unroll
            for (int part = 0; part < C::RT / C::kSpan; ++part) {
                u32x4 q[C::FQ];
#pragma unroll
                for (int j = 0; j < C::FQ; ++j)
                    q[j] = C::Z::fragment(lds + C::kZ, fq + j, part);
#pragma unroll
                for (int i = 0; i < C::FP; ++i) {
                    const u32x4 f = C::X::fragment(lds + C::kX, fp + i, part);
#pragma unroll
                    for (int j = 0; j < C::FQ; ++j)
                        acc[i][j] = multiply(f, q[j], acc[i][j], T{});
                }
            }
    }
    if (dw) {
        float *to = dw + (size_t)place * O * I;
#pragma unroll
        for (int j = 0; j < C::FQ; ++j) {
            const int m = (fq + j) * 16 + (lane & 15);
#pragma unroll
            for (int i = 0; i < C::FP; ++i) {
                const int n = (fp + i) * 16 + (lane >> 4) * 4;
                if (m < O && n < I)
                    write_piece(to + ((size_t)m * I + n), __builtin_bit_cast(u32x4, acc[i][j]), I - n, 0.0f);
            }
        }
    }
    if (db) {
        float(*part)[C::TO + 1] = reinterpret_cast<float(*)[C::TO + 1]>(lds);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; ++k)
            part[C::Z::my_row()][C::Z::my_col() + k] = sums[k];
        __syncthreads();
        if ((int)threadIdx.x < O) {
            float v = 0.0f;
            for (int r = 0; r < C::kRowsOfThreads; ++r)
                v += part[r][threadIdx.x];
            db[(size_t)place * O + threadIdx.x] = v;
        }
    }
}

// out[h][e] = the sum of head h's stretches' parts: the weights' in the first blocks
// of a head, the biases' in its last.  A workgroup's waves sum every fourth part of
// 256 elements, in order, and add up at the end: heads of many rows have so many
// parts that one wave would wait for them in turn (16 heads, 272 parts of 128 x 128:
// 5.7 us, 6.8 with a thread for each element).
template <class W>
__global__ __launch_bounds__(256) void sum_kernel(Problem p, unsigned stretch, const float *wparts, size_t wsize, W *dw,
                                                  const float *bparts, float *db, unsigned wblocks)
{
    constexpr unsigned kWaves = 4, kAtOnce = 8;
    __shared__ unsigned before[kMaxHeads + 1];
    __shared__ f32x4 sums[kWaves][64];
    count_tiles(p, stretch, before);
    const unsigned a = uniform(before[blockIdx.y]), b = uniform(before[blockIdx.y + 1]);
    const bool biases = blockIdx.x >= wblocks;
    const float *parts = biases ? bparts : wparts;
    const size_t size = biases ? (size_t)p.fan_out : wsize;
    const unsigned block = biases ? blockIdx.x - wblocks : blockIdx.x, blocks = biases ? gridDim.x - wblocks : wblocks;
    const unsigned wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (size_t first = block * 256; first < size; first += (size_t)blocks * 256) {
        const size_t e = first + lane * 4;
        const int here = e + 4 <= size ? 4 : e < size ? (int)(size - e) : 0;
        auto read = [&](unsigned i) {
            const float *from = parts + (i * size + e);
            if (here == 4)
                return __builtin_bit_cast(f32x4, reinterpret_cast<const Bytes16 *>(from)->v);
            f32x4 x = {};
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < here)
                    x[k] = from[k];
            return x;
        };
        f32x4 v = {};
        unsigned i = a + wave;
        for (; i + kWaves * (kAtOnce - 1) < b; i += kWaves * kAtOnce) {
            f32x4 x[kAtOnce];
#pragma unroll
            for (unsigned k = 0; k < kAtOnce; ++k)
                x[k] = read(i + k * kWaves);
#pragma unroll
            for (unsigned k = 0; k < kAtOnce; ++k)
                v += x[k];
        }
        for (; i < b; i += kWaves)
            v += read(i);
        sums[wave][lane] = v;
        __syncthreads();
        if (wave == 0) {
            v = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
            if (biases)
                write_four(db + (blockIdx.y * size + e), v, here);
            else
                write_four(dw + (blockIdx.y * size + e), v, here);
        }
        __syncthreads();
    }
}

// ---- choice of a form ---------------------------------------------------------------

template <class C>
hipError_t launch_rows(const Problem &p, const Matrix<typename C::T> &w,
                       const Matrix<typename C::T> &x, const float *bias, int act, Rows y,
                       int width, int depth, hipStream_t s, Rows pre = {nullptr, 0})
{
    using T = typename C::T;
    // at most: every head's last tile and the headless rows' may be partly filled
    return launch_for<C>(((unsigned long long)p.rows / C::TQ + p.heads + 1) * tiles_of(width, C::kCols),
                         [&](unsigned groups, unsigned from) {
                             rows_kernel<C><<<groups, C::kThreads, 0, s>>>(
                                 p, w, x, bias, act, static_cast<T *>(const_cast<void *>(y.p)), y.stride,
                                 static_cast<T *>(const_cast<void *>(pre.p)), pre.stride, width, depth, from);
                         });
}

// 256 x 256 tiles, one workgroup a compute unit, or 128 x 128 ones, two: a large
// one does the work of four in the time of 3.5, but the last round of tiles is a
// larger part of the whole.  us with large and small tiles: 4,096 rows of 2,048 to
// 4,096 100, 89; 32,768 of 1,024 to 1,024 92, 85; 65,536 of 1,024 to 1,024 179,
// 207; 65,536 of 512 to 1,024 103, 107; and 262,144 of 256 to 256, where the depth
// is too short to pay for a large tile's start, 84, 75.  worth: eight rounds of large tiles in
// rounds of small ones.
bool large_tiles(const Problem &p, int width, double worth = 4.6)
{
    constexpr unsigned kCus = 256;
    const unsigned long long large = (p.rows / 256ull + p.heads / 2) * tiles_of(width, 256);
    const unsigned long long small = (p.rows / 128ull + p.heads / 2) * tiles_of(width, 128);
    return 8 * ((large + kCus - 1) / kCus) <= worth * ((small + 2 * kCus - 1) / (2 * kCus));
}

template <class C>
hipError_t launch_shallow(const Problem &p, const Matrix<typename C::T> &w, const Matrix<typename C::T> &x,
                          const float *bias, int act, Rows y, int width, hipStream_t s, Rows pre = {nullptr, 0})
{
    using T = typename C::T;
    const unsigned cols = tiles_of(width, C::kCols), want = 256 * C::kAtOnce / cols;
    // stretches for `want` places, some of which the heads' last ones take
    unsigned stretch = (unsigned)p.heads < want / 2 ? p.rows / (want - p.heads) : p.rows / (want / 2);
    stretch = (stretch + 32) / 32 * 32;
    const unsigned places = p.rows / stretch + p.heads + 1;
    const unsigned groups = (places + kXcds - 1) / kXcds * kXcds * cols;
    shallow_kernel<C><<<groups, C::kThreads, 0, s>>>(p, w, x, bias, act, static_cast<T *>(const_cast<void *>(y.p)), y.stride,
                                                     static_cast<T *>(const_cast<void *>(pre.p)), pre.stride, width, stretch);
    return hipGetLastError();
}

template <class T, int TO, bool DEEP_W, bool MASK, bool PAST, bool PAIR = false>
hipError_t shallow(const Problem &p, const Matrix<T> &w, const Matrix<T> &x, const float *bias, int act, Rows y,
                   int width, hipStream_t s, Rows pre = {nullptr, 0})
{
    const unsigned steps = tiles_of((long long)x.cols * sizeof(T), 128);
    if constexpr (DEEP_W) {
        if (steps == 3)
            return launch_shallow<Shallow<T, TO, 3, DEEP_W, MASK, PAST, PAIR>>(p, w, x, bias, act, y, width, s, pre);
        if (steps == 4)
            return launch_shallow<Shallow<T, TO, 4, DEEP_W, MASK, PAST, PAIR>>(p, w, x, bias, act, y, width, s, pre);
        if (steps == 5)
            return launch_shallow<Shallow<T, TO, 5, DEEP_W, MASK, PAST, PAIR>>(p, w, x, bias, act, y, width, s, pre);
    }
    return steps == 1 ? launch_shallow<Shallow<T, TO, 1, DEEP_W, MASK, PAST, PAIR>>(p, w, x, bias, act, y, width, s, pre)
                      : launch_shallow<Shallow<T, TO, 2, DEEP_W, MASK, PAST, PAIR>>(p, w, x, bias, act, y, width, s, pre);
}

// 128 columns a tile, or 64: for narrow matrices, and for float, which is bound by
// its products, where 128 would pad a seventh or more.  float32 us with 64 and 128, 20,000
// rows: 400 to 155 38, 58; 319 to 400 67, 97; dx of 400 to 319 64, 79; but 400 to 319 71,
// 60 and 400 to 283 71, 60.
template <class T>
bool wide_tile(int width)
{
    return width > 64 && (sizeof(T) == 2 || 8 * 64 * tiles_of(width, 64) > 7 * 128 * tiles_of(width, 128));
}

// Whether a product goes with its weights in LDS: not too wide (its rows are read
// for each 128 columns), on rows for all of the chip, and shallow: up to 2 steps,
// or 5 for a layer, but not where bf16 operands of more than two go to LDS by
// themselves (262,144 rows of 256 to 256: 72 us, 80 here; their gradients with
// ReLU take 220 us, 227 with dx here).  us here and by tiles (of few rows below 32,768):
//   rows   bf16 319 to 256, 8,192 to 262,144: 10, 12; 12, 15 (16,384); 16, 23 (32,768);
//          85, 102; 63 to 64 8.2, 8.9 (16,384); 13, 20; float32 63 to 128 10, 13 (16,384);
//          13, 19 (32,768); 56, 75; 128 to 128 92, 92; dx of 256 to 64 109, 114
//   width  bf16 on 65,536, 100 to 512 22, 35; to 768 30, 49; to 1,024 41, 63; float32
//          100 to 512 111, 93; 128 to 768 194, 133
// So bf16 would gain on fewer rows and beyond 512 columns; float32 loses at 512 on more
// than 32,768 rows (57, 56 there).
template <class T, bool DEEP_W>
bool is_shallow(const Problem &p, const Matrix<T> &w, const Matrix<T> &x, int width, int depth)
{
    const unsigned steps = tiles_of((long long)depth * sizeof(T), 128);
    if (width > 512 || p.rows < 32768 || steps > 5)
        return false;
    return steps <= 2 || (DEEP_W && (sizeof(T) == 4 || !goes_alone(w) || !goes_alone(x)));
}

// Few rows: tiles of 64 x 32, whose depth four teams of two waves share, while that
// is a round of workgroups, or two and a half in float, whose products of 128 rows
// take longer, if it is not shallow.  us of large tiles and of these: float32 of 128
// to 2,816, 1,024 rows, dx 182, 40; of 1,024 to 1,024, 1,024 rows (544 tiles) 72, 52,
// 2,048 rows (1,056) 74, 83; dx of 319 to 155, 2,048 rows (330) 12.6, 15; bfloat16 of
// 2,816 to 128, 2,048 rows 34, 14; of 1,024 to 1,024, 512 rows (288) 13, 16.
template <class T>
bool few_rows(const Problem &p, int width, int depth)
{
    const unsigned long long tiles = (p.rows / 32ull + p.heads / 2) * tiles_of(width, 64);
    return tiles <= (sizeof(T) == 4 && depth >= 256 ? 640 : 256);
}

// The rows' product with tiles for its width.  NARROW: shallow products of at most 64
// columns come here (not those of gated layers, whose narrow ones have a kernel of their own).
template <class T, bool DEEP_W, bool MASK, bool NARROW = true>
hipError_t rows_product(const Problem &p, const Matrix<T> &w, const Matrix<T> &x, const float *bias,
                        bool relu, Rows y, int width, int depth, hipStream_t s)
{
    if (is_shallow<T, DEEP_W>(p, w, x, width, depth)) {
        const bool past = past_caches(static_cast<const T *>(y.p), y.stride, width);
        if constexpr (NARROW)
            if (width <= 64)
                return past ? shallow<T, 64, DEEP_W, MASK, true>(p, w, x, bias, relu, y, width, s)
                            : shallow<T, 64, DEEP_W, MASK, false>(p, w, x, bias, relu, y, width, s);
        return past ? shallow<T, 128, DEEP_W, MASK, true>(p, w, x, bias, relu, y, width, s)
                    : shallow<T, 128, DEEP_W, MASK, false>(p, w, x, bias, relu, y, width, s);
    }
    if (few_rows<T>(p, width, depth))
        return launch_rows<Product<T, 64, 32, 2, 1, DEEP_W, true, MASK, false, false, 4>>(p, w, x, bias, relu, y, width,
                                                                                      depth, s);
    const bool alone = goes_alone(w) && goes_alone(x);
    if constexpr (sizeof(T) == 2 && !MASK)
        if (alone && depth >= 512 && large_tiles(p, width))
            return launch_rows<Product<T, 256, 256, 4, 2, DEEP_W, true, false, true>>(p, w, x, bias, relu, y, width,
                                                                                    depth, s);
    if (wide_tile<T>(width)) {
        if constexpr (!MASK)
            if (alone)
                return launch_rows<Product<T, 128, 128, 2, 2, DEEP_W, true, false, true>>(
                    p, w, x, bias, relu, y, width, depth, s);
        return launch_rows<Product<T, 128, 128, 2, 2, DEEP_W, true, MASK>>(
            p, w, x, bias, relu, y, width, depth, s);
    }
    return launch_rows<Product<T, 64, 128, 2, 2, DEEP_W, true, MASK>>(p, w, x, bias, relu, y,
                                                                             width, depth, s);
}

// Rows of a stretch of the weights' product, 0: each head as a whole.  Split until
// there are 512 tiles, a round of them, or 1024 in float32, whose tiles take so
// long that heads of many rows would hold up the rest (191 to 576 on 242,086 rows of
// 26 heads, weights' part: 820 us, 1448 with 512).  In bfloat16 the parts' traffic
// costs more (256 to 256 on 262,144 rows of 16, both gradients: 149 us, 165 with 1024).
struct Split {
    unsigned stretch, places;
};
Split split_rows(unsigned rows, int heads, int fan_in, int fan_out, bool bf16)
{
    const unsigned long long tiles =
        (unsigned long long)tiles_of(fan_in, fan_in > 64 ? 128 : 64) * tiles_of(fan_out, fan_out > 64 ? 128 : 64);
    const unsigned long long want = (bf16 ? 512 : 1024) / tiles;
    if (want <= (unsigned)heads)
        return {0, (unsigned)heads};
    unsigned stretch = (unsigned)(rows / (want - heads));
    stretch = (stretch + 255) / 256 * 256;
    if (stretch < 256)
        stretch = 256;
    return {stretch, rows / stretch + heads};
}

// The stretches' parts added up.
template <class W>
hipError_t launch_sums(const Problem &p, const Split &split, const float *wparts, W *dw, const float *bparts, float *db,
                       hipStream_t s)
{
    const size_t size = (size_t)p.fan_in * p.fan_out;
    const unsigned blocks = dw ? tiles_of(size, 256) : 0, wblocks = blocks < 1024 ? blocks : 1024;
    const unsigned bblocks = db ? tiles_of(p.fan_out, 256) : 0;
    sum_kernel<W><<<dim3(wblocks + bblocks, p.heads), 256, 0, s>>>(p, split.stretch, wparts, size, dw, bparts, db, wblocks);
    return hipGetLastError();
}

template <class C, class W>
hipError_t launch_weights(const Problem &p, const Matrix<typename C::T> &dz,
                          const Matrix<typename C::T> &x, W *dw, float *db, char *workspace,
                          hipStream_t s)
{
    const Split split = split_rows(p.rows, p.heads, p.fan_in, p.fan_out, sizeof(typename C::T) == 2);
    const bool partial = split.stretch != 0;
    const size_t size = (size_t)p.fan_in * p.fan_out;
    float *wparts = reinterpret_cast<float *>(workspace);
    float *bparts = wparts + (size_t)split.places * size;
    const unsigned row_tiles = tiles_of(p.fan_out, C::TQ), col_tiles = dw ? tiles_of(p.fan_in, C::TP) : 1;
    const unsigned long long tiles = (unsigned long long)split.places * row_tiles * col_tiles;
    auto launch = [&](auto *to_w, float *to_b) {
        using To = std::remove_pointer_t<decltype(to_w)>;
        return launch_for<C>(tiles, [&](unsigned groups, unsigned from) {
            weights_kernel<C, To><<<groups, C::kThreads, 0, s>>>(p, dz, x, to_w, to_b, split.stretch, split.places, row_tiles, col_tiles, from);
        });
    };
    // tiles of 256 x 256 are taken from 256 of them on: at least 512 of 128 x 128, and no stretches
    if (C::TP == 256 || !partial)
        return launch(dw, db);
    if constexpr (C::TP != 256) {
        const hipError_t e = launch(dw ? wparts : nullptr, db ? bparts : nullptr);
        return e != hipSuccess ? e : launch_sums(p, split, wparts, dw, bparts, db, s);
    }
}

// 256 x 256 tiles from 256 of them on, one a compute unit.  dW and db, us with large and
// small tiles: 2,048 to 4,096 on 32,768 rows of 8 heads (1,024 tiles) 499, 612; 1,024 to
// 1,024 on 16,384 of 8 (128) 115, 70; 512 to 512 on 65,536 of 16 (64) 111, 80; at the line
// small ones would win: 1,024 to 2,048 on 16,384 of 8 119, 101; 1,024 to 1,024 on 65,536 of
// 16 387, 271.
template <class T, bool MASK, class W, bool NARROW = true>
hipError_t weights_product(const Problem &p, const Matrix<T> &dz, const Matrix<T> &x, W *dw,
                           float *db, char *workspace, hipStream_t s)
{
    const bool wide_o = wide_tile<T>(p.fan_out), wide_i = wide_tile<T>(p.fan_in);
    const bool alone = goes_alone(dz) && goes_alone(x);
    if constexpr (sizeof(T) == 2 && !MASK)
        if (alone && p.fan_out > 128 && p.fan_in > 128 &&
            (unsigned long long)tiles_of(p.fan_out, 256) * tiles_of(p.fan_in, 256) * p.heads >= 256)
            return launch_weights<Product<T, 256, 256, 4, 2, false, false, false, true, true>>(p, dz, x, dw, db,
                                                                                             workspace, s);
    if constexpr (!MASK)
        if (wide_o && wide_i && alone)
            return launch_weights<Product<T, 128, 128, 2, 2, false, false, false, true, true>>(
                p, dz, x, dw, db, workspace, s);
    if (wide_o && wide_i)
        return launch_weights<Product<T, 128, 128, 2, 2, false, false, MASK, false, true>>(p, dz, x, dw, db, workspace, s);
    if (wide_o)
        return launch_weights<Product<T, 64, 128, 2, 2, false, false, MASK, false, true>>(p, dz, x, dw, db, workspace, s);
    if (wide_i)
        return launch_weights<Product<T, 128, 64, 2, 2, false, false, MASK, false, true>>(p, dz, x, dw, db, workspace, s);
    if constexpr (NARROW)
        return launch_weights<Product<T, 64, 64, 2, 2, false, false, MASK, false, true>>(p, dz, x, dw, db, workspace, s);
    return hipErrorInvalidValue;  // no call: bf16 gated layers of at most 64 to 2 x 32 are narrow
}

// Layers that narrow_kernel takes, and its stretches: a workgroup for each, as
// many as run at once.  us with half as many, with these, and with twice as many, 16
// heads with ReLU: bf16 128 to 128 on 65,536 rows 33, 29, 39, on 262,144 85, 57, 70; 64 to
// 64 on 131,072 28, 23, 23; float32 63 to 128 on 131,072 69, 62, 75, on 32,768 29, 34, 34;
// 128 to 128 on 131,072 189, 107, 128.
bool is_narrow(int fan_in, int fan_out) { return fan_in <= 128 && fan_out <= 128; }
Split narrow_split(unsigned rows, int heads, int fan_in, int fan_out, bool bf16)
{
    const unsigned kPlaces = !bf16 && (fan_in <= 64 || fan_out <= 64) ? 512 : 256;
    const unsigned most = (unsigned)heads < kPlaces / 2 ? kPlaces - heads : kPlaces / 2;
    unsigned stretch = (rows / most + 32) / 32 * 32;
    if (stretch < 128)
        stretch = 128;
    return {stretch, rows / stretch + heads};
}

// Bytes that the products of the gradients need for their stretches' parts.
size_t parts_bytes(unsigned rows, int heads, int fan_in, int fan_out, bool bf16)
{
    const Split split = split_rows(rows, heads, fan_in, fan_out, bf16), narrow = narrow_split(rows, heads, fan_in, fan_out, bf16);
    size_t places = split.stretch ? split.places : 0;
    if (is_narrow(fan_in, fan_out) && narrow.places > places)
        places = narrow.places;
    return places * fan_out * ((size_t)fan_in + 1) * sizeof(float);
}

template <class C, class W>
hipError_t launch_narrow(const Problem &p, const Matrix<typename C::T> &w, const Matrix<typename C::T> &dz,
                         const Matrix<typename C::T> &x, Rows dx, W *dw, float *db, char *workspace, hipStream_t s)
{
    using T = typename C::T;
    const Split split = narrow_split(p.rows, p.heads, p.fan_in, p.fan_out, sizeof(T) == 2);
    float *wparts = reinterpret_cast<float *>(workspace);
    float *bparts = wparts + (size_t)split.places * p.fan_in * p.fan_out;
    narrow_kernel<C><<<split.places + 1, C::kThreads, 0, s>>>(p, w, dz, x, static_cast<T *>(const_cast<void *>(dx.p)), dx.stride,
                                                              dw ? wparts : nullptr, db ? bparts : nullptr, split.stretch);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || (!dw && !db) ? e : launch_sums(p, split, wparts, dw, bparts, db, s);
}

template <class T, bool MASK, class W>
hipError_t narrow(const Problem &p, const Matrix<T> &w, const Matrix<T> &dz, const Matrix<T> &x, Rows dx, W *dw,
                  float *db, char *workspace, hipStream_t s)
{
    if (p.fan_in <= 64)
        return p.fan_out <= 64 ? launch_narrow<Narrow<T, 64, 64, MASK>>(p, w, dz, x, dx, dw, db, workspace, s)
                               : launch_narrow<Narrow<T, 64, 128, MASK>>(p, w, dz, x, dx, dw, db, workspace, s);
    return p.fan_out <= 64 ? launch_narrow<Narrow<T, 128, 64, MASK>>(p, w, dz, x, dx, dw, db, workspace, s)
                           : launch_narrow<Narrow<T, 128, 128, MASK>>(p, w, dz, x, dx, dw, db, workspace, s);
}

template <class CR, class CW, class W>
hipError_t launch_gradients(const Problem &p, const Matrix<typename CR::T> &w, const Matrix<typename CR::T> &dz,
                            const Matrix<typename CR::T> &x, Rows dx, W *dw, float *db, hipStream_t s)
{
    using T = typename CR::T;
    const unsigned long long all =
        ((unsigned long long)p.rows / CR::TQ + p.heads + 1) * tiles_of(p.fan_in, CR::TP) +
        (unsigned long long)p.heads * tiles_of(p.fan_out, CW::TQ) * tiles_of(p.fan_in, CW::TP) + 3 * kXcds * kRun;
    if (all >= 1ull << 23)
        return hipErrorInvalidConfiguration;
    gradients_kernel<CR, CW, W><<<(unsigned)all, CR::kThreads, 0, s>>>(
        p, w, dz, x, static_cast<T *>(const_cast<void *>(dx.p)), dx.stride, dw, db);
    return hipGetLastError();
}

// Whether both gradients go in one launch: where they have two rounds of tiles, so that
// filling up the last one matters, and heads as a whole.  us in one and in two launches,
// 8 heads: 1,024 to 2,048 on 16,384 rows (512 tiles) 131, 177; 1,024 to 1,024 on 32,768
// (640) 164, 180, on 16,384 (384) 106, 103; 512 to 1,024 on 16,384 (192) 86, 84; 16 heads:
// 512 to 1,024 on 32,768 (384) 95, 102.  Where heads would be split: 512 to 512 on 262,144
// rows of 16 915, 474; 256 to 512 on 131,072 531, 117.
bool gradients_together(const Problem &p)
{
    const unsigned long long x_tiles = p.rows / 256ull * tiles_of(p.fan_in, 256);
    const unsigned long long w_tiles = (unsigned long long)p.heads * tiles_of(p.fan_out, 256) * tiles_of(p.fan_in, 256);
    return p.fan_in >= 512 && p.fan_out >= 512 && x_tiles + w_tiles < 1u << 16 && x_tiles + w_tiles >= 512 &&
           split_rows(p.rows, p.heads, p.fan_in, p.fan_out, true).stretch == 0;
}

}  // namespace

}  // namespace derf
