// Orthogonalised updates.  A matrix u (a head's update) becomes X = u / (|u| + 1e-7), |u|
// its Frobenius norm, and goes through steps
//
//   S = X X^T,   Q = b S + c S^2,   X = a X + Q X,     (a, b, c) = (3.4445, -4.7750, 2.0315)
//
// which take every singular value s to a s + b s^3 + c s^5 and leave the directions: from
// (0, 1] they come near 1.  X is taken with its shorter side as rows (u^T for a tall
// matrix), padded with zeros to multiples of 64, which stay zeros.
//
// The products run on the fp16 matrix units.  All singular values stay below 1.21, so no
// entry of X, S or Q is above 3.5 in magnitude, and they are held as fp16 values of 2^12
// times themselves, far from fp16's limits.  For float32 updates each is held as two
// fp16 values, the rounded one and the rest (22 bits), and a product is three.  Float32's
// operands have 24 bits, and its sums lose more the longer they are.  Off in 1e-6 of the
// result's norm (root mean square, normal values) here and by plain products in float32:
// 8 x 8 1.05, 0.77; 16 x 16 0.83, 0.75; 32 x 96 1.64, 1.25; 64 x 64 0.85, 1.19; 64 x 512 1.84,
// 1.64; 128 x 128 0.81, 1.42; 300 x 701 1.35, 2.40; 1,024 x 1,024 1.19, 3.07.  a X is added in
// float32: with a in Q's diagonal the matrix units' sums, whose roundings are those of their
// largest terms, lose twice as much.  bf16 updates, whose own rounding is 2^-9 (1.65e-3 of a
// matrix's norm), multiply the first halves alone: 11 bits, whatever the gradient's type (but
// where a side is below 8: exact_products in heads_api.cpp).  X
// itself keeps both, since a X takes what a step loses of the small singular values' part to
// 3.4 times as much in the next: the results, rounding included, are 2.0e-3 (1,024 x 1,024) to
// 3.2e-3 (8 x 8; one of 20,000 6.2e-3) off, with X in 11 bits too up to 8e-3, with bf16 products
// about ten times that.  Where few singular values make up a matrix they do not average: one by
// itself is 3 to 5e-3 off as a rule and up to 3.3e-2 (two million of them in an emulation), 128 x 200
// matrices of rank 3 4.1e-3, one of 400 1.0e-2.  In memory X keeps both for all but the last
// two steps, after which nothing grows much: as exact, and of 2,048 x 4,096 matrices' last
// products 564 us where both take 680.
#include "product.h"

#include <algorithm>

namespace derf {

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kUnit = 4096.0f;  // what 1 is held as
constexpr double kNormEps = 1e-7;
typedef _Float16 f16;
typedef f16 f16x4 __attribute__((ext_vector_type(4)));

// Matrix k of a set.
__device__ __forceinline__ MuonEntry entry_of(const MuonSet &set, unsigned k)
{
    if (set.table)
        return set.table[set.first + k];
    MuonEntry t = set.one;
    const long long at = (long long)k * t.fan_out * t.fan_in;
    t.param = static_cast<char *>(t.param) + at * (t.param_bf16 ? 2 : 4);
    t.grad = static_cast<const char *>(t.grad) + at * (t.grad_bf16 ? 2 : 4);
    return t;
}

template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Four {
    T v[4];
};
__device__ __forceinline__ f32x4 read4(const void *p, bool bf16, long long i, int here)
{
    f32x4 x = {};
    if (bf16) {
        const __bf16 *a = static_cast<const __bf16 *>(p) + i;
        if (here == 4) {
            const Four<__bf16> f = *reinterpret_cast<const Four<__bf16> *>(a);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                x[k] = (float)f.v[k];
            return x;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < here)
                x[k] = (float)a[k];
        return x;
    }
    const float *a = static_cast<const float *>(p) + i;
    if (here == 4) {
        const Four<float> f = *reinterpret_cast<const Four<float> *>(a);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] = f.v[k];
        return x;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < here)
            x[k] = a[k];
    return x;
}
template <class T>
__device__ __forceinline__ void write4_as(T *a, f32x4 x, int here)
{
    if (here == 4) {
        Four<T> f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            f.v[k] = (T)x[k];
        *reinterpret_cast<Four<T> *>(a) = f;
        return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < here)
            a[k] = (T)x[k];
}
__device__ __forceinline__ void write4(void *p, bool bf16, long long i, f32x4 x, int here)
{
    if (bf16)
        write4_as(static_cast<__bf16 *>(p) + i, x, here);
    else
        write4_as(static_cast<float *>(p) + i, x, here);
}

// The update of four values: u = g, or with momentum m = momentum m + g and u = g +
// momentum m (nesterov) or m.  g: the gradient times *grad_scale.
__device__ __forceinline__ f32x4 update_of(const MuonStep &st, f32x4 g, f32x4 m)
{
    if (!st.has_momentum)
        return g;
    return st.nesterov ? g + m * st.momentum : m;
}

// ---- momentum and norm ------------------------------------------------------------
// A workgroup takes a chunk of a matrix: the new momentum is written and the squares of
// the update summed, in 64 bits: no gradient is too large or too small for its norm.
__global__ __launch_bounds__(256) void momentum_kernel(const MuonSet set, MuonStep st, unsigned chunk,
                                                       double *squares)
{
    __shared__ double sums[4];
    const MuonEntry t = entry_of(set, blockIdx.y);
    const long long n = (long long)t.fan_out * t.fan_in;
    const long long from = (long long)blockIdx.x * chunk, to = from + chunk < n ? from + chunk : n;
    const float scale = st.grad_scale ? *st.grad_scale : 1.0f;
    double sum = 0.0;
    for (long long i = from + threadIdx.x * 4; i < to; i += 1024) {
        const int here = to - i >= 4 ? 4 : (int)(to - i);
        const f32x4 g = read4(t.grad, t.grad_bf16, i, here) * scale;
        f32x4 m = {};
        if (st.has_momentum) {
            m = read4(t.m, false, i, here) * st.momentum + g;
            write4(t.m, false, i, m, here);
        }
        const f32x4 u = update_of(st, g, m);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            sum += (double)u[k] * (double)u[k];  // values that are not there are zero
    }
    for (int off = 32; off; off >>= 1)
        sum += __shfl_xor(sum, off);
    if ((threadIdx.x & 63) == 0)
        sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        squares[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// 1 / (|u| + eps) from the chunks' squares, in every thread.
__device__ __forceinline__ double inverse_norm(const double *squares, unsigned chunks)
{
    __shared__ double sums[4];
    double sum = 0.0;
    for (unsigned i = threadIdx.x; i < chunks; i += 256)
        sum += squares[i];
    for (int off = 32; off; off >>= 1)
        sum += __shfl_xor(sum, off);
    if ((threadIdx.x & 63) == 0)
        sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    return 1.0 / (sqrt(sums[0] + sums[1] + sums[2] + sums[3]) + kNormEps);
}

// ---- X's start, and the end -----------------------------------------------------------
// A workgroup takes 64 x 64 values of the tensor; X holds tall matrices transposed.
// Between the two forms they go through LDS, a row a few banks on from the one before.

constexpr int kTurnRow = 68;  // floats

// The planes of a matrix: rows x cols fp16 each, the rests (X's always, S's and Q's where
// split) behind the rounded values.
struct Planes {
    f16 *p;
    long long matrix;  // values from a matrix to the next
    unsigned rows, cols;
};

__global__ __launch_bounds__(256) void start_kernel(const MuonSet set, MuonStep st, const double *squares,
                                                    unsigned chunks, Planes x)
{
    __shared__ __attribute__((aligned(16))) float tile[64][kTurnRow];
    const MuonEntry t = entry_of(set, blockIdx.z);
    const bool tall = t.fan_out > t.fan_in;
    const unsigned r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;  // of X
    const double inverse = inverse_norm(squares + (size_t)blockIdx.z * chunks, chunks);
    const float scale = st.grad_scale ? *st.grad_scale : 1.0f;
    const int o0 = (int)(tall ? c0 : r0), i0 = (int)(tall ? r0 : c0);  // of the tensor
    const int c = (threadIdx.x & 15) * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k * 16 + threadIdx.x / 16;
        const int left = t.fan_in - i0 - c, here = o0 + r < t.fan_out ? (left >= 4 ? 4 : left > 0 ? left : 0) : 0;
        f32x4 v = {};
        if (here > 0) {
            const long long at = (long long)(o0 + r) * t.fan_in + i0 + c;
            const f32x4 g = read4(t.grad, t.grad_bf16, at, here) * scale;
            const f32x4 m = st.has_momentum ? read4(t.m, false, at, here) : f32x4{};
            const f32x4 u = update_of(st, g, m);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = (float)((double)u[e] * inverse) * kUnit;
        }
        *reinterpret_cast<f32x4 *>(&tile[r][c]) = v;
    }
    __syncthreads();
    f16 *out = x.p + blockIdx.z * x.matrix;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k * 16 + threadIdx.x / 16;
        f32x4 v;
        if (tall)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = tile[c + e][r];
        else
            v = *reinterpret_cast<const f32x4 *>(&tile[r][c]);
        f16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            hi[e] = (f16)v[e];
            lo[e] = (f16)(v[e] - (float)hi[e]);
        }
        const size_t at = (size_t)(r0 + r) * x.cols + c0 + c;
        *reinterpret_cast<f16x4 *>(out + at) = hi;
        *reinterpret_cast<f16x4 *>(out + (size_t)x.rows * x.cols + at) = lo;
    }
}

// The parameters' step along X, or X itself as the result (no parameters).
__global__ __launch_bounds__(256) void finish_kernel(const MuonSet set, MuonStep st, Planes x, bool rest)
{
    __shared__ __attribute__((aligned(16))) float tile[64][kTurnRow];
    const MuonEntry t = entry_of(set, blockIdx.z);
    const bool tall = t.fan_out > t.fan_in;
    const unsigned r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    const int o0 = (int)(tall ? c0 : r0), i0 = (int)(tall ? r0 : c0);
    const int c = (threadIdx.x & 15) * 4;
    const f16 *in = x.p + blockIdx.z * x.matrix;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k * 16 + threadIdx.x / 16;
        const size_t at = (size_t)(r0 + r) * x.cols + c0 + c;
        f32x4 v = __builtin_convertvector(*reinterpret_cast<const f16x4 *>(in + at), f32x4);
        if (rest)
            v += __builtin_convertvector(*reinterpret_cast<const f16x4 *>(in + (size_t)x.rows * x.cols + at), f32x4);
        v *= 1.0f / kUnit;
        if (tall)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                tile[c + e][r] = v[e];
        else
            *reinterpret_cast<f32x4 *>(&tile[r][c]) = v;
    }
    __syncthreads();
    const float rate = st.rate * t.size;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k * 16 + threadIdx.x / 16;
        const int left = t.fan_in - i0 - c, here = o0 + r < t.fan_out ? (left >= 4 ? 4 : left > 0 ? left : 0) : 0;
        if (here <= 0)
            continue;
        const long long at = (long long)(o0 + r) * t.fan_in + i0 + c;
        f32x4 v = *reinterpret_cast<const f32x4 *>(&tile[r][c]);
        if (st.updates)
            v = read4(t.param, t.param_bf16, at, here) * st.decay - v * rate;
        write4(t.param, t.param_bf16, at, v, here);
        if (t.copy)
            write4(t.copy, true, at, v, here);
    }
}

// ---- the steps' products ------------------------------------------------------------

enum Kind { kGram, kSquare, kApply };

// What a wave's results are added to (S or X): read at once where the registers hold it all,
// else row by row of results (all of it before the product, beside the first loads: 5 us of
// 280 more).  RESTS: 1 it has both planes.
template <int KIND, int RESTS, int FP, int FQ>
struct Was {
    static constexpr bool kAll = FP * FQ * (RESTS & 1 ? 2 : 1) <= 16;
    static constexpr int kRows = kAll ? FQ : 1;
    f16x4 hi[kRows][FP], lo[kRows][FP];
    __device__ __forceinline__ void read_row(const f16 *from, unsigned rows, unsigned cols, unsigned r, unsigned c, int j)
    {
        const int lane = threadIdx.x & 63;
        const unsigned row = r + j * 16 + (lane & 15);
#pragma unroll
        for (int i = 0; i < FP; ++i) {
            const unsigned col = c + i * 16 + (lane >> 4) * 4;
            f16x4 &h = hi[j % kRows][i], &l = lo[j % kRows][i];
            h = l = f16x4{};
            if (row < rows && col < cols) {
                const f16 *at = from + ((size_t)row * cols + col);
                h = *reinterpret_cast<const f16x4 *>(at);
                if (RESTS & 1)
                    l = *reinterpret_cast<const f16x4 *>(at + (size_t)rows * cols);
            }
        }
    }
    __device__ __forceinline__ void read(const f16 *from, unsigned rows, unsigned cols, unsigned r, unsigned c)
    {
        if (kAll && KIND != kGram)
#pragma unroll
            for (int j = 0; j < FQ; ++j)
                read_row(from, rows, cols, r, c, j);
    }
};

// 16 rows of results (as write_16_rows) of a symmetric matrix to their columns' rows: turned
// in the wave's place in LDS, 8 rows a piece, a column's two pieces in turn.
template <int FP>
__device__ __forceinline__ void write_turned(const f32x4 (&v)[FP], char *mine, unsigned row0, unsigned c, f16 *to, unsigned size)
{
    const int lane = threadIdx.x & 63;
    auto place = [](int col, int piece) { return col * 32 + (piece ^ (col >> 2 & 1)) * 16; };
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *reinterpret_cast<f16 *>(mine + place(i * 16 + (lane >> 4) * 4 + k, lane >> 3 & 1) + (lane & 7) * 2) = (f16)v[i][k];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int n = 0; n < FP * 32; n += 64) {
        const int col = (n + lane) >> 1, piece = lane & 1;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(mine + place(col, piece));
        const unsigned row = row0 + piece * 8;
        if (row < size && c + col < size)  // both are multiples of 64
            *reinterpret_cast<u32x4 *>(to + ((size_t)(c + col) * size + row)) = x;
    }
    __builtin_amdgcn_wave_barrier();
}

// A wave's results, from row r and column c on, to `to` [rows][cols].  mirror: those of a
// symmetric matrix to the place above the diagonal too.  RESTS: 2 `to` gets both planes.
// PAST: past the caches; small matrices' products are read from them.
template <int KIND, int RESTS, bool PAST, int FP, int FQ>
__device__ __forceinline__ void write_step(const f32x4 (&acc)[FP][FQ], Was<KIND, RESTS, FP, FQ> &was, const f16 *from, f16 *to, unsigned rows,
                                           unsigned cols, unsigned r, unsigned c, char *mine, bool mirror)
{
    const size_t rest = (size_t)rows * cols;
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
        f32x4 v[FP], lo[FP];
        if (KIND != kGram && !was.kAll)
            was.read_row(from, rows, cols, r, c, j);
#pragma unroll
        for (int i = 0; i < FP; ++i) {
            v[i] = acc[i][j] * (1.0f / kUnit);
            if (KIND != kGram) {
                f32x4 old = __builtin_convertvector(was.hi[j % was.kRows][i], f32x4);
                if (RESTS & 1)
                    old += __builtin_convertvector(was.lo[j % was.kRows][i], f32x4);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[i][k] = KIND == kSquare ? fmaf(kC, v[i][k], kB * old[k]) : fmaf(kA, old[k], v[i][k]);
            }
            // rounded once, for all that take it: from a sum's fused multiply-add a second
            // conversion may round to another value, whose rest this is not
            const f32x4 hi = __builtin_convertvector(__builtin_convertvector(v[i], f16x4), f32x4);
            lo[i] = v[i] - hi;
            v[i] = hi;
        }
        write_16_rows<f16, FP * 16, true, PAST>(v, mine, r + j * 16, rows, c, cols, to, cols);
        if (RESTS & 2)
            write_16_rows<f16, FP * 16, true, PAST>(lo, mine, r + j * 16, rows, c, cols, to + rest, cols);
        if (KIND != kApply && mirror) {
            write_turned<FP>(v, mine, r + j * 16, c, to, rows);
            if (RESTS & 2)
                write_turned<FP>(lo, mine, r + j * 16, c, to + rest, rows);
        }
    }
}

// Tile `in` of a matrix: of all row by row in groups, or of a triangle row by row.
template <int TP, int TQ, bool SYMMETRIC>
__device__ __forceinline__ void step_tile(unsigned in, unsigned row_tiles, unsigned col_tiles, unsigned &r0, unsigned &c0)
{
    if (SYMMETRIC) {
        unsigned row = (unsigned)((sqrtf(8.0f * (float)in + 1.0f) - 1.0f) * 0.5f);
        while (row * (row + 1) / 2 > in)
            --row;
        while ((row + 1) * (row + 2) / 2 <= in)
            ++row;
        r0 = uniform(row) * TQ;
        c0 = uniform(in - row * (row + 1) / 2) * TP;
    } else {
        const Place2 where = in_groups(in, row_tiles, col_tiles);
        r0 = where.a * TQ;
        c0 = where.b * TP;
    }
}

// Which tiles a workgroup takes.  A matrix's tiles go to 2^parts XCDs (eight share an L2 of
// their own each): the same ones in every product, so that what they wrote and read is in
// their L2 still.  parts < 0: tiles in order, by runs (by_xcd).
struct Spread {
    unsigned matrices, each;  // tiles of a matrix
    int parts;
};
__host__ __device__ inline unsigned chunk_of(const Spread &sp) { return (sp.each + (1u << sp.parts) - 1) >> sp.parts; }
// Workgroups' numbers end here.
__host__ __device__ inline unsigned long long spread_end(const Spread &sp)
{
    if (sp.parts < 0)
        return (unsigned long long)sp.matrices * sp.each + kXcds * kRun;  // runs_end is not above it
    return (((unsigned long long)sp.matrices << sp.parts) + kXcds - 1) / kXcds * chunk_of(sp) * kXcds;
}
__device__ __forceinline__ bool tile_of(const Spread &sp, unsigned b, unsigned &matrix, unsigned &tile)
{
    if (sp.parts < 0) {
        const unsigned at = by_xcd(b, sp.matrices * sp.each);
        matrix = at / sp.each;
        tile = at - matrix * sp.each;
        return matrix < sp.matrices;
    }
    const unsigned chunk = chunk_of(sp), j = b / kXcds, xcd = b % kXcds, round = j / chunk;
    matrix = (round * kXcds + xcd) >> sp.parts;
    tile = (xcd & ((1u << sp.parts) - 1)) * chunk + j - round * chunk;
    return matrix < sp.matrices && tile < sp.each;
}

// out = a product of P and Q for each matrix: S = X X^T (Gram: P, Q = X), Q = b S +
// c S S (Square: P, Q = S; both results symmetric: tiles on and below the diagonal are
// computed and written to both places), X = a X + Q X (Apply: P = X, depth down its
// columns).
// SPLIT: the products of each operand's rests with the other's rounded values, then of
// those, one after the other into the same registers.
template <class C, int KIND, bool SPLIT, int RESTS>
__global__ __launch_bounds__(C::kThreads, 2) void step_kernel(Planes pm, Planes qm, Planes out, Spread sp)
{
    constexpr bool kSymmetric = KIND != kApply;
    constexpr int kPasses = SPLIT ? 3 : 1, COLS = C::FP * 16;
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    __shared__ __attribute__((aligned(16))) char results[C::WP * C::WQ * 16 * kPieceRow<f16, COLS>];
    const unsigned row_tiles = (out.rows + C::TQ - 1) / C::TQ, col_tiles = (out.cols + C::TP - 1) / C::TP;
    const unsigned end = sp.parts < 0 ? runs_end(sp.matrices * sp.each) : (unsigned)spread_end(sp), depth = qm.cols;
    static_assert(!kSymmetric || C::TP == C::TQ, "square tiles");
    auto tile_at = [&](unsigned b, unsigned &matrix, unsigned &r0, unsigned &c0) {
        unsigned tile;
        if (!tile_of(sp, b, matrix, tile))
            return false;
        step_tile<C::TP, C::TQ, kSymmetric>(tile, row_tiles, col_tiles, r0, c0);
        return true;
    };
    unsigned ahead = blockIdx.x, pass = 0;
    auto next_tile = [&](Pipe<C> &pipe) {
        unsigned matrix, r0, c0;
        for (; ahead < end; ahead += gridDim.x) {
            if (!tile_at(ahead, matrix, r0, c0))
                continue;
            const f16 *p = pm.p + matrix * pm.matrix, *q = qm.p + matrix * qm.matrix;
            if (SPLIT && pass == 0)  // the small ones first
                p += (size_t)pm.rows * pm.cols;
            if (SPLIT && pass == 1)
                q += (size_t)qm.rows * qm.cols;
            const typename C::P::Source ps = {{p, pm.cols, nullptr, 0, pm.rows, (int)pm.cols}, c0};
            const typename C::Q::Source qs = {{q, qm.cols, nullptr, 0, qm.rows, (int)qm.cols}, r0};
            if (++pass == kPasses) {
                pass = 0;
                ahead += gridDim.x;
            }
            pipe.load_tile(ps, qs, depth);
            return;
        }
        pipe.load_nothing();
    };
    const int wave = uniform(threadIdx.x >> 6);
    const int wp = (wave % C::WP) * COLS, wq = (wave / C::WP) * C::FQ * 16;
    char *mine = results + wave * 16 * kPieceRow<f16, COLS>;
    Pipe<C> pipe;
    pipe.start(lds, next_tile);
    for (unsigned b = blockIdx.x; b < end; b += gridDim.x) {
        unsigned matrix, r0, c0;
        if (!tile_at(b, matrix, r0, c0))
            continue;
        f32x4 acc[C::FP][C::FQ] = {};
#pragma unroll 1
        for (int n = 0; n < kPasses; ++n)
#pragma unroll 1
            for (unsigned k = 0; k < depth; k += C::kDepth)
                pipe.step(acc, next_tile, [](auto &) {});
        const f16 *from = pm.p + matrix * pm.matrix;
        Was<KIND, RESTS, C::FP, C::FQ> was;
        was.read(from, out.rows, out.cols, r0 + wq, c0 + wp);
        write_step<KIND, RESTS, (C::TP >= 256), C::FP, C::FQ>(acc, was, from, out.p + matrix * out.matrix, out.rows, out.cols, r0 + wq, c0 + wp, mine,
                                              r0 != c0);
    }
    arrived<0>();
}

// Two results side by side of 16 rows, as 16-byte chunks of a row: a lane of quarter q gets
// chunk q / 2 of result q % 2 from its own half and that of the lane 16 on, or back.
__device__ __forceinline__ void swap_halves(u32x4 &x)
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto both = __builtin_amdgcn_permlane16_swap(x[k], x[2 + k], false, false);
        x[k] = both[0];
        x[2 + k] = both[1];
    }
}
__device__ __forceinline__ u32x4 as_halves(f32x4 a, f32x4 b)
{
    return __builtin_bit_cast(u32x4, __builtin_convertvector(__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), f16x8));
}
__device__ __forceinline__ void from_halves(u32x4 x, f32x4 &a, f32x4 &b)
{
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    const f32x8 v = __builtin_convertvector(__builtin_bit_cast(f16x8, x), f32x8);
    a = __builtin_shufflevector(v, v, 0, 1, 2, 3);
    b = __builtin_shufflevector(v, v, 4, 5, 6, 7);
}
// Where: row `row` of a plane of tiles, results f and f + 1.
template <class TILE>
__device__ __forceinline__ unsigned pair_at(int row, int f)
{
    const int quarter = (threadIdx.x & 63) >> 4;
    return (row >> 6) * TILE::kBytes + TILE::at(row & 63, 2 * (f + (quarter & 1)) + (quarter >> 1));
}
template <class TILE, bool SPLIT>
__device__ __forceinline__ void write_pair(char *plane, int plane_bytes, int row, int f, f32x4 a, f32x4 b)
{
    const unsigned at = pair_at<TILE>(row, f);
    u32x4 hi = as_halves(a, b);
    if (SPLIT) {
        f32x4 c, d;
        from_halves(hi, c, d);
        u32x4 lo = as_halves(a - c, b - d);
        swap_halves(lo);
        *reinterpret_cast<u32x4 *>(plane + plane_bytes + at) = lo;
    }
    swap_halves(hi);
    *reinterpret_cast<u32x4 *>(plane + at) = hi;
}
template <class TILE, bool SPLIT>
__device__ __forceinline__ void read_pair(const char *plane, int plane_bytes, int row, int f, f32x4 &a, f32x4 &b)
{
    const unsigned at = pair_at<TILE>(row, f);
    u32x4 hi = *reinterpret_cast<const u32x4 *>(plane + at);
    swap_halves(hi);
    from_halves(hi, a, b);
    if (SPLIT) {
        u32x4 lo = *reinterpret_cast<const u32x4 *>(plane + plane_bytes + at);
        swap_halves(lo);
        f32x4 c, d;
        from_halves(lo, c, d);
        a += c;
        b += d;
    }
}

// acc[i][j] += sum over DEPTH of P's and Q's 16-row results: p_read, q_read (plane, result, 32
// deep part) give the matrix unit's operands.  SPLIT: products with a rest go to `rest`: beside
// the others their last bits would be lost to each of the sum's roundings (300 x 701: 2.1e-6
// of the norm off, 1.5e-6 with sums of their own).
template <int FP, int FQ, bool SPLIT, int DEPTH, class PRead, class QRead>
__device__ __forceinline__ void small_product(f32x4 (&acc)[FP][FQ], f32x4 (&rest)[FP][FQ], PRead p_read, QRead q_read)
{
#pragma unroll 4
    for (int part = 0; part < DEPTH / 32; ++part) {
        u32x4 p[FP], q[FQ];
#pragma unroll
        for (int j = 0; j < FQ; ++j)
            q[j] = q_read(0, j, part);
#pragma unroll
        for (int i = 0; i < FP; ++i)
            p[i] = p_read(0, i, part);
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FQ; ++j)
                acc[i][j] = multiply(p[i], q[j], acc[i][j], f16{});
        if (SPLIT) {
            u32x4 low[FQ];
#pragma unroll
            for (int j = 0; j < FQ; ++j)
                low[j] = q_read(1, j, part);
#pragma unroll
            for (int i = 0; i < FP; ++i)
#pragma unroll
                for (int j = 0; j < FQ; ++j)
                    rest[i][j] = multiply(p[i], low[j], rest[i][j], f16{});
#pragma unroll
            for (int i = 0; i < FP; ++i)
                p[i] = p_read(1, i, part);
#pragma unroll
            for (int i = 0; i < FP; ++i)
#pragma unroll
                for (int j = 0; j < FQ; ++j)
                    rest[i][j] = multiply(p[i], q[j], rest[i][j], f16{});
        }
    }
}
template <int FP, int FQ, bool SPLIT>
__device__ __forceinline__ void add_rest(f32x4 (&acc)[FP][FQ], const f32x4 (&rest)[FP][FQ])
{
    if (SPLIT)
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
            for (int j = 0; j < FQ; ++j)
                acc[i][j] += rest[i][j];
}

// The same for split matrices of few tiles, one a workgroup: a step brings both planes of
// both operands, so that it has three products to do while the next ones' loads are under
// way, where the passes of step_kernel have one and wait.
template <class C, int KIND>
__global__ __launch_bounds__(C::kThreads, 2) void pair_kernel(Planes pm, Planes qm, Planes out, Spread sp)
{
    constexpr bool kSymmetric = KIND != kApply;
    constexpr int kStage = 2 * C::kStage, kLoads = 2 * C::kLoads, COLS = C::FP * 16;
    __shared__ __attribute__((aligned(16))) char lds[2 * kStage];
    static_assert(C::WP * C::WQ * 16 * kPieceRow<f16, COLS> <= 2 * kStage, "results take the stages' place");
    const unsigned row_tiles = (out.rows + C::TQ - 1) / C::TQ, col_tiles = (out.cols + C::TP - 1) / C::TP;
    unsigned matrix, tile, r0, c0;
    if (!tile_of(sp, blockIdx.x, matrix, tile))
        return;
    step_tile<C::TP, C::TQ, kSymmetric>(tile, row_tiles, col_tiles, r0, c0);
    const f16 *p = pm.p + matrix * pm.matrix, *q = qm.p + matrix * qm.matrix;
    typename C::P::Feed pf[2];
    typename C::Q::Feed qf[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        pf[n].start({{p + n * ((size_t)pm.rows * pm.cols), pm.cols, nullptr, 0, pm.rows, (int)pm.cols}, c0});
        qf[n].start({{q + n * ((size_t)qm.rows * qm.cols), qm.cols, nullptr, 0, qm.rows, (int)qm.cols}, r0});
    }
    const unsigned lds0 = lds_byte(lds);
    // a step's loads; behind the last step they bring what lies there, or zeros, and nothing reads it
    auto bring = [&](unsigned to) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int i = 0; i < C::P::kShare; ++i)
                pf[n].piece(i, lds0 + to + n * C::kStage);
#pragma unroll
            for (int i = 0; i < C::Q::kShare; ++i)
                qf[n].piece(i, lds0 + to + n * C::kStage + C::P::kBytes);
            pf[n].advance();
            qf[n].advance();
        }
    };
    const int wave = uniform(threadIdx.x >> 6);
    const int fp = (wave % C::WP) * C::FP, fq = (wave / C::WP) * C::FQ;
    bring(0);
    bring(kStage);
    f32x4 acc[C::FP][C::FQ] = {}, rest[C::FP][C::FQ] = {};
    unsigned stage = 0;
#pragma unroll 1
    for (unsigned k = 0; k < qm.cols; k += C::kDepth) {
        arrived<kLoads>();
        const char *from = lds + stage;
        small_product<C::FP, C::FQ, true, C::kDepth>(
            acc, rest, [&](int plane, int i, int part) { return C::P::fragment(from + plane * C::kStage, fp + i, part); },
            [&](int plane, int j, int part) { return C::Q::fragment(from + plane * C::kStage + C::P::kBytes, fq + j, part); });
        stored();  // all waves have read the stage
        bring(stage);
        stage ^= kStage;
    }
    Was<KIND, 3, C::FP, C::FQ> was;
    was.read(p, out.rows, out.cols, r0 + fq * 16, c0 + fp * 16);
    arrived<0>();
    add_rest<C::FP, C::FQ, true>(acc, rest);
    write_step<KIND, 3, false, C::FP, C::FQ>(acc, was, p, out.p + matrix * out.matrix, out.rows, out.cols, r0 + fq * 16, c0 + fp * 16,
                                      lds + wave * 16 * kPieceRow<f16, COLS>, r0 != c0);
}

// ---- small matrices, all of it in one launch ----------------------------------------------

// Matrices that fit: a workgroup takes one from its gradient to its parameters, X and S (or
// Q in its place) in LDS.  Both lie in tiles of 64 rows by up to 128 columns, X's by blocks
// of columns: their rows are read as they lie, and X's columns for Q X by transposing reads.
// Bound by waits: a step's three products follow each other, with a barrier after each, and a
// compute unit holds one matrix of 128 rows.  A step of 144 of 128 x 128 (float32) 58 us, in
// steps through memory 327; orthogonalised alone 46, in bf16 28; 24 of 64 x 256 30, 85 (bf16 24).
template <int M_, int N_, bool SPLIT>
struct Small {
    static constexpr int M = M_, N = N_, kPlanes = SPLIT ? 2 : 1 /* of S */, kThreads = M == 128 ? 1024 : 512;
    static constexpr int WP = M == 128 ? 4 : 2, WQ = kThreads / 64 / WP;  // waves over columns and rows
    static constexpr int FQ = M / 16 / WQ, FS = M / 16 / WP, FX = N / 16 / WP;  // 16-row results of each: rows, columns of S and X
    static_assert(WQ * FQ * 16 == M && FS % 2 == 0, "all rows, and columns in pairs");
    static constexpr int kBlock = N < 128 ? N : 128;  // columns
    using X = Tile<f16, kBlock, false, kThreads, false, false, true>;
    using S = Tile<f16, M, false, kThreads, false, false, true>;
    static constexpr int kXBlock = M / 64 * X::kBytes;
    static constexpr int kX = M * N * 2, kS = M * M * 2, kLds = 2 * kX + kPlanes * kS;  // bytes
    static constexpr int kVecs = M * N / 4 / kThreads;  // of a thread
    // workgroups a compute unit: by their LDS, and by registers: 128 of a lane, of long rows 256
    static constexpr int kByLds = 160 * 1024 / (kLds + 256), kByRegisters = N > 256 ? 1 : 1024 / kThreads;
    static constexpr int kAtOnce = kByLds < kByRegisters ? kByLds : kByRegisters;
};

// Four values side by side in a plane of tiles: row r, columns from c on.
template <class C>
__device__ __forceinline__ unsigned lds_at(int r, int c)
{
    using TILE = typename C::X;
    return c / C::kBlock * C::kXBlock + (r >> 6) * TILE::kBytes + TILE::at(r & 63, c % C::kBlock >> 3) + (c & 4) * 2;
}
template <class C>
__device__ __forceinline__ f32x4 read_lds(const char *plane, int r, int c)
{
    const unsigned at = lds_at<C>(r, c);
    f32x4 v = __builtin_convertvector(*reinterpret_cast<const f16x4 *>(plane + at), f32x4);
    v += __builtin_convertvector(*reinterpret_cast<const f16x4 *>(plane + C::kX + at), f32x4);
    return v;
}
template <class C>
__device__ __forceinline__ void write_lds(char *plane, int r, int c, f32x4 v)
{
    const unsigned at = lds_at<C>(r, c);
    const f16x4 hi = __builtin_convertvector(v, f16x4);
    *reinterpret_cast<f16x4 *>(plane + at) = hi;
    *reinterpret_cast<f16x4 *>(plane + C::kX + at) = __builtin_convertvector(v - __builtin_convertvector(hi, f32x4), f16x4);
}

// The products, a wave's part of each: rows from 16 fq on, results from wp FS or wp FX on.
template <class C>
struct Part {
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int wp = wave % C::WP, fq = wave / C::WP * C::FQ;
    const int row = fq * 16 + (lane & 15);  // of the wave's first results; the next 16 on
};
template <class C>
__device__ __forceinline__ auto s_rows(const char *sq, int first)
{
    return [=](int plane, int i, int part) {
        using S = typename C::S;
        const int f = first + i;
        return S::row_fragment(sq + plane * C::kS + (f >> 2) * S::kBytes, f & 3, part);
    };
}
// S's sums: X X^T is added.
template <class C, bool SPLIT>
__device__ __forceinline__ void small_gram(const char *x, f32x4 (&acc)[C::FS][C::FQ], f32x4 (&rest)[C::FS][C::FQ])
{
    const Part<C> my;
    auto x_rows = [&](int first) {
        return [=](int plane, int i, int part) {
            using X = typename C::X;
            constexpr int kParts = C::kBlock / 32;  // of a block
            const int f = first + i;
            return X::row_fragment(x + plane * C::kX + part / kParts * C::kXBlock + (f >> 2) * X::kBytes, f & 3, part % kParts);
        };
    };
    small_product<C::FS, C::FQ, SPLIT, C::N>(acc, rest, x_rows(my.wp * C::FS), x_rows(my.fq));
}
// Sums times `times` to S's (or Q's) place.
template <class C, bool SPLIT>
__device__ __forceinline__ void write_small(char *sq, const f32x4 (&acc)[C::FS][C::FQ], float times)
{
    const Part<C> my;
#pragma unroll
    for (int i = 0; i < C::FS; i += 2)
#pragma unroll
        for (int j = 0; j < C::FQ; ++j)
            write_pair<typename C::S, SPLIT>(sq, C::kS, my.row + j * 16, my.wp * C::FS + i, acc[i][j] * times, acc[i + 1][j] * times);
}
// S becomes Q.
template <class C, bool SPLIT>
__device__ __forceinline__ void small_square(char *sq)
{
    const Part<C> my;
    f32x4 acc[C::FS][C::FQ] = {}, rest[C::FS][C::FQ] = {};
    small_product<C::FS, C::FQ, SPLIT, C::M>(acc, rest, s_rows<C>(sq, my.wp * C::FS), s_rows<C>(sq, my.fq));
    add_rest<C::FS, C::FQ, SPLIT>(acc, rest);
#pragma unroll
    for (int i = 0; i < C::FS; i += 2)
#pragma unroll
        for (int j = 0; j < C::FQ; ++j) {
            f32x4 a, b;
            read_pair<typename C::S, SPLIT>(sq, C::kS, my.row + j * 16, my.wp * C::FS + i, a, b);
            acc[i][j] = acc[i][j] * (kC / kUnit) + a * kB;
            acc[i + 1][j] = acc[i + 1][j] * (kC / kUnit) + b * kB;
        }
    __syncthreads();
    write_small<C, SPLIT>(sq, acc, 1.0f);
}
// X becomes a X + Q X.
template <class C, bool SPLIT>
__device__ __forceinline__ void small_apply(char *x, const char *sq)
{
    using X = typename C::X;
    constexpr int FX = C::FX, FQ = C::FQ, kOfBlock = C::kBlock / 16;
    const Part<C> my;
    f32x4 acc[FX][FQ] = {}, more[FX][FQ] = {};
    auto &rest = FX * FQ > 8 ? acc : more;  // two parts of depth only, and no registers for more
    auto x_columns = [&](int plane, int i, int part) {
        const int f = my.wp * FX + i;
        return X::fragment(x + plane * C::kX + f / kOfBlock * C::kXBlock + (part >> 1) * X::kBytes, f % kOfBlock, part & 1);
    };
    small_product<FX, FQ, SPLIT, C::M>(acc, rest, x_columns, s_rows<C>(sq, my.fq));
    add_rest<FX, FQ, SPLIT && FX * FQ <= 8>(acc, rest);
#pragma unroll
    for (int i = 0; i < FX; i += 2)
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
            f32x4 a, b;
            const int f = my.wp * FX + i;
            read_pair<X, true>(x + f / kOfBlock * C::kXBlock, C::kX, my.row + j * 16, f % kOfBlock, a, b);
            acc[i][j] = acc[i][j] * (1.0f / kUnit) + a * kA;
            acc[i + 1][j] = acc[i + 1][j] * (1.0f / kUnit) + b * kA;
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FX; i += 2)
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
            const int f = my.wp * FX + i;
            write_pair<X, true>(x + f / kOfBlock * C::kXBlock, C::kX, my.row + j * 16, f % kOfBlock, acc[i][j], acc[i + 1][j]);
        }
}

template <class C, bool SPLIT>
__global__ __launch_bounds__(C::kThreads, C::kAtOnce *C::kThreads / 256) void small_kernel(const MuonSet set, MuonStep st)
{
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    __shared__ double sums[C::kThreads / 64];
    char *const x = lds, *const sq = lds + 2 * C::kX;
    const MuonEntry t = entry_of(set, blockIdx.x);
    const bool tall = t.fan_out > t.fan_in;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const float scale = st.grad_scale ? *st.grad_scale : 1.0f;
    const int vecs = (tall ? C::M : C::N) / 4;  // of a row of the tensor, padded
    // vector k of this thread's: row o and column i of the tensor, elements there
    auto place = [&](int k, int &o, int &i) {
        const int n = k * C::kThreads + threadIdx.x;
        o = n / vecs;
        i = n % vecs * 4;
        const int left = t.fan_in - i;
        return o < t.fan_out && left > 0 ? (left < 4 ? left : 4) : 0;
    };
    {
        f32x4 u[C::kVecs];
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < C::kVecs; ++k) {
            int o, i;
            const int here = place(k, o, i);
            u[k] = f32x4{};
            if (here > 0) {
                const long long at = (long long)o * t.fan_in + i;
                const f32x4 g = read4(t.grad, t.grad_bf16, at, here) * scale;
                f32x4 m = {};
                if (st.has_momentum) {
                    m = read4(t.m, false, at, here) * st.momentum + g;
                    write4(t.m, false, at, m, here);
                }
                u[k] = update_of(st, g, m);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum += (double)u[k][e] * (double)u[k][e];
        }
        for (int off = 32; off; off >>= 1)
            sum += __shfl_xor(sum, off);
        if (lane == 0)
            sums[wave] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < C::kThreads / 64; ++w)
            sum += sums[w];
        const double inverse = 1.0 / (sqrt(sum) + kNormEps);
#pragma unroll
        for (int k = 0; k < C::kVecs; ++k) {
            int o, i;
            place(k, o, i);
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = (float)((double)u[k][e] * inverse) * kUnit;
            if (!tall) {
                write_lds<C>(x, o, i, v);
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f16 *to = reinterpret_cast<f16 *>(x + lds_at<C>(i + e, o)) + (o & 3);
                const f16 hi = (f16)v[e];
                to[0] = hi;
                to[C::kX / 2] = (f16)(v[e] - (float)hi);
            }
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int n = 0; n < st.iterations; ++n) {
        {
            f32x4 acc[C::FS][C::FQ] = {}, rest[C::FS][C::FQ] = {};
            small_gram<C, SPLIT>(x, acc, rest);
            add_rest<C::FS, C::FQ, SPLIT>(acc, rest);
            write_small<C, SPLIT>(sq, acc, 1.0f / kUnit);
        }
        __syncthreads();
        small_square<C, SPLIT>(sq);
        __syncthreads();
        small_apply<C, SPLIT>(x, sq);
        __syncthreads();
    }
    const float rate = st.rate * t.size;
#pragma unroll
    for (int k = 0; k < C::kVecs; ++k) {
        int o, i;
        const int here = place(k, o, i);
        if (here <= 0)
            continue;
        f32x4 v;
        if (tall)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f16 *from = reinterpret_cast<const f16 *>(x + lds_at<C>(i + e, o)) + (o & 3);
                v[e] = (float)from[0] + (float)from[C::kX / 2];
            }
        else
            v = read_lds<C>(x, o, i);
        v *= 1.0f / kUnit;
        const long long at = (long long)o * t.fan_in + i;
        if (st.updates)
            v = read4(t.param, t.param_bf16, at, here) * st.decay - v * rate;
        write4(t.param, t.param_bf16, at, v, here);
        if (t.copy)
            write4(t.copy, true, at, v, here);
    }
}

// ---- matrices of up to 128 rows that do not fit -------------------------------------------

// A step in two launches: this one takes columns of X, `per` pieces of 128 of them a
// workgroup, through Q X and the next S's part of those columns, as small_kernel does;
// sum_parts_kernel sums the parts.  S is the same for all of a matrix's workgroups, each of
// which squares it for itself.  apply: there is an S; gram: there is a next step.  Bound by a
// launch's chain of waits (S, its square, Q X, the next S, about 8 us); a call's us so and by the
// products of large matrices, float32 and bf16: 22 of 11 x 1,924 95, 182 and 87, 145; 51 of 123 x
// 1,545 245, 299 and 203, 235; 70 of 96 x 200 128, 136 and 108, 118; 16 of 128 x 16,384 516, 1,252 and
// 410, 1,030; 1,000 of 64 x 600 556, 979 and 454, 655.
template <class C, bool SPLIT>
__global__ __launch_bounds__(C::kThreads, C::kAtOnce *C::kThreads / 256) void columns_kernel(Planes xm, const f16 *s, float *parts,
                                                                                              unsigned per, bool apply, bool gram)
{
    constexpr int M = C::M;
    static_assert(C::N == 128 && C::kBlock == 128, "a piece");
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    char *const x = lds, *const sq = lds + 2 * C::kX;
    const size_t plane = (size_t)xm.rows * xm.cols;
    f16 *const from = xm.p + blockIdx.y * xm.matrix;
    const unsigned pieces = (xm.cols + 127) / 128, first = blockIdx.x * per, last = first + per < pieces ? first + per : pieces;
    if (apply) {
        const f16 *mine = s + blockIdx.y * (size_t)(M * M * C::kPlanes);
        for (int i = threadIdx.x; i < C::kPlanes * M * M / 8; i += C::kThreads) {
            const int r = i / (M / 8) % M, c = i % (M / 8);
            using S = typename C::S;
            *reinterpret_cast<u32x4 *>(sq + i / (M * M / 8) * C::kS + (r >> 6) * S::kBytes + S::at(r & 63, c)) =
                *reinterpret_cast<const u32x4 *>(mine + (size_t)i * 8);
        }
    }
    // 16 bytes of both planes: in LDS, and in memory, where the columns are X's
    auto each = [&](unsigned piece, auto &&what) {
#pragma unroll
        for (int i = threadIdx.x; i < 2 * M * 16; i += C::kThreads) {
            const int r = i / 16 % M, c = i % 16, low = i / (M * 16);
            using X = typename C::X;
            const unsigned col = piece * 128 + c * 8;
            what(x + low * C::kX + (r >> 6) * X::kBytes + X::at(r & 63, c), from + low * plane + ((size_t)r * xm.cols + col), col < xm.cols);
        }
    };
    auto load = [&](char *to, const f16 *at, bool there) {
        *reinterpret_cast<u32x4 *>(to) = there ? *reinterpret_cast<const u32x4 *>(at) : u32x4{};
    };
    f32x4 acc[C::FS][C::FQ] = {}, rest[C::FS][C::FQ] = {};
    each(first, load);
    __syncthreads();
    if (apply) {
        small_square<C, SPLIT>(sq);
        __syncthreads();
    }
#pragma unroll 1
    for (unsigned piece = first; piece < last; ++piece) {
        if (piece != first) {
            __syncthreads();
            each(piece, load);
            __syncthreads();
        }
        if (apply) {
            small_apply<C, SPLIT>(x, sq);
            __syncthreads();
            each(piece, [&](const char *value, f16 *to, bool there) {
                if (there)
                    *reinterpret_cast<u32x4 *>(to) = *reinterpret_cast<const u32x4 *>(value);
            });
        }
        if (gram)
            small_gram<C, SPLIT>(x, acc, rest);
    }
    if (!gram)
        return;
    add_rest<C::FS, C::FQ, SPLIT>(acc, rest);
    const Part<C> my;
    float *to = parts + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * (M * M);
#pragma unroll
    for (int i = 0; i < C::FS; ++i)
#pragma unroll
        for (int j = 0; j < C::FQ; ++j)
            *reinterpret_cast<f32x4 *>(to + (my.row + j * 16) * M + (my.wp * C::FS + i) * 16 + (my.lane >> 4) * 4) = acc[i][j];
}

// S of each matrix from its parts, four values a thread.
template <bool SPLIT>
__global__ __launch_bounds__(256) void sum_parts_kernel(const float *parts, unsigned count, unsigned size, f16 *s)
{
    const unsigned i = (blockIdx.x * 256 + threadIdx.x) * 4;
    const float *from = parts + (size_t)blockIdx.y * count * size + i;
    f32x4 sum = {};
#pragma unroll 8
    for (unsigned n = 0; n < count; ++n)
        sum += *reinterpret_cast<const f32x4 *>(from + (size_t)n * size);
    sum *= 1.0f / kUnit;
    f16 *to = s + (size_t)blockIdx.y * size * (SPLIT ? 2 : 1) + i;
    const f16x4 hi = __builtin_convertvector(sum, f16x4);
    *reinterpret_cast<f16x4 *>(to) = hi;
    if (SPLIT)
        *reinterpret_cast<f16x4 *>(to + size) = __builtin_convertvector(sum - __builtin_convertvector(hi, f32x4), f16x4);
}

// ---- launches --------------------------------------------------------------------------

template <int M, int N, bool SPLIT>
hipError_t launch_small(const MuonSet &set, unsigned matrices, const MuonStep &st, hipStream_t s)
{
    using C = Small<M, N, SPLIT>;
    small_kernel<C, SPLIT><<<matrices, C::kThreads, 0, s>>>(set, st);
    return hipGetLastError();
}

unsigned padded(int n) { return (unsigned)(n + 63) / 64 * 64; }
size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Sizes of a group of matrices of one padded shape.
struct Sizes {
    unsigned m, n;  // of X
    unsigned chunk, chunks;
    size_t squares, x, s;  // bytes of a matrix
};
Sizes sizes_of(int fan_out, int fan_in, bool split)
{
    Sizes z;
    const unsigned o = padded(fan_out), i = padded(fan_in);
    z.m = o < i ? o : i;
    z.n = o < i ? i : o;
    // chunks of the padded matrix, which are enough for every member of the group
    const unsigned long long all = (unsigned long long)z.m * z.n;
    unsigned long long chunk = (all / 256 + 1023) / 1024 * 1024;
    z.chunk = (unsigned)(chunk < 4096 ? 4096 : chunk);
    z.chunks = (unsigned)((all + z.chunk - 1) / z.chunk);
    z.squares = z.chunks * sizeof(double);
    z.x = all * 4;
    z.s = (size_t)z.m * z.m * (split ? 4 : 2);
    return z;
}

// A matrix on as few XCDs as take no more rounds than all would, but for large tiles, whose
// matrices an L2 does not hold; at_once: workgroups a compute unit.  A call's us so and in
// order: float32, 24 of 300 x 701 287, 302; 8 of 512 x 512 192, 234; 4 of 1,024 x 1,024 447, 483;
// one of 300 x 300 112, 116; bf16, 24 of 300 x 701 198, 204; 16 of 2,048 x 4,096 6,160, 6,100.
template <class C, int KIND>
Spread spread(const Planes &out, unsigned matrices, unsigned at_once)
{
    const unsigned rows = (out.rows + C::TQ - 1) / C::TQ, cols = (out.cols + C::TP - 1) / C::TP;
    Spread sp = {matrices, KIND != kApply ? rows * (rows + 1) / 2 : rows * cols, 0};
    const unsigned long long slots = 32 * at_once, all = (unsigned long long)matrices * sp.each;
    const unsigned long long rounds = ((all + kXcds - 1) / kXcds + slots - 1) / slots;
    for (; C::TQ < 256 && sp.parts < 4; ++sp.parts)
        if ((spread_end(sp) / kXcds + slots - 1) / slots <= rounds)
            return sp;
    sp.parts = -1;
    return sp;
}

template <class C, int KIND, bool SPLIT, int RESTS>
hipError_t launch_step(const Planes &p, const Planes &q, const Planes &out, unsigned matrices, hipStream_t s)
{
    const Spread sp = spread<C, KIND>(out, matrices, C::kThreads >= 512 ? 1 : 2);
    return launch_for<C>(spread_end(sp), [&](unsigned groups, unsigned) {
        step_kernel<C, KIND, SPLIT, RESTS><<<groups, C::kThreads, 0, s>>>(p, q, out, sp);
    });
}

template <class C, int KIND>
hipError_t launch_pair(const Planes &p, const Planes &q, const Planes &out, unsigned matrices, hipStream_t s)
{
    const Spread sp = spread<C, KIND>(out, matrices, C::kThreads >= 512 ? 1 : 2);
    const unsigned long long end = spread_end(sp);
    if (end >= 1ull << 31)  // more than any memory holds
        return hipErrorInvalidConfiguration;
    pair_kernel<C, KIND><<<(unsigned)end, C::kThreads, 0, s>>>(p, q, out, sp);
    return hipGetLastError();
}

// Tiles of 64, 128 or 256 rows and columns, by the rounds that they take of the workgroups that
// run at once (512 of 64; 512 of 128, split 256; 256 of 256).  A round of 128 takes as long as
// 1.5 to 1.9 of 64 (split S and Q up to 2, while there are few); from 2,048 of depth on one of
// 256 as long as 1.6 to 2 of 128, split 3.4 (but for split S and Q, where they are no
// faster: 8 of 2,048 x 4,096 494, 282 with 128, 592, 340 with 256).  us of S, Q and Q X with 64,
// 128 and 256 (matrices of m x n; bf16's Q X the mean of its steps):
//   float32  24 of 300 x 701        14, 11, 25       20, 17, 29       Q X 55
//            8 of 512 x 512         11, 13, 13       16, 20, 18       62
//            16 of 512 x 1,024      26, 20, 43       28, 22, 40       68
//            4 of 1,024 x 1,024     29, 32, 40       28, 32, 32       92
//            2 of 2,048 x 2,048     84, 87, 132      91, 98, 101      151
//            16 of 1,024 x 1,024    84, 92, 154      82, 94, 121      124
//            8 of 2,048 x 4,096     652, 311, 1,112  493, 266, 936    726
//   bf16     24 of 300 x 701        10.1, 7.8, 17.6  12.6, 10.8, 16   25, 23, 31
//            8 of 512 x 512         7.4, 8.4, 9.7    9.8, 11.4, 13    23, 29, 33
//            16 of 512 x 1,024      20, 13.5, 28     16, 12.8, 20     33, 31, 36
//            2 of 2,048 x 2,048     50, 52, 74       36, 40, 46       54, 63, 66
//            16 of 1,024 x 1,024    44, 48, 83       33, 38, 53       39, 48, 56
//            8 of 2,048 x 4,096     397, 156, 615    188, 99, 366     208, 133, 297
//            16 of 2,048 x 4,096    -                330, 188, -      312, 202, 564
// Calls: 8 of 2,048 x 4,096 7,885 us in float32 (the products at the library's rate 6,950), 24 of
// 300 x 701 257, in bf16 183 (58 % of S's wave cycles waiting, matrix units 5 % busy); a step of 112
// of 256 x 256 in float32 383.
template <int KIND, bool SPLIT, int RESTS>
hipError_t step(const Planes &p, const Planes &q, const Planes &out, unsigned matrices, hipStream_t s)
{
    constexpr bool kDeep = KIND != kApply;
    auto tiles = [&](unsigned size) {
        const unsigned long long rows = (out.rows + size - 1) / size, cols = (out.cols + size - 1) / size;
        return matrices * (kDeep ? rows * (rows + 1) / 2 : rows * cols);
    };
    auto rounds = [&](unsigned size, unsigned at_once) { return (double)((tiles(size) + at_once - 1) / at_once); };
    const double middle = rounds(128, SPLIT ? 256 : 512);
    const bool small = rounds(64, 512) <= std::max(1.7 * middle, SPLIT && kDeep ? 2.0 : 0.0);
    if constexpr (!SPLIT || !kDeep) {
        if (!small && q.cols >= 2048 && (SPLIT ? 3.4 : 1.65) * rounds(256, 256) <= middle)
            return launch_step<Product<f16, 256, 256, 4, 2, kDeep, true, false, true>, KIND, SPLIT, RESTS>(p, q, out, matrices, s);
    }
    if constexpr (SPLIT)
        return small ? launch_pair<Product<f16, 64, 64, 2, 2, kDeep, true, false, true>, KIND>(p, q, out, matrices, s)
                     : launch_pair<Product<f16, 128, 128, 2, 4, kDeep, true, false, true>, KIND>(p, q, out, matrices, s);
    else
        return small ? launch_step<Product<f16, 64, 64, 2, 2, kDeep, true, false, true>, KIND, false, RESTS>(p, q, out, matrices, s)
                     : launch_step<Product<f16, 128, 128, 2, 2, kDeep, true, false, true>, KIND, false, RESTS>(p, q, out, matrices, s);
}

// Whether a matrix's X and S fit a compute unit's LDS.
bool is_small(const Sizes &z)
{
    return z.m == 64 ? z.n <= 512 : z.m == 128 && z.n == 128;
}
template <bool SPLIT>
hipError_t small(const MuonSet &set, unsigned matrices, const Sizes &z, const MuonStep &st, hipStream_t s)
{
    if (z.m == 128)
        return launch_small<128, 128, SPLIT>(set, matrices, st, s);
    if (z.n > 128)
        return z.n > 256 ? launch_small<64, 512, SPLIT>(set, matrices, st, s) : launch_small<64, 256, SPLIT>(set, matrices, st, s);
    return z.n > 64 ? launch_small<64, 128, SPLIT>(set, matrices, st, s) : launch_small<64, 64, SPLIT>(set, matrices, st, s);
}

// Matrices of up to 128 rows that do not fit: pieces of 128 columns, and how many a workgroup
// takes so that as many run as at once can: 512, or 256 of 128 rows (51 of 123 x 1,545 245 us, 297
// with 512).
bool is_long(const Sizes &z) { return z.m <= 128 && !is_small(z); }
struct Pieces {
    unsigned per, parts;
};
Pieces pieces_of(const Sizes &z, unsigned matrices)
{
    const unsigned pieces = (z.n + 127) / 128, want = matrices ? (z.m == 64 ? 512 : 256) / matrices : 1, parts = want < 1 ? 1 : want < pieces ? want : pieces;
    const unsigned per = (pieces + parts - 1) / parts;
    return {per, (pieces + per - 1) / per};
}
size_t parts_bytes(const Sizes &z, unsigned matrices)
{
    return whole((size_t)matrices * pieces_of(z, matrices).parts * z.m * z.m * sizeof(float));
}
template <int M, bool SPLIT>
hipError_t columns(const Planes &x, unsigned matrices, const Sizes &z, int iterations, f16 *gram, float *parts, hipStream_t s)
{
    using C = Small<M, 128, SPLIT>;
    const Pieces p = pieces_of(z, matrices);
    for (int i = 0; i <= iterations; ++i) {
        columns_kernel<C, SPLIT><<<dim3(p.parts, matrices), C::kThreads, 0, s>>>(x, gram, parts, p.per, i > 0, i < iterations);
        if (i < iterations)
            sum_parts_kernel<SPLIT><<<dim3(M * M / 1024, matrices), 256, 0, s>>>(parts, p.parts, M * M, gram);
    }
    return hipGetLastError();
}

template <bool SPLIT>
hipError_t orthogonalise(const MuonSet &set, unsigned matrices, const Sizes &z, const MuonStep &st, char *ws,
                         hipStream_t s)
{
    auto take = [&](size_t bytes) {
        char *p = ws;
        ws += whole(bytes * matrices);
        return p;
    };
    double *squares = reinterpret_cast<double *>(take(z.squares));
    auto planes = [&](size_t bytes, unsigned rows, unsigned cols) {
        return Planes{reinterpret_cast<f16 *>(take(bytes)), (long long)(bytes / sizeof(f16)), rows, cols};
    };
    Planes x = planes(z.x, z.m, z.n);
    if (is_long(z)) {
        f16 *gram = reinterpret_cast<f16 *>(take(z.s));
        float *parts = reinterpret_cast<float *>(ws);
        momentum_kernel<<<dim3(z.chunks, matrices), 256, 0, s>>>(set, st, z.chunk, squares);
        const dim3 tiles(z.n / 64, z.m / 64, matrices);
        start_kernel<<<tiles, 256, 0, s>>>(set, st, squares, z.chunks, x);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess)
            e = z.m == 64 ? columns<64, SPLIT>(x, matrices, z, st.iterations, gram, parts, s)
                          : columns<128, SPLIT>(x, matrices, z, st.iterations, gram, parts, s);
        if (e != hipSuccess)
            return e;
        finish_kernel<<<tiles, 256, 0, s>>>(set, st, x, true);
        return hipGetLastError();
    }
    Planes y = planes(z.x, z.m, z.n);
    const Planes gram = planes(z.s, z.m, z.m), poly = planes(z.s, z.m, z.m);
    momentum_kernel<<<dim3(z.chunks, matrices), 256, 0, s>>>(set, st, z.chunk, squares);
    const dim3 tiles(z.n / 64, z.m / 64, matrices);
    start_kernel<<<tiles, 256, 0, s>>>(set, st, squares, z.chunks, x);
    hipError_t e = hipGetLastError();
    for (int i = 0; i < st.iterations && e == hipSuccess; ++i) {
        constexpr int kRests = SPLIT ? 3 : 0;
        e = step<kGram, SPLIT, kRests>(x, x, gram, matrices, s);
        if (e == hipSuccess)
            e = step<kSquare, SPLIT, kRests>(gram, gram, poly, matrices, s);
        if (e != hipSuccess)
            break;
        const int left = st.iterations - i;
        if (SPLIT || left > 3)
            e = step<kApply, SPLIT, 3>(x, poly, y, matrices, s);
        else if (left == 3)
            e = step<kApply, SPLIT, SPLIT ? 3 : 1>(x, poly, y, matrices, s);
        else
            e = step<kApply, SPLIT, kRests>(x, poly, y, matrices, s);
        const Planes was = x;
        x = y;
        y = was;
    }
    if (e != hipSuccess)
        return e;
    finish_kernel<<<tiles, 256, 0, s>>>(set, st, x, SPLIT);
    return hipGetLastError();
}

}  // namespace

size_t muon_workspace_bytes(int fan_out, int fan_in, bool split, unsigned matrices)
{
    const Sizes z = sizes_of(fan_out, fan_in, split);
    if (is_small(z))
        return 0;  // all in LDS
    const size_t both = whole(z.squares * matrices) + whole(z.x * matrices) + whole(z.s * matrices);
    return both + (is_long(z) ? parts_bytes(z, matrices) : whole(z.x * matrices) + whole(z.s * matrices));
}

hipError_t launch_muon(const MuonSet &set, unsigned matrices, int fan_out, int fan_in, bool split,
                       const MuonStep &st, void *workspace, hipStream_t s)
{
    const Sizes z = sizes_of(fan_out, fan_in, split);
    if (is_small(z))
        return split ? small<true>(set, matrices, z, st, s) : small<false>(set, matrices, z, st, s);
    char *ws = static_cast<char *>(workspace);
    return split ? orthogonalise<true>(set, matrices, z, st, ws, s)
                 : orthogonalise<false>(set, matrices, z, st, ws, s);
}

}  // namespace derf
