// Products on the matrix units, tile by tile, and what their kernels share: which rows
// of which head a workgroup takes, operands from memory to LDS and registers, results
// back.  Included by the units whose kernels are made of them.
//
// tile_product below: operand P (TP rows of the matrix unit's first operand) times
// operand Q (TQ of its second), reduced over steps of 128 bytes of depth.  Each
// operand lies in memory either with its depth side by side ("deep") or with its
// tile's rows side by side.
#pragma once
#include "ops_internal.h"

namespace derf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned uniform(unsigned x)
{
    return (unsigned)__builtin_amdgcn_readfirstlane((int)x);
}

struct Problem {
    const int *offsets;
    unsigned rows;
    int heads, fan_in, fan_out;
};

__device__ __forceinline__ unsigned bound(const Problem &p, int h)
{
    const int v = p.offsets[h];
    return v < 0 ? 0u : (unsigned)v < p.rows ? (unsigned)v : p.rows;
}

// ---- which rows a workgroup takes ---------------------------------------------

// Rows [first, last) of one head (or of none: head = number of heads).
struct RowTile {
    unsigned first, last;
    int head;
};

// before[h] (h <= heads): the tiles of `tile_rows` rows of the heads before h, in
// LDS; never more than rows / tile_rows + heads in all, what grids and workspaces
// are made for, whatever the offsets.  At least 256 threads, all call it.
constexpr int kMaxHeads = 256;
__device__ __forceinline__ void count_tiles(const Problem &p, unsigned tile_rows, unsigned *before)
{
    const int h = threadIdx.x, lane = h & 63, wave = h >> 6;
    unsigned mine = 0;
    if (h < p.heads) {
        const unsigned a = bound(p, h), b = bound(p, h + 1);
        mine = b > a ? (b - a + tile_rows - 1) / tile_rows : 0;
    }
    unsigned incl = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned y = __shfl_up(incl, off);
        if (lane >= off)
            incl += y;
    }
    __shared__ unsigned tmp[kMaxHeads / 64];
    if (lane == 63 && wave < kMaxHeads / 64)
        tmp[wave] = incl;
    __syncthreads();
    for (int w = 0; w < wave && w < kMaxHeads / 64; ++w)
        incl += tmp[w];
    const unsigned most = p.rows / tile_rows + p.heads;
    if (h < p.heads)
        before[h + 1] = incl < most ? incl : most;
    if (h == 0)
        before[0] = 0;
    __syncthreads();
}

// Rows of tile number `tile`, which is below before[heads].
__device__ __forceinline__ RowTile head_tile(const Problem &p, const unsigned *before, unsigned tile,
                                             unsigned tile_rows)
{
    int lo = 0, hi = p.heads - 1;  // the last head with before[h] <= tile
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (uniform(before[mid]) <= tile)
            lo = mid;
        else
            hi = mid - 1;
    }
    const unsigned first = uniform(bound(p, lo)) + (tile - uniform(before[lo])) * tile_rows;
    const unsigned last = uniform(bound(p, lo + 1));
    return {first, last - first > tile_rows ? first + tile_rows : last, lo};
}

// Number b, in the order in which they are taken, of `all` tiles: consecutive
// workgroups go to the 8 XCDs in turn; each XCD gets runs of up to 32 tiles (its
// compute units), neighbours that share operands in its L2, and short ones where
// there are few tiles, so that none gets much more than another.  us with runs of 32
// and of 1: bf16 256 to 256 on 262,144 rows 68, 73, both gradients 130, 163; gradients
// of 2,048 to 4,096 on 16,384 498, 511, the layer on 32,768 489, 480 (of 128: 461);
// float32 319 to 640 on 65,536 272, 282 (of 128: 290).  Some b beyond `all` give tiles
// too, and some below none; none from runs_end(all) on does.
constexpr unsigned kXcds = 8, kRun = 32;
__device__ __forceinline__ unsigned run_of(unsigned all)
{
    return all >= 64 * kRun ? kRun : all >= 64 ? all / 64 : 1;
}
__device__ __forceinline__ unsigned by_xcd(unsigned b, unsigned all)
{
    const unsigned run = run_of(all), j = b / kXcds;
    return (j / run * kXcds + b % kXcds) * run + j % run;
}
__device__ __forceinline__ unsigned runs_end(unsigned all)
{
    const unsigned round = run_of(all) * kXcds;
    return (all + round - 1) / round * round;
}

// Tile `at` of rows x cols ones: in groups of 4 rows, a group column by column.
struct Place2 {
    unsigned a, b;
};
__device__ __forceinline__ Place2 in_groups(unsigned at, unsigned rows, unsigned cols)
{
    const unsigned group = at / (4 * cols), in = at - group * 4 * cols;
    const unsigned tall = rows - group * 4 < 4 ? rows - group * 4 : 4;
    return {group * 4 + in % tall, in / tall};
}

// ---- operands -------------------------------------------------------------------

template <class T>
struct Type;
template <>
struct Type<__bf16> {
    static constexpr int kVec = 8;  // elements of 16 bytes
};
template <>
struct Type<_Float16> {
    static constexpr int kVec = 8;
};
template <>
struct Type<float> {
    static constexpr int kVec = 4;
};

struct __attribute__((packed, aligned(2))) Bytes16 {
    u32x4 v;
};

// x without its first `n` elements, zeros behind (n >= the elements: all zero).
template <class T>
__device__ __forceinline__ u32x4 drop_first(u32x4 x, int n)
{
    const int bits = n * (int)sizeof(T) * 8;
    unsigned long long lo = x[0] | (unsigned long long)x[1] << 32;
    unsigned long long hi = x[2] | (unsigned long long)x[3] << 32;
    const int s = bits & 63;
    if (bits >= 64) {
        lo = hi;
        hi = 0;
    }
    if (bits >= 128)
        lo = 0;
    if (s) {
        lo = lo >> s | hi << (64 - s);
        hi >>= s;
    }
    return u32x4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}

// x where y > 0, zero elsewhere (bf16: a value is positive and no NaN if its
// bits less one are below those of infinity).
__device__ __forceinline__ u32x4 where_positive(u32x4 x, u32x4 y, __bf16)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned lo = ((y[i] & 0xFFFFu) - 1u) < 0x7F80u ? 0xFFFFu : 0u;
        const unsigned hi = ((y[i] >> 16) - 1u) < 0x7F80u ? 0xFFFF0000u : 0u;
        x[i] &= lo | hi;
    }
    return x;
}
__device__ __forceinline__ u32x4 where_positive(u32x4 x, u32x4 y, float)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[i] = __uint_as_float(y[i]) > 0.0f ? x[i] : 0u;
    return x;
}

// An operand in memory: element (row, col) at p[row * stride + col], `rows` by
// `cols`; what lies outside counts as zero.  With a mask of the same shape,
// elements count where the mask's are positive.  All of it is the same for the
// whole workgroup.
template <class T>
struct Matrix {
    const T *p;
    long long stride;
    const T *mask;
    long long mask_stride;
    unsigned rows;
    int cols;
};

// A stretch of memory that a workgroup reads at 32-bit offsets: what starts at
// or behind its end reads as zero, and no read that starts in front of it (a
// whole 16-byte piece of a row) reaches over it.  At most 2^31 - 1 bytes, which
// a tile's 256 rows do not exceed (row strides are below 2^21 elements); an
// offset of kOutside is behind every window's end.
typedef u32x4 Window;
constexpr long long kMostBytes = 0x7FFFFFFF;
constexpr unsigned kOutside = 0xFFFFFFF0u;
constexpr unsigned kWindowFlags = 0x00020000u;  // untyped, rows of no fixed length
template <class T>
__device__ __forceinline__ Window window(const T *p, long long stride, unsigned rows, int cols,
                                         unsigned row0, int col0)
{
    const unsigned long long at = reinterpret_cast<unsigned long long>(p + (row0 * stride + col0));
    const long long end = row0 < rows && col0 < cols
                              ? ((long long)(rows - row0 - 1) * stride + cols - col0) * (long long)sizeof(T)
                              : 0;
    const unsigned records = end < kMostBytes ? (unsigned)end : (unsigned)kMostBytes;
    return Window{uniform((unsigned)at), uniform((unsigned)(at >> 32)), uniform(records), kWindowFlags};
}
__device__ __forceinline__ u32x4 read16(const Window &w, unsigned offset)
{
    const void *p = reinterpret_cast<const void *>(w[0] | (unsigned long long)w[1] << 32);
    return __builtin_amdgcn_raw_buffer_load_b128(
        __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, w[2], w[3]), offset, 0, 0);
}
// 64 x 16 bytes to LDS: lane l's piece at `offset` lands at byte lds + 16 l of
// LDS.  Written as asm so that the compiler does not wait for it at the next
// read of LDS; it is waited for where its tile is needed (arrived).
__device__ __forceinline__ void read16_to_lds(const Window &w, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 ::"s"(lds), "v"(offset), "s"(w)
                 : "memory");
}
// The same with 64 x 4 bytes.
__device__ __forceinline__ void read4_to_lds(const Window &w, unsigned offset, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 ::"s"(lds), "v"(offset), "s"(w)
                 : "memory");
}
__device__ __forceinline__ unsigned lds_byte(const char *p)
{
    return uniform((unsigned)(unsigned long)(__attribute__((address_space(3))) const char *)p);
}
// Waits until at most N of this wave's loads and none of its LDS accesses are
// under way, and for the other waves to get here.
template <int N>
__device__ __forceinline__ void arrived()
{
    static_assert(N < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The same for LDS accesses alone.
__device__ __forceinline__ void stored() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Tile of an operand: DEEP: TILE rows by D columns, else D rows by TILE columns;
// one depth step's, D elements being 128 bytes.  In LDS it lies row by row in
// 16-byte chunks, a row's chunks permuted by the row so that reads touch every
// bank once (64 of 4 bytes; no conflicts counted): 16 lanes read 16 bytes at a
// time (lanes 0-3, 12-15, 20-23, 24-27 for one), or 32 lanes 8 bytes where they
// transpose.  A thread brings kShare chunks, all of the same columns.
// PAIR: a deep tile of rows of two halves of a matrix, 16 of the first and 16 of the
// second in turn, so that a wave has both results of a column in the same lanes.
// BOTH: not deep, but read (row_fragment) and written by rows as much as by columns: b128
// reads and transposing ones without bank conflicts in either form, b128 writes of 16 rows
// 8 cycles with TILE 128, 16 without.
constexpr int kChunks = 8;
template <class T, int TILE, bool DEEP, int THREADS, bool MASK, bool PAIR = false, bool BOTH = false>
struct Tile {
    static_assert(DEEP || !PAIR, "pairs are of rows");
    static constexpr int V = Type<T>::kVec, D = kChunks * V;
    static constexpr int kShare = TILE * kChunks / THREADS;
    static constexpr int kBytes = TILE * kChunks * 16;
    static constexpr int kPerRow = DEEP ? kChunks : TILE / V;
    static constexpr int kRowStep = THREADS / kPerRow;
    static_assert(TILE * kChunks % THREADS == 0 && (kRowStep % 16 == 0 || (sizeof(T) == 4 && !DEEP)),
                  "whole shares, of one permutation");
    struct S {
        u32x4 x[kShare];
        u32x4 y[MASK ? kShare : 1];
    };

    // the permutation of row r's chunks: chunk c lies at c ^ turn(r)
    static __device__ __forceinline__ unsigned turn(unsigned r)
    {
        if (DEEP)
            return r >> 1 & 7;
        if (BOTH)  // 8 lanes write 16 bytes at a time, within 128: rows 0-7 differ in their lowest bits
            return TILE == 64 ? (r & 3) | (r >> 1 & 4) : (r & 3) << 1 | ((r << 1 ^ r) & 8) | (r >> 2 & 1);
        if (sizeof(T) == 2)  // in pairs of chunks: rows 0-3 and 8-11 are read at once
            return (TILE == 64 ? (r >> 1 & 1) | (r >> 2 & 2) : (r & 3) | (r >> 1 & 4)) << 1;
        return kRowStep % 16 == 0 ? ((r & 3) | (r >> 1 & 4)) << 1 : 0;
    }
    static __device__ __forceinline__ unsigned my_thread() { return threadIdx.x % THREADS; }  // of a team
    static __device__ __forceinline__ unsigned my_row() { return my_thread() / kPerRow; }
    static __device__ __forceinline__ int my_col()
    {
        return (int)((my_thread() % kPerRow) ^ turn(my_row())) * V;
    }

    // This workgroup's tiles of a matrix, from tile row (or column) t0 on.
    struct Source {
        Matrix<T> m;
        unsigned t0;
        unsigned half;  // PAIR: rows from a row of the first half to the second's
    };
    // Row of the matrix, from t0 on, that is the tile's row r.
    static __device__ __forceinline__ unsigned matrix_row(const Source &s, unsigned r)
    {
        return PAIR ? (r >> 5) * 16 + (r & 15) + (r & 16 ? s.half : 0) : r;
    }
    // First column of the step at depth k, columns from there on, and its window.
    static __device__ __forceinline__ int cols_left(const Source &s, unsigned k)
    {
        return s.m.cols - (int)(DEEP ? k : s.t0);
    }
    static __device__ __forceinline__ int first_col(const Source &s, unsigned k)
    {
        return (int)(DEEP ? k : s.t0);
    }
    // `back`: elements in front of the step's first column to see as well
    static __device__ __forceinline__ Window view(const Source &s, const T *p, long long stride,
                                                  unsigned k, int back = 0)
    {
        return window(p, stride, s.m.rows, s.m.cols, DEEP ? s.t0 : k, first_col(s, k) - back);
    }

    // Starts the loads of the step at depth k.
    static __device__ __forceinline__ void load(S &s, const Source &src, unsigned k)
    {
        const int left = cols_left(src, k);
        const int col = my_col();
        if (src.m.cols >= V) {
            // a chunk that reaches over its row's end is read where it ends with it
            const int back = first_col(src, k) > 0 ? V : 0;
            const unsigned c = (unsigned)(back + (col + V <= left ? col : left - V));
            const unsigned row_bytes = (unsigned)src.m.stride * sizeof(T);
            const Window w = view(src, src.m.p, src.m.stride, k, back);
            const unsigned offset = (PAIR ? 0 : my_row() * row_bytes) + c * (unsigned)sizeof(T);
#pragma unroll
            for (int i = 0; i < kShare; ++i)
                s.x[i] = read16(w, offset + (PAIR ? matrix_row(src, my_row() + i * kRowStep) : i * kRowStep) * row_bytes);
            if (MASK) {
                const unsigned mask_bytes = (unsigned)src.m.mask_stride * sizeof(T);
                const Window y = view(src, src.m.mask, src.m.mask_stride, k, back);
                const unsigned at = my_row() * mask_bytes + c * (unsigned)sizeof(T);
#pragma unroll
                for (int i = 0; i < kShare; ++i)
                    s.y[i] = read16(y, at + i * kRowStep * mask_bytes);
            }
            return;
        }
        // rows shorter than 16 bytes
        const unsigned row0 = (DEEP ? src.t0 : k) + my_row();
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
            const unsigned r = PAIR ? src.t0 + matrix_row(src, my_row() + i * kRowStep) : row0 + i * kRowStep;
            const bool in = r < src.m.rows && col == 0 && left == src.m.cols;
            unsigned x[V] = {}, y[V] = {};
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (in && e < src.m.cols) {
                    x[e] = bits(src.m.p[r * src.m.stride + e]);
                    if (MASK)
                        y[e] = bits(src.m.mask[r * src.m.mask_stride + e]);
                }
            s.x[i] = pack(x);
            if (MASK)
                s.y[i] = pack(y);
        }
    }
    static __device__ __forceinline__ unsigned bits(float x) { return __float_as_uint(x); }
    static __device__ __forceinline__ unsigned bits(__bf16 x) { return __builtin_bit_cast(unsigned short, x); }
    static __device__ __forceinline__ unsigned bits(_Float16 x) { return __builtin_bit_cast(unsigned short, x); }
    static __device__ __forceinline__ u32x4 pack(const unsigned (&x)[V])
    {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = V == 4 ? x[i] : x[2 * i] | x[(2 * i + 1) % V] << 16;
        return v;
    }

    // What was loaded, zero outside the matrix and where its mask says so.
    static __device__ __forceinline__ void settle(S &s, const Source &src, unsigned k)
    {
        if (MASK)
#pragma unroll
            for (int i = 0; i < kShare; ++i)
                s.x[i] = where_positive(s.x[i], s.y[i], T{});
        const int left = cols_left(src, k);
        if (left < (DEEP ? D : TILE) && src.m.cols >= V) {
            const int over = my_col() + V - left;
            if (over > 0)
#pragma unroll
                for (int i = 0; i < kShare; ++i)
                    s.x[i] = drop_first<T>(s.x[i], over);
        }
    }
    static __device__ __forceinline__ void store(const S &s, char *lds)
    {
#pragma unroll
        for (int i = 0; i < kShare; ++i)
            *reinterpret_cast<u32x4 *>(lds + (my_thread() + i * THREADS) * 16) = s.x[i];
    }

    // The same without registers in between, for matrices without a mask whose
    // rows start at multiples of 16 bytes and are as long: steps one after
    // another, with little work for each.
    struct Feed {
        Window w;
        long long left;  // bytes of the matrix from the window's start on
        unsigned step, more;
        int cols;
        unsigned offset[kShare];
        __device__ __forceinline__ void start(const Source &s)
        {
            w = view(s, s.m.p, s.m.stride, 0);
            const unsigned row_bytes = (unsigned)s.m.stride * sizeof(T);
            const int col = my_col();
            cols = cols_left(s, 0);
            more = 0;
            left = s.m.rows ? ((long long)(s.m.rows - 1) * s.m.stride + cols) * (long long)sizeof(T) : 0;
            step = D * row_bytes;
            // a tile's columns that are not the matrix's are outside in every step
#pragma unroll
            for (int i = 0; i < kShare; ++i)
                offset[i] = DEEP || col < cols ? matrix_row(s, my_row() + i * kRowStep) * row_bytes + col * (unsigned)sizeof(T) : kOutside;
        }
        // The steps from here on bring zeros: an empty window, whether or not
        // there was a tile before.
        __device__ __forceinline__ void stop()
        {
            w = Window{0u, 0u, 0u, kWindowFlags};
            left = 0;
            step = more = 0;
            cols = 0;
#pragma unroll
            for (int i = 0; i < kShare; ++i)
                offset[i] = kOutside;
        }
        // Brings piece i of the step to the LDS tile that starts at byte `lds`.
        __device__ __forceinline__ void piece(int i, unsigned lds) const
        {
            const unsigned to = lds + uniform(threadIdx.x & ~63u) * 16 + i * THREADS * 16;
            if (DEEP)
                read16_to_lds(w, my_col() < cols ? offset[i] + more : kOutside, to);
            else
                read16_to_lds(w, offset[i], to);
        }
        __device__ __forceinline__ void advance()
        {
            if (DEEP) {
                cols -= D;
                more += D * sizeof(T);
            } else {
                const unsigned long long at = (w[0] | (unsigned long long)w[1] << 32) + step;
                left -= step;
                w[0] = (unsigned)at;
                w[1] = (unsigned)(at >> 32);
                w[2] = left > kMostBytes ? (unsigned)kMostBytes : left > 0 ? (unsigned)left : 0u;
            }
        }
    };

    // 16-byte chunk `c` of row `r`, in bytes.
    static __device__ __forceinline__ unsigned at(unsigned r, unsigned c)
    {
        return (r * kPerRow + (c ^ turn(r))) * 16;
    }

    // Of an operand whose tile's rows lie side by side, read as a deep one: rows
    // [16 f, 16 f + 16), 64 bytes from byte 64 part on.
    static __device__ __forceinline__ u32x4 row_fragment(const char *lds, int f, int part)
    {
        static_assert(!DEEP, "the other kind");
        const int quarter = (threadIdx.x & 63) >> 4, l = threadIdx.x & 15;
        return *reinterpret_cast<const u32x4 *>(lds + at(f * 16 + l, part * 4 + quarter));
    }

    // The matrix unit's operand: tile rows [16 f, 16 f + 16), half `part` of the
    // step.  bf16: 32 deep, 8 side by side a lane.  float: 16 deep, lane quarter h
    // has depths 4 h + (0 .. 3): the unit takes them four (one of each) at a time.
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int f, int part)
    {
        const int quarter = (threadIdx.x & 63) >> 4, l = threadIdx.x & 15;
        if (DEEP)
            return *reinterpret_cast<const u32x4 *>(lds + at(f * 16 + l, part * 4 + quarter));
        if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 rows of 16 elements and get them by columns
            const unsigned r = part * 32 + quarter * 8 + (l >> 2);
            const unsigned e = f * 16 + (l & 3) * 4;
            typedef __attribute__((address_space(3))) i16x4 *Lds;
            const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(lds + at(r, e / 8) + (e & 4) * 2));
            const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(lds + at(r + 4, e / 8) + (e & 4) * 2));
            return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            u32x4 x;
            const unsigned e = f * 16 + l;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = *reinterpret_cast<const unsigned *>(
                    lds + at(part * 16 + quarter * 4 + j, e / 4) + (e & 3) * 4);
            return x;
        }
    }
};

// 16 x 16 results: of the matrix unit's forms the one of least power, which is
// what bounds it (random bf16 values in registers: 2,060 TFLOP/s, 32 x 32 x 16:
// 1,780).  Lane 16 h + l has column l (of Q), rows 4 h + (0 .. 3) (of P).
__device__ __forceinline__ f32x4 multiply(u32x4 p, u32x4 q, f32x4 c, __bf16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p),
                                                   __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(u32x4 p, u32x4 q, f32x4 c, _Float16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(u32x4 p, u32x4 q, f32x4 c, float)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(p[j]), __uint_as_float(q[j]), c, 0, 0, 0);
    return c;
}

// Sizes of a product: a workgroup's tile TP x TQ, by WP x WQ waves.  MASK: Q has
// a mask.  ASYNC: operands go from memory to LDS by themselves (Tile::Feed).
// EACH_Q: tile_product shows its caller the Q tiles.  TEAMS: of so many waves each;
// they take the depth's steps in turn, in LDS of their own, and add up at the end.
// PAIR: P's tiles are of pairs (Tile).
template <class T_, int TP_, int TQ_, int WP_, int WQ_, bool DEEP_P, bool DEEP_Q, bool MASK,
          bool ASYNC = false, bool EACH_Q = false, int TEAMS = 1, bool PAIR = false>
struct Product {
    using T = T_;
    static constexpr int TP = TP_, TQ = TQ_, WP = WP_, WQ = WQ_;
    static constexpr int kTeams = TEAMS, kTeam = WP * WQ * 64, kThreads = kTeam * TEAMS;
    static constexpr bool kAsync = ASYNC, kEachQ = EACH_Q, kPair = PAIR;
    static_assert(TEAMS == 1 || !ASYNC, "teams bring their operands through registers");
    using P = Tile<T, TP, DEEP_P, kTeam, false, PAIR>;
    using Q = Tile<T, TQ, DEEP_Q, kTeam, MASK>;
    static constexpr int kDepth = P::D;
    static constexpr int FP = TP / WP / 16, FQ = TQ / WQ / 16;  // a wave's 16 x 16 results
    static constexpr int kStage = P::kBytes + Q::kBytes, kLds = 2 * kStage * TEAMS;
    static constexpr int kLoads = P::kShare + Q::kShare;  // of a thread for a step
    // tile_product's sets of registers: a second one costs masked 128 x 128 tiles
    // spills and narrow ones a workgroup more on the compute unit (262,144 rows of
    // 64 to 64 24 us, 18 with one; of 319 to 256 132, 147 with one)
    static constexpr int kSets = TEAMS > 1 || (!MASK && FP * FQ >= 16) ? 2 : 1;
    static constexpr int kCols = PAIR ? TP / 2 : TP;  // of a result's row
    static_assert(FP * WP * 16 == TP && FQ * WQ * 16 == TQ && (!PAIR || FP % 2 == 0), "whole results a wave");
};

// What of `all` things to do in turn n of `turns`, spread evenly: do_one(i).
template <class F>
__device__ __forceinline__ void share_out(int n, int turns, int all, F do_one)
{
#pragma unroll
    for (int i = 0; i < all; ++i)
        if (i * turns / all == n)
            do_one(i);
}

// acc += the products of p and q.  Meanwhile the next part's operands come from
// half `part` of the stage at `lds` to p_next and, each where it has been used, to q
// (READ), and load(i) is called for each of kLoads (LOAD).
template <class C, bool LOAD, class Load>
__device__ __forceinline__ void multiply_part(const u32x4 (&p)[C::FP], u32x4 (&q)[C::FQ], u32x4 (&p_next)[C::FP],
                                              bool read, const char *lds, int fp, int fq, int part,
                                              f32x4 (&acc)[C::FP][C::FQ], Load load)
{
    constexpr int kAll = C::FP * C::FQ;
#pragma unroll
    for (int j = 0; j < C::FQ; ++j)
#pragma unroll
        for (int i = 0; i < C::FP; ++i) {
            const int n = j * C::FP + i;
            acc[i][j] = multiply(p[i], q[j], acc[i][j], typename C::T{});
            if (read) {
                if (i == C::FP - 1)
                    q[j] = C::Q::fragment(lds + C::P::kBytes, fq + j, part);
                share_out(n, kAll, C::FP, [&](int k) { p_next[k] = C::P::fragment(lds, fp + k, part); });
            }
            if (LOAD)
                share_out(n, kAll, C::kLoads, load);
            __builtin_amdgcn_sched_barrier(0);
        }
}

// The first part's operands, from the stage at `lds`.
template <class C>
__device__ __forceinline__ void read_first(u32x4 (&p)[C::FP], u32x4 (&q)[C::FQ], const char *lds, int fp, int fq)
{
#pragma unroll
    for (int i = 0; i < C::FP; ++i)
        p[i] = C::P::fragment(lds, fp + i, 0);
#pragma unroll
    for (int j = 0; j < C::FQ; ++j)
        q[j] = C::Q::fragment(lds + C::P::kBytes, fq + j, 0);
}

// A step has two parts; operands are read a part ahead of their products, the
// next step's first behind the barrier between the parts.  There all of the step
// has been read, and the loads of the step after the next overwrite it.

// Products whose operands go to LDS by themselves: a workgroup's tiles one after
// another, with the loads two steps ahead of the products, across the tiles.
template <class C>
struct Pipe {
    char *lds;
    unsigned lds0, stage, left;  // left: steps of the tile being loaded that are not yet
    int fp, fq;
    typename C::P::Feed pf;
    typename C::Q::Feed qf;
    u32x4 pa[C::FP], pb[C::FP], q[C::FQ];

    __device__ __forceinline__ void piece(int i, unsigned to)
    {
        if (i < C::P::kShare)
            pf.piece(i, to);
        else
            qf.piece(i - C::P::kShare, to + C::P::kBytes);
    }
    // next_tile(*this): calls load_tile with the next tile of more than no steps, or
    // load_nothing.
    __device__ __forceinline__ void load_tile(const typename C::P::Source &p, const typename C::Q::Source &q_,
                                              unsigned depth)
    {
        pf.start(p);
        qf.start(q_);
        left = (depth + C::kDepth - 1) / C::kDepth;
    }
    __device__ __forceinline__ void load_nothing()
    {
        pf.stop();
        qf.stop();
        left = 0xFFFFFFFFu;
    }
    template <class Next>
    __device__ __forceinline__ void start(char *lds_, Next next_tile)
    {
        const int wave = uniform(threadIdx.x >> 6);
        fp = (wave % C::WP) * C::FP;
        fq = (wave / C::WP) * C::FQ;
        lds = lds_;
        lds0 = lds_byte(lds);
        stage = 0;
        left = 0;
        for (int n = 0; n < 2; ++n) {
            if (left == 0)
                next_tile(*this);
#pragma unroll
            for (int i = 0; i < C::kLoads; ++i)
                piece(i, lds0 + n * C::kStage);
            advance();
        }
        arrived<C::kLoads>();
        read_first<C>(pa, q, lds, fp, fq);
    }
    __device__ __forceinline__ void advance()
    {
        pf.advance();
        qf.advance();
        --left;
    }
    // The next step's products.
    template <class Next, class EachQ>
    __device__ __forceinline__ void step(f32x4 (&acc)[C::FP][C::FQ], Next next_tile, EachQ each_q)
    {
        const unsigned used = stage * C::kStage;
        if constexpr (C::kEachQ) {
            typename C::Q::S s;
#pragma unroll
            for (int i = 0; i < C::Q::kShare; ++i)
                s.x[i] = *reinterpret_cast<const u32x4 *>(lds + used + C::P::kBytes + (threadIdx.x + i * C::kThreads) * 16);
            each_q(s);
        }
        if (left == 0)
            next_tile(*this);
        multiply_part<C, false>(pa, q, pb, true, lds + used, fp, fq, 1, acc, [](int) {});
        arrived<0>();
        stage ^= 1;
        multiply_part<C, true>(pb, q, pa, true, lds + stage * C::kStage, fp, fq, 0, acc,
                               [&](int i) { piece(i, lds0 + used); });
        advance();
    }
};

// Through registers, one tile: acc = sum over `depth` of P(p, k) Q(q, k).  A step's
// loads begin two steps before it is stored, into two sets of registers in turn
// (one step is shorter than a load takes), or one where there is no room for two.
// each_q(share): called with each of the Q tiles that this thread brings.  A team's
// steps are every kTeams-th; all teams make as many, of zeros behind the last.
template <class C, class EachQ>
__device__ __forceinline__ void tile_product(const typename C::P::Source &ps, const typename C::Q::Source &qs,
                                             unsigned depth, char *lds,
                                             f32x4 (&acc)[C::FP][C::FQ], EachQ each_q)
{
    constexpr unsigned kStep = C::kDepth * C::kTeams;
    const int wave = uniform(threadIdx.x >> 6) % (C::kTeam / 64);
    const int fp = (wave % C::WP) * C::FP, fq = (wave / C::WP) * C::FQ;
    if (depth == 0)
        return;
    const unsigned team = C::kTeams > 1 ? uniform(threadIdx.x / C::kTeam) : 0, mine = team * C::kDepth;
    lds += team * 2 * C::kStage;
    struct Set {
        typename C::P::S p;
        typename C::Q::S q;
    } sets[C::kSets];
    Set &even = sets[0], &odd = sets[C::kSets - 1];  // steps 0, 2, ... and 1, 3, ...
    u32x4 pa[C::FP], pb[C::FP], q[C::FQ];
    auto load = [&](Set &s, unsigned k) {
        if (k + mine < depth) {
            C::P::load(s.p, ps, k + mine);
            C::Q::load(s.q, qs, k + mine);
        } else if (C::kTeams > 1) {
            s = Set{};
        }
    };
    auto bring = [&](Set &s, unsigned k, unsigned to) {
        if (k >= depth)
            return;
        if (C::kTeams == 1 || k + mine < depth) {
            C::P::settle(s.p, ps, k + mine);
            C::Q::settle(s.q, qs, k + mine);
        }
        if constexpr (C::kEachQ)
            each_q(s.q);
        C::P::store(s.p, lds + to * C::kStage);
        C::Q::store(s.q, lds + to * C::kStage + C::P::kBytes);
    };
    // the step at k, whose successor is in `next`
    auto step = [&](unsigned k, unsigned stage, Set &next) {
        multiply_part<C, false>(pa, q, pb, true, lds + stage * C::kStage, fp, fq, 1, acc, [](int) {});
        bring(next, k + kStep, stage ^ 1);
        load(next, k + (1 + C::kSets) * kStep);
        stored();
        multiply_part<C, false>(pb, q, pa, k + kStep < depth, lds + (stage ^ 1) * C::kStage, fp, fq, 0, acc, [](int) {});
    };
    load(even, 0);
    if constexpr (C::kSets == 2)
        load(odd, kStep);
    bring(even, 0, 0);
    load(even, C::kSets * kStep);
    stored();
    read_first<C>(pa, q, lds, fp, fq);
#pragma unroll 1
    for (unsigned k = 0; k < depth; k += 2 * kStep) {
        step(k, 0, odd);
        if (k + kStep < depth)
            step(k + kStep, 1, even);
    }
}

// The teams' results added up in the first one's registers, in the teams' order.
// `lds` is that of the stages, which all have been read.  True for the first team.
template <class C>
__device__ __forceinline__ bool join_teams(char *lds, f32x4 (&acc)[C::FP][C::FQ])
{
    constexpr int kAll = C::FP * C::FQ;
    const int team = uniform(threadIdx.x / C::kTeam);
    f32x4 *parts = reinterpret_cast<f32x4 *>(lds) + threadIdx.x % C::kTeam;
    stored();
    if (team > 0)
#pragma unroll
        for (int n = 0; n < kAll; ++n)
            parts[((team - 1) * kAll + n) * C::kTeam] = acc[n / C::FQ][n % C::FQ];
    stored();
    if (team > 0)
        return false;
#pragma unroll
    for (int t = 0; t < C::kTeams - 1; ++t)
#pragma unroll
        for (int n = 0; n < kAll; ++n)
            acc[n / C::FQ][n % C::FQ] += parts[(t * kAll + n) * C::kTeam];
    return true;
}
template <class C>
constexpr int kJoinBytes = (C::kTeams - 1) * C::FP * C::FQ * C::kTeam * 16;

// ---- rows: the layer, and its rows' gradient --------------------------------------

// A wave's results as rows of 16 FP elements: lane 16 h + l has, of row 16 j + l
// of Q, elements 4 h + (0 .. 3) of each 16 of P.  float results are written from the
// registers, 16 bytes a lane.  bf16 ones go through LDS, 16 rows at a time, to be
// written in 16-byte pieces; kResultRow: bytes of a row there (4 of 64 banks further
// on for the next row).
template <class C>
constexpr int kResultRow = C::FP * (C::kPair ? 8 : 16) * (int)sizeof(typename C::T) + 16;
template <class C>
constexpr int kResultBytes = sizeof(typename C::T) == 2 ? C::WP * C::WQ * 16 * kResultRow<C> : 16;
template <class T>
__device__ __forceinline__ void store_values(char *to, f32x4 v, T)
{
    union {
        T e[4];
        unsigned long long u;
    } x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x.e[i] = (T)v[i];
    *reinterpret_cast<unsigned long long *>(to) = x.u;
}
__device__ __forceinline__ void store_values(char *to, f32x4 v, float) { *reinterpret_cast<f32x4 *>(to) = v; }

// The first `left` (at most 16 bytes' worth) elements of v.
template <class T>
__device__ __forceinline__ void write_piece(T *to, u32x4 v, int left, T)
{
    constexpr int V = Type<T>::kVec;
    if (left >= V) {
        reinterpret_cast<Bytes16 *>(to)->v = v;
        return;
    }
    union {
        u32x4 v;
        T e[V];
    } piece = {v};
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (k < left)
            to[k] = piece.e[k];
}

// Whether results go past the caches (nontemporal): their rows are whole 128-byte
// lines.  bf16 us so and with ordinary stores: 2,048 to 4,096 on 32,768 rows 468, 521;
// 256 to 256 on 262,139 67, 76, its dx alone 62, 71; 319 to 256 83, 103.  Rows that
// share lines: both gradients of 319 to 256 252 either way, with ReLU 319, 318, though
// dx alone would take 124 instead of 147 and a layer of 256 to 319 97 instead of 118.
template <class T>
__host__ __device__ __forceinline__ bool past_caches(const T *y, long long ys, int width)
{
    return ((unsigned)reinterpret_cast<unsigned long long>(y) | (unsigned)ys * (unsigned)sizeof(T) |
            (unsigned)width * (unsigned)sizeof(T)) % 128 == 0;
}
template <class T>
__device__ __forceinline__ void write_result(T *to, u32x4 v, int left, bool past)
{
    if (past)
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(to));
    else
        write_piece(to, v, left, T{});
}

// 16 rows from row0 on of a wave's COLS results from column n0 on, below `last` and
// `width`: lane 16 h + l has, of row l, columns 4 h + (0 .. 3) of each 16.  bf16 through
// the wave's place in LDS (kPieceRow a row), for pieces of 16 bytes.  PAST: past the caches
// where whole lines allow it.
template <class T, int COLS>
constexpr int kPieceRow = COLS * (int)sizeof(T) + 16;
template <class T, int COLS, bool STAGE = sizeof(T) == 2, bool PAST = true>
__device__ __forceinline__ void write_16_rows(const f32x4 (&v)[COLS / 16], char *mine, unsigned row0, unsigned last, int n0,
                                              int width, T *y, long long ys)
{
    constexpr int V = Type<T>::kVec, kPieces = COLS / V;  // of a row
    const int lane = threadIdx.x & 63;
    if constexpr (!STAGE) {
        const unsigned row = row0 + (lane & 15);
#pragma unroll
        for (int i = 0; i < COLS / 16; ++i) {
            const int n = n0 + i * 16 + (lane >> 4) * 4;
            if (row < last && n < width)
                write_piece(y + (row * ys + n), __builtin_bit_cast(u32x4, v[i]), width - n, T{});
        }
        return;
    }
    const bool past = PAST && COLS * sizeof(T) >= 128 && past_caches(y, ys, width);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < COLS / 16; ++i)
        store_values(mine + (lane & 15) * kPieceRow<T, COLS> + (i * 16 + (lane >> 4) * 4) * (int)sizeof(T), v[i], T{});
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < (16 * kPieces + 63) / 64; ++i) {
        const int r = (i * 64 + lane) / kPieces, c = (i * 64 + lane) % kPieces * V;
        if (16 * kPieces % 64 && r >= 16)
            continue;
        const u32x4 piece = *reinterpret_cast<const u32x4 *>(mine + r * kPieceRow<T, COLS> + c * (int)sizeof(T));
        const unsigned row = row0 + r;
        const int n = n0 + c;
        if (row < last && n < width)
            write_result(y + (row * ys + n), piece, width - n, past);
    }
    __builtin_amdgcn_wave_barrier();
}

// ---- launches ---------------------------------------------------------------------

unsigned tiles_of(long long n, int tile) { return (unsigned)((n + tile - 1) / tile); }

// Launches for at most `all` tiles: launch(workgroups, from).  Where workgroups
// take tiles one after another (ASYNC), as many as run at once; else one a tile,
// within a launch's limits.
template <class C, class F>
hipError_t launch_for(unsigned long long all, F launch)
{
    if (all >= 1ull << 31)  // more than any memory holds
        return hipErrorInvalidConfiguration;
    const unsigned end = (unsigned)all + kXcds * kRun;  // runs_end of as many or fewer is not above it
    if (C::kAsync) {
        int device, cus;
        hipError_t e = hipGetDevice(&device);
        if (e == hipSuccess)
            e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device);
        if (e != hipSuccess)
            return e;
        const unsigned most = (unsigned)cus * (C::kThreads >= 512 ? 1 : 2);
        launch(end < most ? end : most, 0u);
    } else {
        constexpr unsigned kMost = 1u << 22;
        for (unsigned from = 0; from < end; from += kMost)
            launch(end - from < kMost ? end - from : kMost, from);
    }
    return hipGetLastError();
}

// Whether an operand can go from memory to LDS by itself (Tile::Feed).
template <class T>
bool goes_alone(const Matrix<T> &m)
{
    return !m.mask && reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.stride % Type<T>::kVec == 0 &&
           m.cols % Type<T>::kVec == 0;
}

}  // namespace

}  // namespace derf
