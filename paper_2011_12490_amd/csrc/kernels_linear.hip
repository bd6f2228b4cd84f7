// The heads' linear layers and their gradients: products of matrices whose
// rows come in groups, one group a head, with bounds known on the device only.
//
//   layer      y[r][o]  = act(sum_i x[r][i] W[o][i] + b[o])
//   rows       dx[r][i] = sum_o dz[r][o] W[o][i]
//   weights    dW[o][i] = sum_r dz[r][o] x[r][i],  db[o] = sum_r dz[r][o]
//
// One tile product serves all three (tile_product below): operand P (TP
// rows of the matrix unit's first operand) times operand Q (TQ of its second),
// reduced over steps of 128 bytes of depth.  Each operand lies in memory either
// with its depth side by side ("deep": x, dz, and W for a layer) or with its
// tile's rows side by side (W for the rows' gradient; dz and x for the weights').
#include "ops_internal.h"

namespace derf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
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
constexpr int kChunks = 8;
template <class T, int TILE, bool DEEP, int THREADS, bool MASK>
struct Tile {
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
    };
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
            const unsigned offset = my_row() * row_bytes + c * (unsigned)sizeof(T);
#pragma unroll
            for (int i = 0; i < kShare; ++i)
                s.x[i] = read16(w, offset + i * kRowStep * row_bytes);
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
            const unsigned r = row0 + i * kRowStep;
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
                offset[i] = DEEP || col < cols ? (my_row() + i * kRowStep) * row_bytes + col * (unsigned)sizeof(T) : kOutside;
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
template <class T_, int TP_, int TQ_, int WP_, int WQ_, bool DEEP_P, bool DEEP_Q, bool MASK,
          bool ASYNC = false, bool EACH_Q = false, int TEAMS = 1>
struct Product {
    using T = T_;
    static constexpr int TP = TP_, TQ = TQ_, WP = WP_, WQ = WQ_;
    static constexpr int kTeams = TEAMS, kTeam = WP * WQ * 64, kThreads = kTeam * TEAMS;
    static constexpr bool kAsync = ASYNC, kEachQ = EACH_Q;
    static_assert(TEAMS == 1 || !ASYNC, "teams bring their operands through registers");
    using P = Tile<T, TP, DEEP_P, kTeam, false>;
    using Q = Tile<T, TQ, DEEP_Q, kTeam, MASK>;
    static constexpr int kDepth = P::D;
    static constexpr int FP = TP / WP / 16, FQ = TQ / WQ / 16;  // a wave's 16 x 16 results
    static constexpr int kStage = P::kBytes + Q::kBytes, kLds = 2 * kStage * TEAMS;
    static constexpr int kLoads = P::kShare + Q::kShare;  // of a thread for a step
    // tile_product's sets of registers: a second one costs masked 128 x 128 tiles
    // spills and narrow ones a workgroup more on the compute unit (262,144 rows of
    // 64 to 64 24 us, 18 with one; of 319 to 256 132, 147 with one)
    static constexpr int kSets = TEAMS > 1 || (!MASK && FP * FQ >= 16) ? 2 : 1;
    static_assert(FP * WP * 16 == TP && FQ * WQ * 16 == TQ, "whole results a wave");
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
constexpr int kResultRow = C::FP * 16 * (int)sizeof(typename C::T) + 16;
template <class C>
constexpr int kResultBytes = sizeof(typename C::T) == 2 ? C::WP * C::WQ * 16 * kResultRow<C> : 16;
__device__ __forceinline__ void store_values(char *to, f32x4 v, __bf16)
{
    union {
        __bf16 e[4];
        unsigned long long u;
    } x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x.e[i] = (__bf16)v[i];
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

// P: the weights (width columns of the result), Q: rows.  Where operands go to LDS by
// themselves a workgroup goes on from tile to tile with its loads two steps ahead;
// tiles that share rows or weights run on one XCD.  2,048 to 4,096 on 32,768 rows of
// bf16: 493 us, 1,115 TFLOP/s; what depth adds runs at 1,430, the rest is a tile's
// start and its results' stores.  1,024 to 4,096 on 26 rows of 16 heads, the weights'
// reading: 18 us.
template <class C>
__global__ __launch_bounds__(C::kThreads, 2) void rows_kernel(
    Problem p, Matrix<typename C::T> w, Matrix<typename C::T> x, const float *bias, int relu,
    typename C::T *y, long long ys, int width, int depth, unsigned from)
{
    using T = typename C::T;
    constexpr int kBiases = C::kAsync ? 4 : 1;  // of the tiles under way
    __shared__ __attribute__((aligned(16))) char lds[C::kLds];
    __shared__ __attribute__((aligned(16))) char results[C::kAsync ? kResultBytes<C> : 16];
    __shared__ __attribute__((aligned(16))) float biases[kBiases][C::TP];
    __shared__ unsigned before[kMaxHeads + 1];
    static_assert(C::kAsync || kJoinBytes<C> + kResultBytes<C> <= C::kLds, "parts and results take the stages' place");
    count_tiles(p, C::TQ, before);
    const unsigned headed = uniform(before[p.heads]), headless = bound(p, p.heads);
    const unsigned tail = (unsigned)(((unsigned long long)(p.rows - headless) + C::TQ - 1) / C::TQ);
    const unsigned row_tiles = headed + tail, col_tiles = (width + C::TP - 1) / C::TP;
    const unsigned all = row_tiles * col_tiles, end = runs_end(all);
    const size_t head_size = (size_t)p.fan_in * p.fan_out;
    // what workgroup number b does: false if nothing
    auto tile_at = [&](unsigned b, RowTile &t, int &n0) {
        const unsigned at = by_xcd(b, all);
        if (at >= all)
            return false;
        const Place2 where = in_groups(at, row_tiles, col_tiles);
        n0 = (int)where.b * C::TP;
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
        ps = {w, (unsigned)n0};
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
                    const Window b = window(bias + (size_t)u.head * width, width, 1, width, 0, m0);
                    const unsigned wave = uniform(threadIdx.x >> 6);
                    read4_to_lds(b, threadIdx.x * 4, lds_byte(reinterpret_cast<const char *>(biases[loaded & 3])) + wave * 256);
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
            write_rows<C>(t, n0, width, acc, has && bias ? biases[done & 3] : nullptr, has && relu, results, y, ys);
            done += has;
        }
        arrived<0>();
    } else {
        if (!tile_at(from + blockIdx.x, t, n0))
            return;
        f32x4 acc[C::FP][C::FQ] = {};
        const bool has = t.head < p.heads;
        if (has) {
            if (bias && threadIdx.x < C::TP)
                biases[0][threadIdx.x] =
                    n0 + (int)threadIdx.x < width ? bias[(size_t)t.head * width + n0 + threadIdx.x] : 0.0f;
            typename C::P::Source ps;
            typename C::Q::Source qs;
            sources(t, n0, ps, qs);
            tile_product<C>(ps, qs, depth, lds, acc, [](auto &) {});
        }
        if constexpr (C::kTeams > 1)
            if (!join_teams<C>(lds, acc))
                return;
        write_rows<C>(t, n0, width, acc, has && bias ? biases[0] : nullptr, has && relu, lds + kJoinBytes<C>, y, ys);
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

// A tile of dW [O][I], rows from m0 on, columns from n0 on.
template <class C>
__device__ __forceinline__ void write_weights(float *to, int m0, int n0, int O, int I, const f32x4 (&acc)[C::FP][C::FQ])
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
            write_piece(to + ((size_t)m * I + n), __builtin_bit_cast(u32x4, acc[i][j]), I - n, 0.0f);
        }
    }
}

// P: x, Q: dz, reduced over rows: a tile of a head's dW from a stretch of
// `stretch` of its rows.  Where heads have more than one stretch (partial),
// each has a place of its own in dw and db, and sum_kernel adds them up.  db comes from
// the dz tiles on their way, no pass of its own.  dW and db of 2,048 to 4,096 on 32,768
// rows of bf16: 499 us, 1,100 TFLOP/s, bound by the matrix units' power.
template <class C>
__global__ __launch_bounds__(C::kThreads, 2) void weights_kernel(Problem p, Matrix<typename C::T> dz,
                                                                 Matrix<typename C::T> x, float *dw,
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
template <class T_, int TO_, int STEPS, bool DEEP_W, bool MASK, bool PAST>
struct Shallow {
    using T = T_;
    static constexpr bool kPast = PAST;  // asked in the loop instead, it costs what it brings
    static constexpr int TO = TO_, kSteps = STEPS, kThreads = 512, kColGroups = TO / 64, RT = 16 * 8 / kColGroups;
    using W = Tile<T, TO, DEEP_W, kThreads, false>;
    using X = Tile<T, RT, true, kThreads, MASK>;
    static constexpr int FP = 4;  // a wave's: 64 outputs of 16 rows
    static constexpr int kRowBytes = 64 * (int)sizeof(T) + 16;
    static constexpr int kX = STEPS * W::kBytes, kOut = kX + STEPS * X::kBytes, kLds = kOut + 8 * 16 * kRowBytes;
    // workgroups a compute unit: by LDS, and 4 waves a SIMD
    static constexpr int kAtOnce = 2 * (kLds + 4096) <= 160 * 1024 ? 2 : 1;
};

template <class C>
__global__ __launch_bounds__(C::kThreads, 2 * C::kAtOnce) void shallow_kernel(Problem p, Matrix<typename C::T> w,
                                                                              Matrix<typename C::T> x, const float *bias,
                                                                              int relu, typename C::T *y, long long ys, int width,
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
    const unsigned cols = (O + C::TO - 1) / C::TO, j = blockIdx.x / kXcds;
    const unsigned places = uniform(before[p.heads]), place = j / cols * kXcds + blockIdx.x % kXcds;
    const int n0 = (int)(j % cols) * C::TO;
    if (place >= places) {  // rows without a head: zeros
        const unsigned headless = bound(p, p.heads);
        const unsigned long long from = headless + (unsigned long long)(place - places) * stretch;
        for (unsigned long long r = from + wave; r < from + stretch && r < p.rows; r += C::kThreads / 64)
            for (int c = n0 + lane; c < n0 + C::TO && c < O; c += 64)
                y[r * ys + c] = (T)0.0f;
        return;
    }
    const RowTile t = head_tile(p, before, place, stretch);
    typename C::W::Source ws = {w, (unsigned)n0};
    ws.m.p += t.head * ((size_t)p.fan_in * p.fan_out);
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
    if (threadIdx.x < C::TO)
        biases[threadIdx.x] =
            bias && n0 + (int)threadIdx.x < O ? bias[(size_t)t.head * O + n0 + threadIdx.x] : 0.0f;
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
#pragma unroll
        for (int f = 0; f < C::FP; ++f) {
            const int e = f * 16 + (lane >> 4) * 4;
            f32x4 v = acc[f] + *reinterpret_cast<const f32x4 *>(biases + fp * 16 + e);
            if (relu)
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
template <class CR, class CW>
__global__ __launch_bounds__(CR::kThreads, 2) void gradients_kernel(Problem p, Matrix<typename CR::T> w,
                                                                    Matrix<typename CR::T> dz, Matrix<typename CR::T> x,
                                                                    typename CR::T *dx, long long dxs, float *dw, float *db)
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
__global__ __launch_bounds__(256) void sum_kernel(Problem p, unsigned stretch, const float *wparts, size_t wsize, float *dw,
                                                  const float *bparts, float *db, unsigned wblocks)
{
    constexpr unsigned kWaves = 4, kAtOnce = 8;
    __shared__ unsigned before[kMaxHeads + 1];
    __shared__ f32x4 sums[kWaves][64];
    count_tiles(p, stretch, before);
    const unsigned a = uniform(before[blockIdx.y]), b = uniform(before[blockIdx.y + 1]);
    const bool biases = blockIdx.x >= wblocks;
    const float *parts = biases ? bparts : wparts;
    float *out = biases ? db : dw;
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
            write_piece(out + (blockIdx.y * size + e), __builtin_bit_cast(u32x4, v), here, 0.0f);
        }
        __syncthreads();
    }
}

// ---- a masked copy -------------------------------------------------------------------

// out[r][c] = x[r][c] where y[r][c] > 0, else zero; rows of `cols`, a multiple of 8.
// Three passes over rows of fan_out, bound by their bytes.
__global__ __launch_bounds__(256) void mask_kernel(const __bf16 *x, long long xs, const __bf16 *y, long long ys,
                                                   unsigned rows, int cols, __bf16 *out)
{
    const unsigned vecs = cols / 8;
    for (unsigned r = blockIdx.x; r < rows; r += gridDim.x)
        for (unsigned c = threadIdx.x; c < vecs; c += 256) {
            const u32x4 a = reinterpret_cast<const Bytes16 *>(x + r * xs + c * 8)->v;
            const u32x4 b = reinterpret_cast<const Bytes16 *>(y + r * ys + c * 8)->v;
            *reinterpret_cast<u32x4 *>(out + (size_t)r * cols + c * 8) = where_positive(a, b, __bf16{});
        }
}

// ---- choice of a form ---------------------------------------------------------------

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

template <class C>
hipError_t launch_rows(const Problem &p, const Matrix<typename C::T> &w,
                       const Matrix<typename C::T> &x, const float *bias, bool relu, Rows y,
                       int width, int depth, hipStream_t s)
{
    using T = typename C::T;
    // at most: every head's last tile and the headless rows' may be partly filled
    return launch_for<C>(((unsigned long long)p.rows / C::TQ + p.heads + 1) * tiles_of(width, C::TP),
                         [&](unsigned groups, unsigned from) {
                             rows_kernel<C><<<groups, C::kThreads, 0, s>>>(
                                 p, w, x, bias, relu, static_cast<T *>(const_cast<void *>(y.p)), y.stride, width, depth, from);
                         });
}

// Whether an operand can go from memory to LDS by itself (Tile::Feed).
template <class T>
bool goes_alone(const Matrix<T> &m)
{
    return !m.mask && reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.stride % Type<T>::kVec == 0 &&
           m.cols % Type<T>::kVec == 0;
}

// 256 x 256 tiles, one workgroup a compute unit, or 128 x 128 ones, two: a large
// one does the work of four in the time of 3.5, but the last round of tiles is a
// larger part of the whole.  us with large and small tiles: 4,096 rows of 2,048 to
// 4,096 100, 89; 32,768 of 1,024 to 1,024 92, 85; 65,536 of 1,024 to 1,024 179,
// 207; 65,536 of 512 to 1,024 103, 107; and 262,144 of 256 to 256, where the depth
// is too short to pay for a large tile's start, 84, 75.
bool large_tiles(const Problem &p, int width)
{
    constexpr unsigned kCus = 256;
    const unsigned long long large = (p.rows / 256ull + p.heads / 2) * tiles_of(width, 256);
    const unsigned long long small = (p.rows / 128ull + p.heads / 2) * tiles_of(width, 128);
    return 8 * ((large + kCus - 1) / kCus) <= 4.6 * ((small + 2 * kCus - 1) / (2 * kCus));
}

template <class C>
hipError_t launch_shallow(const Problem &p, const Matrix<typename C::T> &w, const Matrix<typename C::T> &x,
                          const float *bias, bool relu, Rows y, int width, hipStream_t s)
{
    using T = typename C::T;
    const unsigned cols = tiles_of(width, C::TO), want = 256 * C::kAtOnce / cols;
    // stretches for `want` places, some of which the heads' last ones take
    unsigned stretch = (unsigned)p.heads < want / 2 ? p.rows / (want - p.heads) : p.rows / (want / 2);
    stretch = (stretch + 32) / 32 * 32;
    const unsigned places = p.rows / stretch + p.heads + 1;
    const unsigned groups = (places + kXcds - 1) / kXcds * kXcds * cols;
    shallow_kernel<C><<<groups, C::kThreads, 0, s>>>(p, w, x, bias, relu, static_cast<T *>(const_cast<void *>(y.p)), y.stride,
                                                     width, stretch);
    return hipGetLastError();
}

template <class T, int TO, bool DEEP_W, bool MASK, bool PAST>
hipError_t shallow(const Problem &p, const Matrix<T> &w, const Matrix<T> &x, const float *bias, bool relu, Rows y,
                   int width, hipStream_t s)
{
    const unsigned steps = tiles_of((long long)x.cols * sizeof(T), 128);
    if constexpr (DEEP_W) {
        if (steps == 3)
            return launch_shallow<Shallow<T, TO, 3, DEEP_W, MASK, PAST>>(p, w, x, bias, relu, y, width, s);
        if (steps == 4)
            return launch_shallow<Shallow<T, TO, 4, DEEP_W, MASK, PAST>>(p, w, x, bias, relu, y, width, s);
        if (steps == 5)
            return launch_shallow<Shallow<T, TO, 5, DEEP_W, MASK, PAST>>(p, w, x, bias, relu, y, width, s);
    }
    return steps == 1 ? launch_shallow<Shallow<T, TO, 1, DEEP_W, MASK, PAST>>(p, w, x, bias, relu, y, width, s)
                      : launch_shallow<Shallow<T, TO, 2, DEEP_W, MASK, PAST>>(p, w, x, bias, relu, y, width, s);
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

// The rows' product with tiles for its width.
template <class T, bool DEEP_W, bool MASK>
hipError_t rows_product(const Problem &p, const Matrix<T> &w, const Matrix<T> &x, const float *bias,
                        bool relu, Rows y, int width, int depth, hipStream_t s)
{
    if (is_shallow<T, DEEP_W>(p, w, x, width, depth)) {
        const bool past = past_caches(static_cast<const T *>(y.p), y.stride, width);
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
hipError_t launch_sums(const Problem &p, const Split &split, const float *wparts, float *dw, const float *bparts, float *db,
                       hipStream_t s)
{
    const size_t size = (size_t)p.fan_in * p.fan_out;
    const unsigned blocks = dw ? tiles_of(size, 256) : 0, wblocks = blocks < 1024 ? blocks : 1024;
    const unsigned bblocks = db ? tiles_of(p.fan_out, 256) : 0;
    sum_kernel<<<dim3(wblocks + bblocks, p.heads), 256, 0, s>>>(p, split.stretch, wparts, size, dw, bparts, db, wblocks);
    return hipGetLastError();
}

template <class C>
hipError_t launch_weights(const Problem &p, const Matrix<typename C::T> &dz,
                          const Matrix<typename C::T> &x, float *dw, float *db, char *workspace,
                          hipStream_t s)
{
    const Split split = split_rows(p.rows, p.heads, p.fan_in, p.fan_out, sizeof(typename C::T) == 2);
    const bool partial = split.stretch != 0;
    const size_t size = (size_t)p.fan_in * p.fan_out;
    float *wparts = reinterpret_cast<float *>(workspace);
    float *bparts = wparts + (size_t)split.places * size;
    float *to_w = dw ? (partial ? wparts : dw) : nullptr, *to_b = db ? (partial ? bparts : db) : nullptr;
    const unsigned row_tiles = tiles_of(p.fan_out, C::TQ), col_tiles = dw ? tiles_of(p.fan_in, C::TP) : 1;
    const hipError_t e = launch_for<C>(
        (unsigned long long)split.places * row_tiles * col_tiles, [&](unsigned groups, unsigned from) {
            weights_kernel<C><<<groups, C::kThreads, 0, s>>>(p, dz, x, to_w, to_b, split.stretch, split.places, row_tiles, col_tiles, from);
        });
    if (e != hipSuccess)
        return e;
    return partial ? launch_sums(p, split, wparts, dw, bparts, db, s) : hipSuccess;
}

// 256 x 256 tiles from 256 of them on, one a compute unit.  dW and db, us with large and
// small tiles: 2,048 to 4,096 on 32,768 rows of 8 heads (1,024 tiles) 499, 612; 1,024 to
// 1,024 on 16,384 of 8 (128) 115, 70; 512 to 512 on 65,536 of 16 (64) 111, 80; at the line
// small ones would win: 1,024 to 2,048 on 16,384 of 8 119, 101; 1,024 to 1,024 on 65,536 of
// 16 387, 271.
template <class T, bool MASK>
hipError_t weights_product(const Problem &p, const Matrix<T> &dz, const Matrix<T> &x, float *dw,
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
    return launch_weights<Product<T, 64, 64, 2, 2, false, false, MASK, false, true>>(p, dz, x, dw, db, workspace, s);
}

Problem problem(const LinearShape &sh) { return {sh.offsets, sh.rows, sh.heads, sh.fan_in, sh.fan_out}; }

template <class T>
hipError_t forward(const LinearShape &sh, Rows x, const void *w, const float *bias, bool relu,
                   Rows y, hipStream_t s)
{
    const Matrix<T> mw = {static_cast<const T *>(w), sh.fan_in, nullptr, 0, (unsigned)sh.fan_out, sh.fan_in};
    const Matrix<T> mx = {static_cast<const T *>(x.p), x.stride, nullptr, 0, sh.rows, sh.fan_in};
    return rows_product<T, true, false>(problem(sh), mw, mx, bias, relu, y, sh.fan_out, sh.fan_in, s);
}

size_t masked_bytes(unsigned rows, int fan_out) { return ((size_t)rows * fan_out * 2 + 255) / 256 * 256; }

// Whether a masked dz is laid out by a pass of its own, so that the products'
// operands go to LDS by themselves: where both read it often.  us without and
// with: 16,384 rows of 512 to 1,024 123, 103; 262,144 rows of 256 to 256 218, 234.
bool mask_apart(int fan_in, int fan_out, bool bf16)
{
    return bf16 && fan_in >= 512 && fan_out >= 512 && fan_in % 8 == 0 && fan_out % 8 == 0;
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

template <class C>
hipError_t launch_narrow(const Problem &p, const Matrix<typename C::T> &w, const Matrix<typename C::T> &dz,
                         const Matrix<typename C::T> &x, Rows dx, float *dw, float *db, char *workspace, hipStream_t s)
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

template <class T, bool MASK>
hipError_t narrow(const Problem &p, const Matrix<T> &w, const Matrix<T> &dz, const Matrix<T> &x, Rows dx, float *dw,
                  float *db, char *workspace, hipStream_t s)
{
    if (p.fan_in <= 64)
        return p.fan_out <= 64 ? launch_narrow<Narrow<T, 64, 64, MASK>>(p, w, dz, x, dx, dw, db, workspace, s)
                               : launch_narrow<Narrow<T, 64, 128, MASK>>(p, w, dz, x, dx, dw, db, workspace, s);
    return p.fan_out <= 64 ? launch_narrow<Narrow<T, 128, 64, MASK>>(p, w, dz, x, dx, dw, db, workspace, s)
                           : launch_narrow<Narrow<T, 128, 128, MASK>>(p, w, dz, x, dx, dw, db, workspace, s);
}

template <class CR, class CW>
hipError_t launch_gradients(const Problem &p, const Matrix<typename CR::T> &w, const Matrix<typename CR::T> &dz,
                            const Matrix<typename CR::T> &x, Rows dx, float *dw, float *db, hipStream_t s)
{
    using T = typename CR::T;
    const unsigned long long all =
        ((unsigned long long)p.rows / CR::TQ + p.heads + 1) * tiles_of(p.fan_in, CR::TP) +
        (unsigned long long)p.heads * tiles_of(p.fan_out, CW::TQ) * tiles_of(p.fan_in, CW::TP) + 3 * kXcds * kRun;
    if (all >= 1ull << 23)
        return hipErrorInvalidConfiguration;
    gradients_kernel<CR, CW><<<(unsigned)all, CR::kThreads, 0, s>>>(
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

template <class T>
hipError_t backward(const LinearShape &sh, Rows dy, Rows x, const void *w, Rows y, Rows dx,
                    float *dw, float *db, char *workspace, hipStream_t s)
{
    const Problem p = problem(sh);
    Matrix<T> mz = {static_cast<const T *>(dy.p), dy.stride, static_cast<const T *>(y.p), y.stride, sh.rows, sh.fan_out};
    const Matrix<T> mw = {static_cast<const T *>(w), sh.fan_in, nullptr, 0, (unsigned)sh.fan_out, sh.fan_in};
    Matrix<T> mx = {static_cast<const T *>(x.p), x.stride, nullptr, 0, sh.rows, sh.fan_in};
    if constexpr (sizeof(T) == 2)
        if (y.p && sh.rows > 0 && mask_apart(sh.fan_in, sh.fan_out, true)) {
            __bf16 *dz = reinterpret_cast<__bf16 *>(workspace);
            mask_kernel<<<sh.rows < (1u << 20) ? sh.rows : 1u << 20, 256, 0, s>>>(mz.p, mz.stride, mz.mask, mz.mask_stride,
                                                                                 sh.rows, sh.fan_out, dz);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess)
                return e;
            workspace += masked_bytes(sh.rows, sh.fan_out);
            mz = {dz, sh.fan_out, nullptr, 0, sh.rows, sh.fan_out};
        }
    if constexpr (sizeof(T) == 2)
        if (dx.p && dw && sh.rows > 0 && goes_alone(mz) && goes_alone(mw) && goes_alone(mx) && gradients_together(p))
            return launch_gradients<Product<T, 256, 256, 4, 2, false, true, false, true>,
                                    Product<T, 256, 256, 4, 2, false, false, false, true, true>>(p, mw, mz, mx, dx, dw, db, s);
    if (is_narrow(sh.fan_in, sh.fan_out) && sh.rows > 0 && (dx.p ? dw || db : dw != nullptr)) {
        if (!dw)  // nothing needs x
            mx = {mz.p, mz.stride, nullptr, 0, mz.rows, mz.cols};
        return mz.mask ? narrow<T, true>(p, mw, mz, mx, dx, dw, db, workspace, s)
                       : narrow<T, false>(p, mw, mz, mx, dx, dw, db, workspace, s);
    }
    if (dx.p && sh.rows > 0) {
        const hipError_t e =
            mz.mask ? rows_product<T, false, true>(p, mw, mz, nullptr, false, dx, sh.fan_in, sh.fan_out, s)
                    : rows_product<T, false, false>(p, mw, mz, nullptr, false, dx, sh.fan_in, sh.fan_out, s);
        if (e != hipSuccess)
            return e;
    }
    if (!dw && !db)
        return hipSuccess;
    if (!dw) {  // nothing needs x: the product's other operand is any matrix of these rows
        mx = mz;
        mx.mask = nullptr;
    }
    return mz.mask ? weights_product<T, true>(p, mz, mx, dw, db, workspace, s)
                   : weights_product<T, false>(p, mz, mx, dw, db, workspace, s);
}

}  // namespace

hipError_t launch_heads_linear(const LinearShape &sh, Rows x, const void *w, const float *bias,
                               bool relu, bool bf16, Rows y, hipStream_t s)
{
    return bf16 ? forward<__bf16>(sh, x, w, bias, relu, y, s) : forward<float>(sh, x, w, bias, relu, y, s);
}

size_t heads_linear_workspace_bytes(unsigned rows, int heads, int fan_in, int fan_out, bool relu, bool bf16)
{
    const Split split = split_rows(rows, heads, fan_in, fan_out, bf16), narrow = narrow_split(rows, heads, fan_in, fan_out, bf16);
    size_t places = split.stretch ? split.places : 0;
    if (is_narrow(fan_in, fan_out) && narrow.places > places)
        places = narrow.places;
    return (relu && mask_apart(fan_in, fan_out, bf16) ? masked_bytes(rows, fan_out) : 0) +
           places * fan_out * ((size_t)fan_in + 1) * sizeof(float);
}

hipError_t launch_heads_linear_backward(const LinearShape &sh, Rows dy, Rows x, const void *w,
                                        Rows y, bool bf16, Rows dx, float *dw, float *db,
                                        void *workspace, hipStream_t s)
{
    char *ws = static_cast<char *>(workspace);
    return bf16 ? backward<__bf16>(sh, dy, x, w, y, dx, dw, db, ws, s)
                : backward<float>(sh, dy, x, w, y, dx, dw, db, ws, s);
}

}  // namespace derf
