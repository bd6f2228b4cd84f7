// The heads' linear layers and their gradients: products of matrices whose
// rows come in groups, one group a head, with bounds known on the device only.
#include "ops_internal.h"

namespace derf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kTile = 64;  // rows and columns of a workgroup's tile of the result

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

// The rows [first, last) of tile `tile` and their head (p.heads: rows without
// one, p.heads + 1: there is no such tile).  256 threads, all call it.
struct TileRows {
    unsigned first, last;
    int head;
};
__device__ TileRows find_tile(const Problem &p, unsigned tile, unsigned tile_rows, TileRows *found,
                              unsigned *tmp)
{
    const int h = threadIdx.x, lane = h & 63, wave = h >> 6;
    unsigned a = 0, b = 0;
    if (h < p.heads) {
        a = bound(p, h);
        b = bound(p, h + 1);
    }
    const unsigned mine = b > a ? (b - a + tile_rows - 1) / tile_rows : 0;
    unsigned incl = mine;
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned y = __shfl_up(incl, off);
        if (lane >= off)
            incl += y;
    }
    if (lane == 63)
        tmp[wave] = incl;
    __syncthreads();
    if (h == 0)
        found->head = p.heads + 1;  // until the tile's thread says otherwise, below
    __syncthreads();
    unsigned before = incl - mine, total = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave)
            before += tmp[w];
        total += tmp[w];
    }
    if (tile >= before && tile - before < mine) {
        found->first = a + (tile - before) * tile_rows;
        found->last = found->first + tile_rows < b ? found->first + tile_rows : b;
        found->head = h;
    }
    if (h == 0 && tile >= total) {
        const unsigned from = bound(p, p.heads);
        const unsigned long long at = from + (unsigned long long)(tile - total) * tile_rows;
        if (at < p.rows) {
            found->first = (unsigned)at;
            found->last = at + tile_rows < p.rows ? (unsigned)at + tile_rows : p.rows;
            found->head = p.heads;
        }
    }
    __syncthreads();
    return *found;
}

template <class T>
struct Kind;
template <>
struct Kind<__bf16> {
    static constexpr int kDepth = 32;  // of one step through LDS
    static __device__ __forceinline__ f32x4 step(const __bf16 *a, const __bf16 *b, int q, f32x4 c)
    {
        bf16x8 x, y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = a[q * 8 + i];
            y[i] = b[q * 8 + i];
        }
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    }
};
template <>
struct Kind<float> {
    static constexpr int kDepth = 16;
    static __device__ __forceinline__ f32x4 step(const float *a, const float *b, int q, f32x4 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i * 4 + q], b[i * 4 + q], c, 0, 0, 0);
        return c;
    }
};

// C[m][n] = sum_k A(m, k) B(n, k) over a 64 x 64 tile, four waves of 16 rows.
template <class T, class LoadA, class LoadB>
__device__ __forceinline__ void tile_product(unsigned depth, LoadA load_a, LoadB load_b,
                                             T (*As)[Kind<T>::kDepth + 8], T (*Bs)[Kind<T>::kDepth + 8],
                                             f32x4 (&acc)[4], float *row_sum)
{
    constexpr int kDepth = Kind<T>::kDepth;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (unsigned k0 = 0; k0 < depth; k0 += kDepth) {
        for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
            const int r = i / kDepth, k = i % kDepth;
            As[r][k] = k0 + k < depth ? load_a(r, k0 + k) : (T)0.0f;
            Bs[r][k] = k0 + k < depth ? load_b(r, k0 + k) : (T)0.0f;
        }
        __syncthreads();
        const T *a = As[wave * 16 + (lane & 15)];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc[j] = Kind<T>::step(a, Bs[j * 16 + (lane & 15)], lane >> 4, acc[j]);
        if (row_sum && threadIdx.x < kTile)
            for (int k = 0; k < kDepth; ++k)
                *row_sum += (float)As[threadIdx.x][k];
        __syncthreads();
    }
}

// y = act(x W^T + b) (BACK = false), or dx = dz W (BACK = true).
template <class T, bool BACK>
__global__ __launch_bounds__(kThreads) void rows_kernel(Problem p, const T *x, long long xs,
                                                        const T *w, const float *bias, bool relu,
                                                        const T *mask, long long ms, T *y,
                                                        long long ys)
{
    __shared__ T As[kTile][Kind<T>::kDepth + 8], Bs[kTile][Kind<T>::kDepth + 8];
    __shared__ TileRows found;
    __shared__ unsigned tmp[4];
    const int depth = BACK ? p.fan_out : p.fan_in, width = BACK ? p.fan_in : p.fan_out;
    const int n0 = blockIdx.y * kTile;
  for (unsigned tile = blockIdx.x;; tile += gridDim.x) {
    const TileRows t = find_tile(p, tile, kTile, &found, tmp);
    if (t.head > p.heads)
        return;
    f32x4 acc[4] = {};
    const bool headed = t.head < p.heads;
    if (headed) {
        const T *wh = w + (size_t)t.head * p.fan_out * p.fan_in;
        tile_product<T>(
            depth,
            [&](int r, int k) -> T {
                if (t.first + r >= t.last)
                    return (T)0.0f;
                if (BACK && mask && !((float)mask[(t.first + r) * ms + k] > 0.0f))
                    return (T)0.0f;
                return x[(t.first + r) * xs + k];
            },
            [&](int r, int k) -> T {
                if (n0 + r >= width)
                    return (T)0.0f;
                return BACK ? wh[(size_t)k * p.fan_in + n0 + r] : wh[(size_t)(n0 + r) * p.fan_in + k];
            },
            As, Bs, acc, nullptr);
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + j * 16 + (lane & 15);
        for (int i = 0; i < 4; ++i) {
            const unsigned r = t.first + wave * 16 + (lane >> 4) * 4 + i;
            if (r >= t.last || n >= width)
                continue;
            float v = acc[j][i];
            if (!BACK && headed) {
                if (bias)
                    v += bias[(size_t)t.head * width + n];
                if (relu)
                    v = v < 0.0f ? 0.0f : v;
            }
            y[r * ys + n] = (T)v;
        }
    }
  }
}

// dW[o][i] = sum_r dz[r][o] x[r][i] of head blockIdx.z, and db[o] = sum_r dz[r][o].
template <class T>
__global__ __launch_bounds__(kThreads) void weights_kernel(Problem p, const T *dy, long long ds,
                                                           const T *x, long long xs, const T *mask,
                                                           long long ms, float *dw, float *db)
{
    __shared__ T As[kTile][Kind<T>::kDepth + 8], Bs[kTile][Kind<T>::kDepth + 8];
    const int h = blockIdx.z, m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
    const unsigned first = bound(p, h), last = bound(p, h + 1);
    f32x4 acc[4] = {};
    float sum = 0.0f;
    tile_product<T>(
        last > first ? last - first : 0,
        [&](int m, unsigned k) -> T {
            if (m0 + m >= p.fan_out)
                return (T)0.0f;
            if (mask && !((float)mask[(first + k) * ms + m0 + m] > 0.0f))
                return (T)0.0f;
            return dy[(first + k) * ds + m0 + m];
        },
        [&](int n, unsigned k) -> T {
            return dw && n0 + n < p.fan_in ? x[(first + k) * xs + n0 + n] : (T)0.0f;
        },
        As, Bs, acc, db && n0 == 0 ? &sum : nullptr);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (dw)
        for (int j = 0; j < 4; ++j)
            for (int i = 0; i < 4; ++i) {
                const int m = m0 + wave * 16 + (lane >> 4) * 4 + i, n = n0 + j * 16 + (lane & 15);
                if (m < p.fan_out && n < p.fan_in)
                    dw[((size_t)h * p.fan_out + m) * p.fan_in + n] = acc[j][i];
            }
    if (db && n0 == 0 && threadIdx.x < kTile && m0 + (int)threadIdx.x < p.fan_out)
        db[(size_t)h * p.fan_out + m0 + threadIdx.x] = sum;
}

unsigned tiles(int n) { return (unsigned)((n + kTile - 1) / kTile); }

// Tiles of rows: each head's last one may be partly filled, and so may the last
// of the rows without a head.
unsigned row_tiles(const LinearShape &sh)
{
    const unsigned n = sh.rows / kTile + sh.heads + 1;
    return n < (1u << 20) ? n : 1u << 20;
}

template <class T>
hipError_t forward(const LinearShape &sh, Rows x, const void *w, const float *bias, bool relu,
                   Rows y, hipStream_t s)
{
    const Problem p = {sh.offsets, sh.rows, sh.heads, sh.fan_in, sh.fan_out};
    rows_kernel<T, false><<<dim3(row_tiles(sh), tiles(sh.fan_out)), kThreads, 0, s>>>(
        p, static_cast<const T *>(x.p), x.stride, static_cast<const T *>(w), bias, relu, nullptr, 0,
        static_cast<T *>(const_cast<void *>(y.p)), y.stride);
    return hipGetLastError();
}

template <class T>
hipError_t backward(const LinearShape &sh, Rows dy, Rows x, const void *w, Rows y, Rows dx,
                    float *dw, float *db, hipStream_t s)
{
    const Problem p = {sh.offsets, sh.rows, sh.heads, sh.fan_in, sh.fan_out};
    const T *dyp = static_cast<const T *>(dy.p), *yp = static_cast<const T *>(y.p);
    if (dx.p && sh.rows > 0)
        rows_kernel<T, true><<<dim3(row_tiles(sh), tiles(sh.fan_in)), kThreads, 0, s>>>(
            p, dyp, dy.stride, static_cast<const T *>(w), nullptr, false, yp, y.stride,
            static_cast<T *>(const_cast<void *>(dx.p)), dx.stride);
    if (dw || db)
        weights_kernel<T><<<dim3(dw ? tiles(sh.fan_in) : 1, tiles(sh.fan_out), sh.heads), kThreads, 0, s>>>(
            p, dyp, dy.stride, static_cast<const T *>(x.p), x.stride, yp, y.stride, dw, db);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_heads_linear(const LinearShape &sh, Rows x, const void *w, const float *bias,
                               bool relu, bool bf16, Rows y, hipStream_t s)
{
    return bf16 ? forward<__bf16>(sh, x, w, bias, relu, y, s) : forward<float>(sh, x, w, bias, relu, y, s);
}

size_t heads_linear_workspace_bytes(unsigned, int, int, int, bool) { return 0; }

hipError_t launch_heads_linear_backward(const LinearShape &sh, Rows dy, Rows x, const void *w,
                                        Rows y, bool bf16, Rows dx, float *dw, float *db,
                                        void *, hipStream_t s)
{
    return bf16 ? backward<__bf16>(sh, dy, x, w, y, dx, dw, db, s)
                : backward<float>(sh, dy, x, w, y, dx, dw, db, s);
}

}  // namespace derf
