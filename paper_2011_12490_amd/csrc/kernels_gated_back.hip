// The gradients of the heads' gated layers.  With the gates g and ups u that the
// layer kept, dz = [dg; du]:
//
//   dg = dy u act'(g),   du = dy act(g)
//
// and the rest is the gradient of a linear layer of 2 fan_out outputs without an
// activation: dx = W^T dz, dW = dz^T x, db = sum dz.  One pass over the rows makes dz
// in the rows' type for the products, and sums db from its float32 values.
#include "layers.h"

namespace derf {

namespace {

// act(g) and its slope.
template <class T>
__device__ __forceinline__ void act_and_slope(float g, int act, float &value, float &slope)
{
    if (act == DERF_ACT_RELU) {
        value = g < 0.0f ? 0.0f : g;
        slope = g > 0.0f ? 1.0f : 0.0f;
    } else if (act == DERF_ACT_GELU) {
        const float part = below(g);
        value = g * part;
        slope = part + g * 0.39894228f * exp_of(-0.5f * g * g, T{});
    } else {
        const float e = exp_of(-g, T{});
        const float part = sizeof(T) == 2 ? __builtin_amdgcn_rcpf(1.0f + e) : 1.0f / (1.0f + e);
        const float rest = e < 1e30f ? e * part : 1.0f;  // 1 - part, without its cancellation
        value = act == DERF_ACT_SILU ? g * part : part;
        slope = act == DERF_ACT_SILU ? part * (1.0f + g * rest) : part * rest;
    }
}

// V elements from a row's column on, `left` of which are the row's.
template <class T>
__device__ __forceinline__ u32x4 read_piece(const T *from, int left)
{
    constexpr int V = Type<T>::kVec;
    if (left >= V)
        return reinterpret_cast<const Bytes16 *>(from)->v;
    union {
        u32x4 v;
        T e[V];
    } piece = {};
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (k < left)
            piece.e[k] = from[k];
    return piece.v;
}

// dz [rows][2 O] and the sums of its columns over a stretch of a head's rows, at the
// stretch's place in parts.  2^log_lanes lanes side by side take 16 bytes of a row each,
// a workgroup 256 >> log_lanes rows at a time.  Bound by its bytes: three pieces read
// for two written.
template <class T>
__global__ __launch_bounds__(256) void gate_gradient_kernel(Problem p, const T *dy, long long dys, const T *pre, long long pres,
                                                            int act, T *dz, long long dzs, float *parts, unsigned stretch,
                                                            int log_lanes)
{
    constexpr int V = Type<T>::kVec;
    __shared__ unsigned before[kMaxHeads + 1];
    __shared__ float sums[256][2 * V + 1];
    const int O = p.fan_out;
    count_tiles(p, stretch, before);
    if (blockIdx.x >= uniform(before[p.heads]))
        return;
    const RowTile t = head_tile(p, before, blockIdx.x, stretch);
    const unsigned lanes = 1u << log_lanes, rows = 256 >> log_lanes;
    const int c = (int)(blockIdx.y * lanes + threadIdx.x % lanes) * V, left = O - c;
    float dg_sum[V] = {}, du_sum[V] = {};
    if (left > 0)
#pragma unroll 2
        for (unsigned r = t.first + threadIdx.x / lanes; r < t.last; r += rows) {
            union Piece {
                u32x4 v;
                T e[V];
            };
            const Piece y = {read_piece(dy + (r * dys + c), left)};
            const Piece g = {read_piece(pre + (r * pres + c), left)};
            const Piece u = {read_piece(pre + (r * pres + O + c), left)};
            Piece dg, du;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float value, slope;
                act_and_slope<T>((float)g.e[k], act, value, slope);
                const float a = (float)y.e[k] * (float)u.e[k] * slope, b = (float)y.e[k] * value;
                dg_sum[k] += a;
                du_sum[k] += b;
                dg.e[k] = (T)a;
                du.e[k] = (T)b;
            }
            if (dz) {
                write_piece(dz + (r * dzs + c), dg.v, left, T{});
                write_piece(dz + (r * dzs + O + c), du.v, left, T{});
            }
        }
    if (!parts)
        return;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        sums[threadIdx.x][k] = dg_sum[k];
        sums[threadIdx.x][V + k] = du_sum[k];
    }
    __syncthreads();
    for (unsigned i = threadIdx.x; i < lanes * 2 * V; i += 256) {
        const unsigned half = i / (lanes * V), e = i % (lanes * V);
        float x = 0.0f;
        for (unsigned r = 0; r < rows; ++r)
            x += sums[r * lanes + e / V][half * V + e % V];
        const int n = (int)(blockIdx.y * lanes * V + e);
        if (n < O)
            parts[((size_t)blockIdx.x * 2 + half) * O + n] = x;
    }
}

// Stretches of the pass over the rows: about 2,048 workgroups.
struct Stretches {
    int log_lanes;
    unsigned chunks, stretch, places;
};
Stretches stretches(unsigned rows, int heads, int fan_out, bool bf16)
{
    const int V = bf16 ? 8 : 4;
    Stretches s = {0, 0, 0, 0};
    while (s.log_lanes < 5 && V << s.log_lanes < fan_out)
        ++s.log_lanes;
    s.chunks = tiles_of(fan_out, V << s.log_lanes);
    const unsigned want = s.chunks < 1024 ? 2048 / s.chunks : 2, each = 256u >> s.log_lanes;
    s.stretch = (rows / want / each + 1) * each;
    if (s.stretch < 2 * each)
        s.stretch = 2 * each;
    s.places = rows / s.stretch + heads;
    return s;
}

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }
long long dz_stride(int fan_out) { return (2LL * fan_out + 7) / 8 * 8; }
size_t dz_bytes(unsigned rows, int fan_out, bool bf16) { return whole((size_t)rows * dz_stride(fan_out) * (bf16 ? 2 : 4)); }
size_t sums_bytes(unsigned rows, int heads, int fan_out, bool bf16)
{
    return whole((size_t)stretches(rows, heads, fan_out, bf16).places * 2 * fan_out * sizeof(float));
}

template <class T>
hipError_t gated_backward(const LinearShape &sh, Rows dy, Rows pre, Rows x, const void *w, int act, Rows dx, T *dw, float *db,
                          char *workspace, hipStream_t s)
{
    constexpr bool bf16 = sizeof(T) == 2;
    const Problem p = {sh.offsets, sh.rows, sh.heads, sh.fan_in, 2 * sh.fan_out};
    const bool rows = sh.rows > 0;
    float *parts = reinterpret_cast<float *>(workspace);
    workspace += sums_bytes(sh.rows, sh.heads, sh.fan_out, bf16);
    T *dz = dx.p || dw ? reinterpret_cast<T *>(workspace) : nullptr;
    workspace += dz_bytes(sh.rows, sh.fan_out, bf16);
    hipError_t e = hipSuccess;
    const Stretches st = stretches(sh.rows, sh.heads, sh.fan_out, bf16);
    if (rows && (dz || db)) {
        const Problem half = {sh.offsets, sh.rows, sh.heads, sh.fan_in, sh.fan_out};
        gate_gradient_kernel<T><<<dim3(st.places, st.chunks), 256, 0, s>>>(
            half, static_cast<const T *>(dy.p), dy.stride, static_cast<const T *>(pre.p), pre.stride, act, dz,
            dz_stride(sh.fan_out), db ? parts : nullptr, st.stretch, st.log_lanes);
        e = hipGetLastError();
    }
    if (e == hipSuccess && db)
        e = launch_sums<float>(p, {st.stretch, st.places}, nullptr, nullptr, parts, db, s);
    if (e != hipSuccess || !dz)
        return e;
    const Matrix<T> mz = {dz, dz_stride(sh.fan_out), nullptr, 0, sh.rows, p.fan_out};
    const Matrix<T> mw = {static_cast<const T *>(w), sh.fan_in, nullptr, 0, (unsigned)p.fan_out, sh.fan_in};
    const Matrix<T> mx = {static_cast<const T *>(x.p), x.stride, nullptr, 0, sh.rows, sh.fan_in};
    if constexpr (bf16)
        if (rows && dx.p && dw && goes_alone(mz) && goes_alone(mw) && goes_alone(mx) && gradients_together(p))
            return launch_gradients<Product<T, 256, 256, 4, 2, false, true, false, true>,
                                    Product<T, 256, 256, 4, 2, false, false, false, true, true>>(p, mw, mz, mx, dx, dw,
                                                                                               (float *)nullptr, s);
    if (rows && dw && is_narrow(p.fan_in, p.fan_out))
        return narrow<T, false>(p, mw, mz, mx, dx, dw, nullptr, workspace, s);
    if (rows && dx.p)
        e = rows_product<T, false, false>(p, mw, mz, nullptr, false, dx, sh.fan_in, p.fan_out, s);
    if (e != hipSuccess || !dw)
        return e;
    return weights_product<T, false>(p, mz, mx, dw, (float *)nullptr, workspace, s);
}

}  // namespace

size_t heads_gated_workspace_bytes(unsigned rows, int heads, int fan_in, int fan_out, bool bf16)
{
    return sums_bytes(rows, heads, fan_out, bf16) + dz_bytes(rows, fan_out, bf16) +
           parts_bytes(rows, heads, fan_in, 2 * fan_out, bf16);
}

hipError_t launch_heads_gated_backward(const LinearShape &sh, Rows dy, Rows pre, Rows x, const void *w, int act, bool bf16,
                                       Rows dx, void *dw, float *db, void *workspace, hipStream_t s)
{
    char *ws = static_cast<char *>(workspace);
    return bf16 ? gated_backward<__bf16>(sh, dy, pre, x, w, act, dx, static_cast<__bf16 *>(dw), db, ws, s)
                : gated_backward<float>(sh, dy, pre, x, w, act, dx, static_cast<float *>(dw), db, ws, s);
}

}  // namespace derf
