// The gradients of the heads' gated layers.  With the gates g and ups u that the
// layer kept, dz = [dg; du]:
//
//   dg = dy u act'(g),   du = dy act(g)
//
// and the rest is the gradient of a linear layer of 2 fan_out outputs without an
// activation: dx = W^T dz, dW = dz^T x, db = sum dz.  One pass over the rows makes dz
// in the rows' type for the products, and sums db from its float32 values.  In bf16 that
// rounding, half a step, is as large as the results' own: dx and dW are 2.3e-3 of their norm
// off, 1.7e-3 without it.  A second plane with dz's rest would make two products of each one,
// and the products bound the wide layers (52 % of the matrix units' cycles, at their power).
#include "layers.h"

namespace derf {

namespace {

// dg = dy u act'(g) and du = dy act(g) of a piece of a row; the activation is chosen once
// for all of it, so that its elements' instructions interleave.
template <class T>
struct Grads {
    static constexpr int V = Type<T>::kVec;
    float g[V], u[V];
};
template <class T>
__device__ __forceinline__ Grads<T> gradients_of(u32x4 dy, u32x4 gate, u32x4 up, int act)
{
    constexpr int V = Type<T>::kVec;
    union Piece {
        u32x4 v;
        T e[V];
    };
    const Piece y = {dy}, g = {gate}, u = {up};
    Grads<T> d;
    if (act == DERF_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float x = (float)g.e[k];
            d.g[k] = (float)y.e[k] * (float)u.e[k] * (x > 0.0f ? 1.0f : 0.0f);
            d.u[k] = (float)y.e[k] * (x < 0.0f ? 0.0f : x);
        }
    } else if (act == DERF_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float bell;
            const float x = (float)g.e[k], part = below(x, bell);
            d.g[k] = (float)y.e[k] * (float)u.e[k] * (part + x * 0.39894228f * bell);
            d.u[k] = (float)y.e[k] * (x * part);
        }
    } else if (act == DERF_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float x = (float)g.e[k], part = logistic(x), both = (float)y.e[k] * part;
            d.g[k] = both * (float)u.e[k] * (1.0f + x * (1.0f - part));  // x (1 - part): 2^-24 |x| off, beside 1
            d.u[k] = both * x;
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float e = exp_of(-(float)g.e[k]);
            const float part = __builtin_amdgcn_rcpf(1.0f + e);
            const float rest = e < 1e30f ? e * part : 1.0f;  // 1 - part, without its cancellation
            d.g[k] = (float)y.e[k] * (float)u.e[k] * (part * rest);
            d.u[k] = (float)y.e[k] * part;
        }
    }
    return d;
}
// V values rounded.
template <class T>
__device__ __forceinline__ u32x4 rounded(const float (&v)[Type<T>::kVec])
{
    union {
        u32x4 v;
        T e[Type<T>::kVec];
    } piece;
#pragma unroll
    for (int k = 0; k < Type<T>::kVec; ++k)
        piece.e[k] = (T)v[k];
    return piece.v;
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
// for two written: 16,384 rows of 4,096 bf16 values, 671 MB, in 132 us (5.1 TB/s).
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
            const u32x4 y = read_piece(dy + (r * dys + c), left), g = read_piece(pre + (r * pres + c), left);
            const Grads<T> d = gradients_of<T>(y, g, read_piece(pre + (r * pres + O + c), left), act);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                dg_sum[k] += d.g[k];
                du_sum[k] += d.u[k];
            }
            if (dz) {
                write_piece(dz + (r * dzs + c), rounded<T>(d.g), left, T{});
                write_piece(dz + (r * dzs + O + c), rounded<T>(d.u), left, T{});
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

// ---- narrow layers, all gradients in one pass over the rows --------------------------

// Layers of at most 128 to 2 x 128 (float: where one of both is at most 64, whose weights
// fit): as narrow_kernel, a workgroup a compute unit keeps its head's weights in LDS and its
// part of dW in registers and goes through a stretch of the head's rows, RT at a time, the
// next ones' loads under way.  dz is made on the way from the registers to LDS, where both
// products read it: dx by rows, dW by columns.  128 to 128 in bf16 on 131,072 rows 59 us with
// the parts' sums (102 by dz in memory), 63 to 128 in float32 on 98,301 rows 91 (161).  Bound by
// LDS, a third of the time, and waits between its barriers: the 168 MB would take 36 us.
template <class T_, int TI_, int TO_>
struct GatedNarrow {
    using T = T_;
    static constexpr int TI = TI_, TO = TO_, kThreads = 512, V = Type<T>::kVec;
    static constexpr bool kBoth = sizeof(T) == 2;
    using X = Tile<T, TI, false, kThreads, false, false, kBoth>;
    using Z = Tile<T, TO, false, kThreads, false, false, kBoth>;  // dg, and du
    static constexpr int RT = X::D, kSpan = RT / 2;               // rows of a step, a fragment's depth
    static_assert(Z::D == RT, "a tile of rows a step");
    static constexpr int FP = TI / 32, FQ = 2 * TO / 64;  // dW: 2 waves over fan_in, 4 over gates and ups
    static constexpr int kRowGroups = RT / 16, kColGroups = 8 / kRowGroups, FX = TI / 16 / kColGroups;  // dx
    static constexpr int kWeights = 2 * TO / RT;  // tiles of RT outputs
    static constexpr int kZ = 0, kX = kZ + 2 * Z::kBytes, kW = kX + X::kBytes, kOut = kW + kWeights * X::kBytes;
    static constexpr int kRowsOfThreads = kThreads / Z::kPerRow;
    static constexpr int kSums = kRowsOfThreads * (2 * TO + 1) * 4;
    static constexpr int kAll = kOut + (sizeof(T) == 2 ? 8 * 16 * kPieceRow<T, FX * 16> : 0), kLds = kAll > kSums ? kAll : kSums;
};

template <class C>
__global__ __launch_bounds__(C::kThreads, 2) void gated_narrow_kernel(Problem p, Matrix<typename C::T> w, Matrix<typename C::T> dy,
                                                                      Matrix<typename C::T> pre, int act, Matrix<typename C::T> x,
                                                                      typename C::T *dx, long long dxs, float *dw, float *db,
                                                                      unsigned stretch)
{
    using T = typename C::T;
    using X = typename C::X;
    using Z = typename C::Z;
    constexpr int V = C::V;
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
    typename X::Source xs = {x, 0};
    typename Z::Source ys = {dy, 0}, gs = {pre, 0}, us = {pre, 0};
    us.m.p += O;
    xs.m.p += t.first * x.stride;
    ys.m.p += t.first * dy.stride;
    gs.m.p += t.first * pre.stride;
    us.m.p += t.first * pre.stride;
    gs.m.cols = us.m.cols = O;
    xs.m.rows = ys.m.rows = gs.m.rows = us.m.rows = t.last - t.first;
    typename X::S sx;
    typename Z::S sy, sg, su;
    auto load = [&](unsigned k) {
        Z::load(sg, gs, k);
        Z::load(su, us, k);
        Z::load(sy, ys, k);
        X::load(sx, xs, k);
    };
    if (dx) {
#pragma unroll
        for (int i = 0; i < C::kWeights; ++i) {
            typename X::S sw;
            const int half = i * C::RT / C::TO, k = i * C::RT % C::TO;
            typename X::Source ws = {w, 0};
            ws.m.p += t.head * ((size_t)2 * I * O) + (size_t)half * I * O;
            ws.m.rows = O;
            X::load(sw, ws, k);
            X::settle(sw, ws, k);
            X::store(sw, lds + C::kW + i * X::kBytes);
        }
    }
    load(0);
    float g_sums[V], u_sums[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        g_sums[k] = u_sums[k] = 0.0f;
    f32x4 acc[C::FP][C::FQ] = {};
    const int fp = wave % 2 * C::FP, fq = wave / 2 * C::FQ;  // of dW; results fq on are of the ups from TO / 16 on
    const int fr = wave / C::kColGroups, fc = wave % C::kColGroups * C::FX;  // of dx
    char *mine = lds + C::kOut + wave * 16 * kPieceRow<T, C::FX * 16>;
    constexpr int kOfHalf = C::TO / 16;
    const char *const z_of_dw = lds + C::kZ + (fq >= kOfHalf ? Z::kBytes : 0);
    const int fz = fq >= kOfHalf ? fq - kOfHalf : fq;
#pragma unroll 1
    for (unsigned k = 0; k < t.last - t.first; k += C::RT) {
        stored();
        Z::settle(sg, gs, k);
        Z::settle(su, us, k);
        Z::settle(sy, ys, k);
        X::settle(sx, xs, k);
        X::store(sx, lds + C::kX);
#pragma unroll
        for (int j = 0; j < Z::kShare; ++j) {
            const Grads<T> d = gradients_of<T>(sy.x[j], sg.x[j], su.x[j], act);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                g_sums[e] += d.g[e];
                u_sums[e] += d.u[e];
            }
            *reinterpret_cast<u32x4 *>(lds + C::kZ + (threadIdx.x + j * C::kThreads) * 16) = rounded<T>(d.g);
            *reinterpret_cast<u32x4 *>(lds + C::kZ + Z::kBytes + (threadIdx.x + j * C::kThreads) * 16) = rounded<T>(d.u);
        }
        stored();
        if (k + C::RT < t.last - t.first)
            load(k + C::RT);
        if (dx) {
            f32x4 rows[C::FX] = {};
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int part = 0; part < C::TO / C::kSpan; ++part) {
                    const u32x4 q = Z::row_fragment(lds + C::kZ + half * Z::kBytes, fr, part);
#pragma unroll
                    for (int i = 0; i < C::FX; ++i)
                        rows[i] = multiply(X::fragment(lds + C::kW + (half * C::TO + part * C::kSpan) / C::RT * X::kBytes, fc + i, part & 1),
                                           q, rows[i], T{});
                }
            write_16_rows<T, C::FX * 16>(rows, mine, t.first + k + fr * 16, t.last, fc * 16, I, dx, dxs);
        }
        if (dw)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                u32x4 q[C::FQ];
#pragma unroll
                for (int j = 0; j < C::FQ; ++j)
                    q[j] = Z::fragment(z_of_dw, fz + j, part);
#pragma unroll
                for (int i = 0; i < C::FP; ++i) {
                    const u32x4 f = X::fragment(lds + C::kX, fp + i, part);
#pragma unroll
                    for (int j = 0; j < C::FQ; ++j)
                        acc[i][j] = multiply(f, q[j], acc[i][j], T{});
                }
            }
    }
    if (dw) {
        float *to = dw + (size_t)place * 2 * O * I + (fq >= kOfHalf ? (size_t)O * I : 0);
#pragma unroll
        for (int j = 0; j < C::FQ; ++j) {
            const int m = (fz + j) * 16 + (lane & 15);
#pragma unroll
            for (int i = 0; i < C::FP; ++i) {
                const int n = (fp + i) * 16 + (lane >> 4) * 4;
                if (m < O && n < I)
                    write_piece(to + ((size_t)m * I + n), __builtin_bit_cast(u32x4, acc[i][j]), I - n, 0.0f);
            }
        }
    }
    if (db) {
        float(*part)[2 * C::TO + 1] = reinterpret_cast<float(*)[2 * C::TO + 1]>(lds);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) {
            part[Z::my_row()][Z::my_col() + e] = g_sums[e];
            part[Z::my_row()][C::TO + Z::my_col() + e] = u_sums[e];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * C::TO; i += C::kThreads) {
            float v = 0.0f;
            for (int r = 0; r < C::kRowsOfThreads; ++r)
                v += part[r][i];
            const int half = i / C::TO, o = i % C::TO;
            if (o < O)
                db[((size_t)place * 2 + half) * O + o] = v;
        }
    }
}

template <class T, int TI, int TO>
hipError_t gated_narrow(const Problem &p, const Matrix<T> &w, const Matrix<T> &dy, const Matrix<T> &pre, int act,
                        const Matrix<T> &x, Rows dx, T *dw, float *db, char *workspace, hipStream_t s)
{
    using C = GatedNarrow<T, TI, TO>;
    const Split split = narrow_split(p.rows, p.heads, p.fan_in, p.fan_out, true);
    float *wparts = reinterpret_cast<float *>(workspace);
    float *bparts = wparts + (size_t)split.places * 2 * p.fan_out * p.fan_in;
    gated_narrow_kernel<C><<<split.places + 1, C::kThreads, 0, s>>>(p, w, dy, pre, act, x, static_cast<T *>(const_cast<void *>(dx.p)),
                                                                    dx.stride, dw ? wparts : nullptr, db ? bparts : nullptr, split.stretch);
    const hipError_t e = hipGetLastError();
    const Problem both = {p.offsets, p.rows, p.heads, p.fan_in, 2 * p.fan_out};
    return e != hipSuccess || (!dw && !db) ? e : launch_sums(both, split, wparts, dw, bparts, db, s);
}

bool is_gated_narrow(int fan_in, int fan_out, bool bf16)
{
    return fan_in <= 128 && fan_out <= 128 && (bf16 || fan_in <= 64 || fan_out <= 64);
}
size_t gated_narrow_bytes(unsigned rows, int heads, int fan_in, int fan_out)
{
    return (size_t)narrow_split(rows, heads, fan_in, fan_out, true).places * 2 * fan_out * ((size_t)fan_in + 1) * sizeof(float);
}

// ---- launches --------------------------------------------------------------------------

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
    const Matrix<T> mw = {static_cast<const T *>(w), sh.fan_in, nullptr, 0, (unsigned)p.fan_out, sh.fan_in};
    Matrix<T> mx = {static_cast<const T *>(x.p), x.stride, nullptr, 0, sh.rows, sh.fan_in};
    if (rows && is_gated_narrow(sh.fan_in, sh.fan_out, bf16)) {
        const Problem one = {sh.offsets, sh.rows, sh.heads, sh.fan_in, sh.fan_out};
        const Matrix<T> my = {static_cast<const T *>(dy.p), dy.stride, nullptr, 0, sh.rows, sh.fan_out};
        const Matrix<T> mp = {static_cast<const T *>(pre.p), pre.stride, nullptr, 0, sh.rows, sh.fan_out};
        if (!dw)  // nothing needs x
            mx = {my.p, my.stride, nullptr, 0, my.rows, my.cols < mx.cols ? my.cols : mx.cols};
        if (sh.fan_in <= 64)
            return sh.fan_out <= 64 ? gated_narrow<T, 64, 64>(one, mw, my, mp, act, mx, dx, dw, db, workspace, s)
                                    : gated_narrow<T, 64, 128>(one, mw, my, mp, act, mx, dx, dw, db, workspace, s);
        if (sh.fan_out <= 64)
            return gated_narrow<T, 128, 64>(one, mw, my, mp, act, mx, dx, dw, db, workspace, s);
        if constexpr (bf16)
            return gated_narrow<T, 128, 128>(one, mw, my, mp, act, mx, dx, dw, db, workspace, s);
    }
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
    if constexpr (bf16)
        if (rows && dx.p && dw && goes_alone(mz) && goes_alone(mw) && goes_alone(mx) && gradients_together(p))
            return launch_gradients<Product<T, 256, 256, 4, 2, false, true, false, true>,
                                    Product<T, 256, 256, 4, 2, false, false, false, true, true>>(p, mw, mz, mx, dx, dw,
                                                                                               (float *)nullptr, s);
    // float32: 256 to 256 on 65,536 rows 394 us: dz 61, dx 178, dW 204 (each product alone 114)
    if (rows && dx.p)
        e = rows_product<T, false, false, false>(p, mw, mz, nullptr, false, dx, sh.fan_in, p.fan_out, s);
    if (e != hipSuccess || !dw)
        return e;
    // without rows narrow layers come here too: what is theirs is zeros
    if (!rows)
        return launch_sums(p, Split{256, (unsigned)sh.heads}, (const float *)nullptr, dw, nullptr, nullptr, s);
    return weights_product<T, false, T, !bf16>(p, mz, mx, dw, (float *)nullptr, workspace, s);
}

}  // namespace

size_t heads_gated_workspace_bytes(unsigned rows, int heads, int fan_in, int fan_out, bool bf16)
{
    if (rows > 0 && is_gated_narrow(fan_in, fan_out, bf16))
        return gated_narrow_bytes(rows, heads, fan_in, fan_out);
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
