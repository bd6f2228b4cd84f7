// The heads' linear layers and their gradients: products of matrices whose
// rows come in groups, one group a head, with bounds known on the device only.
//
//   layer      y[r][o]  = act(sum_i x[r][i] W[o][i] + b[o])
//   rows       dx[r][i] = sum_o dz[r][o] W[o][i]
//   weights    dW[o][i] = sum_r dz[r][o] x[r][i],  db[o] = sum_r dz[r][o]
//
// One tile product serves all three (tile_product in product.h): "deep" operands
// have their depth side by side (x, dz, and W for a layer), the others their tile's
// rows (W for the rows' gradient; dz and x for the weights').  The kernels are in
// layers.h.
#include "layers.h"

namespace derf {

namespace {

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
    return (relu && mask_apart(fan_in, fan_out, bf16) ? masked_bytes(rows, fan_out) : 0) +
           parts_bytes(rows, heads, fan_in, fan_out, bf16);
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
