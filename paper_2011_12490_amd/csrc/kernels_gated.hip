// The heads' gated layers: y[r][o] = act(g) u with the gates and ups
//
//   g = sum_i x[r][i] Wg[o][i] + bg[o],   u = sum_i x[r][i] Wu[o][i] + bu[o]
//
// The layer of kernels_linear.hip with both weights in one matrix of 2 fan_out rows:
// a tile takes 16 rows of Wg and the 16 of Wu that belong to them in turn, so a lane
// holds a gate and its up in the same place of two results, and the activation and the
// product are taken on the way out of the registers.  x is read once for both.
#include "layers.h"

namespace derf {

namespace {

// The forms of a layer of 2 fan_out outputs (rows_product), with tiles of pairs.
template <class T>
hipError_t gated(const LinearShape &sh, Rows x, const void *w, const float *bias, int act, Rows y, Rows pre, hipStream_t s)
{
    const Problem p = {sh.offsets, sh.rows, sh.heads, sh.fan_in, sh.fan_out};
    const int O = sh.fan_out, depth = sh.fan_in;
    const Matrix<T> mw = {static_cast<const T *>(w), depth, nullptr, 0, 2 * (unsigned)O, depth};
    const Matrix<T> mx = {static_cast<const T *>(x.p), x.stride, nullptr, 0, sh.rows, depth};
    if (is_shallow<T, true>(p, mw, mx, 2 * O, depth)) {
        if (O <= 32)
            return shallow<T, 64, true, false, false, true>(p, mw, mx, bias, act, y, O, s, pre);
        return shallow<T, 128, true, false, false, true>(p, mw, mx, bias, act, y, O, s, pre);
    }
    if (few_rows<T>(p, 2 * O, depth))
        return launch_rows<Product<T, 64, 32, 2, 1, true, true, false, false, false, 4, true>>(p, mw, mx, bias, act, y, O, depth,
                                                                                            s, pre);
    const bool alone = goes_alone(mw) && goes_alone(mx);
    if constexpr (sizeof(T) == 2) {
        // large tiles as in large_tiles, and from a depth of 256 to 512 only where they leave little
        // of their last round empty (their gain there is less); in both sizes a wave has 64
        // columns, whole lines.  us, rows of bf16 with gates and ups kept, 256 and 128: 256 to 256
        // on 262,139 130, 136, on 131,072 76, 69; 320 to 512 on 65,536 80, 77 (64 heads 91, 81), on
        // 131,072 148, 150; 384 to 384 131, 126; 448 to 640 on 65,536 122, 116; 512 to 512 103, 99;
        // 768 to 768 188, 194; 1,024 to 1,024 on 32,768 152, 155; 2,048 to 2,048 on 16,384 256, 281;
        // 2,048 to 4,096 on 32,768 1,003, 1,224.  262,139 rows of 256 to 256 move 537 MB: 4.1 TB/s (197
        // us past weights in LDS), the four steps of a tile's loads waiting for its results'
        // stores; wide ones are bound by the matrix units' power (1,096 TFLOP/s)
        if (alone && depth >= 256 && large_tiles(p, 2 * O, depth < 512 ? 4.25 : 4.6))
            return launch_rows<Product<T, 256, 256, 2, 4, true, true, false, true, false, 1, true>>(p, mw, mx, bias, act, y, O,
                                                                                                 depth, s, pre);
        if (alone && wide_tile<T>(2 * O))
            return launch_rows<Product<T, 128, 128, 1, 4, true, true, false, true, false, 1, true>>(p, mw, mx, bias, act, y, O,
                                                                                                 depth, s, pre);
    }
    if (wide_tile<T>(2 * O)) {
        // float32, all kept: 256 to 256 on 65,536 rows 164 us (its products alone 114), 1,024 to
        // 1,024 on 32,768 1,058 (910): matrix units, 65 % busy
        if constexpr (sizeof(T) == 4)
            if (alone)
                return launch_rows<Product<T, 128, 128, 2, 2, true, true, false, true, false, 1, true>>(p, mw, mx, bias, act, y,
                                                                                                     O, depth, s, pre);
        return launch_rows<Product<T, 128, 128, 2, 2, true, true, false, false, false, 1, true>>(p, mw, mx, bias, act, y, O,
                                                                                              depth, s, pre);
    }
    return launch_rows<Product<T, 64, 128, 2, 2, true, true, false, false, false, 1, true>>(p, mw, mx, bias, act, y, O, depth, s,
                                                                                         pre);
}

}  // namespace

hipError_t launch_heads_gated(const LinearShape &sh, Rows x, const void *w, const float *bias, int act, bool bf16, Rows y,
                              Rows pre, hipStream_t s)
{
    return bf16 ? gated<__bf16>(sh, x, w, bias, act, y, pre, s) : gated<float>(sh, x, w, bias, act, y, pre, s);
}

}  // namespace derf
