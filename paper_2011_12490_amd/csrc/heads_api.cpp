// Host side of the heads' gated layers, table lookups and orthogonalised updates
// declared in include/derf.h: argument checks before any HIP call, then the launches.
#include "ops_checks.h"

#include <math.h>

using namespace derf;

namespace {

// A gated layer: a head's weights are read at 32-bit offsets from a row of a tile on.
bool gated_sizes_valid(long long rows, int heads, int fan_in, int fan_out, int precision)
{
    return linear_sizes_valid(rows, heads, fan_in, fan_out) && is_precision(precision) &&
           (2LL * fan_out + 256) * fan_in * (precision == DERF_PREC_BF16 ? 2 : 4) < (1LL << 31);
}

int check_gated(long long rows, int heads, int fan_in, int fan_out, int act, int precision)
{
    TRY(check_linear(rows, heads, fan_in, fan_out, precision));
    if (!gated_sizes_valid(rows, heads, fan_in, fan_out, precision))
        return report(DERF_ERR_INVALID_ARG, "a head's weights from %d to 2 x %d take 2^31 bytes or more", fan_in, fan_out);
    if (act < DERF_ACT_SILU || act > DERF_ACT_SIGMOID)
        return report(DERF_ERR_INVALID_ARG, "unknown activation %d", act);
    return DERF_OK;
}

bool lookup_sizes_valid(long long samples, long long rows, int dim)
{
    return samples >= 0 && samples < kMaxRows && rows >= 1 && rows < kMaxRows && dim >= 1 && dim <= kMaxDim;
}

int check_lookup(long long samples, long long rows, int dim, float scale, int precision)
{
    if (!lookup_sizes_valid(samples, rows, dim))
        return report(DERF_ERR_INVALID_ARG, "need 0 <= num_samples < 2^31, 1 <= num_rows < 2^31, 1 <= dim <= %d", kMaxDim);
    if (!is_precision(precision))
        return report(DERF_ERR_INVALID_ARG, "unknown precision %d", precision);
    if (!isfinite(scale))
        return report(DERF_ERR_INVALID_ARG, "scale is not finite");
    return DERF_OK;
}

}  // namespace

extern "C" {

int derf_heads_gated(const void *x, long long x_stride, const void *w, const float *bias,
                     const int *offsets, long long num_rows, int num_heads, int fan_in,
                     int fan_out, int act, int precision, void *y, long long y_stride, void *pre,
                     long long pre_stride, void *hip_stream)
{
    TRY(check_gated(num_rows, num_heads, fan_in, fan_out, act, precision));
    if (num_rows == 0)
        return DERF_OK;
    TRY(check_layer_rows("x", x, x_stride, fan_in, precision));
    TRY(check_array("w", w, precision == DERF_PREC_BF16 ? 2 : 4));
    if (bias)
        TRY(check_array("bias", bias, 4));
    TRY(check_array("offsets", offsets, 4));
    TRY(check_layer_rows("y", y, y_stride, fan_out, precision));
    if (pre)
        TRY(check_layer_rows("pre", pre, pre_stride, 2 * fan_out, precision));
    const LinearShape sh = {offsets, (unsigned)num_rows, num_heads, fan_in, fan_out};
    return launched(launch_heads_gated(sh, {x, x_stride}, w, bias, act, precision == DERF_PREC_BF16, {y, y_stride},
                                       {pre, pre_stride}, static_cast<hipStream_t>(hip_stream)),
                    "derf_heads_gated");
}

long long derf_heads_gated_workspace(long long num_rows, int num_heads, int fan_in, int fan_out,
                                     int precision)
{
    if (!gated_sizes_valid(num_rows, num_heads, fan_in, fan_out, precision))
        return -1;
    return (long long)heads_gated_workspace_bytes((unsigned)num_rows, num_heads, fan_in, fan_out,
                                                  precision == DERF_PREC_BF16);
}

int derf_heads_gated_backward(const void *dy, long long dy_stride, const void *pre,
                              long long pre_stride, const void *x, long long x_stride,
                              const void *w, const int *offsets, long long num_rows,
                              int num_heads, int fan_in, int fan_out, int act, int precision,
                              void *out_x, long long out_x_stride, void *out_w, float *out_bias,
                              void *workspace, long long workspace_bytes, void *hip_stream)
{
    TRY(check_gated(num_rows, num_heads, fan_in, fan_out, act, precision));
    const unsigned align = precision == DERF_PREC_BF16 ? 2 : 4;
    if (num_rows > 0) {
        TRY(check_layer_rows("dy", dy, dy_stride, fan_out, precision));
        TRY(check_layer_rows("pre", pre, pre_stride, 2 * fan_out, precision));
        if (out_x) {
            TRY(check_array("w", w, align));
            TRY(check_layer_rows("out_x", out_x, out_x_stride, fan_in, precision));
        }
        if (out_w)
            TRY(check_layer_rows("x", x, x_stride, fan_in, precision));
    }
    if (out_w)
        TRY(check_array("out_w", out_w, align));
    if (out_bias)
        TRY(check_array("out_bias", out_bias, 4));
    TRY(check_array("offsets", offsets, 4));
    TRY(check_workspace(workspace, workspace_bytes,
                        derf_heads_gated_workspace(num_rows, num_heads, fan_in, fan_out, precision)));
    const LinearShape sh = {offsets, (unsigned)num_rows, num_heads, fan_in, fan_out};
    return launched(launch_heads_gated_backward(sh, {dy, dy_stride}, {pre, pre_stride}, {x, x_stride}, w, act,
                                                precision == DERF_PREC_BF16, {out_x, out_x_stride}, out_w, out_bias,
                                                workspace, static_cast<hipStream_t>(hip_stream)),
                    "derf_heads_gated_backward");
}

int derf_lookup(const void *table, long long table_stride, const int *ids, long long num_samples,
                long long num_rows, int dim, float scale, int precision, void *out,
                long long out_stride, void *hip_stream)
{
    TRY(check_lookup(num_samples, num_rows, dim, scale, precision));
    if (num_samples == 0)
        return DERF_OK;
    TRY(check_rows("table", table, table_stride, dim, precision));
    TRY(check_array("ids", ids, 4));
    TRY(check_rows("out", out, out_stride, dim, precision));
    return launched(launch_lookup({table, table_stride}, ids, num_samples, num_rows, dim, scale, precision == DERF_PREC_BF16,
                                  {out, out_stride}, static_cast<hipStream_t>(hip_stream)),
                    "derf_lookup");
}

long long derf_lookup_workspace(long long num_samples, long long num_rows, int dim)
{
    if (!lookup_sizes_valid(num_samples, num_rows, dim))
        return -1;
    return (long long)lookup_workspace_bytes((unsigned)num_samples, (unsigned)num_rows, dim);
}

int derf_lookup_backward(const void *dout, long long dout_stride, const int *ids,
                         long long num_samples, long long num_rows, int dim, float scale,
                         int precision, float *out, void *workspace, long long workspace_bytes,
                         void *hip_stream)
{
    TRY(check_lookup(num_samples, num_rows, dim, scale, precision));
    if (num_samples > 0) {
        TRY(check_rows("dout", dout, dout_stride, dim, precision));
        TRY(check_array("ids", ids, 4));
    }
    TRY(check_array("out", out, 4));
    TRY(check_workspace(workspace, workspace_bytes, derf_lookup_workspace(num_samples, num_rows, dim)));
    return launched(launch_lookup_backward({dout, dout_stride}, ids, (unsigned)num_samples, (unsigned)num_rows, dim, scale,
                                           precision == DERF_PREC_BF16, out, workspace, static_cast<hipStream_t>(hip_stream)),
                    "derf_lookup_backward");
}

}  // extern "C"
