// Host side of the training operators declared in include/derf.h: argument
// checks before any HIP call, then the launches.
#include "ops_checks.h"

#include <math.h>

#include <new>
#include <vector>

using namespace derf;

struct derf_adamw {
    AdamWEntry *table = nullptr;  // device memory
    int device = -1;              // of the table
    int tensors = 0;
    int state_bits = 32;
    unsigned items = 0;
};

extern "C" {

long long derf_route_workspace(long long num_tokens, int top_k, int num_heads)
{
    if (!pairs_valid(num_tokens, top_k) || num_heads < 1 || num_heads > kMaxHeads)
        return -1;
    return (long long)route_workspace_bytes((unsigned)(num_tokens * top_k), num_heads);
}

int derf_route(const int *heads, long long num_tokens, int top_k, int num_heads, int *out_offsets,
               int *out_pair, int *out_row, void *workspace, long long workspace_bytes,
               void *hip_stream)
{
    TRY(check_pairs(num_tokens, top_k, 1, DERF_PREC_FP32));
    if (num_heads < 1 || num_heads > kMaxHeads)
        return report(DERF_ERR_INVALID_ARG, "need 1 <= num_heads <= %d", kMaxHeads);
    TRY(check_array("out_offsets", out_offsets, 4));
    if (num_tokens > 0) {
        TRY(check_array("heads", heads, 4));
        TRY(check_array("out_pair", out_pair, 4));
        TRY(check_array("out_row", out_row, 4));
    }
    TRY(check_workspace(workspace, workspace_bytes,
                        derf_route_workspace(num_tokens, top_k, num_heads)));
    return launched(launch_route(heads, (unsigned)(num_tokens * top_k), num_heads, out_offsets,
                                 out_pair, out_row, static_cast<unsigned *>(workspace),
                                 static_cast<hipStream_t>(hip_stream)),
                    "derf_route");
}

int derf_dispatch(const void *x, long long x_stride, const int *row, long long num_tokens,
                  int top_k, int dim, int precision, void *out, long long out_stride,
                  void *hip_stream)
{
    TRY(check_pairs(num_tokens, top_k, dim, precision));
    if (num_tokens == 0)
        return DERF_OK;
    TRY(check_rows("x", x, x_stride, dim, precision));
    TRY(check_array("row", row, 4));
    TRY(check_rows("out", out, out_stride, dim, precision));
    return launched(launch_dispatch({x, x_stride}, row, num_tokens, top_k, dim,
                                    precision == DERF_PREC_BF16, {out, out_stride},
                                    static_cast<hipStream_t>(hip_stream)),
                    "derf_dispatch");
}

int derf_combine(const void *rows, long long rows_stride, const float *weights, const int *row,
                 long long num_tokens, int top_k, int dim, int precision, void *out,
                 long long out_stride, void *hip_stream)
{
    TRY(check_pairs(num_tokens, top_k, dim, precision));
    if (num_tokens == 0)
        return DERF_OK;
    TRY(check_rows("rows", rows, rows_stride, dim, precision));
    if (weights)
        TRY(check_array("weights", weights, 4));
    TRY(check_array("row", row, 4));
    TRY(check_rows("out", out, out_stride, dim, precision));
    return launched(launch_combine({rows, rows_stride}, weights, row, num_tokens, top_k, dim,
                                   precision == DERF_PREC_BF16, {out, out_stride},
                                   static_cast<hipStream_t>(hip_stream)),
                    "derf_combine");
}

int derf_combine_backward(const void *dout, long long dout_stride, const void *rows,
                          long long rows_stride, const float *weights, const int *row,
                          long long num_tokens, int top_k, int dim, int precision,
                          void *out_rows, long long out_rows_stride, float *out_weights,
                          void *hip_stream)
{
    TRY(check_pairs(num_tokens, top_k, dim, precision));
    if (num_tokens == 0)
        return DERF_OK;
    TRY(check_rows("dout", dout, dout_stride, dim, precision));
    if (out_weights) {
        TRY(check_array("out_weights", out_weights, 4));
        TRY(check_rows("rows", rows, rows_stride, dim, precision));
    }
    if (weights)
        TRY(check_array("weights", weights, 4));
    TRY(check_array("row", row, 4));
    TRY(check_rows("out_rows", out_rows, out_rows_stride, dim, precision));
    return launched(launch_combine_backward({dout, dout_stride}, {rows, rows_stride}, weights, row,
                                            num_tokens, top_k, dim, precision == DERF_PREC_BF16,
                                            {out_rows, out_rows_stride}, out_weights,
                                            static_cast<hipStream_t>(hip_stream)),
                    "derf_combine_backward");
}

int derf_heads_linear(const void *x, long long x_stride, const void *w, const float *bias,
                      const int *offsets, long long num_rows, int num_heads, int fan_in,
                      int fan_out, int relu, int precision, void *y, long long y_stride,
                      void *hip_stream)
{
    TRY(check_linear(num_rows, num_heads, fan_in, fan_out, precision));
    if (num_rows == 0)
        return DERF_OK;
    TRY(check_layer_rows("x", x, x_stride, fan_in, precision));
    TRY(check_array("w", w, precision == DERF_PREC_BF16 ? 2 : 4));
    if (bias)
        TRY(check_array("bias", bias, 4));
    TRY(check_array("offsets", offsets, 4));
    TRY(check_layer_rows("y", y, y_stride, fan_out, precision));
    const LinearShape sh = {offsets, (unsigned)num_rows, num_heads, fan_in, fan_out};
    return launched(launch_heads_linear(sh, {x, x_stride}, w, bias, relu != 0,
                                        precision == DERF_PREC_BF16, {y, y_stride},
                                        static_cast<hipStream_t>(hip_stream)),
                    "derf_heads_linear");
}

long long derf_heads_linear_workspace(long long num_rows, int num_heads, int fan_in, int fan_out,
                                      int relu, int precision)
{
    if (!linear_sizes_valid(num_rows, num_heads, fan_in, fan_out) || !is_precision(precision))
        return -1;
    return (long long)heads_linear_workspace_bytes((unsigned)num_rows, num_heads, fan_in, fan_out,
                                                   relu != 0, precision == DERF_PREC_BF16);
}

int derf_heads_linear_backward(const void *dy, long long dy_stride, const void *x,
                               long long x_stride, const void *w, const void *y,
                               long long y_stride, const int *offsets, long long num_rows,
                               int num_heads, int fan_in, int fan_out, int precision, void *out_x,
                               long long out_x_stride, float *out_w, float *out_bias,
                               void *workspace, long long workspace_bytes, void *hip_stream)
{
    TRY(check_linear(num_rows, num_heads, fan_in, fan_out, precision));
    if (num_rows > 0) {
        TRY(check_layer_rows("dy", dy, dy_stride, fan_out, precision));
        if (y)
            TRY(check_layer_rows("y", y, y_stride, fan_out, precision));
        if (out_x) {
            TRY(check_array("w", w, precision == DERF_PREC_BF16 ? 2 : 4));
            TRY(check_layer_rows("out_x", out_x, out_x_stride, fan_in, precision));
        }
        if (out_w)
            TRY(check_layer_rows("x", x, x_stride, fan_in, precision));
    }
    if (out_w)
        TRY(check_array("out_w", out_w, 4));
    if (out_bias)
        TRY(check_array("out_bias", out_bias, 4));
    TRY(check_array("offsets", offsets, 4));
    TRY(check_workspace(workspace, workspace_bytes,
                        derf_heads_linear_workspace(num_rows, num_heads, fan_in, fan_out,
                                                    y != nullptr, precision)));
    const LinearShape sh = {offsets, (unsigned)num_rows, num_heads, fan_in, fan_out};
    return launched(launch_heads_linear_backward(sh, {dy, dy_stride}, {x, x_stride}, w,
                                                 {y, y_stride}, precision == DERF_PREC_BF16,
                                                 {out_x, out_x_stride}, out_w, out_bias, workspace,
                                                 static_cast<hipStream_t>(hip_stream)),
                    "derf_heads_linear_backward");
}

int derf_adamw_create(derf_adamw **out, const derf_adamw_tensor *tensors, int num_tensors,
                      int state_bits)
{
    if (!out)
        return report(DERF_ERR_INVALID_ARG, "null out");
    *out = nullptr;
    if (num_tensors < 0 || num_tensors > 65536 || (num_tensors > 0 && !tensors))
        return report(DERF_ERR_INVALID_ARG, "need 0 <= num_tensors <= 65536 and their array");
    if (state_bits != 8 && state_bits != 32)
        return report(DERF_ERR_INVALID_ARG, "state_bits is %d, not 8 or 32", state_bits);
    try {
        std::vector<AdamWEntry> table;
        table.reserve(num_tensors);
        long long values = 0;
        unsigned long long items = 0;
        for (int i = 0; i < num_tensors; ++i) {
            const derf_adamw_tensor &t = tensors[i];
            if (t.n < 0 || t.n >= (1LL << 40) || (values += t.n) >= (1LL << 40))
                return report(DERF_ERR_INVALID_ARG, "tensor %d: %lld values", i, t.n);
            if (!is_precision(t.param_precision) || !is_precision(t.grad_precision))
                return report(DERF_ERR_INVALID_ARG, "tensor %d: unknown precision", i);
            if (t.n == 0)
                continue;
            const unsigned pa = t.param_precision == DERF_PREC_BF16 ? 2 : 4;
            const unsigned ga = t.grad_precision == DERF_PREC_BF16 ? 2 : 4;
            const unsigned ma = state_bits == 32 ? 4 : 1;
            if (!t.param || !t.grad || !t.m || !t.v)
                return report(DERF_ERR_INVALID_ARG, "tensor %d: a null array", i);
            if (state_bits == 8 && (!t.m_scale || !t.v_scale))
                return report(DERF_ERR_INVALID_ARG, "tensor %d: null scales", i);
            if (misaligned(t.param, pa) || misaligned(t.grad, ga) || misaligned(t.m, ma) ||
                misaligned(t.v, ma) || misaligned(t.copy, 2) ||
                (state_bits == 8 && (misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4))))
                return report(DERF_ERR_INVALID_ARG, "tensor %d: an array is not aligned to its elements", i);
            AdamWEntry e;
            e.t = t;
            e.first = (unsigned)items;
            // four values at a time
            e.aligned = !misaligned(t.param, 4 * pa) && !misaligned(t.grad, 4 * ga) &&
                        !misaligned(t.m, 4 * ma) && !misaligned(t.v, 4 * ma) && !misaligned(t.copy, 8);
            table.push_back(e);
            items += adamw_items(t.n);
            if (items >= (1ull << 31))
                return report(DERF_ERR_INVALID_ARG, "too many values");
        }
        derf_adamw *opt = new derf_adamw;
        opt->tensors = (int)table.size();
        opt->state_bits = state_bits;
        opt->items = (unsigned)items;
        if (!table.empty()) {
            const size_t bytes = table.size() * sizeof(AdamWEntry);
            hipError_t e = hipGetDevice(&opt->device);
            if (e != hipSuccess) {
                delete opt;
                return report(DERF_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
            }
            e = device_alloc(reinterpret_cast<void **>(&opt->table), bytes);
            if (e != hipSuccess) {
                (void)hipGetLastError();
                delete opt;
                if (e == hipErrorOutOfMemory)
                    return report(DERF_ERR_OOM, "optimizer table of %zu bytes", bytes);
                return report(DERF_ERR_HIP, "hipMalloc: %s", hipGetErrorString(e));
            }
            e = hipMemcpy(opt->table, table.data(), bytes, hipMemcpyHostToDevice);
            if (e != hipSuccess) {
                (void)device_free(opt->table);
                delete opt;
                return report(DERF_ERR_HIP, "hipMemcpy: %s", hipGetErrorString(e));
            }
        }
        *out = opt;
        return DERF_OK;
    } catch (const std::bad_alloc &) {
        return report(DERF_ERR_OOM, "host memory");
    }
}

int derf_adamw_step(derf_adamw *opt, double lr, double beta1, double beta2, double eps,
                    double weight_decay, long long step, const float *grad_scale,
                    void *hip_stream)
{
    if (!opt)
        return report(DERF_ERR_INVALID_ARG, "null optimizer");
    if (!(lr >= 0) || !isfinite(lr) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) ||
        !(eps >= 0) || !isfinite(eps) || !(weight_decay >= 0) || !isfinite(weight_decay))
        return report(DERF_ERR_INVALID_ARG, "need finite lr, eps, weight_decay >= 0 and betas in [0, 1)");
    if (step < 1)
        return report(DERF_ERR_INVALID_ARG, "step %lld: the first is 1", step);
    if (grad_scale && misaligned(grad_scale, 4))
        return report(DERF_ERR_INVALID_ARG, "grad_scale is not aligned to its elements");
    if (opt->items == 0)
        return DERF_OK;
    const OnDevice on(opt->device);
    if (on.status != hipSuccess)
        return launched(on.status, "the optimizer's device");
    // Step number and rates go into the launch, which a graph would repeat as it is.  Where
    // the runtime does not tell (another stream's capture), the launch says what is wrong.
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(static_cast<hipStream_t>(hip_stream), &capture) != hipSuccess)
        (void)hipGetLastError();
    else if (capture != hipStreamCaptureStatusNone)
        return report(DERF_ERR_INVALID_ARG, "the stream is being captured: a graph would repeat step %lld", step);
    AdamWScalars c;
    c.decay = (float)(1.0 - lr * weight_decay);
    c.beta1 = (float)beta1;
    c.one_minus_beta1 = (float)(1.0 - beta1);
    c.beta2 = (float)beta2;
    c.one_minus_beta2 = (float)(1.0 - beta2);
    c.rate = (float)(lr / (1.0 - pow(beta1, (double)step)));
    c.root_scale = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
    c.eps = (float)eps;
    return launched(launch_adamw(opt->table, opt->tensors, opt->items, opt->state_bits, c,
                                 grad_scale, static_cast<hipStream_t>(hip_stream)),
                    "derf_adamw_step");
}

void derf_adamw_destroy(derf_adamw *opt)
{
    if (!opt)
        return;
    if (opt->table) {
        const OnDevice on(opt->device);
        (void)hipDeviceSynchronize();
        (void)device_free(opt->table);
    }
    delete opt;
}

}  // extern "C"
