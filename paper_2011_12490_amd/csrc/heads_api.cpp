// Host side of the heads' gated layers, table lookups and orthogonalised updates
// declared in include/derf.h: argument checks before any HIP call, then the launches.
#include "ops_checks.h"

#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

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

constexpr long long kMaxMatrices = 32768;
constexpr int kMaxSide = 16384;
constexpr int kMaxIterations = 20;
constexpr size_t kMostWorkspace = 8ull << 30;  // of an optimizer, but for a matrix that needs more

bool matrices_valid(long long matrices, int fan_out, int fan_in)
{
    return matrices >= 0 && matrices <= kMaxMatrices && fan_out >= 1 && fan_out <= kMaxSide && fan_in >= 1 && fan_in <= kMaxSide;
}

// Whether a matrix's products take 22 bits: float32's, and those of few rows (or columns).  Of
// few singular values the roundings of 11 bits do not average out: of 20,000 matrices of bf16 normal
// values the worst was off, rounding included, by 1.9e-2 of its norm (2 x 2), 1.4e-2 (4 x 4), 8.1e-3
// (6 x 6), 6.2e-3 (8 x 8; 3.2e-3 root mean square), where a rounding alone is 3.9e-3 at most.  200
// such matrices take 14 us, with 11 bits 10.
bool exact_products(int fan_out, int fan_in, bool bf16) { return !bf16 || std::min(fan_out, fan_in) < 8; }

// Matrices of a table that go together: of one padded shape and exactness.
struct MuonGroup {
    unsigned first, count;
    int fan_out, fan_in;
    bool split;
};

int padded_side(int n) { return (n + 63) / 64 * 64; }

// An array of a tensor, in bytes.
struct Span {
    uintptr_t from, to;
    bool written;
    int tensor;
};
void add_span(std::vector<Span> &spans, const void *p, long long bytes, bool written, int tensor)
{
    if (p && bytes > 0)
        spans.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes, written, tensor});
}
// A tensor with an array that is written and shares memory with another array, or -1.
int overlapping(std::vector<Span> &spans)
{
    std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.from < b.from; });
    uintptr_t any = 0, written = 0;  // the furthest ends so far
    for (const Span &s : spans) {
        if (s.from < (s.written ? any : written))
            return s.tensor;
        any = std::max(any, s.to);
        if (s.written)
            written = std::max(written, s.to);
    }
    return -1;
}

}  // namespace

struct derf_muon {
    MuonEntry *table = nullptr;  // device memory, as the workspace
    void *workspace = nullptr;
    int device = -1;
    std::vector<MuonGroup> groups;
};

namespace {

void free_muon(derf_muon *opt)
{
    if (opt->table)
        (void)device_free(opt->table);
    if (opt->workspace)
        (void)device_free(opt->workspace);
    delete opt;
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
    TRY(check_apart({rows_area("y", y, num_rows, y_stride, fan_out, precision),
                     rows_area("pre", pre, num_rows, pre_stride, 2 * fan_out, precision)},
                    {rows_area("x", x, num_rows, x_stride, fan_in, precision),
                     rows_area("w", w, num_heads * 2LL * fan_out, fan_in, fan_in, precision),
                     array_area("bias", bias, num_heads * 8LL * fan_out), array_area("offsets", offsets, (num_heads + 1) * 4LL)}));
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
    const long long need = derf_heads_gated_workspace(num_rows, num_heads, fan_in, fan_out, precision);
    TRY(check_workspace(workspace, workspace_bytes, need));
    const long long weights = num_heads * 2LL * fan_out;
    TRY(check_apart({rows_area("out_x", out_x, num_rows, out_x_stride, fan_in, precision),
                     rows_area("out_w", out_w, weights, fan_in, fan_in, precision), array_area("out_bias", out_bias, weights * 4),
                     array_area("workspace", workspace, need)},
                    {rows_area("dy", dy, num_rows, dy_stride, fan_out, precision),
                     rows_area("pre", pre, num_rows, pre_stride, 2 * fan_out, precision),
                     rows_area("x", out_w ? x : nullptr, num_rows, x_stride, fan_in, precision),
                     rows_area("w", out_x ? w : nullptr, weights, fan_in, fan_in, precision),
                     array_area("offsets", offsets, (num_heads + 1) * 4LL)}));
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
    TRY(check_apart({rows_area("out", out, num_samples, out_stride, dim, precision)},
                    {rows_area("table", table, num_rows, table_stride, dim, precision), array_area("ids", ids, num_samples * 4)}));
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
    const long long need = derf_lookup_workspace(num_samples, num_rows, dim);
    TRY(check_workspace(workspace, workspace_bytes, need));
    TRY(check_apart({rows_area("out", out, num_rows, dim, dim, DERF_PREC_FP32), array_area("workspace", workspace, need)},
                    {rows_area("dout", dout, num_samples, dout_stride, dim, precision), array_area("ids", ids, num_samples * 4)}));
    return launched(launch_lookup_backward({dout, dout_stride}, ids, (unsigned)num_samples, (unsigned)num_rows, dim, scale,
                                           precision == DERF_PREC_BF16, out, workspace, static_cast<hipStream_t>(hip_stream)),
                    "derf_lookup_backward");
}

long long derf_orthogonalise_workspace(long long num_matrices, int fan_out, int fan_in,
                                       int precision)
{
    if (!matrices_valid(num_matrices, fan_out, fan_in) || !is_precision(precision))
        return -1;
    return (long long)muon_workspace_bytes(fan_out, fan_in, exact_products(fan_out, fan_in, precision == DERF_PREC_BF16),
                                           (unsigned)num_matrices);
}

int derf_orthogonalise(const void *x, long long num_matrices, int fan_out, int fan_in,
                       int iterations, int precision, void *out, void *workspace,
                       long long workspace_bytes, void *hip_stream)
{
    if (!matrices_valid(num_matrices, fan_out, fan_in))
        return report(DERF_ERR_INVALID_ARG, "need 0 <= num_matrices <= %lld, fan_out and fan_in in [1, %d]", kMaxMatrices, kMaxSide);
    if (!is_precision(precision))
        return report(DERF_ERR_INVALID_ARG, "unknown precision %d", precision);
    if (iterations < 1 || iterations > kMaxIterations)
        return report(DERF_ERR_INVALID_ARG, "iterations is %d, not in [1, %d]", iterations, kMaxIterations);
    if (num_matrices == 0)
        return DERF_OK;
    const bool bf16 = precision == DERF_PREC_BF16;
    TRY(check_array("x", x, bf16 ? 2 : 4));
    TRY(check_array("out", out, bf16 ? 2 : 4));
    const long long need = derf_orthogonalise_workspace(num_matrices, fan_out, fan_in, precision);
    TRY(check_workspace(workspace, workspace_bytes, need));
    // x itself is read before any of it is written
    const Area from = rows_area("x", x, num_matrices * fan_out, fan_in, fan_in, precision);
    TRY(check_apart({rows_area("out", out, num_matrices * fan_out, fan_in, fan_in, precision), array_area("workspace", workspace, need)},
                    {x == out ? Area{} : from}));
    const MuonSet set = {nullptr, 0, {out, x, nullptr, nullptr, fan_out, fan_in, bf16, bf16, 1.0f}};
    const MuonStep st = {0.0f, 1.0f, 0.0f, 0, 0, 0, iterations, nullptr};
    return launched(launch_muon(set, (unsigned)num_matrices, fan_out, fan_in, exact_products(fan_out, fan_in, bf16), st, workspace,
                                static_cast<hipStream_t>(hip_stream)),
                    "derf_orthogonalise");
}

int derf_muon_create(derf_muon **out, const derf_muon_tensor *tensors, int num_tensors)
{
    if (!out)
        return report(DERF_ERR_INVALID_ARG, "null out");
    *out = nullptr;
    if (num_tensors < 0 || num_tensors > 65536 || (num_tensors > 0 && !tensors))
        return report(DERF_ERR_INVALID_ARG, "need 0 <= num_tensors <= 65536 and their array");
    derf_muon *opt = nullptr;
    try {
        std::vector<MuonEntry> table;
        std::vector<Span> spans;
        long long matrices = 0;
        for (int i = 0; i < num_tensors; ++i) {
            const derf_muon_tensor &t = tensors[i];
            if (!matrices_valid(t.num_matrices, t.fan_out, t.fan_in) || (matrices += t.num_matrices) > kMaxMatrices)
                return report(DERF_ERR_INVALID_ARG, "tensor %d: %d matrices of %d x %d", i, t.num_matrices, t.fan_out, t.fan_in);
            if (!is_precision(t.param_precision) || !is_precision(t.grad_precision))
                return report(DERF_ERR_INVALID_ARG, "tensor %d: unknown precision", i);
            const unsigned pa = t.param_precision == DERF_PREC_BF16 ? 2 : 4, ga = t.grad_precision == DERF_PREC_BF16 ? 2 : 4;
            if (t.num_matrices > 0 && (!t.param || !t.grad || !t.m))
                return report(DERF_ERR_INVALID_ARG, "tensor %d: a null array", i);
            if (misaligned(t.param, pa) || misaligned(t.grad, ga) || misaligned(t.m, 4) || misaligned(t.copy, 2))
                return report(DERF_ERR_INVALID_ARG, "tensor %d: an array is not aligned to its elements", i);
            const long long size = (long long)t.fan_out * t.fan_in;
            const long long all = size * t.num_matrices;
            add_span(spans, t.param, all * pa, true, i);
            add_span(spans, t.m, all * 4, true, i);
            add_span(spans, t.copy, all * 2, true, i);
            add_span(spans, t.grad, all * ga, false, i);
            for (int k = 0; k < t.num_matrices; ++k)
                table.push_back({static_cast<char *>(t.param) + k * size * pa, static_cast<const char *>(t.grad) + k * size * ga,
                                 t.m + k * size, t.copy ? static_cast<char *>(t.copy) + k * size * 2 : nullptr, t.fan_out, t.fan_in,
                                 t.param_precision == DERF_PREC_BF16, t.grad_precision == DERF_PREC_BF16,
                                 (float)sqrt(std::max(1.0, (double)t.fan_out / t.fan_in))});
        }
        const int twice = overlapping(spans);
        if (twice >= 0)
            return report(DERF_ERR_INVALID_ARG, "tensor %d: an array shares memory with another", twice);
        auto small = [](const MuonEntry &e) { return e.fan_out <= 128 && e.fan_in <= 128; };
        // Few small matrices run at once, in places of the largest: 128 of 128 x 128 and 16 of
        // 128 x 63 take 58 us (91 where the 16 went alone, in places of 64 x 128, and 68 this
        // way, with eight waves a matrix).
        struct {
            int count, m, n;
        } places[2] = {};  // of 11 bits, of 22
        auto exact = [](const MuonEntry &e) { return exact_products(e.fan_out, e.fan_in, e.param_bf16); };
        for (const MuonEntry &e : table)
            if (small(e)) {
                const int o = padded_side(e.fan_out), i = padded_side(e.fan_in);
                auto &p = places[exact(e)];
                p = {p.count + 1, std::max(p.m, std::min(o, i)), std::max(p.n, std::max(o, i))};
            }
        auto key = [&](const MuonEntry &e) {
            const int o = padded_side(e.fan_out), i = padded_side(e.fan_in);
            const auto &p = places[exact(e)];
            const bool as_largest = small(e) && p.count <= 256;
            const long long m = as_largest ? p.m : std::min(o, i), n = as_largest ? p.n : std::max(o, i);
            return (m << 32 | n << 1) + (exact(e) ? 1 : 0);
        };
        std::stable_sort(table.begin(), table.end(), [&](const MuonEntry &a, const MuonEntry &b) { return key(a) < key(b); });
        opt = new derf_muon;
        size_t workspace = 0;
        for (size_t i = 0; i < table.size();) {
            const long long shape = key(table[i]) >> 1;  // padded sides
            MuonGroup g = {(unsigned)i, 1, (int)(shape >> 31), (int)(shape & 0x7FFFFFFF), exact(table[i])};
            while (i + g.count < table.size() && key(table[i + g.count]) == key(table[i]) &&
                   muon_workspace_bytes(g.fan_out, g.fan_in, g.split, g.count + 1) <= kMostWorkspace)
                ++g.count;
            workspace = std::max(workspace, muon_workspace_bytes(g.fan_out, g.fan_in, g.split, g.count));
            opt->groups.push_back(g);
            i += g.count;
        }
        hipError_t e = hipSuccess;
        if (!table.empty()) {
            const size_t bytes = table.size() * sizeof(MuonEntry);
            e = hipGetDevice(&opt->device);
            if (e == hipSuccess)
                e = device_alloc(reinterpret_cast<void **>(&opt->table), bytes);
            if (e == hipSuccess && workspace > 0)
                e = device_alloc(&opt->workspace, workspace);
            if (e == hipSuccess)
                e = hipMemcpy(opt->table, table.data(), bytes, hipMemcpyHostToDevice);
        }
        if (e != hipSuccess) {
            (void)hipGetLastError();
            free_muon(opt);
            if (e == hipErrorOutOfMemory)
                return report(DERF_ERR_OOM, "optimizer workspace of %zu bytes", workspace);
            return report(DERF_ERR_HIP, "derf_muon_create: %s", hipGetErrorString(e));
        }
        *out = opt;
        return DERF_OK;
    } catch (const std::bad_alloc &) {
        delete opt;  // nothing on the device yet
        return report(DERF_ERR_OOM, "host memory");
    }
}

int derf_muon_step(derf_muon *opt, double lr, double momentum, int nesterov, double weight_decay,
                   int iterations, const float *grad_scale, void *hip_stream)
{
    if (!opt)
        return report(DERF_ERR_INVALID_ARG, "null optimizer");
    if (!(lr >= 0) || !isfinite(lr) || !(momentum >= 0 && momentum < 1) || !(weight_decay >= 0) || !isfinite(weight_decay))
        return report(DERF_ERR_INVALID_ARG, "need finite lr, weight_decay >= 0 and momentum in [0, 1)");
    if (iterations < 1 || iterations > kMaxIterations)
        return report(DERF_ERR_INVALID_ARG, "iterations is %d, not in [1, %d]", iterations, kMaxIterations);
    if (misaligned(grad_scale, 4))
        return report(DERF_ERR_INVALID_ARG, "grad_scale is not aligned to its elements");
    if (opt->groups.empty())
        return DERF_OK;
    const OnDevice on(opt->device);
    if (on.status != hipSuccess)
        return launched(on.status, "the optimizer's device");
    // the rate goes into the launches, which a graph would repeat as it is
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(static_cast<hipStream_t>(hip_stream), &capture) != hipSuccess)
        (void)hipGetLastError();
    else if (capture != hipStreamCaptureStatusNone)
        return report(DERF_ERR_INVALID_ARG, "the stream is being captured: a graph would repeat this step's rate");
    const MuonStep st = {(float)momentum, (float)(1.0 - lr * weight_decay), (float)lr, 1, nesterov != 0, 1, iterations, grad_scale};
    for (const MuonGroup &g : opt->groups) {
        const MuonSet set = {opt->table, g.first, {}};
        TRY(launched(launch_muon(set, g.count, g.fan_out, g.fan_in, g.split, st, opt->workspace,
                                 static_cast<hipStream_t>(hip_stream)),
                     "derf_muon_step"));
    }
    return DERF_OK;
}

void derf_muon_destroy(derf_muon *opt)
{
    if (!opt)
        return;
    if (opt->device >= 0) {
        const OnDevice on(opt->device);
        (void)hipDeviceSynchronize();
        free_muon(opt);
    } else {
        delete opt;
    }
}

}  // extern "C"
