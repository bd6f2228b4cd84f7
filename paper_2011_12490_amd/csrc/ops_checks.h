// Argument checks that the entry points of the training operators share.
#pragma once
#include "ops_internal.h"

namespace derf {

namespace {

#define TRY(expr)                  \
    do {                           \
        const int rc_ = (expr);    \
        if (rc_ != DERF_OK)        \
            return rc_;            \
    } while (0)

constexpr int kMaxHeads = 256;
constexpr int kMaxDim = 65536;
constexpr long long kMaxRows = 1LL << 31;

int launched(hipError_t e, const char *what)
{
    return e == hipSuccess ? DERF_OK : report(DERF_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool is_precision(int p) { return p == DERF_PREC_FP32 || p == DERF_PREC_BF16; }

bool pairs_valid(long long tokens, int top_k)
{
    return tokens >= 0 && top_k >= 1 && top_k <= DERF_MAX_TOP_K && tokens < kMaxRows / top_k;
}

bool misaligned(const void *p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// A row array: there, aligned to its type, and rows that do not overlap.
int check_rows(const char *name, const void *p, long long stride, int dim, int precision)
{
    if (!p)
        return report(DERF_ERR_INVALID_ARG, "null %s", name);
    if (misaligned(p, precision == DERF_PREC_BF16 ? 2 : 4))
        return report(DERF_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    if (stride < dim || stride >= (1LL << 40))
        return report(DERF_ERR_INVALID_ARG, "%s: stride %lld for rows of %d", name, stride, dim);
    return DERF_OK;
}

// The rows of a linear layer: a tile of them is read at 32-bit offsets.
constexpr long long kMaxLayerStride = 1LL << 21;
int check_layer_rows(const char *name, const void *p, long long stride, int dim, int precision)
{
    if (stride >= kMaxLayerStride)
        return report(DERF_ERR_INVALID_ARG, "%s: stride %lld, a layer takes less than 2^21", name, stride);
    return check_rows(name, p, stride, dim, precision);
}

int check_array(const char *name, const void *p, unsigned align)
{
    if (!p)
        return report(DERF_ERR_INVALID_ARG, "null %s", name);
    if (misaligned(p, align))
        return report(DERF_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    return DERF_OK;
}

int check_pairs(long long tokens, int top_k, int dim, int precision)
{
    if (!pairs_valid(tokens, top_k))
        return report(DERF_ERR_INVALID_ARG,
                      "need num_tokens >= 0, 1 <= top_k <= %d, num_tokens * top_k < 2^31",
                      DERF_MAX_TOP_K);
    if (dim < 1 || dim > kMaxDim)
        return report(DERF_ERR_INVALID_ARG, "need 1 <= dim <= %d", kMaxDim);
    if (!is_precision(precision))
        return report(DERF_ERR_INVALID_ARG, "unknown precision %d", precision);
    return DERF_OK;
}

bool linear_sizes_valid(long long rows, int heads, int fan_in, int fan_out)
{
    return rows >= 0 && rows < kMaxRows && heads >= 1 && heads <= kMaxHeads && fan_in >= 1 &&
           fan_in <= kMaxDim && fan_out >= 1 && fan_out <= kMaxDim;
}

int check_linear(long long rows, int heads, int fan_in, int fan_out, int precision)
{
    if (!linear_sizes_valid(rows, heads, fan_in, fan_out))
        return report(DERF_ERR_INVALID_ARG,
                      "need 0 <= num_rows < 2^31, 1 <= num_heads <= %d, fan_in and fan_out in [1, %d]",
                      kMaxHeads, kMaxDim);
    if (!is_precision(precision))
        return report(DERF_ERR_INVALID_ARG, "unknown precision %d", precision);
    return DERF_OK;
}

int check_workspace(const void *p, long long have, long long need)
{
    if (have < need)
        return report(DERF_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", have, need);
    if (need > 0 && (!p || misaligned(p, 16)))
        return report(DERF_ERR_INVALID_ARG, "workspace is null or not 16-byte aligned");
    return DERF_OK;
}

// Makes a device the current one, and the one before again at its end.
struct OnDevice {
    int device, before = -1;
    hipError_t status;
    explicit OnDevice(int device_) : device(device_)
    {
        status = hipGetDevice(&before);
        if (status == hipSuccess && before != device)
            status = hipSetDevice(device);
    }
    ~OnDevice()
    {
        if (before >= 0 && before != device)
            (void)hipSetDevice(before);
    }
};

}  // namespace

}  // namespace derf
