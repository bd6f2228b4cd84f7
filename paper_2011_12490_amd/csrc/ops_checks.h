// Argument checks that the entry points of the training operators share.
#pragma once
#include "ops_internal.h"

#include <algorithm>
#include <initializer_list>

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

typedef __int128 Wide;

// Rows of an array in memory, in bytes; p null or no rows: none.
struct Area {
    const char *name = "";
    const void *p = nullptr;
    long long rows = 0, row = 0, stride = 0;
    uintptr_t from = 0, to = 0;  // of all

    Area() = default;
    Area(const char *name_, const void *p_, long long rows_, long long row_, long long stride_)
        : name(name_), p(p_), rows(row_ > 0 ? rows_ : 0), row(row_), stride(rows > 1 ? stride_ : row_)
    {
        if (!p || rows <= 0)
            return;
        from = reinterpret_cast<uintptr_t>(p);
        const Wide end = from + (Wide)(rows - 1) * stride + row;
        to = end < (Wide)UINTPTR_MAX ? (uintptr_t)end : UINTPTR_MAX;
    }
};
Area rows_area(const char *name, const void *p, long long rows, long long stride, long long dim, int precision)
{
    const int bytes = precision == DERF_PREC_BF16 ? 2 : 4;
    return {name, p, rows, dim * bytes, stride * bytes};
}
Area array_area(const char *name, const void *p, long long bytes) { return {name, p, 1, bytes, bytes}; }

// The sum of floor((a i + b) / m) over i in [0, n), a, b >= 0: whole parts taken out, what is
// left counted along the other axis, as Euclid's algorithm goes.
Wide floor_sum(Wide n, Wide m, Wide a, Wide b)
{
    Wide sum = 0;
    while (n > 0) {
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const Wide top = a * n + b;
        n = top / m;
        b = top % m;
        std::swap(a, m);
    }
    return sum;
}

// Whether a byte is in a row of both.  Row i of one begins at x = i sa - d behind the other's
// first, and has bytes of its rows j with x - lb < j sb < x + la: floor((x + la - 1) / sb) -
// floor((x - lb) / sb) of them, all of which, or their neighbours, are there while x is within
// (-la, (nb - 1) sb + lb).
bool share_memory(const Area &one, const Area &other)
{
    if (one.from >= other.to || other.from >= one.to)  // as most are; or one is none
        return false;
    const Wide la = one.row, lb = other.row, na = one.rows, nb = other.rows, sa = one.stride, sb = other.stride;
    const Wide d = (Wide)other.from - (Wide)one.from, end_b = (nb - 1) * sb + lb;
    const Wide from = d < la ? 0 : (d - la) / sa + 1, to = std::min(na, (end_b + d + sa - 1) / sa);
    if (from >= to)
        return false;
    const Wide x = from * sa - d, up = ((la + lb) / sb + 1) * sb;  // no operand below zero
    return floor_sum(to - from, sb, sa, x + la - 1 + up) > floor_sum(to - from, sb, sa, x - lb + up);
}

// What is written shares memory neither with what is read nor with each other.
int check_apart(std::initializer_list<Area> written, std::initializer_list<Area> read)
{
    for (const Area *w = written.begin(); w != written.end(); ++w) {
        for (const Area &r : read)
            if (share_memory(*w, r))
                return report(DERF_ERR_INVALID_ARG, "%s overlaps %s", w->name, r.name);
        for (const Area *v = w + 1; v != written.end(); ++v)
            if (share_memory(*w, *v))
                return report(DERF_ERR_INVALID_ARG, "%s overlaps %s", w->name, v->name);
    }
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
