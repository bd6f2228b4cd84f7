// Which arrays of the gated layers, lookups and orthogonalised matrices the host code
// (csrc/heads_api.cpp) takes, on launches of this file's own that run nothing: the check
// for shared memory against a map of bytes, then the entry points.
// Prints one line per failed expectation; exit status 0 without any.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <random>
#include <vector>

#include "ops_checks.h"

namespace {

int failures = 0, launches = 0;
char last_error[512];

void expect(bool ok, const char *what)
{
    if (!ok) {
        printf("FAILED: %s (last error: %s)\n", what, last_error);
        ++failures;
    }
}

}  // namespace

extern "C" {
hipError_t hipGetDevice(int *) { return hipErrorNoDevice; }
hipError_t hipSetDevice(int) { return hipErrorNoDevice; }
hipError_t hipDeviceSynchronize(void) { return hipErrorNoDevice; }
hipError_t hipMemcpy(void *, const void *, size_t, hipMemcpyKind) { return hipErrorNoDevice; }
hipError_t hipGetLastError(void) { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *) { return hipErrorNoDevice; }
}

namespace derf {

int report(int status, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(last_error, sizeof(last_error), fmt, ap);
    va_end(ap);
    return status;
}
hipError_t device_alloc(void **, size_t) { return hipErrorOutOfMemory; }
hipError_t device_free(void *) { return hipSuccess; }
size_t muon_workspace_bytes(int, int, bool, unsigned) { return 256; }
hipError_t launch_muon(const MuonSet &, unsigned, int, int, bool, const MuonStep &, void *, hipStream_t)
{
    ++launches;
    return hipSuccess;
}
hipError_t launch_heads_gated(const LinearShape &, Rows, const void *, const float *, int, bool, Rows, Rows, hipStream_t)
{
    ++launches;
    return hipSuccess;
}
size_t heads_gated_workspace_bytes(unsigned, int, int, int, bool) { return 256; }
hipError_t launch_heads_gated_backward(const LinearShape &, Rows, Rows, Rows, const void *, int, bool, Rows, void *, float *, void *,
                                       hipStream_t)
{
    ++launches;
    return hipSuccess;
}
hipError_t launch_lookup(Rows, const int *, long long, long long, int, float, bool, Rows, hipStream_t)
{
    ++launches;
    return hipSuccess;
}
size_t lookup_workspace_bytes(unsigned, unsigned, int) { return 256; }
hipError_t launch_lookup_backward(Rows, const int *, unsigned, unsigned, int, float, bool, float *, void *, hipStream_t)
{
    ++launches;
    return hipSuccess;
}

}  // namespace derf

namespace {

using derf::Area;

char *at(long long address) { return reinterpret_cast<char *>(address); }

bool by_bytes(const Area &a, const Area &b)
{
    std::vector<char> taken(4096, 0);
    for (long long i = 0; i < a.rows; ++i)
        for (long long k = 0; k < a.row; ++k)
            taken[(size_t)a.p + i * a.stride + k] = 1;
    for (long long j = 0; j < b.rows; ++j)
        for (long long k = 0; k < b.row; ++k)
            if (taken[(size_t)b.p + j * b.stride + k])
                return true;
    return false;
}

void against_bytes()
{
    std::mt19937 rng(1);
    int both[2] = {0, 0};
    auto area = [&] {
        const long long row = 1 + rng() % 12, stride = row + rng() % (rng() % 2 ? 40 : 4);
        return Area{"", at(1 + rng() % 200), (long long)(rng() % 14), row, stride};
    };
    for (int n = 0; n < 400000; ++n) {
        Area a = area(), b = area();
        if (n % 2) {  // columns of one buffer
            const long long stride = std::max(a.stride, b.stride);
            a = {"", a.p, a.rows, a.row, stride};
            b = {"", b.p, b.rows, b.row, stride};
        }
        const bool want = by_bytes(a, b);
        ++both[want];
        if (share_memory(a, b) != want || share_memory(b, a) != want) {
            printf("FAILED: %p %lld rows of %lld, %lld apart, and %p %lld of %lld, %lld apart\n", a.p, a.rows, a.row, a.stride, b.p, b.rows,
                   b.row, b.stride);
            ++failures;
            return;
        }
    }
    expect(both[0] > 50000 && both[1] > 50000, "both answers are met");
    // large ones: 2^31 rows far apart, and the same one byte on
    const Area far = {"", at(1 << 20), (1LL << 31) - 1, 1000, 1LL << 14}, beside = {"", at((1 << 20) + 1000), (1LL << 31) - 1, 15384, 1LL << 14};
    expect(!share_memory(far, beside) && !share_memory(beside, far), "rows between rows");
    const Area on = {"", at((1 << 20) + 999), beside.rows, beside.row, beside.stride};
    expect(share_memory(far, on) && share_memory(on, far), "one byte of each");
    auto moving = [](long long rows) { return Area{"", at((1 << 20) + 1000), rows, 8, (1LL << 14) + 1}; };  // one byte on with every row
    expect(share_memory(far, moving(1 << 20)), "the last of the gap's rows");
    expect(!share_memory(far, moving(15376)), "none yet");  // row i ends at 1008 + i, the next far one begins at 16384
    expect(share_memory(far, moving(15378)), "the first");
    // more than any memory holds: no sum may turn over
    expect(share_memory(Area{"", at(64), 1LL << 30, 8, 1LL << 42}, Area{"", at(1LL << 47), 4, 1 << 20, 1 << 20}), "beyond 64 bits");
    expect(!share_memory(Area{"", at(64), 0, 8, 8}, far) && !share_memory(far, Area{"", nullptr, 5, 1 << 30, 1 << 30}), "no rows, no array");
}

// Arguments that lie far apart, but for one.
long long apart = 1 << 20;
char *fresh() { return at(apart += 1 << 20); }

void entry_points()
{
    const int R = 8, K = 4, I = 16, O = 24, bf = DERF_PREC_BF16;
    char *x = fresh(), *w = fresh(), *b = fresh(), *off = fresh(), *y = fresh(), *pre = fresh(), *dy = fresh(), *dx = fresh(),
         *dw = fresh(), *db = fresh(), *ws = fresh();
    const long long wide = 200;
    auto gated = [&](char *x_, char *y_, char *pre_) {
        return derf_heads_gated(x_, wide, w, reinterpret_cast<float *>(b), reinterpret_cast<int *>(off), R, K, I, O, 0, bf, y_, wide, pre_, wide, nullptr);
    };
    auto refused = [&](int status, const char *message) {
        expect(status == DERF_ERR_INVALID_ARG && !strcmp(last_error, message), message);
        expect(launches == 0, "nothing is launched");
    };
    auto taken = [&](int status, const char *what) {
        expect(status == DERF_OK && launches == 1, what);
        launches = 0;
    };
    taken(gated(x, y, pre), "gated");
    taken(gated(x, y, nullptr), "gated without pre");
    taken(gated(x, x + I * 2, x + (I + O) * 2), "columns of one buffer");
    taken(gated(x, x + R * wide * 2, nullptr), "rows of one buffer");
    refused(gated(x, x, nullptr), "y overlaps x");
    refused(gated(x, x + I * 2 - 2, nullptr), "y overlaps x");
    refused(gated(x, y, y + O * 2 - 2), "y overlaps pre");
    refused(gated(x, w + K * 2 * O * I * 2 - 2, nullptr), "y overlaps w");
    taken(gated(x, w + K * 2 * O * I * 2, nullptr), "behind the weights");
    refused(gated(x, y, b), "pre overlaps bias");
    refused(gated(x, off + 16, nullptr), "y overlaps offsets");
    taken(gated(x, off + 20, nullptr), "behind the offsets");

    auto backward = [&](char *x_, char *w_, char *dx_, char *dw_, char *db_, char *ws_) {
        return derf_heads_gated_backward(dy, O, pre, 2 * O, x_, I, w_, reinterpret_cast<int *>(off), R, K, I, O, 0, bf, dx_, I, dw_,
                                         reinterpret_cast<float *>(db_), ws_, 256, nullptr);
    };
    taken(backward(x, w, dx, dw, db, ws), "gradients");
    refused(backward(x, w, x, dw, db, ws), "out_x overlaps x");
    taken(backward(x, w, x, nullptr, db, ws), "x is not read");
    refused(backward(x, w, dy, dw, db, ws), "out_x overlaps dy");
    refused(backward(x, w, dx, w, db, ws), "out_w overlaps w");
    taken(backward(x, w, nullptr, w, db, ws), "w is not read");
    refused(backward(x, w, dx, dw, off, ws), "out_bias overlaps offsets");
    refused(backward(x, w, dx, dw, dw + K * 2 * O * I * 2 - 4, ws), "out_w overlaps out_bias");
    taken(backward(x, w, dx, dw, dw + K * 2 * O * I * 2, ws), "one behind the other");
    refused(backward(x, w, dx, dw, db, pre), "workspace overlaps pre");
    refused(backward(x, w, dx, dw, db, dx - 240), "out_x overlaps workspace");

    int *ids = reinterpret_cast<int *>(fresh());
    char *table = fresh(), *out = fresh();
    auto lookup = [&](char *out_) { return derf_lookup(table, 24, ids, 6, 5, 12, 1.0f, DERF_PREC_FP32, out_, 24, nullptr); };
    taken(lookup(out), "lookup");
    taken(lookup(table + 48 - 96), "gaps of as many values as a row has");
    refused(lookup(table + 44), "out overlaps table");
    refused(lookup(reinterpret_cast<char *>(ids) - 5 * 96 - 44), "out overlaps ids");
    auto gradient = [&](char *out_, char *ws_) {
        return derf_lookup_backward(table, 20, ids, 6, 5, 12, 1.0f, DERF_PREC_FP32, reinterpret_cast<float *>(out_), ws_, 256, nullptr);
    };
    taken(gradient(out, ws), "the table's gradient");
    refused(gradient(table, ws), "out overlaps dout");
    refused(gradient(out, out + 224), "out overlaps workspace");
    refused(gradient(out, reinterpret_cast<char *>(ids)), "workspace overlaps ids");

    auto orthogonalise = [&](char *x_, char *out_, char *ws_) {
        return derf_orthogonalise(x_, 3, 8, 10, 5, DERF_PREC_FP32, out_, ws_, 256, nullptr);
    };
    taken(orthogonalise(table, out, ws), "orthogonalise");
    taken(orthogonalise(table, table, ws), "in place");
    refused(orthogonalise(table, table + 4, ws), "out overlaps x");
    refused(orthogonalise(table, table - 320, ws), "out overlaps x");
    refused(orthogonalise(table, out, table), "workspace overlaps x");
    refused(orthogonalise(table, table, table + 944), "out overlaps workspace");
}

}  // namespace

int main()
{
    against_bytes();
    entry_points();
    printf("heads arrays driver: %d failure(s)\n", failures);
    return failures ? 1 : 0;
}
