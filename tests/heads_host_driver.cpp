// The host code of the gated layers, lookups and orthogonalised updates
// (csrc/heads_api.cpp) on a HIP runtime of this file's own: two devices, allocations that
// may fail, streams that may be capturing, and launches that are counted.  It shows what
// the host does where no GPU, or a second one, is at hand.
// Prints one line per failed expectation; exit status 0 without any.
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <set>

#include "ops_internal.h"

namespace {

int current = 0;  // device
int waited_for = -1, launched_on = -1;
hipStreamCaptureStatus capture_status = hipStreamCaptureStatusNone;  // of every stream
hipError_t capture_query = hipSuccess, copy_status = hipSuccess;
int launches = 0, allocations_left = 1000, freed_elsewhere = 0;
std::set<void *> live;
derf::MuonStep last_step;
unsigned matrices_launched = 0;

int failures = 0;
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
hipError_t hipGetDevice(int *device)
{
    *device = current;
    return hipSuccess;
}
hipError_t hipSetDevice(int device)
{
    current = device;
    return hipSuccess;
}
hipError_t hipDeviceSynchronize(void)
{
    waited_for = current;
    return hipSuccess;
}
hipError_t hipMemcpy(void *to, const void *from, size_t bytes, hipMemcpyKind)
{
    if (copy_status == hipSuccess)
        memcpy(to, from, bytes);
    return copy_status;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status)
{
    *status = capture_status;
    return capture_query;
}
}  // extern "C"

namespace derf {

int report(int status, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(last_error, sizeof(last_error), fmt, ap);
    va_end(ap);
    return status;
}
hipError_t device_alloc(void **p, size_t bytes)
{
    if (allocations_left-- <= 0)
        return hipErrorOutOfMemory;
    *p = malloc(bytes);
    live.insert(*p);
    return hipSuccess;
}
hipError_t device_free(void *p)
{
    freed_elsewhere += current != 1;
    live.erase(p);
    free(p);
    return hipSuccess;
}
size_t muon_workspace_bytes(int fan_out, int fan_in, bool, unsigned matrices)
{
    return fan_out <= 128 && fan_in <= 128 ? 0 : (size_t)matrices * 64;
}
hipError_t launch_muon(const MuonSet &set, unsigned matrices, int, int, bool, const MuonStep &st, void *, hipStream_t)
{
    ++launches;
    launched_on = current;
    last_step = st;
    matrices_launched += matrices;
    expect(!set.table || set.table[set.first].param != nullptr, "a launch's first matrix is in the table");
    return hipSuccess;
}

// not called here
hipError_t launch_heads_gated(const LinearShape &, Rows, const void *, const float *, int, bool, Rows, Rows, hipStream_t) { abort(); }
size_t heads_gated_workspace_bytes(unsigned, int, int, int, bool) { abort(); }
hipError_t launch_heads_gated_backward(const LinearShape &, Rows, Rows, Rows, const void *, int, bool, Rows, void *, float *, void *,
                                       hipStream_t)
{
    abort();
}
hipError_t launch_lookup(Rows, const int *, long long, long long, int, float, bool, Rows, hipStream_t) { abort(); }
size_t lookup_workspace_bytes(unsigned, unsigned, int) { abort(); }
hipError_t launch_lookup_backward(Rows, const int *, unsigned, unsigned, int, float, bool, float *, void *, hipStream_t) { abort(); }

}  // namespace derf

int main()
{
    static float p[3][3 * 200 * 300], g[3][3 * 200 * 300], m[3][3 * 200 * 300];
    derf_muon_tensor tensors[3] = {};
    for (int i = 0; i < 3; ++i)
        tensors[i] = {p[i], g[i], m[i], nullptr, 3, i == 1 ? 200 : 100, i == 2 ? 300 : 90, DERF_PREC_FP32, DERF_PREC_FP32};
    derf_muon *opt = nullptr;

    // every allocation that fails leaves nothing behind
    current = 1;
    for (int at = 0; at < 2; ++at) {
        allocations_left = at;
        expect(derf_muon_create(&opt, tensors, 3) == DERF_ERR_OOM && !opt, "a failed allocation is out of memory");
        expect(live.empty(), "and frees what there was");
    }
    allocations_left = 1000;
    copy_status = hipErrorUnknown;
    expect(derf_muon_create(&opt, tensors, 3) == DERF_ERR_HIP && !opt && live.empty(), "a failed copy frees both");
    copy_status = hipSuccess;

    // an optimizer works on the device that it was made on, and leaves the current one alone
    expect(derf_muon_create(&opt, tensors, 3) == DERF_OK && opt, "made on device 1");
    current = 0;
    expect(derf_muon_step(opt, 0.1, 0.9, 1, 0.5, 5, nullptr, nullptr) == DERF_OK, "a step from device 0");
    expect(launched_on == 1 && current == 0, "runs on device 1");
    expect(launches == 3 && matrices_launched == 9, "three shapes, nine matrices");
    expect(last_step.decay == (float)(1.0 - 0.1 * 0.5) && last_step.rate == 0.1f && last_step.momentum == 0.9f && last_step.updates &&
               last_step.iterations == 5,
           "its scalars");

    // a capturing stream is refused, with nothing launched
    launches = 0;
    for (hipStreamCaptureStatus status : {hipStreamCaptureStatusActive, hipStreamCaptureStatusInvalidated}) {
        capture_status = status;
        expect(derf_muon_step(opt, 0.1, 0.9, 1, 0.0, 5, nullptr, nullptr) == DERF_ERR_INVALID_ARG, "a capture is refused");
        expect(launches == 0 && current == 0, "and nothing runs");
    }
    capture_status = hipStreamCaptureStatusNone;
    capture_query = hipErrorUnknown;
    expect(derf_muon_step(opt, 0.1, 0.9, 0, 0.0, 5, nullptr, nullptr) == DERF_OK, "no answer: the launch says what is wrong");
    capture_query = hipSuccess;

    freed_elsewhere = 0;
    derf_muon_destroy(opt);
    expect(waited_for == 1 && freed_elsewhere == 0 && current == 0 && live.empty(), "its end waits for and frees on device 1");

    // small matrices of any shapes go together while they run at once
    static float small[300][3][64];
    derf_muon_tensor many[300];
    for (int i = 0; i < 300; ++i)
        many[i] = {small[i][0], small[i][1], small[i][2], nullptr, 1, i % 2 ? 8 : 4, i % 2 ? 8 : 16, DERF_PREC_FP32, DERF_PREC_FP32};
    current = 1;
    expect(derf_muon_create(&opt, many, 256) == DERF_OK, "256 small ones");
    expect(live.size() == 1, "need no workspace");
    launches = 0;
    derf_muon_step(opt, 0.1, 0.9, 1, 0.0, 5, nullptr, nullptr);
    expect(launches == 1, "in one launch");
    derf_muon_destroy(opt);
    for (int i = 0; i < 300; ++i)
        if (i % 2)
            many[i].param_precision = DERF_PREC_BF16;
    expect(derf_muon_create(&opt, many, 300) == DERF_OK, "of two types");
    launches = 0;
    derf_muon_step(opt, 0.1, 0.9, 1, 0.0, 5, nullptr, nullptr);
    expect(launches == 2, "each type in one launch");
    derf_muon_destroy(opt);
    expect(live.empty(), "nothing left");
    printf("heads host driver: %d failure(s)\n", failures);
    return failures ? 1 : 0;
}
