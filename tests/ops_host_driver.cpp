// The training operators' host code (csrc/ops_api.cpp) on a HIP runtime of this
// file's own: two devices that hold nothing, streams that may be capturing, and
// launches that are counted.  It shows what the host does where no GPU, or a
// second one, is at hand.
// Prints one line per failed expectation; exit status 0 without any.
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "ops_internal.h"

namespace {

int current = 0;                                                     // device
int waited_for = -1, freed_on = -1, launched_on = -1;                // the device that was current
hipStreamCaptureStatus capture_status = hipStreamCaptureStatusNone;  // of every stream
hipError_t capture_query = hipSuccess;
int launches = 0;

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

// ---- the runtime ------------------------------------------------------------------

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
    memcpy(to, from, bytes);
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status)
{
    *status = capture_status;
    return capture_query;
}
}  // extern "C"

// ---- the rest of the library ------------------------------------------------------

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
    *p = malloc(bytes);
    return hipSuccess;
}
hipError_t device_free(void *p)
{
    freed_on = current;
    free(p);
    return hipSuccess;
}

unsigned adamw_items(long long n) { return (unsigned)((n + 4095) / 4096); }
hipError_t launch_adamw(const AdamWEntry *, int, unsigned, int, const AdamWScalars &, const float *, hipStream_t)
{
    ++launches;
    launched_on = current;
    return hipSuccess;
}

// not called here
size_t route_workspace_bytes(unsigned, int) { abort(); }
hipError_t launch_route(const int *, unsigned, int, int *, int *, int *, unsigned *, hipStream_t) { abort(); }
hipError_t launch_dispatch(Rows, const int *, long long, int, int, bool, Rows, hipStream_t) { abort(); }
hipError_t launch_combine(Rows, const float *, const int *, long long, int, int, bool, Rows, hipStream_t) { abort(); }
hipError_t launch_combine_backward(Rows, Rows, const float *, const int *, long long, int, int, bool, Rows, float *,
                                   hipStream_t)
{
    abort();
}
hipError_t launch_heads_linear(const LinearShape &, Rows, const void *, const float *, bool, bool, Rows, hipStream_t)
{
    abort();
}
size_t heads_linear_workspace_bytes(unsigned, int, int, int, bool, bool) { abort(); }
hipError_t launch_heads_linear_backward(const LinearShape &, Rows, Rows, const void *, Rows, bool, Rows, float *, float *,
                                        void *, hipStream_t)
{
    abort();
}

}  // namespace derf

// ---- what is expected ---------------------------------------------------------------

namespace {

float values[64];

derf_adamw *optimizer()
{
    const derf_adamw_tensor t = {values, values + 16, values + 32, values + 48, nullptr, nullptr, nullptr, 16,
                                 DERF_PREC_FP32, DERF_PREC_FP32};
    derf_adamw *opt = nullptr;
    expect(derf_adamw_create(&opt, &t, 1, 32) == DERF_OK && opt, "an optimizer of one tensor");
    return opt;
}

int step(derf_adamw *opt)
{
    return derf_adamw_step(opt, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1, nullptr, nullptr);
}

// A recorded step would repeat its step number and rate: it is refused, and
// nothing is recorded.
void capture()
{
    derf_adamw *opt = optimizer();
    launches = 0;
    for (hipStreamCaptureStatus s : {hipStreamCaptureStatusActive, hipStreamCaptureStatusInvalidated}) {
        capture_status = s;
        expect(step(opt) == DERF_ERR_INVALID_ARG && strstr(last_error, "captur"), "a step on a capturing stream is refused");
        expect(launches == 0, "nothing is recorded");
    }
    capture_status = hipStreamCaptureStatusNone;
    expect(step(opt) == DERF_OK && launches == 1, "the next step is taken");
    // a stream whose state the runtime does not tell: the launch decides
    capture_query = hipErrorStreamCaptureImplicit;
    expect(step(opt) == DERF_OK && launches == 2, "a step where the query fails");
    capture_query = hipSuccess;
    derf_adamw_destroy(opt);
}

// An optimizer works on the device that it was made on, whichever is current, and
// leaves the current one as it was.
void devices()
{
    current = 1;
    derf_adamw *opt = optimizer();
    current = 0;
    launched_on = waited_for = freed_on = -1;
    expect(step(opt) == DERF_OK && launched_on == 1, "a step runs on the optimizer's device");
    expect(current == 0, "a step leaves the current device");
    derf_adamw_destroy(opt);
    expect(waited_for == 1, "destroy waits for the optimizer's device");
    expect(freed_on == 1, "destroy frees there");
    expect(current == 0, "destroy leaves the current device");
}

}  // namespace

int main()
{
    capture();
    devices();
    printf("ops host driver: %d failure(s)\n", failures);
    return failures != 0;
}
