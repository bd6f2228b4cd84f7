// How an optimizer of orthogonalised updates (csrc/heads_api.cpp) puts its matrices into
// launches, on a HIP runtime of this file's own that allocates addresses and runs nothing:
// every matrix once, in a launch of a shape that holds it and of its exactness, with no
// more workspace than there is.
// Prints one line per failed expectation; exit status 0 without any.
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <map>
#include <vector>

#include "ops_internal.h"

namespace {

constexpr size_t kGiB = 1ull << 30;

struct Launch {
    unsigned first, count;
    int fan_out, fan_in;
    bool split;
};
std::vector<Launch> launches;
std::vector<derf::MuonEntry> launched;  // matrices, in order
std::map<const void *, size_t> allocated;
const void *workspace_of_all = nullptr;
size_t per_matrix = 0;  // bytes of workspace

int failures = 0;
char last_error[512];

void expect(bool ok, const char *what)
{
    if (!ok) {
        printf("FAILED: %s (last error: %s)\n", what, last_error);
        ++failures;
    }
}

int padded(int n) { return (n + 63) / 64 * 64; }

}  // namespace

extern "C" {
hipError_t hipGetDevice(int *device)
{
    *device = 0;
    return hipSuccess;
}
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceSynchronize(void) { return hipSuccess; }
hipError_t hipMemcpy(void *to, const void *from, size_t bytes, hipMemcpyKind)
{
    expect(allocated.count(to) && allocated[to] >= bytes, "the table fits its memory");
    memcpy(to, from, bytes);
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "an error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *status)
{
    *status = hipStreamCaptureStatusNone;
    return hipSuccess;
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
// The first allocation of an optimizer is its table, the second its workspace, of which
// only the size counts.
hipError_t device_alloc(void **p, size_t bytes)
{
    *p = malloc(allocated.empty() ? bytes : 16);
    allocated[*p] = bytes;
    return hipSuccess;
}
hipError_t device_free(void *p)
{
    allocated.erase(p);
    free(p);
    return hipSuccess;
}
size_t muon_workspace_bytes(int fan_out, int fan_in, bool, unsigned matrices)
{
    return fan_out <= 128 && fan_in <= 128 ? 0 : matrices * per_matrix;
}
hipError_t launch_muon(const MuonSet &set, unsigned matrices, int fan_out, int fan_in, bool split, const MuonStep &, void *workspace,
                       hipStream_t)
{
    launches.push_back({set.first, matrices, fan_out, fan_in, split});
    expect(set.first == launched.size() && matrices > 0, "one launch's matrices behind the other's");
    const size_t need = muon_workspace_bytes(fan_out, fan_in, split, matrices);
    expect(need == 0 || (allocated.count(workspace) && allocated[workspace] >= need), "its workspace is there");
    expect(need <= 8 * kGiB || matrices == 1, "8 GiB at most, but for one matrix");
    for (unsigned k = 0; k < matrices; ++k) {
        const MuonEntry e = set.table[set.first + k];
        const int o = padded(e.fan_out), i = padded(e.fan_in), m = std::min(fan_out, fan_in), n = std::max(fan_out, fan_in);
        expect(std::min(o, i) <= m && std::max(o, i) <= n, "the launch's shape holds the matrix");
        expect((o <= 128 && i <= 128) || (std::min(o, i) == m && std::max(o, i) == n), "a large one's is its own");
        expect(split == (!e.param_bf16 || std::min(e.fan_out, e.fan_in) < 8), "exactness by the parameters' type and the shorter side");
        launched.push_back(e);
    }
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

namespace {

// Tensors whose arrays lie far apart.
struct Tensors {
    std::vector<derf_muon_tensor> all;
    long long matrices = 0;
    void add(int count, int fan_out, int fan_in, int precision = DERF_PREC_FP32)
    {
        auto place = [&](int which) { return reinterpret_cast<char *>((all.size() * 3 + which + 1) << 36); };
        all.push_back({place(0), place(1), reinterpret_cast<float *>(place(2)), nullptr, count, fan_out, fan_in, precision, DERF_PREC_FP32});
        matrices += count;
    }
};

// A step's launches; every matrix of every tensor is in one.
std::vector<Launch> step(const Tensors &t)
{
    launches.clear();
    launched.clear();
    derf_muon *opt = nullptr;
    expect(derf_muon_create(&opt, t.all.data(), (int)t.all.size()) == DERF_OK, "made");
    expect(derf_muon_step(opt, 0.1, 0.9, 1, 0.0, 5, nullptr, nullptr) == DERF_OK, "a step");
    derf_muon_destroy(opt);
    expect(allocated.empty(), "nothing left");
    expect((long long)launched.size() == t.matrices, "as many matrices as there are");
    std::map<const void *, int> seen;
    for (const derf::MuonEntry &e : launched)
        ++seen[e.param];
    for (const derf_muon_tensor &x : t.all)
        for (int k = 0; k < x.num_matrices; ++k) {
            const long long at = (long long)k * x.fan_out * x.fan_in;
            const void *param = static_cast<char *>(x.param) + at * (x.param_precision == DERF_PREC_BF16 ? 2 : 4);
            expect(seen[param] == 1, "each of them once");
            for (const derf::MuonEntry &e : launched)
                if (e.param == param) {
                    expect(e.fan_out == x.fan_out && e.fan_in == x.fan_in && e.m == x.m + at &&
                               e.grad == static_cast<const char *>(x.grad) + at * 4,
                           "with its own arrays");
                    break;
                }
        }
    return launches;
}
bool is(const Launch &l, unsigned count, int m, int n, bool split = true)
{
    return l.count == count && std::min(l.fan_out, l.fan_in) == m && std::max(l.fan_out, l.fan_in) == n && l.split == split;
}

}  // namespace

int main()
{
    per_matrix = 64;
    // small ones of three padded shapes: together up to 256 of a type, in places of the largest
    Tensors t;
    t.add(100, 8, 8);
    t.add(100, 100, 20);
    t.add(56, 128, 128);
    std::vector<Launch> l = step(t);
    expect(l.size() == 1 && is(l[0], 256, 128, 128), "256 of three shapes in one launch");
    t.add(1, 20, 100);
    l = step(t);
    expect(l.size() == 3 && is(l[0], 100, 64, 64) && is(l[1], 101, 64, 128) && is(l[2], 56, 128, 128), "257: one for each padded shape");
    // the limit is of each type by itself
    t = {};
    t.add(200, 8, 8);
    t.add(56, 65, 65);
    t.add(200, 8, 8, DERF_PREC_BF16);
    t.add(56, 8, 128, DERF_PREC_BF16);
    l = step(t);
    expect(l.size() == 2 && is(l[0], 256, 64, 128, false) && is(l[1], 256, 128, 128), "256 of each type in two launches");
    // few rows or columns go with the exact ones
    t = {};
    t.add(2, 8, 128, DERF_PREC_BF16);
    t.add(3, 7, 128, DERF_PREC_BF16);
    t.add(4, 100, 7, DERF_PREC_BF16);
    t.add(5, 64, 64);
    t.add(2, 7, 700, DERF_PREC_BF16);
    t.add(2, 8, 700, DERF_PREC_BF16);
    l = step(t);
    expect(l.size() == 4 && is(l[0], 2, 64, 128, false) && is(l[1], 12, 64, 128) && is(l[2], 2, 64, 704, false) && is(l[3], 2, 64, 704),
           "by exactness, then shape");
    // places are as large as the largest of each side asks for
    t = {};
    t.add(2, 128, 3);
    t.add(2, 64, 64);
    l = step(t);
    expect(l.size() == 1 && is(l[0], 4, 64, 128), "64 x 128");
    // large ones are not among them
    t.add(3, 300, 200);
    t.add(2, 200, 300);
    t.add(1, 129, 128);
    l = step(t);
    expect(l.size() == 3 && is(l[0], 4, 64, 128) && is(l[1], 1, 128, 192) && is(l[2], 5, 256, 320), "large ones by their padded shapes");

    // workspace: as many of a shape together as 8 GiB hold
    per_matrix = 3 * kGiB;
    t = {};
    t.add(7, 300, 200);
    t.add(4, 8, 8);
    l = step(t);
    expect(l.size() == 5 && is(l[0], 4, 64, 64) && is(l[1], 2, 256, 320) && is(l[2], 2, 256, 320) && is(l[3], 2, 256, 320) && is(l[4], 1, 256, 320),
           "twice 3 GiB at a time");
    per_matrix = 8 * kGiB;
    t = {};
    t.add(2, 300, 200);
    l = step(t);
    expect(l.size() == 2 && is(l[0], 1, 256, 320) && is(l[1], 1, 256, 320), "8 GiB each");
    per_matrix = 20 * kGiB;
    l = step(t);
    expect(l.size() == 2 && is(l[0], 1, 256, 320), "a larger one by itself");
    per_matrix = kGiB;
    t.add(9, 500, 400);
    t.add(3, 400, 500, DERF_PREC_BF16);
    l = step(t);
    expect(l.size() == 4 && is(l[0], 2, 256, 320) && is(l[1], 3, 448, 512, false) && is(l[2], 8, 448, 512) && is(l[3], 1, 448, 512),
           "eight of one shape and type, then the rest");
    printf("muon groups driver: %d failure(s)\n", failures);
    return failures ? 1 : 0;
}
