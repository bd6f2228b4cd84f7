// Which kernels the gated layers, the table lookups and the orthogonalised updates
// launch: the library's launchers, as built, on a HIP runtime of this file's own that
// writes down the kernels by name and runs nothing.
//
// stdin: one call a line,
//   gated    bf16 rows heads fan_in fan_out pad shift keep
//   backward bf16 rows heads fan_in fan_out pad shift outputs
//   lookup   bf16 samples rows dim pad shift
//   gradient bf16 samples rows dim pad shift
//   matrices float32 count fan_out fan_in
// pad elements between rows, which start shift elements behind an aligned place;
// outputs: 1 dx + 2 dW + 4 db.  stdout: "has NAME" for every kernel of the units, then for
// each call a line "call" and "ran NAME" for every launch.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <map>
#include <string>

#include "ops_internal.h"

namespace {

std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> m;
    return m;
}

}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *)
{
    static void *module;
    return &module;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *,
                           int *)
{
    names()[host] = name;
}
void __hipRegisterVar(void **, void *, char *, const char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *s)
{
    *grid = *block = dim3(1);
    *lds = 0;
    *s = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *host, dim3, dim3, void **, size_t, hipStream_t)
{
    printf("ran %s\n", names()[host].c_str());
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipGetDevice(int *device)
{
    *device = 0;
    return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int *value, hipDeviceAttribute_t, int)
{
    *value = 256;  // compute units
    return hipSuccess;
}
}  // extern "C"

int main()
{
    for (const auto &n : names())
        printf("has %s\n", n.second.c_str());
    char op[16];
    int type;
    while (scanf("%15s %d", op, &type) == 2) {
        char *const at = reinterpret_cast<char *>(1 << 20);
        float *const f = reinterpret_cast<float *>(at);
        const int *const offsets = reinterpret_cast<const int *>(at);
        const int bytes = type ? 2 : 4;
        hipError_t e = hipErrorInvalidValue;
        long long a[8];
        const int numbers = !strcmp(op, "gated") || !strcmp(op, "backward") ? 7 : !strcmp(op, "matrices") ? 3 : 5;
        for (int i = 0; i < numbers; ++i)
            if (scanf("%lld", &a[i]) != 1)
                return 2;
        printf("call\n");
        if (numbers == 7) {
            const int I = (int)a[2], O = (int)a[3];
            char *const shifted = at + a[5] * bytes;
            const derf::LinearShape sh = {offsets, (unsigned)a[0], (int)a[1], I, O};
            const derf::Rows x = {shifted, I + a[4]}, y = {shifted, O + a[4]}, pre = {shifted, 2 * O + a[4]}, none = {nullptr, 0};
            if (!strcmp(op, "gated"))
                e = derf::launch_heads_gated(sh, x, at, f, 0, type, y, a[6] ? pre : none, nullptr);
            else
                e = derf::launch_heads_gated_backward(sh, y, pre, x, at, 0, type, a[6] & 1 ? derf::Rows{at, I} : none,
                                                      a[6] & 2 ? at : nullptr, a[6] & 4 ? f : nullptr, at, nullptr);
        } else if (numbers == 5) {
            const derf::Rows rows = {at + a[4] * bytes, a[2] + a[3]};
            e = !strcmp(op, "lookup") ? derf::launch_lookup(rows, offsets, a[0], a[1], (int)a[2], 1.0f, type, rows, nullptr)
                                      : derf::launch_lookup_backward(rows, offsets, (unsigned)a[0], (unsigned)a[1], (int)a[2], 1.0f,
                                                                     type, f, at, nullptr);
        } else {
            const derf::MuonSet set = {nullptr, 0, {at, at, f, nullptr, (int)a[1], (int)a[2], 0, 0, 1.0f}};
            const derf::MuonStep st = {0.9f, 1.0f, 0.1f, 1, 1, 1, 5, nullptr};
            e = derf::launch_muon(set, (unsigned)a[0], (int)a[1], (int)a[2], type, st, at, nullptr);
        }
        if (e != hipSuccess)
            return 1;
    }
    return 0;
}
