// Which kernels the heads' layers launch: the library's launchers
// (csrc/kernels_linear.hip, as built) on a HIP runtime of this file's own that
// writes down the kernels by name and runs nothing.
//
// stdin: one call a line,
//   forward  bf16 rows heads fan_in fan_out pad shift
//   backward bf16 rows heads fan_in fan_out pad shift relu outputs
// pad elements between rows of x, y and dy, which start shift elements behind an
// aligned place; outputs: 1 dx + 2 dW + 4 db.  stdout: "has NAME" for every kernel of
// the library, then for each call a line "call" and "ran NAME" for every launch.
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
    int bf16, heads, fan_in, fan_out, pad, shift;
    unsigned rows;
    while (scanf("%15s %d %u %d %d %d %d %d", op, &bf16, &rows, &heads, &fan_in, &fan_out, &pad, &shift) == 8) {
        char *const at = reinterpret_cast<char *>(1 << 20);
        char *const shifted = at + shift * (bf16 ? 2 : 4);
        float *const f = reinterpret_cast<float *>(at);
        const derf::LinearShape sh = {reinterpret_cast<const int *>(at), rows, heads, fan_in, fan_out};
        const derf::Rows in = {shifted, fan_in + pad}, out = {shifted, fan_out + pad};
        printf("call\n");
        hipError_t e;
        if (!strcmp(op, "forward")) {
            e = derf::launch_heads_linear(sh, in, at, f, true, bf16, out, nullptr);
        } else {
            int relu, outputs;
            if (scanf("%d %d", &relu, &outputs) != 2)
                return 2;
            const derf::Rows none = {nullptr, 0}, dx = {at, fan_in};
            e = derf::launch_heads_linear_backward(sh, out, in, at, relu ? out : none, bf16, outputs & 1 ? dx : none,
                                                   outputs & 2 ? f : nullptr, outputs & 4 ? f : nullptr, at, nullptr);
        }
        if (e != hipSuccess)
            return 1;
    }
    return 0;
}
