// Internal interfaces between the host side of the training operators
// (ops_api.cpp) and their kernels.  Nothing here is part of the public C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "derf.h"

namespace derf {

// Records `fmt` as the calling thread's last error and returns `status`.
int report(int status, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
// Every device allocation of the library (counted and made to fail in test builds).
hipError_t device_alloc(void **p, size_t bytes);
hipError_t device_free(void *p);

// ---- routing (kernels_route.hip) -------------------------------------------
size_t route_workspace_bytes(unsigned pairs, int num_heads);
hipError_t launch_route(const int *heads, unsigned pairs, int num_heads, int *offsets, int *pair,
                        int *row, unsigned *workspace, hipStream_t s);

// Rows of `dim` elements, `stride` elements apart.
struct Rows {
    const void *p;
    long long stride;
};
hipError_t launch_dispatch(Rows x, const int *row, long long tokens, int top_k, int dim, bool bf16,
                           Rows out, hipStream_t s);
hipError_t launch_combine(Rows rows, const float *weights, const int *row, long long tokens,
                          int top_k, int dim, bool bf16, Rows out, hipStream_t s);
hipError_t launch_combine_backward(Rows dout, Rows rows, const float *weights, const int *row,
                                   long long tokens, int top_k, int dim, bool bf16, Rows drows,
                                   float *dweights, hipStream_t s);

// ---- the heads' linear layers (kernels_linear.hip) --------------------------
struct LinearShape {
    const int *offsets;
    unsigned rows;
    int heads, fan_in, fan_out;
};
hipError_t launch_heads_linear(const LinearShape &sh, Rows x, const void *w, const float *bias,
                               bool relu, bool bf16, Rows y, hipStream_t s);
size_t heads_linear_workspace_bytes(unsigned rows, int heads, int fan_in, int fan_out, bool relu, bool bf16);
// y.p: null without ReLU.  dx.p, dw, db may be null.
hipError_t launch_heads_linear_backward(const LinearShape &sh, Rows dy, Rows x, const void *w,
                                        Rows y, bool bf16, Rows dx, float *dw, float *db,
                                        void *workspace, hipStream_t s);

// ---- AdamW (kernels_adamw.hip) ----------------------------------------------
// Values of an 8-bit moment that share a scale.
constexpr int kMomentBlock = 256;
struct AdamWScalars {
    float decay, beta1, one_minus_beta1, beta2, one_minus_beta2, rate, root_scale, eps;
};
// Tensors as the kernel reads them: `first` is the tensor's first work item
// among all tensors' (adamw_items(n) each).
struct AdamWEntry {
    derf_adamw_tensor t;
    unsigned first;
    unsigned aligned;  // every array starts at a multiple of its widest load
};
unsigned adamw_items(long long n);
hipError_t launch_adamw(const AdamWEntry *table, int tensors, unsigned items, int state_bits,
                        const AdamWScalars &c, const float *grad_scale, hipStream_t s);

}  // namespace derf
