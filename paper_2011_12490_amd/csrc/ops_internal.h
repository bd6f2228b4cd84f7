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

// ---- the heads' gated layers (kernels_gated.hip, kernels_gated_back.hip) -------
// pre.p may be null.
hipError_t launch_heads_gated(const LinearShape &sh, Rows x, const void *w, const float *bias, int act, bool bf16, Rows y,
                              Rows pre, hipStream_t s);
size_t heads_gated_workspace_bytes(unsigned rows, int heads, int fan_in, int fan_out, bool bf16);
// dx.p, dw, db may be null.
hipError_t launch_heads_gated_backward(const LinearShape &sh, Rows dy, Rows pre, Rows x, const void *w, int act, bool bf16,
                                       Rows dx, void *dw, float *db, void *workspace, hipStream_t s);

// ---- table lookups (kernels_lookup.hip) -----------------------------------------
hipError_t launch_lookup(Rows table, const int *ids, long long samples, long long rows, int dim, float scale, bool bf16, Rows out,
                         hipStream_t s);
size_t lookup_workspace_bytes(unsigned samples, unsigned rows, int dim);
hipError_t launch_lookup_backward(Rows dout, const int *ids, unsigned samples, unsigned rows, int dim, float scale, bool bf16,
                                  float *out, void *workspace, hipStream_t s);

// ---- orthogonalised updates (kernels_muon.hip) ----------------------------------
// A matrix: its parameters (or where the result goes), gradient, momentum and copy.
struct MuonEntry {
    void *param;
    const void *grad;
    float *m;
    void *copy;
    int fan_out, fan_in, param_bf16, grad_bf16;
    float size;  // of its steps
};
// Matrices from table[first] on (device memory), or, without a table, some like `one`
// that lie one after another.
struct MuonSet {
    const MuonEntry *table;
    unsigned first;
    MuonEntry one;
};
struct MuonStep {
    float momentum, decay, rate;
    int has_momentum, nesterov;
    int updates;  // 0: the result itself is written
    int iterations;
    const float *grad_scale;  // device, or null
};
// Of matrices of one padded shape, those of fan_out x fan_in being one of them.  split:
// products as exact as float32's.
size_t muon_workspace_bytes(int fan_out, int fan_in, bool split, unsigned matrices);
hipError_t launch_muon(const MuonSet &set, unsigned matrices, int fan_out, int fan_in, bool split, const MuonStep &st,
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
