// AdamW over many tensors in one launch, moments in float or in e4m3 with a
// float scale for each 256 values.
//
// Every operation is rounded on its own (nothing is contracted into a fused
// multiply-add), so the codes of an 8-bit moment are a function of the formula
// alone and not of how the compiler schedules it.
#include "ops_internal.h"

#pragma clang fp contract(off)

namespace derf {

namespace {

constexpr int kThreads = 256;
constexpr int kItem = 1024;  // values of a work item: a workgroup's share

__device__ __forceinline__ float load_value(const void *p, long long i, int precision)
{
    return precision == DERF_PREC_BF16 ? (float)static_cast<const __bf16 *>(p)[i]
                                       : static_cast<const float *>(p)[i];
}

// The tensor that work item `item` belongs to: the last whose first is <= item.
__device__ __forceinline__ int find_tensor(const AdamWEntry *table, int tensors, unsigned item)
{
    int lo = 0, hi = tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table[mid].first <= item)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float wave_max(float x)
{
    for (int off = 32; off > 0; off >>= 1)
        x = fmaxf(x, __shfl_xor(x, off));
    return x;
}

__device__ __forceinline__ float finite_abs(float x) { return isfinite(x) ? fabsf(x) : 0.0f; }

// x / scale as an e4m3 code; is_root: a positive value keeps the smallest code.
__device__ __forceinline__ unsigned char encode8(float x, float inv_scale, bool is_root)
{
    if (!isfinite(x))
        return 0x7F;
    float q = fminf(fmaxf(x * inv_scale, -448.0f), 448.0f);
    if (is_root && x > 0.0f)
        q = fmaxf(q, 0x1p-9f);
    return (unsigned char)(__builtin_amdgcn_cvt_pk_fp8_f32(q, 0.0f, 0, false) & 0xFF);
}

__device__ __forceinline__ float decode8(unsigned char c, float scale)
{
    return __builtin_amdgcn_cvt_f32_fp8((int)c, 0) * scale;
}

// One wave takes 256 values (a moment block), four a lane.
template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamWEntry *table, int tensors,
                                                         AdamWScalars c, const float *grad_scale)
{
    const AdamWEntry &e = table[find_tensor(table, tensors, blockIdx.x)];
    const float gs = grad_scale ? *grad_scale : 1.0f;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const long long block = (long long)(blockIdx.x - e.first) * (kItem / kMomentBlock) + wave;
    const long long base = block * kMomentBlock;
    const long long n = e.t.n;
    if (base >= n)
        return;
    float ms = 0.0f, vs = 0.0f;
    if (BITS == 8) {
        ms = e.t.m_scale[block];
        vs = e.t.v_scale[block];
    }
    float m[4], root[4];
    float mmax = 0.0f, rmax = 0.0f;
    for (int j = 0; j < 4; ++j) {
        const long long i = base + lane * 4 + j;
        m[j] = root[j] = 0.0f;
        if (i >= n)
            continue;
        const float g = load_value(e.t.grad, i, e.t.grad_precision) * gs;
        float p = load_value(e.t.param, i, e.t.param_precision);
        float mo, vo;
        if (BITS == 8) {
            mo = decode8(static_cast<const unsigned char *>(e.t.m)[i], ms);
            const float r = decode8(static_cast<const unsigned char *>(e.t.v)[i], vs);
            vo = r * r;
        } else {
            mo = static_cast<const float *>(e.t.m)[i];
            vo = static_cast<const float *>(e.t.v)[i];
        }
        m[j] = mo * c.beta1 + g * c.one_minus_beta1;
        const float v = vo * c.beta2 + (g * g) * c.one_minus_beta2;
        root[j] = sqrtf(v);
        p = p * c.decay - m[j] / (root[j] * c.root_scale + c.eps) * c.rate;
        if (e.t.param_precision == DERF_PREC_BF16)
            static_cast<__bf16 *>(e.t.param)[i] = (__bf16)p;
        else
            static_cast<float *>(e.t.param)[i] = p;
        if (e.t.copy)
            static_cast<__bf16 *>(e.t.copy)[i] = (__bf16)p;
        if (BITS == 32) {
            static_cast<float *>(e.t.m)[i] = m[j];
            static_cast<float *>(e.t.v)[i] = v;
        }
        mmax = fmaxf(mmax, finite_abs(m[j]));
        rmax = fmaxf(rmax, finite_abs(root[j]));
    }
    if (BITS == 8) {
        ms = fmaxf(wave_max(mmax) * (1.0f / 448.0f), 0x1p-120f);
        vs = fmaxf(wave_max(rmax) * (1.0f / 448.0f), 0x1p-120f);
        const float mi = 1.0f / ms, vi = 1.0f / vs;
        for (int j = 0; j < 4; ++j) {
            const long long i = base + lane * 4 + j;
            if (i >= n)
                continue;
            static_cast<unsigned char *>(e.t.m)[i] = encode8(m[j], mi, false);
            static_cast<unsigned char *>(e.t.v)[i] = encode8(root[j], vi, true);
        }
        if (lane == 0) {
            e.t.m_scale[block] = ms;
            e.t.v_scale[block] = vs;
        }
    }
}

}  // namespace

unsigned adamw_items(long long n)
{
    return (unsigned)((n + kItem - 1) / kItem);
}

hipError_t launch_adamw(const AdamWEntry *table, int tensors, unsigned items, int state_bits,
                        const AdamWScalars &c, const float *grad_scale, hipStream_t s)
{
    if (state_bits == 8)
        adamw_kernel<8><<<items, kThreads, 0, s>>>(table, tensors, c, grad_scale);
    else
        adamw_kernel<32><<<items, kThreads, 0, s>>>(table, tensors, c, grad_scale);
    return hipGetLastError();
}

}  // namespace derf
