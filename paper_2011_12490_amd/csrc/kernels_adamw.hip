// AdamW over many tensors in one launch, moments in float or in e4m3 with a
// float scale for each 256 values:
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// One pass over the bytes: 28 a float value with float moments, 14 with e4m3 ones and
// bf16 gradients.  Of v the codes hold the square root, whose exponents span half of
// v's.  A wave has a block of 256 values, so a scale is a wave's maximum, and reads its
// next block before it computes.  2.4 M values with a bf16 copy, 32 bits: 14.6 us, 4.9 TB/s;
// 200 M, 8 bits: 490 us, 5.7 TB/s, its vector units as busy as memory.
//
// Every operation is rounded on its own (nothing is contracted into a fused
// multiply-add), so the codes of an 8-bit moment are a function of the formula
// alone and not of how the compiler schedules it.
#include "ops_internal.h"

#pragma clang fp contract(off)

namespace derf {

namespace {

constexpr int kThreads = 256;
constexpr int kItem = 4096;  // values of a work item, a workgroup's: 4 blocks a wave

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// Four values of an array at i, converted to and from float.  WHOLE: all of
// them are there and lie at a multiple of their size; else those below n, one by one.
template <bool WHOLE, class T>
__device__ __forceinline__ f32x4 read4(const void *p, long long i, long long n)
{
    typedef T Four __attribute__((ext_vector_type(4)));
    const T *a = static_cast<const T *>(p) + i;
    if constexpr (WHOLE)
        return __builtin_convertvector(__builtin_nontemporal_load(reinterpret_cast<const Four *>(a)), f32x4);
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n)
            x[j] = (float)a[j];
    return x;
}
template <bool WHOLE, class T>
__device__ __forceinline__ void write4(void *p, long long i, long long n, f32x4 x)
{
    typedef T Four __attribute__((ext_vector_type(4)));
    T *a = static_cast<T *>(p) + i;
    const Four y = __builtin_convertvector(x, Four);
    if constexpr (WHOLE) {
        __builtin_nontemporal_store(y, reinterpret_cast<Four *>(a));
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n)
            a[j] = y[j];
}
// The same for four codes, one in each byte.
template <bool WHOLE>
__device__ __forceinline__ unsigned read_codes(const void *p, long long i, long long n)
{
    const unsigned char *a = static_cast<const unsigned char *>(p) + i;
    if constexpr (WHOLE)
        return __builtin_nontemporal_load(reinterpret_cast<const unsigned *>(a));
    unsigned x = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n)
            x |= (unsigned)a[j] << 8 * j;
    return x;
}
template <bool WHOLE>
__device__ __forceinline__ void write_codes(void *p, long long i, long long n, unsigned x)
{
    unsigned char *a = static_cast<unsigned char *>(p) + i;
    if constexpr (WHOLE) {
        __builtin_nontemporal_store(x, reinterpret_cast<unsigned *>(a));
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n)
            a[j] = (unsigned char)(x >> 8 * j);
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
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        x = fmaxf(x, __shfl_xor(x, off));
    return x;
}

__device__ __forceinline__ float finite_abs(float x)
{
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.0f;  // a NaN compares false
}

// Four values over their block's scale as e4m3 codes (what is not finite: NaN);
// is_root: a positive value keeps the smallest code.
__device__ __forceinline__ unsigned encode8(f32x4 x, float inv_scale, bool is_root)
{
    float q[4];
    unsigned bad = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        q[j] = fminf(fmaxf(x[j] * inv_scale, -448.0f), 448.0f);
        if (is_root && x[j] > 0.0f)
            q[j] = fmaxf(q[j], 0x1p-9f);
        if (!(fabsf(x[j]) < INFINITY))
            bad |= 0x7Fu << 8 * j;
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
    return (unsigned)c | bad;
}
__device__ __forceinline__ f32x4 decode8(unsigned c, float scale)
{
    return f32x4{__builtin_amdgcn_cvt_f32_fp8((int)c, 0) * scale, __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * scale,
                 __builtin_amdgcn_cvt_f32_fp8((int)c, 2) * scale, __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * scale};
}

// What a lane reads of a block: four values of each array.
struct Block {
    f32x4 g, p, m, v;  // 8 bits: m[0], v[0] hold the codes
    float ms, vs;
};
template <int BITS, bool WHOLE, class P, class G>
__device__ __forceinline__ Block read_block(const derf_adamw_tensor &t, long long base)
{
    const long long i = base + (threadIdx.x & 63) * 4, block = base / kMomentBlock;
    Block b;
    b.g = read4<WHOLE, G>(t.grad, i, t.n);
    b.p = read4<WHOLE, P>(t.param, i, t.n);
    if (BITS == 8) {
        b.ms = t.m_scale[block];
        b.vs = t.v_scale[block];
        b.m[0] = __uint_as_float(read_codes<WHOLE>(t.m, i, t.n));
        b.v[0] = __uint_as_float(read_codes<WHOLE>(t.v, i, t.n));
    } else {
        b.m = read4<WHOLE, float>(t.m, i, t.n);
        b.v = read4<WHOLE, float>(t.v, i, t.n);
    }
    return b;
}

// One wave's step on the 256 values from `base` on.
template <int BITS, bool WHOLE, class P>
__device__ __forceinline__ void step_block(const derf_adamw_tensor &t, long long base, const Block &b,
                                           const AdamWScalars &c, float gs)
{
    const int lane = threadIdx.x & 63;
    const long long i = base + lane * 4, n = t.n, block = base / kMomentBlock;
    const f32x4 g = b.g * gs;
    f32x4 m = b.m, v = b.v;
    if (BITS == 8) {
        m = decode8(__float_as_uint(b.m[0]), b.ms);
        v = decode8(__float_as_uint(b.v[0]), b.vs);
        v = v * v;
    }
    m = m * c.beta1 + g * c.one_minus_beta1;
    v = v * c.beta2 + (g * g) * c.one_minus_beta2;
    f32x4 root;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        root[j] = sqrtf(v[j]);
    const f32x4 p = b.p * c.decay - m / (root * c.root_scale + c.eps) * c.rate;
    write4<WHOLE, P>(t.param, i, n, p);
    if (t.copy)
        write4<WHOLE, __bf16>(t.copy, i, n, p);
    if (BITS == 32) {
        write4<WHOLE, float>(t.m, i, n, m);
        write4<WHOLE, float>(t.v, i, n, v);
        return;
    }
    // lanes past the end have zeros
    float mmax = 0.0f, rmax = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        mmax = fmaxf(mmax, finite_abs(m[j]));
        rmax = fmaxf(rmax, finite_abs(root[j]));
    }
    const float ms = fmaxf(wave_max(mmax) * (1.0f / 448.0f), 0x1p-120f);
    const float vs = fmaxf(wave_max(rmax) * (1.0f / 448.0f), 0x1p-120f);
    write_codes<WHOLE>(t.m, i, n, encode8(m, 1.0f / ms, false));
    write_codes<WHOLE>(t.v, i, n, encode8(root, 1.0f / vs, true));
    if (lane == 0) {
        t.m_scale[block] = ms;
        t.v_scale[block] = vs;
    }
}

// A work item: each wave takes every fourth of its blocks, and reads one ahead.
template <int BITS, class P, class G>
__device__ __forceinline__ void step_item(const derf_adamw_tensor &t, bool aligned, long long base,
                                          const AdamWScalars &c, float gs)
{
    constexpr int kStep = 4 * kMomentBlock;
    const long long end = base + kItem < t.n ? base + kItem : t.n;
    base += (threadIdx.x >> 6) * kMomentBlock;
    if (aligned && base + kMomentBlock <= end) {
        Block b = read_block<BITS, true, P, G>(t, base);
#pragma unroll 1
        for (; base + kStep + kMomentBlock <= end; base += kStep) {
            const Block next = read_block<BITS, true, P, G>(t, base + kStep);
            step_block<BITS, true, P>(t, base, b, c, gs);
            b = next;
        }
        step_block<BITS, true, P>(t, base, b, c, gs);
        base += kStep;
    }
#pragma unroll 1
    for (; base < end; base += kStep)
        step_block<BITS, false, P>(t, base, read_block<BITS, false, P, G>(t, base), c, gs);
}

template <int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamWEntry *table, int tensors,
                                                         AdamWScalars c, const float *grad_scale)
{
    const AdamWEntry e = table[find_tensor(table, tensors, blockIdx.x)];
    const float gs = grad_scale ? *grad_scale : 1.0f;
    const long long base = (long long)(blockIdx.x - e.first) * kItem;
    const bool pb = e.t.param_precision == DERF_PREC_BF16, gb = e.t.grad_precision == DERF_PREC_BF16;
    if (pb && gb)
        step_item<BITS, __bf16, __bf16>(e.t, e.aligned, base, c, gs);
    else if (pb)
        step_item<BITS, __bf16, float>(e.t, e.aligned, base, c, gs);
    else if (gb)
        step_item<BITS, float, __bf16>(e.t, e.aligned, base, c, gs);
    else
        step_item<BITS, float, float>(e.t, e.aligned, base, c, gs);
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
