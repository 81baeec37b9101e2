// One AdamW step over a list of tensors, states in 32 or in 8 bits.
//
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2
//     p -= lr wd p + lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// The list travels as a kernel parameter (no copy to the device, nothing that a captured graph could lose); a
// block takes CHUNK elements of one tensor and finds it by a search over the tensors' first chunks.
//
// 8-bit states: a warp has the 256 elements that share a scale, 8 per lane.  m and sqrt(v) are e4m3 codes
// times a power of two, so scaling is exact and the rounding to a code looks at the fp32 number's own bits:
// adding 20 random bits below the three mantissa bits that stay and cutting the rest off rounds up with the
// probability of the fraction.  (Numbers below 2^-6, where e4m3's spacing is even, get 2^-6 added first.)
// The new m and v are formed in fp64 and rounded once to fp32, so that the codes do not depend on how the
// arithmetic is ordered.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>

#include "peagle_internal.h"

namespace peagle {

namespace {

constexpr int AW_THREADS = 256;
constexpr int AW_BLOCK = PEAGLE_ADAMW_BLOCK;
constexpr int CHUNK = (AW_THREADS / 32) * AW_BLOCK; // elements per thread block
constexpr uint32_t GOLDEN = 0x9E3779B9u;            // 2^32 / golden ratio

struct Tensor {
    void *param;
    const void *grad;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t count;
    uint32_t first; // chunk
    float weight_decay;
    int8_t param_dtype, grad_dtype;
};

struct How {
    double beta1, beta2, log_beta1, log_beta2;
    float lr, eps;
    const float *lr_dev, *grad_scale_dev;
    const int64_t *step_dev;
    int64_t step;
    uint32_t seed, ordinal; // place of the first tensor in the caller's list
    int n;
};

template <int N>
struct Table {
    How how;
    Tensor t[N];
};
static_assert(sizeof(Table<PEAGLE_ADAMW_TENSORS>) <= 32764, "kernel parameters");

// Scrambles 32 bits: two rounds of shift-xor and multiplication by an odd number, each of them one to one.
__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ x >> 16;
}

__device__ __forceinline__ float load_any(const void *p, int dtype, int64_t i)
{
    return dtype == PEAGLE_F32 ? static_cast<const float *>(p)[i]
                               : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ float decode(uint8_t c)
{
    __nv_fp8_e4m3 f;
    f.__x = c;
    return (float)f;
}

// y rounded up or down to an e4m3 number, by 16 random bits; |y| <= 256.  `keep`: not to zero (y >= 0).
__device__ __forceinline__ uint8_t encode(float y, uint32_t bits16, bool keep)
{
    float z = fabsf(y);
    if (!(z <= 256.f))
        return 0x7f; // NaN
    const bool small = z < 0.015625f;
    if (small)
        z += 0.015625f;
    z = __uint_as_float((__float_as_uint(z) + (bits16 << 4) + 8u) & 0xfff00000u);
    if (small)
        z -= 0.015625f;
    if (keep)
        z = fmaxf(z, 0.001953125f); // 2^-9
    return __nv_fp8_e4m3(copysignf(z, y)).__x;
}

// Power of two that brings `largest` into [128, 256), at least 2^-107; and its reciprocal.
__device__ __forceinline__ float2 scale_of(float largest)
{
    const int e = max((int)(__float_as_uint(largest) >> 23) - 127, -100) - 7;
    return make_float2(__uint_as_float((uint32_t)(e + 127) << 23), __uint_as_float((uint32_t)(127 - e) << 23));
}

__device__ __forceinline__ float warp_max(float v)
{
    for (int o = 16; o; o >>= 1)
        v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

struct Factors {
    float lr, step_size, root_scale; // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float grad_scale;
    uint32_t key;
};

__device__ __forceinline__ Factors factors(const How &h)
{
    Factors f;
    const int64_t step = h.step_dev ? *h.step_dev : h.step;
    f.lr = h.lr_dev ? *h.lr_dev : h.lr;
    f.step_size = (float)(f.lr / -expm1((double)step * h.log_beta1));
    f.root_scale = (float)(1.0 / sqrt(-expm1((double)step * h.log_beta2)));
    f.grad_scale = h.grad_scale_dev ? *h.grad_scale_dev : 1.f;
    f.key = mix(h.seed + (uint32_t)step * GOLDEN);
    return f;
}

template <int N>
__global__ void __launch_bounds__(AW_THREADS) adamw_kernel(const __grid_constant__ Table<N> table)
{
    const How &how = table.how;
    __shared__ Factors shared_f;
    if (threadIdx.x == 0)
        shared_f = factors(how);
    __syncthreads();
    const Factors f = shared_f;
    int lo = 0, hi = how.n - 1; // the last tensor whose first chunk is not past this one
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table.t[mid].first <= blockIdx.x)
            lo = mid;
        else
            hi = mid - 1;
    }
    const Tensor &t = table.t[lo];
    const int lane = threadIdx.x & 31;
    const int64_t base = (int64_t)(blockIdx.x - t.first) * CHUNK + (threadIdx.x >> 5) * AW_BLOCK;
    if (base >= t.count)
        return; // a whole warp
    const int64_t block = base / AW_BLOCK;
    const bool eight = t.m_scale != nullptr;
    const float b1 = (float)how.beta1, c1 = (float)(1.0 - how.beta1), b2 = (float)how.beta2, c2 = (float)(1.0 - how.beta2);
    float m[8], root[8];
    const float ms = eight ? t.m_scale[block] : 1.f, vs = eight ? t.v_scale[block] : 1.f;
    float m_max = 0.f, r_max = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t i = base + lane + 32 * k;
        m[k] = root[k] = 0.f;
        if (i >= t.count)
            continue;
        const float g = load_any(t.grad, t.grad_dtype, i) * f.grad_scale;
        float v;
        if (eight) {
            const float m0 = decode(static_cast<const uint8_t *>(t.m)[i]) * ms;
            const float r0 = decode(static_cast<const uint8_t *>(t.v)[i]) * vs;
            m[k] = (float)__dadd_rn(__dmul_rn(how.beta1, (double)m0), __dmul_rn(1.0 - how.beta1, (double)g));
            v = (float)__dadd_rn(__dmul_rn(how.beta2, (double)(r0 * r0)),
                                 __dmul_rn(__dmul_rn(1.0 - how.beta2, (double)g), (double)g));
        } else {
            float *mp = static_cast<float *>(t.m) + i, *vp = static_cast<float *>(t.v) + i;
            *mp = m[k] = fmaf(b1, *mp, c1 * g);
            *vp = v = fmaf(b2, *vp, c2 * g * g);
        }
        root[k] = __fsqrt_rn(v);
        const float update = m[k] / fmaf(root[k], f.root_scale, (float)how.eps) * f.step_size;
        float p = t.master ? t.master[i] : load_any(t.param, t.param_dtype, i);
        p = fmaf(-f.lr * t.weight_decay, p, p) - update;
        if (t.master)
            t.master[i] = p;
        if (t.param_dtype == PEAGLE_F32)
            static_cast<float *>(t.param)[i] = p;
        else
            static_cast<__nv_bfloat16 *>(t.param)[i] = __float2bfloat16_rn(p);
        if (fabsf(m[k]) <= 3.4028235e38f)
            m_max = fmaxf(m_max, fabsf(m[k]));
        if (root[k] <= 3.4028235e38f)
            r_max = fmaxf(r_max, root[k]);
    }
    if (!eight)
        return;
    const float2 sm = scale_of(warp_max(m_max)), sv = scale_of(warp_max(r_max));
    uint32_t key = mix(f.key ^ (how.ordinal + (uint32_t)lo + 1u));
    if (base >> 32)
        key = mix(key ^ (uint32_t)(base >> 32));
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t i = base + lane + 32 * k;
        if (i >= t.count)
            continue;
        const uint32_t bits = mix(key + (uint32_t)i * GOLDEN);
        static_cast<uint8_t *>(t.m)[i] = encode(m[k] * sm.y, bits & 0xffffu, false);
        static_cast<uint8_t *>(t.v)[i] = encode(root[k] * sv.y, bits >> 16, root[k] > 0.f);
    }
    if (lane == 0) {
        t.m_scale[block] = sm.x;
        t.v_scale[block] = sv.x;
    }
}

} // namespace

int launch_adamw(const peagle_adamw_t &how, const peagle_adamw_tensor_t *tensors, int n, int n_sm, cudaStream_t s)
{
    (void)n_sm;
    int launches = 0;
    for (int from = 0; from < n;) {
        Table<PEAGLE_ADAMW_TENSORS> table = {};
        How &h = table.how;
        h.beta1 = how.beta1;
        h.beta2 = how.beta2;
        h.log_beta1 = std::log(how.beta1);
        h.log_beta2 = std::log(how.beta2);
        h.lr = (float)how.lr;
        h.eps = (float)how.eps;
        h.lr_dev = how.lr_dev;
        h.grad_scale_dev = how.grad_scale_dev;
        h.step_dev = how.step_dev;
        h.step = how.step;
        h.seed = how.seed;
        h.ordinal = (uint32_t)from;
        uint32_t chunks = 0;
        for (; h.n < PEAGLE_ADAMW_TENSORS && from < n; ++from) {
            const peagle_adamw_tensor_t &t = tensors[from];
            Tensor &d = table.t[h.n++];
            d.param = t.param;
            d.grad = t.grad;
            d.master = t.master;
            d.m = t.m;
            d.v = t.v;
            d.m_scale = t.m_scale;
            d.v_scale = t.v_scale;
            d.count = t.count;
            d.first = chunks;
            d.weight_decay = t.weight_decay;
            d.param_dtype = (int8_t)t.param_dtype;
            d.grad_dtype = (int8_t)t.grad_dtype;
            chunks += (uint32_t)((t.count + CHUNK - 1) / CHUNK);
        }
        if (chunks) {
            adamw_kernel<PEAGLE_ADAMW_TENSORS><<<chunks, AW_THREADS, 0, s>>>(table);
            ++launches;
        }
    }
    return launches;
}

} // namespace peagle
