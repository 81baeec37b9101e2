// One AdamW step over a list of tensors, states in 32 or in 8 bits.
//
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2
//     p -= lr wd p + lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: every element of p, g, m and v is read once and, but for g, written once.  The list travels as a
// kernel parameter (no copy to the device, nothing that a captured graph could lose); a block takes CHUNK elements
// of one tensor, which it finds by a search over the tensors' first chunks, and a thread 8 neighbouring ones, in
// 16-byte accesses where the tensor's addresses allow.
//
// 8-bit states: a warp has the 256 elements that share a scale.  m and sqrt(v) are e4m3 codes times a power of two,
// so scaling is exact and the rounding to a code looks at the fp32 number's own bits: adding 20 random bits below
// the three mantissa bits that stay and cutting the rest off rounds up with the probability of the fraction.
// (Numbers below 2^-6, where e4m3's spacing is even, get 2^-6 added first.)  The new m and v are formed in fp64 and
// rounded once to fp32, so that the codes do not depend on how the arithmetic is ordered.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "peagle_internal.h"
#include "sm100_ptx.cuh"

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
    bool aligned; // 16-byte pieces of all (8-byte ones of codes)
};

// What a step multiplies by; on the host, or by every block where lr or the step's number are on the device.
struct Factors {
    float lr, step_size, root_scale; // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    uint32_t key;                    // of the random bits: seed and step
};

struct How {
    double beta1, beta2;
    float eps;
    uint32_t seed, ordinal; // place of the first tensor in the caller's list
    uint32_t chunks;
    int n;
    const float *grad_scale_dev;
    Factors factors;
    // with lr_dev or step_dev
    const float *lr_dev;
    const int64_t *step_dev;
    int64_t step;
    float lr;
    double log_beta1, log_beta2;
};

template <int N>
struct Table {
    How how;
    Tensor t[N];
};
constexpr int SHORT_LIST = 32; // tensors of a smaller kernel parameter, which takes less time to launch with
static_assert(sizeof(Table<PEAGLE_ADAMW_TENSORS>) <= 32764, "kernel parameters");

// Scrambles 32 bits: two rounds of shift-xor and multiplication by an odd number, each of them one to one.
__host__ __device__ inline uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ x >> 16;
}

// 8 neighbouring numbers as fp32, `left` of which are there (the others 0); VEC: all are, on 16-byte addresses (8-byte
// ones for codes).
template <bool VEC>
__device__ __forceinline__ void load8(const void *p, int dtype, int64_t i, int left, float (&f)[8])
{
    if (dtype == PEAGLE_F32) {
        const float *q = static_cast<const float *>(p) + i;
        if (VEC) {
            const float4 a = reinterpret_cast<const float4 *>(q)[0], b = reinterpret_cast<const float4 *>(q)[1];
            f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                f[k] = k < left ? q[k] : 0.f;
        }
    } else {
        const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p) + i;
        if (VEC) {
            const uint4 a = *reinterpret_cast<const uint4 *>(q);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[2 * k] = __uint_as_float(w[k] << 16);
                f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                f[k] = k < left ? __bfloat162float(q[k]) : 0.f;
        }
    }
}

template <bool VEC>
__device__ __forceinline__ void store8(void *p, int dtype, int64_t i, int left, const float (&f)[8])
{
    if (dtype == PEAGLE_F32) {
        float *q = static_cast<float *>(p) + i;
        if (VEC) {
            reinterpret_cast<float4 *>(q)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4 *>(q)[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left)
                    q[k] = f[k];
        }
    } else {
        __nv_bfloat16 *q = static_cast<__nv_bfloat16 *>(p) + i;
        if (VEC) {
            *reinterpret_cast<uint4 *>(q) =
                make_uint4(sm100::pack_bf16x2(f[0], f[1]), sm100::pack_bf16x2(f[2], f[3]), sm100::pack_bf16x2(f[4], f[5]),
                           sm100::pack_bf16x2(f[6], f[7]));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < left)
                    q[k] = __float2bfloat16_rn(f[k]);
        }
    }
}

template <bool VEC>
__device__ __forceinline__ uint2 load_codes(const void *p, int64_t i, int left)
{
    const uint8_t *q = static_cast<const uint8_t *>(p) + i;
    if constexpr (VEC) {
        return *reinterpret_cast<const uint2 *>(q);
    } else {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < left)
                w[k / 4] |= (uint32_t)q[k] << k % 4 * 8;
        return make_uint2(w[0], w[1]);
    }
}

template <bool VEC>
__device__ __forceinline__ void store_codes(void *p, int64_t i, int left, uint2 c)
{
    uint8_t *q = static_cast<uint8_t *>(p) + i;
    if constexpr (VEC) {
        *reinterpret_cast<uint2 *>(q) = c;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < left)
                q[k] = (uint8_t)((k < 4 ? c.x : c.y) >> k % 4 * 8);
    }
}

// Four codes as fp32.
__device__ __forceinline__ void decode4(uint32_t c, float (&f)[8], int at)
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(c >> 16 * k)));
        const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        f[at + 2 * k] = v.x;
        f[at + 2 * k + 1] = v.y;
    }
}

// Four fp32 numbers that are e4m3 numbers, or NaN, as codes.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)hi << 16 | lo;
}

// y rounded up or down to an e4m3 number, by 16 random bits; |y| <= 256, anything else gives NaN.  `keep`: not to
// zero (y >= 0).
__device__ __forceinline__ float to_e4m3(float y, uint32_t bits16, bool keep)
{
    const float a = fabsf(y);
    const float shift = a < 0.015625f ? 0.015625f : 0.f;
    float z = __uint_as_float((__float_as_uint(a + shift) + (bits16 << 4) + 8u) & 0xfff00000u) - shift;
    if (keep)
        z = fmaxf(z, 0.001953125f); // 2^-9
    return a <= 256.f ? copysignf(z, y) : __int_as_float(0x7fffffff);
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

__host__ __device__ inline Factors factors(const How &h, float lr, int64_t step)
{
    Factors f;
    f.lr = lr;
    f.step_size = (float)(lr / -expm1((double)step * h.log_beta1));
    f.root_scale = (float)(1.0 / sqrt(-expm1((double)step * h.log_beta2)));
    f.key = mix(h.seed + (uint32_t)step * GOLDEN);
    return f;
}

// One thread's 8 elements of a tensor, from i on; `left` of them are there.  EIGHT: states in 8 bits, a whole warp
// with a block of PEAGLE_ADAMW_BLOCK elements, the thread's 8 perhaps none.
template <bool VEC, bool EIGHT>
__device__ __forceinline__ void step8(const Tensor &t, const How &how, const Factors &f, float grad_scale,
                                      uint32_t ordinal, int64_t i, int left)
{
    float g[8], m[8], v[8], p[8];
    const int64_t block = i / AW_BLOCK;
    float ms, vs;
    uint2 mc, vc;
    if (EIGHT) {
        mc = load_codes<VEC>(t.m, i, left);
        vc = load_codes<VEC>(t.v, i, left);
        ms = t.m_scale[block];
        vs = t.v_scale[block];
    } else {
        load8<VEC>(t.m, PEAGLE_F32, i, left, m);
        load8<VEC>(t.v, PEAGLE_F32, i, left, v);
    }
    load8<VEC>(t.grad, t.grad_dtype, i, left, g);
    load8<VEC>(t.master ? t.master : t.param, t.master ? PEAGLE_F32 : t.param_dtype, i, left, p);
    if (EIGHT) {
        decode4(mc.x, m, 0);
        decode4(mc.y, m, 4);
        decode4(vc.x, v, 0);
        decode4(vc.y, v, 4);
    }
    const float b1 = (float)how.beta1, c1 = (float)(1.0 - how.beta1), b2 = (float)how.beta2, c2 = (float)(1.0 - how.beta2);
    float m_max = 0.f, r_max = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        g[k] *= grad_scale;
        if (EIGHT) {
            const float m0 = m[k] * ms, r0 = v[k] * vs;
            const double gd = (double)g[k];
            m[k] = (float)__dadd_rn(__dmul_rn(how.beta1, (double)m0), __dmul_rn(1.0 - how.beta1, gd));
            v[k] = (float)__dadd_rn(__dmul_rn(how.beta2, (double)(r0 * r0)), __dmul_rn(__dmul_rn(1.0 - how.beta2, gd), gd));
        } else {
            m[k] = fmaf(b1, m[k], c1 * g[k]);
            v[k] = fmaf(b2, v[k], c2 * g[k] * g[k]);
        }
        const float root = __fsqrt_rn(v[k]);
        const float update = __fdividef(m[k], fmaf(root, f.root_scale, how.eps)) * f.step_size;
        p[k] = fmaf(-f.lr * t.weight_decay, p[k], p[k]) - update;
        if (EIGHT) {
            v[k] = root;
            if (fabsf(m[k]) <= 3.4028235e38f)
                m_max = fmaxf(m_max, fabsf(m[k]));
            if (root <= 3.4028235e38f)
                r_max = fmaxf(r_max, root);
        }
    }
    if (t.master)
        store8<VEC>(t.master, PEAGLE_F32, i, left, p);
    store8<VEC>(t.param, t.param_dtype, i, left, p);
    if (!EIGHT) {
        store8<VEC>(t.m, PEAGLE_F32, i, left, m);
        store8<VEC>(t.v, PEAGLE_F32, i, left, v);
        return;
    }
    const float2 sm = scale_of(warp_max(m_max)), sv = scale_of(warp_max(r_max));
    uint32_t key = mix(f.key ^ (ordinal + 1u));
    if (i >> 32)
        key = mix(key ^ (uint32_t)(i >> 32));
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t bits = mix(key + (uint32_t)(i + k) * GOLDEN);
        m[k] = to_e4m3(m[k] * sm.y, bits & 0xffffu, false);
        v[k] = to_e4m3(v[k] * sv.y, bits >> 16, v[k] > 0.f);
    }
    store_codes<VEC>(t.m, i, left, make_uint2(encode4(m[0], m[1], m[2], m[3]), encode4(m[4], m[5], m[6], m[7])));
    store_codes<VEC>(t.v, i, left, make_uint2(encode4(v[0], v[1], v[2], v[3]), encode4(v[4], v[5], v[6], v[7])));
    if (threadIdx.x % 32 == 0) {
        t.m_scale[block] = sm.x;
        t.v_scale[block] = sv.x;
    }
}

template <int N>
__global__ void __launch_bounds__(AW_THREADS) adamw_kernel(const __grid_constant__ Table<N> table)
{
    const How &how = table.how;
    Factors f = how.factors;
    if (how.lr_dev || how.step_dev) { // in fp64, so by one thread
        __shared__ Factors shared_f;
        if (threadIdx.x == 0)
            shared_f = factors(how, how.lr_dev ? *how.lr_dev : how.lr, how.step_dev ? *how.step_dev : how.step);
        __syncthreads();
        f = shared_f;
    }
    const float grad_scale = how.grad_scale_dev ? *how.grad_scale_dev : 1.f;
    for (uint32_t chunk = blockIdx.x; chunk < how.chunks; chunk += gridDim.x) {
        int lo = 0, hi = how.n - 1; // the last tensor whose first chunk is not past this one
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (table.t[mid].first <= chunk)
                lo = mid;
            else
                hi = mid - 1;
        }
        const Tensor &t = table.t[lo];
        const int64_t i = (int64_t)(chunk - t.first) * CHUNK + threadIdx.x * 8;
        const int64_t rest = t.count - i;
        const int left = rest >= 8 ? 8 : rest > 0 ? (int)rest : 0;
        const bool vec = t.aligned && rest >= 8;
        if (t.m_scale) {
            // a warp stays together, for its block's scales
            if (__all_sync(~0u, vec))
                step8<true, true>(t, how, f, grad_scale, how.ordinal + lo, i, left);
            else if (__any_sync(~0u, left > 0))
                step8<false, true>(t, how, f, grad_scale, how.ordinal + lo, i, left);
        } else if (vec) {
            step8<true, false>(t, how, f, grad_scale, how.ordinal + lo, i, left);
        } else if (left) {
            step8<false, false>(t, how, f, grad_scale, how.ordinal + lo, i, left);
        }
    }
}

template <int N>
void launch_table(const How &how, const Tensor *t, int n_sm, cudaStream_t s)
{
    Table<N> table;
    table.how = how;
    for (int i = 0; i < how.n; ++i)
        table.t[i] = t[i];
    // a block per chunk; where each has to form the factors, no more than fit the GPU
    const uint32_t most = how.lr_dev || how.step_dev ? 4u * n_sm : how.chunks;
    adamw_kernel<N><<<how.chunks < most ? how.chunks : most, AW_THREADS, 0, s>>>(table);
}

} // namespace

int launch_adamw(const peagle_adamw_t &how, const peagle_adamw_tensor_t *tensors, int n, int n_sm, cudaStream_t s)
{
    How h = {};
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
    if (!how.lr_dev && !how.step_dev)
        h.factors = factors(h, h.lr, h.step);
    int launches = 0;
    for (int from = 0; from < n;) {
        Tensor list[PEAGLE_ADAMW_TENSORS];
        h.ordinal = (uint32_t)from;
        h.chunks = 0;
        for (h.n = 0; h.n < PEAGLE_ADAMW_TENSORS && from < n; ++from) {
            const peagle_adamw_tensor_t &t = tensors[from];
            Tensor &d = list[h.n++];
            d.param = t.param;
            d.grad = t.grad;
            d.master = t.master;
            d.m = t.m;
            d.v = t.v;
            d.m_scale = t.m_scale;
            d.v_scale = t.v_scale;
            d.count = t.count;
            d.first = h.chunks;
            d.weight_decay = t.weight_decay;
            d.param_dtype = (int8_t)t.param_dtype;
            d.grad_dtype = (int8_t)t.grad_dtype;
            const uintptr_t states = reinterpret_cast<uintptr_t>(t.m) | reinterpret_cast<uintptr_t>(t.v);
            d.aligned = ((reinterpret_cast<uintptr_t>(t.param) | reinterpret_cast<uintptr_t>(t.grad) |
                          reinterpret_cast<uintptr_t>(t.master)) % 16 == 0) &&
                        states % (t.m_scale ? 8 : 16) == 0;
            h.chunks += (uint32_t)((t.count + CHUNK - 1) / CHUNK);
        }
        if (h.chunks) {
            if (h.n <= SHORT_LIST)
                launch_table<SHORT_LIST>(h, list, n_sm, s);
            else
                launch_table<PEAGLE_ADAMW_TENSORS>(h, list, n_sm, s);
            ++launches;
        }
    }
    return launches;
}

} // namespace peagle
