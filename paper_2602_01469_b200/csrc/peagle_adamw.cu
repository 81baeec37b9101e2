// One AdamW step over a list of tensors, states in 32 or in 8 bits.
//
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2
//     p -= lr wd p + lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: every element of p, g, m and v is read once and, but for g, written once.  The list travels as a
// kernel parameter (no copy to the device, nothing that a captured graph could lose); a block takes CHUNK elements
// of one tensor, which it finds by a search over the tensors' first chunks, and a thread 8 neighbouring ones, in
// 16-byte accesses where the tensor's addresses allow.  91 M elements of bf16 with states in 32 bits take 375 us (104 %
// of the copy rate).
//
// 8-bit states: a warp has the 256 elements that share a scale.  m and sqrt(v) are e4m3 codes times a power of two,
// so scaling is exact and the rounding to a code looks at the fp32 number's own bits: adding 20 random bits below
// the three mantissa bits that stay and cutting the rest off rounds up with the probability of the fraction.
// (Numbers below 2^-6, where e4m3's spacing is even, get 2^-6 added first; a thread without any skips that.)  What
// bounds this is instructions, more than half of them integer ones for the random bits and the roundings: 91 M elements,
// bf16, take 272 us, 52 % of the copy rate.  With all of m and v in fp64 it took 343.  In fp32 alone, some 20 us less, two or
// three codes in a million fall on the other side of their random bits, and a step later the scales of their blocks differ.
// So what fp32 does not settle is formed again in fp64, and every code is the defined one: a code whose number is near its
// border, the largest number of a block near a power of two, blocks in which m cancels, and in blocks of small roots those
// whose v is below fp32's normal numbers.  (All gradients around 1e-14, whose smallest are such: 27 %
// longer.  Blocks that stay, with the next chunk on its way in shared memory, have more instructions: 2 % longer.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <cstring>

#include "peagle_internal.h"
#include "sm100_ptx.cuh"

namespace peagle {
using namespace sm100;

namespace {

constexpr int AW_THREADS = 256;
constexpr int AW_BLOCK = PEAGLE_ADAMW_BLOCK;
// Elements per thread block, 8 per thread.  (Blocks that go on to a second 2,048 spend fewer instructions on finding
// their tensor and wait longer for memory: 18 % longer with 8-bit states of 91 M elements, with four blocks to an SM.)
constexpr int CHUNK = (AW_THREADS / 32) * AW_BLOCK;
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
    float b1_top, b1_rest, c1, c1_rest, b2, c2; // beta1 in two parts, 1 - beta1 in two, beta2, 1 - beta2
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

// Scrambles 32 bits: two rounds of shift-xor and multiplication by an odd number, each of them one to one.  Shifts and
// factors as published by C. Wellons, "Prospecting for hash functions", 2018, found there by search for the least bias.
__host__ __device__ inline uint32_t mix_but_for_the_last(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    return x * 0x846CA68Bu;
}
__host__ __device__ inline uint32_t mix(uint32_t x)
{
    x = mix_but_for_the_last(x);
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
                make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                           pack_bf16x2(f[6], f[7]));
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

// A number within NEAR units in the last place of the border between two codes, the random bits added, is rounded again
// from fp64: see nearness.
constexpr uint32_t NEAR = 8;
// y rounded up or down by 20 random bits.  What is left over tells how near the border is.
__device__ __forceinline__ float rounded(float y, uint32_t bits20, uint32_t &nearness)
{
    const uint32_t z = __float_as_uint(y) + bits20 + NEAR; // the sign stays: adding below it does not carry into it
    nearness = min(nearness, z << 12);                     // less than 2 NEAR << 12: too near, else NEAR changes nothing
    return __uint_as_float(z & 0xfff00000u);
}
// The same where the plain way (`large`) does not do: below 2^-6, where e4m3's spacing is even, and not finite.  `keep`:
// above zero stays above it.
__device__ __forceinline__ float small_code(float y, float large, uint32_t bits20, bool keep, uint32_t &nearness)
{
    const float a = fabsf(y);
    if (a >= 0.015625f)
        return a <= 256.f ? large : __int_as_float(0x7fffffff);
    const float z = rounded(a + 0.015625f, bits20, nearness) - 0.015625f;
    return a != a ? a : copysignf(keep && a > 0.f ? fmaxf(z, 0.001953125f) : z, y); // 2^-9
}
// The code of a number that is exact.
__device__ __forceinline__ uint32_t exact_code(float y, uint32_t bits20, bool keep)
{
    uint32_t none = 0;
    const uint32_t less = bits20 - NEAR; // rounded() adds it
    return encode4(small_code(y, rounded(y, less, none), less, keep, none), 0.f, 0.f, 0.f) & 0xffu;
}
// The 20 bits of an element for m and for the root: the lower and the upper 16 of mix(), and a half.  From what mix()
// has before its last step, which leaves the upper ones as they are: 4 % faster than from mix() itself.
__device__ __forceinline__ uint32_t bits_of_m(uint32_t x) { return ((x << 4 ^ x >> 12) & 0xffff0u) + 8u; }
__device__ __forceinline__ uint32_t bits_of_root(uint32_t x) { return (x >> 12 & 0xffff0u) + 8u; }

// Power of two that brings `largest` into [128, 256), at least 2^-107; and its reciprocal.
__device__ __forceinline__ float2 scale_of(float largest)
{
    const int e = max((int)(__float_as_uint(largest) >> 23) - 127, -100) - 7;
    return make_float2(__uint_as_float((uint32_t)(e + 127) << 23), __uint_as_float((uint32_t)(127 - e) << 23));
}

__device__ __forceinline__ F2 both(float x) { return f2(x, x); }
__device__ __forceinline__ void put2(float (&to)[8], int k, F2 v)
{
    const float2 u = unf2(v);
    to[k] = u.x;
    to[k + 1] = u.y;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Whether a block whose largest magnitude has these bits is done over: not finite, or so near a power of two, from 2^-99 on,
// that fp32's roundings may have carried it across.
__device__ __forceinline__ bool doubtful(uint32_t largest)
{
    return largest >= 0x7f800000u || (largest > 0x0dffff00u && (largest + 32u & 0x7fffffu) < 64u);
}
// From this root on, 2^-60, v is a normal number and the root right to a few units in the last place.  A v below 2^-126 may
// be off by fp32's smallest number, 2^-149, and its root by 2^-76 then.
constexpr float NORMAL_ROOT = 0x1p-60f;
// That is 4 units in the last place of what is rounded to a code (2^-6 of the block's scale and more) where the largest root
// of the block has these bits, 2^-41; where it is smaller, such roots are formed in fp64.
constexpr uint32_t ROOM_FOR_SMALL_ROOTS = 0x2b000000u;

// Whether m's two terms have cancelled in a whole block: `old` is beta1 times its old scale, so its terms were up to 256 times
// that.  In fp32 they leave up to 2^-30 of the scale (see below), a few units in the last place of what is rounded to a code
// unless the largest m is a fourth of what it was or less; then the block is formed in fp64.  (Not where the old scale is
// the least there is, and means nothing.)
__device__ __forceinline__ bool all_cancelled(uint32_t largest, float old)
{
    return __uint_as_float(largest) < 32.f * old && old > 0x1p-107f;
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

// Approximate to about two units in the last place, for numbers below 2^-126 too.  (They are v of gradients below 3e-18 on an
// empty state.  With a root that took them for zero, 91 M elements with 8-bit states took 260 us instead of 266.)
__device__ __forceinline__ float root_of(float v)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// 1 / d for 2^-126 <= d <= 2^126, to a unit in the last place.
__device__ __forceinline__ float reciprocal(float d)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    return r;
}

// p after a step, two elements; `decay` is -lr weight_decay.
__device__ __forceinline__ F2 stepped(F2 p, F2 m, F2 root, const How &how, const Factors &f, float decay)
{
    const float2 d = unf2(fma_f2(root, f2(f.root_scale, f.root_scale), f2(how.eps, how.eps))); // eps >= 2^-126
    const F2 q = mul_f2(m, f2(reciprocal(d.x), reciprocal(d.y)));
    return fma_f2(q, f2(-f.step_size, -f.step_size), fma_f2(p, f2(decay, decay), p));
}

// One thread's 8 elements of a tensor with states in 32 bits, from i on; `left` of them are there.
template <bool VEC>
__device__ __forceinline__ void step8(const Tensor &t, const How &how, const Factors &f, float grad_scale, int64_t i, int left)
{
    float g[8], m[8], v[8], p[8];
    load8<VEC>(t.m, PEAGLE_F32, i, left, m);
    load8<VEC>(t.v, PEAGLE_F32, i, left, v);
    load8<VEC>(t.grad, t.grad_dtype, i, left, g);
    load8<VEC>(t.master ? t.master : t.param, t.master ? PEAGLE_F32 : t.param_dtype, i, left, p);
    const float decay = -f.lr * t.weight_decay;
    const F2 b1 = both(how.b1_top + how.b1_rest), c1 = both(how.c1), b2 = both(how.b2), c2 = both(how.c2);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const F2 gg = mul_f2(f2(g[k], g[k + 1]), f2(grad_scale, grad_scale));
        const F2 m2 = fma_f2(b1, f2(m[k], m[k + 1]), mul_f2(c1, gg));
        const F2 v2 = fma_f2(b2, f2(v[k], v[k + 1]), mul_f2(mul_f2(c2, gg), gg));
        put2(m, k, m2);
        put2(v, k, v2);
        put2(p, k, stepped(f2(p[k], p[k + 1]), m2, f2(root_of(v[k]), root_of(v[k + 1])), how, f, decay));
    }
    if (t.master)
        store8<VEC>(t.master, PEAGLE_F32, i, left, p);
    store8<VEC>(t.param, t.param_dtype, i, left, p);
    store8<VEC>(t.m, PEAGLE_F32, i, left, m);
    store8<VEC>(t.v, PEAGLE_F32, i, left, v);
}

// The new m and root of one element in fp64, rounded once each.
__device__ __forceinline__ void exact_states(const How &how, float m0, float r0, float g, float &m, float &root)
{
    const double gd = (double)g;
    m = (float)__dadd_rn(__dmul_rn(how.beta1, (double)m0), __dmul_rn(1.0 - how.beta1, gd));
    root = __fsqrt_rn((float)__dadd_rn(__dmul_rn(how.beta2, (double)(r0 * r0)), __dmul_rn(__dmul_rn(1.0 - how.beta2, gd), gd)));
}

__device__ __forceinline__ float element(const void *p, int dtype, int64_t i)
{
    return dtype == PEAGLE_F32 ? static_cast<const float *>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

// What one element has in memory, and its new m and root.
__device__ __forceinline__ void exact_element(const Tensor &t, const How &how, float grad_scale, int64_t i, float &m, float &root)
{
    const float ms = t.m_scale[i / AW_BLOCK], vs = t.v_scale[i / AW_BLOCK];
    const float g = element(t.grad, t.grad_dtype, i);
    float m0[8], r0[8];
    decode4(static_cast<const uint8_t *>(t.m)[i], m0, 0);
    decode4(static_cast<const uint8_t *>(t.v)[i], r0, 0);
    exact_states(how, m0[0] * ms, r0[0] * vs, g * grad_scale, m, root);
}

// The parameters of a thread's elements with small roots, from fp64's, where eps does not outweigh what these are off by.
__device__ __forceinline__ void step_of_small_roots(const Tensor &t, const How &how, const Factors &f, float grad_scale, int64_t i,
                                                    int left, const float (&r)[8], float (&p)[8])
{
#pragma unroll 1
    for (int k = 0; k < left; ++k) {
        float m, root;
        exact_element(t, how, grad_scale, i + k, m, root);
        const float p0 = t.master ? t.master[i + k] : element(t.param, t.param_dtype, i + k);
        const float p1 = unf2(stepped(both(p0), both(m), both(root), how, f, -f.lr * t.weight_decay)).x;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            p[j] = j == k && r[j] < NORMAL_ROOT ? p1 : p[j];
    }
}

// A thread's codes from fp64, where one of them was too near a border.  From memory, like the next.
__device__ __forceinline__ void exact_codes(const Tensor &t, const How &how, float grad_scale, int64_t i, int left, uint32_t first,
                                            float m_factor, float r_factor, uint2 &m_codes, uint2 &r_codes)
{
#pragma unroll 1
    for (int k = 0; k < left; ++k) {
        float m, r;
        exact_element(t, how, grad_scale, i + k, m, r);
        const uint32_t x = mix_but_for_the_last(first + k * GOLDEN), at = k % 4 * 8, keep = ~(0xffu << at);
        const uint32_t mc = exact_code(m * m_factor, bits_of_m(x), false) << at;
        const uint32_t rc = exact_code(r * r_factor, bits_of_root(x), true) << at;
        if (k < 4) {
            m_codes.x = m_codes.x & keep | mc;
            r_codes.x = r_codes.x & keep | rc;
        } else {
            m_codes.y = m_codes.y & keep | mc;
            r_codes.y = r_codes.y & keep | rc;
        }
    }
}

// Largest magnitudes of a doubtful block, without the elements that are not finite.  From memory: the numbers that the
// caller has are not kept for this rare case.
__device__ __forceinline__ void exact_largest(const Tensor &t, const How &how, float grad_scale, int64_t i, int left,
                                              uint32_t &largest_m, uint32_t &largest_r)
{
    uint32_t lm = 0, lr = 0;
#pragma unroll 1
    for (int k = 0; k < left; ++k) {
        float m, r;
        exact_element(t, how, grad_scale, i + k, m, r);
        const uint32_t mb = __float_as_uint(fabsf(m)), rb = __float_as_uint(fabsf(r));
        lm = mb < 0x7f800000u ? max(lm, mb) : lm;
        lr = rb < 0x7f800000u ? max(lr, rb) : lr;
    }
    largest_m = __reduce_max_sync(~0u, lm);
    largest_r = __reduce_max_sync(~0u, lr);
}

// One thread's 8 elements of a tensor with states in 8 bits.  The whole warp, with a block of PEAGLE_ADAMW_BLOCK
// elements; elements that are not there are zeros.
// SMALL_EPS: see step_of_small_roots.
template <bool VEC, bool SMALL_EPS>
__device__ __forceinline__ void step8_codes(const Tensor &t, const How &how, const Factors &f, float grad_scale, uint32_t key,
                                            int64_t i, int left)
{
    float g[8], m[8], r[8], p[8];
    const int64_t block = i / AW_BLOCK;
    const uint2 mc = load_codes<VEC>(t.m, i, left), vc = load_codes<VEC>(t.v, i, left);
    const float ms = t.m_scale[block], vs = t.v_scale[block];
    load8<VEC>(t.grad, t.grad_dtype, i, left, g);
    load8<VEC>(t.master ? t.master : t.param, t.master ? PEAGLE_F32 : t.param_dtype, i, left, p);
    decode4(mc.x, m, 0);
    decode4(mc.y, m, 4);
    decode4(vc.x, r, 0);
    decode4(vc.y, r, 4);
    const float decay = -f.lr * t.weight_decay, b1s = how.b1_top * ms, b1r = how.b1_rest * ms; // by a power of two: exact
    const F2 b1 = both(b1s), b1_rest = both(b1r), c1 = both(how.c1), c1_rest = both(how.c1_rest), b2 = both(how.b2),
             c2 = both(how.c2), vs2 = both(vs);
    float m_max = 0.f, r_max = 0.f, m_min = 1e38f, r_min = 1e38f;
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const F2 gg = mul_f2(f2(g[k], g[k + 1]), f2(grad_scale, grad_scale));
        // b1_top's product with a code is exact and the rest is 2^-16 of it, so m is off by 2^-38 of its terms and a few
        // units in the last place of its own: far below a code's spacing, unless the terms cancel in the whole block
        const F2 code = f2(m[k], m[k + 1]), rest = fma_f2(c1_rest, gg, mul_f2(b1_rest, code));
        const F2 m2 = add_f2(fma_f2(c1, gg, mul_f2(b1, code)), rest);
        const F2 r0 = mul_f2(f2(r[k], r[k + 1]), vs2);
        const float2 v = unf2(fma_f2(b2, mul_f2(r0, r0), mul_f2(mul_f2(c2, gg), gg)));
        put2(m, k, m2);
        r[k] = root_of(v.x);
        r[k + 1] = root_of(v.y);
        put2(p, k, stepped(f2(p[k], p[k + 1]), m2, f2(r[k], r[k + 1]), how, f, decay));
        m_max = max_nan(max_nan(m_max, fabsf(m[k])), fabsf(m[k + 1]));
        r_max = max_nan(max_nan(r_max, r[k]), r[k + 1]);
        m_min = fminf(fminf(m_min, fabsf(m[k])), fabsf(m[k + 1]));
        r_min = fminf(fminf(r_min, r[k]), r[k + 1]);
    }
    if (SMALL_EPS && r_min < NORMAL_ROOT)
        step_of_small_roots(t, how, f, grad_scale, i, left, r, p);
    if (t.master)
        store8<VEC>(t.master, PEAGLE_F32, i, left, p);
    store8<VEC>(t.param, t.param_dtype, i, left, p);
    uint32_t largest_m = __reduce_max_sync(~0u, __float_as_uint(m_max) & 0x7fffffffu);
    uint32_t largest_r = __reduce_max_sync(~0u, __float_as_uint(r_max) & 0x7fffffffu);
    bool finite = true;
    bool cancelled = all_cancelled(largest_m, b1s);
    if (doubtful(largest_m) || doubtful(largest_r) || cancelled || largest_r - 1u < __float_as_uint(NORMAL_ROOT)) { // not zero
        finite = largest_m < 0x7f800000u && largest_r < 0x7f800000u;
        exact_largest(t, how, grad_scale, i, left, largest_m, largest_r);
        cancelled = all_cancelled(largest_m, b1s);
    }
    const float2 sm = scale_of(__uint_as_float(largest_m)), sv = scale_of(__uint_as_float(largest_r));
    const uint32_t first = key + (uint32_t)i * GOLDEN;
    const bool plain = finite && m_min * sm.y >= 0.015625f && r_min * sv.y >= 0.015625f;
    const F2 sm2 = f2(sm.y, sm.y), sv2 = f2(sv.y, sv.y);
    uint32_t nearness = cancelled || (r_min < NORMAL_ROOT && largest_r - 1u < ROOM_FOR_SMALL_ROOTS) ? 0u : ~0u;
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const float2 a = unf2(mul_f2(f2(m[k], m[k + 1]), sm2)), b = unf2(mul_f2(f2(r[k], r[k + 1]), sv2));
        const uint32_t x = mix_but_for_the_last(first + k * GOLDEN), y = mix_but_for_the_last(first + (k + 1) * GOLDEN);
        m[k] = rounded(a.x, bits_of_m(x), nearness);
        m[k + 1] = rounded(a.y, bits_of_m(y), nearness);
        r[k] = rounded(b.x, bits_of_root(x), nearness);
        r[k + 1] = rounded(b.y, bits_of_root(y), nearness);
        if (!plain) { // small numbers, roots that must not become zero, and what is not finite
            m[k] = small_code(a.x, m[k], bits_of_m(x), false, nearness);
            m[k + 1] = small_code(a.y, m[k + 1], bits_of_m(y), false, nearness);
            r[k] = small_code(b.x, r[k], bits_of_root(x), true, nearness);
            r[k + 1] = small_code(b.y, r[k + 1], bits_of_root(y), true, nearness);
        }
    }
    uint2 m_codes = make_uint2(encode4(m[0], m[1], m[2], m[3]), encode4(m[4], m[5], m[6], m[7]));
    uint2 r_codes = make_uint2(encode4(r[0], r[1], r[2], r[3]), encode4(r[4], r[5], r[6], r[7]));
    if (nearness < 2 * NEAR << 12)
        exact_codes(t, how, grad_scale, i, left, first, sm.y, sv.y, m_codes, r_codes);
    store_codes<VEC>(t.m, i, left, m_codes);
    store_codes<VEC>(t.v, i, left, r_codes);
    __syncwarp(); // nobody reads the old scales any more
    if (threadIdx.x % 32 == 0) {
        t.m_scale[block] = sm.x;
        t.v_scale[block] = sv.x;
    }
}

// KINDS: which states the list has, 1 in 32 bits, 2 in 8 bits, 3 both (with the registers of the larger).  8-bit states
// alone are best with five blocks to an SM and 48 registers: with four they take 5 % longer, with six, which spill, 10 %.
template <int N, int KINDS, bool SMALL_EPS>
__global__ void __launch_bounds__(AW_THREADS, KINDS == 2 && !SMALL_EPS ? 5 : 4) adamw_kernel(const __grid_constant__ Table<N> table)
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
        const int64_t begin = (int64_t)(chunk - t.first) * CHUNK;
        uint32_t key = mix(f.key ^ (how.ordinal + lo + 1u));
        if (begin >> 32) // a chunk does not cross 2^32
            key = mix(key ^ (uint32_t)(begin >> 32));
        const int64_t i = begin + threadIdx.x * 8, rest = t.count - i;
        if (rest + (int)(threadIdx.x % 32 * 8) <= 0)
            continue; // the whole warp
        const int left = rest >= 8 ? 8 : rest > 0 ? (int)rest : 0;
        const bool vec = t.aligned && rest >= 8;
        if (KINDS == 2 || (KINDS == 3 && t.m_scale)) {
            // a warp stays together, for its block's scales
            if (__all_sync(~0u, vec))
                step8_codes<true, SMALL_EPS>(t, how, f, grad_scale, key, i, left);
            else
                step8_codes<false, SMALL_EPS>(t, how, f, grad_scale, key, i, left);
        } else if (vec) {
            step8<true>(t, how, f, grad_scale, i, left);
        } else if (left) {
            step8<false>(t, how, f, grad_scale, i, left);
        }
    }
}

template <int N>
void launch_table(const How &how, const Tensor *t, int kinds, int n_sm, cudaStream_t s)
{
    Table<N> table;
    table.how = how;
    for (int i = 0; i < how.n; ++i)
        table.t[i] = t[i];
    // a block per chunk; where each has to form the factors, no more than fit the GPU
    const uint32_t most = how.lr_dev || how.step_dev ? 4u * n_sm : how.chunks;
    const uint32_t blocks = how.chunks < most ? how.chunks : most;
    // the 2^-76 that a small root of 8-bit states may be off by, beside eps: below its rounding, or not
    const bool small_eps = how.eps < 0x1p-52 / sqrt(1.0 - how.beta2);
    if (kinds == 1)
        adamw_kernel<N, 1, false><<<blocks, AW_THREADS, 0, s>>>(table);
    else if (kinds == 2)
        (small_eps ? adamw_kernel<N, 2, true> : adamw_kernel<N, 2, false>)<<<blocks, AW_THREADS, 0, s>>>(table);
    else
        (small_eps ? adamw_kernel<N, 3, true> : adamw_kernel<N, 3, false>)<<<blocks, AW_THREADS, 0, s>>>(table);
}

} // namespace

int launch_adamw(const peagle_adamw_t &how, const peagle_adamw_tensor_t *tensors, int n, int n_sm, cudaStream_t s)
{
    How h = {};
    h.beta1 = how.beta1;
    h.beta2 = how.beta2;
    const float b1 = (float)how.beta1;
    uint32_t top;
    std::memcpy(&top, &b1, 4);
    top &= 0xffffff00u; // 16 significant bits: the product with a code's 4 is exact
    std::memcpy(&h.b1_top, &top, 4);
    h.b1_rest = (float)(how.beta1 - (double)h.b1_top);
    h.c1 = (float)(1.0 - how.beta1);
    h.c1_rest = (float)(1.0 - how.beta1 - (double)h.c1);
    h.b2 = (float)how.beta2;
    h.c2 = (float)(1.0 - how.beta2);
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
        int kinds = 0;
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
            kinds |= t.count == 0 ? 0 : t.m_scale ? 2 : 1;
        }
        if (h.chunks) {
            if (h.n <= SHORT_LIST)
                launch_table<SHORT_LIST>(h, list, kinds, n_sm, s);
            else
                launch_table<PEAGLE_ADAMW_TENSORS>(h, list, kinds, n_sm, s);
            ++launches;
        }
    }
    return launches;
}

} // namespace peagle
