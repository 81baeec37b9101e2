// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the gradient.
//
// With m the row's maximum, t_j = scale (x_j - m), S = sum exp(t_j), E = sum exp(t_j) t_j:
//     lse = scale m + log S,   logprob = t_token - log S,   entropy = log S - E / S
// (the differences to m are formed first, so that logprob and entropy do not lose the digits that a large
// m would take).  Backward, with log p = scale x - lse:
//     dx_j = scale ( g ([j = token] - p_j) - h p_j (log p_j + entropy) ).
#include <cuda_bf16.h>

#include "peagle_internal.h"
#include "sm100_ptx.cuh"

namespace peagle {
using namespace sm100;

namespace {

constexpr int LP_THREADS = 256;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float T_FLOOR = -300.f; // below this, in powers of two, a probability is zero in fp32
constexpr float LSE_LARGE = 8192.f; // from here on fp32 keeps less than 2^-10 of a log-sum-exp
constexpr float NEG_INF = -__builtin_huge_valf();

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f32(float *p, float v) { *p = v; }
__device__ __forceinline__ void from_f32(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// Whole numbers in the order of the floats; -0 becomes 0.  Never 0 for a number.
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_key(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }

// Larger value first, then the lower id.
__device__ __forceinline__ uint64_t rank_key(float x, int id) { return (uint64_t)order_key(x) << 32 | (uint32_t)~id; }

template <class V, class F>
__device__ __forceinline__ V block_join(V v, F f)
{
    __shared__ V part[LP_THREADS / 32];
    for (int o = 16; o; o >>= 1)
        v = f(v, __shfl_xor_sync(~0u, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
    for (int i = 1; i < LP_THREADS / 32; ++i)
        v = f(v, part[i]);
    return v;
}

// Writes a row's outputs but the top alternatives; log S as it returns is what they need.
__device__ __forceinline__ float write_row(const LogprobArgs &a, int r, float m, float S, float E, float x_token, int token)
{
    const float ms = m * a.scale;
    float lse, logS = logf(S), H = logS - E * LN2 / S, lp = (x_token - m) * a.scale - logS;
    lse = ms + logS;
    if (ms == -NEG_INF || !(S == S))
        lse = H = lp = logS = __int_as_float(0x7fffffff);
    else if (ms == NEG_INF) {
        lse = lp = NEG_INF;
        H = 0.f;
    }
    if (token == -1)
        lp = 0.f;
    else if (token < 0 || token >= a.vocab) {
        lp = __int_as_float(0x7fffffff);
        if (a.logprob)
            atomicCAS(a.status, 0, PEAGLE_ERR_BAD_META);
    }
    if (a.logprob)
        a.logprob[r] = lp;
    if (a.lse)
        a.lse[r] = lse;
    if (a.entropy)
        a.entropy[r] = H;
    return logS;
}

// One of the top alternatives of a row: its place in the order, its logit and id.
__device__ __forceinline__ void write_top(const LogprobArgs &a, int r, int place, uint64_t key, float m, float logS)
{
    const float x = from_key((uint32_t)(key >> 32));
    const bool none = logS != logS, empty = m * a.scale == NEG_INF;
    a.top[(size_t)r * a.top_k + place] = none ? logS : empty ? NEG_INF : (x - m) * a.scale - logS;
    a.ids[(size_t)r * a.top_k + place] = none ? -1 : (int)~(uint32_t)key;
}

template <class T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_fwd_rows(const LogprobArgs a)
{
    const int r = blockIdx.x;
    const T *x = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
    float m = NEG_INF;
    for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS)
        m = fmaxf(m, to_f32(x[j]));
    m = block_join(m, [](float p, float q) { return fmaxf(p, q); });
    const float from = m == NEG_INF ? 0.f : m, sl = a.scale * LOG2E;
    float S = 0.f, E = 0.f;
    for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS) {
        const float t = (to_f32(x[j]) - from) * sl, e = exp2f(t);
        S += e;
        E = fmaf(e, fmaxf(t, T_FLOOR), E);
    }
    S = block_join(S, [](float p, float q) { return p + q; });
    E = block_join(E, [](float p, float q) { return p + q; });
    const int token = a.tokens ? a.tokens[r] : -1;
    float logS = 0.f;
    __shared__ float shared_logS;
    if (threadIdx.x == 0)
        shared_logS = write_row(a, r, m, S, E, token >= 0 && token < a.vocab ? to_f32(x[token]) : 0.f, token);
    __syncthreads();
    logS = shared_logS;
    uint64_t last = ~0ull;
    for (int i = 0; i < a.top_k; ++i) {
        uint64_t best = 0;
        for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS) {
            const uint64_t k = rank_key(to_f32(x[j]), j);
            if (k < last && k > best)
                best = k;
        }
        last = block_join(best, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
        if (threadIdx.x == 0)
            write_top(a, r, i, last, m, logS);
    }
}

template <class T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_bwd_rows(const LogprobArgs a)
{
    const int r = blockIdx.x;
    const T *x = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
    T *d = static_cast<T *>(a.dlogits) + (size_t)r * a.ldd;
    const int token = a.g_lp ? a.tokens[r] : -1;
    const bool given = token >= 0 && token < a.vocab;
    const float g = given ? a.g_lp[r] : 0.f, h = a.g_h ? a.g_h[r] : 0.f, lse = a.lse_in[r];
    const float H = a.g_h ? a.entropy_in[r] : 0.f;
    const bool zero = (g == 0.f && h == 0.f) || lse == NEG_INF;
    // t = (x - from) scale - off; from the row itself where lse has no digits left for p
    float from = 0.f, off = lse;
    const bool again = !zero && fabsf(lse) >= LSE_LARGE;
    if (again) {
        float m = NEG_INF, S = 0.f;
        for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS)
            m = fmaxf(m, to_f32(x[j]));
        from = block_join(m, [](float p, float q) { return fmaxf(p, q); });
        for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS)
            S += exp2f((to_f32(x[j]) - from) * a.scale * LOG2E);
        off = logf(block_join(S, [](float p, float q) { return p + q; }));
    }
    for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS) {
        float v = 0.f;
        if (!zero) {
            const float xj = to_f32(x[j]);
            const float t = again ? (xj - from) * a.scale - off : fmaf(xj, a.scale, -off), p = exp2f(t * LOG2E);
            v = p * (-g - h * (fmaxf(t, T_FLOOR) + H));
            if (j == token) // 1 - p without the digits that p near 1 would take
                v = -g * expm1f(t) - p * h * (fmaxf(t, T_FLOOR) + H);
        }
        from_f32(d + j, v * a.scale);
    }
}

} // namespace

int launch_logprobs_fwd(const LogprobArgs &a, int n_sm, cudaStream_t s)
{
    (void)n_sm;
    if (a.dtype == PEAGLE_F32)
        logprobs_fwd_rows<float><<<a.rows, LP_THREADS, 0, s>>>(a);
    else
        logprobs_fwd_rows<__nv_bfloat16><<<a.rows, LP_THREADS, 0, s>>>(a);
    return 1;
}

int launch_logprobs_bwd(const LogprobArgs &a, int n_sm, cudaStream_t s)
{
    (void)n_sm;
    if (a.dtype == PEAGLE_F32)
        logprobs_bwd_rows<float><<<a.rows, LP_THREADS, 0, s>>>(a);
    else
        logprobs_bwd_rows<__nv_bfloat16><<<a.rows, LP_THREADS, 0, s>>>(a);
    return 1;
}

} // namespace peagle
