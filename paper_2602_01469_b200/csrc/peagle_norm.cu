// Layer norm and RMS norm of rows, forward and backward.
//
// Forward: one read of the row for its mean, one for the mean square of what is left, one to write
// y = (x - mu) rstd w + b.  Backward, with xh = (x - mu) rstd and u = dy w:
//     dx = rstd (u - mean(u) - xh mean(u xh)),   dw += sum_rows dy xh,   db += sum_rows dy.
// All sums are fp32 and have a fixed order.
#include <cuda_bf16.h>

#include <algorithm>

#include "peagle_internal.h"

namespace peagle {

namespace {

constexpr int ROW_THREADS = 256;
constexpr int COL_PARTS = 64; // parts of the rows that the column sums are made in

template <class T>
__device__ __forceinline__ float load1(const T *p);
template <>
__device__ __forceinline__ float load1(const float *p) { return *p; }
template <>
__device__ __forceinline__ float load1(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float load_w(const void *w, int dtype, int c, float absent)
{
    if (!w)
        return absent;
    return dtype == PEAGLE_F32 ? static_cast<const float *>(w)[c]
                               : __bfloat162float(static_cast<const __nv_bfloat16 *>(w)[c]);
}

__device__ __forceinline__ float2 block_sum(float a, float b)
{
    __shared__ float2 part[ROW_THREADS / 32];
    for (int o = 16; o; o >>= 1) {
        a += __shfl_xor_sync(~0u, a, o);
        b += __shfl_xor_sync(~0u, b, o);
    }
    __syncthreads(); // an earlier sum has been read
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 s = part[0];
    for (int i = 1; i < ROW_THREADS / 32; ++i) {
        s.x += part[i].x;
        s.y += part[i].y;
    }
    return s;
}

template <class T>
__global__ void __launch_bounds__(ROW_THREADS) norm_fwd_rows(const NormArgs a)
{
    for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.X) + (size_t)r * a.ldx;
        T *y = static_cast<T *>(a.Y) + (size_t)r * a.ldy;
        float mu = 0.f;
        if (a.kind == PEAGLE_NORM_LAYER) {
            float s = 0.f;
            for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS)
                s += load1(x + c);
            mu = block_sum(s, 0.f).x / a.cols;
        }
        float s = 0.f, q = 0.f;
        for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS) {
            const float d = load1(x + c) - mu;
            s += d;
            q = fmaf(d, d, q);
        }
        const float2 t = block_sum(s, q);
        // the rounding of mu is taken out of both
        const float left = a.kind == PEAGLE_NORM_LAYER ? t.x / a.cols : 0.f;
        mu += left;
        const float var = t.y / a.cols - left * left;
        const float rstd = rsqrtf((var < 0.f ? 0.f : var) + a.eps); // a NaN stays one
        for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS)
            store1(y + c, fmaf((load1(x + c) - mu) * rstd, load_w(a.weight, a.w_dtype, c, 1.f),
                               load_w(a.bias, a.w_dtype, c, 0.f)));
        if (threadIdx.x == 0) {
            if (a.mean)
                a.mean[r] = mu;
            if (a.rstd)
                a.rstd[r] = rstd;
        }
    }
}

template <class T>
__global__ void __launch_bounds__(ROW_THREADS) norm_bwd_rows(const NormArgs a)
{
    for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.X) + (size_t)r * a.ldx;
        const T *dy = static_cast<const T *>(a.dY) + (size_t)r * a.lddy;
        T *dx = static_cast<T *>(a.dX) + (size_t)r * a.lddx;
        const float mu = a.mean_in ? a.mean_in[r] : 0.f, rstd = a.rstd_in[r];
        float s0 = 0.f, s1 = 0.f;
        for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS) {
            const float u = load1(dy + c) * load_w(a.weight, a.w_dtype, c, 1.f);
            s0 += u;
            s1 = fmaf(u, (load1(x + c) - mu) * rstd, s1);
        }
        const float2 t = block_sum(s0, s1);
        const float c0 = a.mean_in ? t.x / a.cols : 0.f, c1 = t.y / a.cols;
        for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS) {
            const float u = load1(dy + c) * load_w(a.weight, a.w_dtype, c, 1.f);
            const float xh = (load1(x + c) - mu) * rstd;
            store1(dx + c, rstd * (u - c0 - xh * c1));
        }
    }
}

// Column sums of dy xh and dy over one part of the rows: a thread has a column, neighbours neighbouring ones.
template <class T>
__global__ void __launch_bounds__(ROW_THREADS) norm_bwd_cols(const NormArgs a, int parts)
{
    const int c = blockIdx.x * ROW_THREADS + threadIdx.x, part = blockIdx.y;
    if (c >= a.cols)
        return;
    float sw = 0.f, sb = 0.f;
    for (int r = part; r < a.rows; r += parts) {
        const float mu = a.mean_in ? a.mean_in[r] : 0.f, rstd = a.rstd_in[r];
        const float dy = load1(static_cast<const T *>(a.dY) + (size_t)r * a.lddy + c);
        const float xh = (load1(static_cast<const T *>(a.X) + (size_t)r * a.ldx + c) - mu) * rstd;
        sw = fmaf(dy, xh, sw);
        sb += dy;
    }
    a.partial[(size_t)part * a.cols + c] = sw;
    a.partial[(size_t)(parts + part) * a.cols + c] = sb;
}

__global__ void __launch_bounds__(ROW_THREADS) norm_bwd_join(const NormArgs a, int parts)
{
    const int c = blockIdx.x * ROW_THREADS + threadIdx.x;
    if (c >= a.cols)
        return;
    float sw = 0.f, sb = 0.f;
    for (int p = 0; p < parts; ++p) {
        sw += a.partial[(size_t)p * a.cols + c];
        sb += a.partial[(size_t)(parts + p) * a.cols + c];
    }
    if (a.dw)
        a.dw[c] += sw;
    if (a.db)
        a.db[c] += sb;
}

} // namespace

int launch_norm_fwd(const NormArgs &a, int n_sm, cudaStream_t s)
{
    const int grid = std::min(a.rows, n_sm * 8);
    if (a.x_dtype == PEAGLE_F32)
        norm_fwd_rows<float><<<grid, ROW_THREADS, 0, s>>>(a);
    else
        norm_fwd_rows<__nv_bfloat16><<<grid, ROW_THREADS, 0, s>>>(a);
    return 1;
}

size_t norm_bwd_scratch(const NormArgs &a, int n_sm)
{
    (void)n_sm;
    return a.dw || a.db ? (size_t)2 * std::min(a.rows, COL_PARTS) * a.cols * sizeof(float) : 0;
}

int launch_norm_bwd(const NormArgs &a, int n_sm, cudaStream_t s)
{
    int launches = 0;
    if (a.dw || a.db) { // before the rows: dX may be dY or X
        const int parts = std::min(a.rows, COL_PARTS);
        const dim3 grid((a.cols + ROW_THREADS - 1) / ROW_THREADS, parts);
        if (a.x_dtype == PEAGLE_F32)
            norm_bwd_cols<float><<<grid, ROW_THREADS, 0, s>>>(a, parts);
        else
            norm_bwd_cols<__nv_bfloat16><<<grid, ROW_THREADS, 0, s>>>(a, parts);
        norm_bwd_join<<<grid.x, ROW_THREADS, 0, s>>>(a, parts);
        launches += 2;
    }
    const int grid = std::min(a.rows, n_sm * 8);
    if (a.x_dtype == PEAGLE_F32)
        norm_bwd_rows<float><<<grid, ROW_THREADS, 0, s>>>(a);
    else
        norm_bwd_rows<__nv_bfloat16><<<grid, ROW_THREADS, 0, s>>>(a);
    return launches + 1;
}

} // namespace peagle
