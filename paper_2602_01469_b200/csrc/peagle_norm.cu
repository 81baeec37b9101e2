// Layer norm and RMS norm of rows, forward and backward.
//
// Forward: y = (x - mu) rstd w + b; mean first, then the mean square of what is left.  Backward, with
// xh = (x - mu) rstd and u = dy w:
//     dx = rstd (u - mean(u) - xh mean(u xh)),   dw += sum_rows dy xh,   db += sum_rows dy.
// All sums are fp32 and have a fixed order.
//
// Bound by memory: forward a read and a write of every element, backward two reads and a write.  A row is held
// in the registers of a group of threads (8 of them for up to 64 columns, 1,024 for up to 16,384; at most 16
// elements each), so it is read once; a block has several groups, and blocks stay for many rows, with the
// weights as fp32 in shared memory.  In the backward the threads keep the same columns from row to row and
// hold the column sums in registers; a block's groups join theirs in shared memory at the end, and a second
// kernel adds up the blocks.  Rows of more columns go through kernels that read them again for every pass.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "peagle_internal.h"
#include "sm100_ptx.cuh"

namespace peagle {
using namespace sm100;

namespace {

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

// ------------------------------------------------------------------ rows in registers

// What thread t of a group has of a row: E elements, in 16-byte pieces TPR pieces apart (VEC: base addresses and
// row strides are multiples of 16 bytes), or single elements TPR apart.
template <class T, bool VEC, int TPR, int E>
struct Part {
    static constexpr int PIECE = VEC ? 16 / (int)sizeof(T) : 1;
    static constexpr int N = E / PIECE;
    static constexpr bool PACKED = VEC && sizeof(T) == 2; // bf16 pairs stay packed
    static constexpr int WORDS = PACKED ? E / 2 : E;
    uint32_t raw[WORDS];

    static __device__ __forceinline__ int col(int t, int e) { return ((e / PIECE) * TPR + t) * PIECE + e % PIECE; }
    // Where the weight of element e lies in shared memory: thread t + 1 has the 16 bytes behind thread t's.
    static __device__ __forceinline__ int place(int t, int e)
    {
        constexpr int Q = PIECE < 4 ? 1 : 4; // floats per access
        return ((e / Q) * TPR + t) * Q + e % Q;
    }

    // Starts to fetch the share of a row, into the thread's own places in `stage` (shared memory, 16 bytes x threads
    // for every piece); single elements are fetched when they are taken.  cols = 0: zeros.
    static __device__ __forceinline__ void fetch(const T *row, int t, int cols, uint32_t stage)
    {
        if constexpr (VEC) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = (n * TPR + t) * PIECE;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(stage + n * blockDim.x * 16),
                             "l"(c < cols ? row + c : row), "r"(c < cols ? 16 : 0)
                             : "memory");
            }
        }
    }
    __device__ __forceinline__ void take(const T *row, int t, int cols, const uint4 *stage)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (VEC) {
                const uint4 v = stage[n * blockDim.x];
                raw[4 * n] = v.x;
                raw[4 * n + 1] = v.y;
                raw[4 * n + 2] = v.z;
                raw[4 * n + 3] = v.w;
            } else {
                const int c = n * TPR + t;
                raw[n] = c < cols ? __float_as_uint(load1(row + c)) : 0u;
            }
        }
    }
    // What was made of the elements before is not kept in registers past here; the elements are.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            asm volatile("" : "+r"(raw[i]));
    }
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (PACKED)
            return __uint_as_float(e & 1 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
        else
            return __uint_as_float(raw[e]);
    }
    // elements e and e + 1, e even
    __device__ __forceinline__ void set2(int e, float a, float b)
    {
        if constexpr (PACKED) {
            raw[e / 2] = pack_bf16x2(a, b);
        } else {
            raw[e] = __float_as_uint(a);
            raw[e + 1] = __float_as_uint(b);
        }
    }
    __device__ __forceinline__ void store(T *row, int t, int cols) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = (n * TPR + t) * PIECE;
            if (c < cols) {
                if constexpr (VEC)
                    *reinterpret_cast<uint4 *>(row + c) = make_uint4(raw[4 * n], raw[4 * n + 1], raw[4 * n + 2], raw[4 * n + 3]);
                else
                    store1(row + c, __uint_as_float(raw[n]));
            }
        }
    }
};

// Rows that are on their way to a thread while it works on one: two, where the block's shared memory allows (of
// the widest groups' 227 KB, fp32 weights and bias take 128).
template <class T, bool VEC, int TPR, int E, int TENSORS>
struct Ring {
    static constexpr int PIECES = VEC ? TENSORS * E * (int)sizeof(T) / 16 : 0;
    static constexpr int DEPTH = !VEC || (TPR == 1024 && sizeof(T) == 4) ? 1 : 2;
    static constexpr int BYTES = DEPTH * PIECES * 16; // per thread
};
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Threads of a block: whole groups.
__host__ __device__ constexpr int block_threads(int tpr) { return tpr == 192 ? 384 : tpr < 256 ? 256 : tpr; }

// Sums over the threads of a group.  `red` has two halves that take turns, so that one barrier is enough.
template <int TPR>
__device__ __forceinline__ float2 group_sum(float a, float b, float2 (*red)[block_threads(TPR) / 32], int &turn)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1) {
        a += __shfl_xor_sync(~0u, a, o);
        b += __shfl_xor_sync(~0u, b, o);
    }
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, group = warp / W;
        if ((threadIdx.x & 31) == 0)
            red[turn][warp] = make_float2(a, b);
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
        a = b = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float2 v = red[turn][group * W + i];
            a += v.x;
            b += v.y;
        }
        turn ^= 1;
    }
    return make_float2(a, b);
}

// Blocks that an SM should hold: about 768 threads; 512 where a thread holds 48 words of elements and sums or more.
constexpr int blocks_per_sm(int threads, int words) { return threads >= 512 ? 1 : (words >= 48 ? 512 : 768) / threads; }

template <class T, bool VEC, int TPR, int E>
__global__ void __launch_bounds__(block_threads(TPR)) norm_fwd_kernel(const NormArgs a)
{
    using Row = Part<T, VEC, TPR, E>;
    using Stages = Ring<T, VEC, TPR, E, 1>;
    constexpr int BT = block_threads(TPR), G = BT / TPR, D = Stages::DEPTH;
    extern __shared__ float4 smem[];
    uint4 *ring = reinterpret_cast<uint4 *>(smem) + threadIdx.x;
    float *sw = reinterpret_cast<float *>(smem + D * Stages::PIECES * BT), *sb = sw + TPR * E;
    __shared__ float2 red[2][BT / 32];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const bool layer = a.kind == PEAGLE_NORM_LAYER;
    const T *X = static_cast<const T *>(a.X);
    const int64_t step = (int64_t)gridDim.x * G;
    const int64_t first = (int64_t)blockIdx.x * G + g;
    const uint32_t ring_at = smem_u32(ring);
#pragma unroll
    for (int i = 0; i < D; ++i) {
        const int64_t r = first + i * step;
        Row::fetch(r < a.rows ? X + r * a.ldx : X, t, r < a.rows ? a.cols : 0, ring_at + i * Stages::PIECES * BT * 16);
        copies_commit();
    }
    // group g brings every G-th element of each thread's share
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = Row::col(t, e);
        if (e % G == g && c < a.cols) {
            sw[Row::place(t, e)] = load_w(a.weight, a.w_dtype, c, 1.f);
            if (a.bias)
                sb[Row::place(t, e)] = load_w(a.bias, a.w_dtype, c, 0.f);
        }
    }
    __syncthreads();
    const float n = (float)a.cols;
    int turn = 0, stage = 0;
    for (int64_t r = first; r - g < a.rows; r += step) {
        const bool live = r < a.rows;
        Row x;
        copies_wait<D - 1>();
        x.take(X + r * a.ldx, t, live ? a.cols : 0, ring + stage * Stages::PIECES * BT);
        float mu = 0.f;
        if (layer) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e)
                s += x.get(e);
            mu = group_sum<TPR>(s, 0.f, red, turn).x / n;
        }
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (Row::col(t, e) < a.cols) {
                const float d = x.get(e) - mu;
                s += d;
                q = fmaf(d, d, q);
            }
        const float2 sq = group_sum<TPR>(s, q, red, turn);
        // the sums are formed, so the stage has been read
        const int64_t ahead = r + D * step;
        Row::fetch(ahead < a.rows ? X + ahead * a.ldx : X, t, ahead < a.rows ? a.cols : 0,
                   ring_at + stage * Stages::PIECES * BT * 16);
        copies_commit();
        stage = stage + 1 == D ? 0 : stage + 1;
        // the rounding of mu is taken out of both
        const float left = layer ? sq.x / n : 0.f;
        mu += left;
        const float var = sq.y / n - left * left;
        const float rstd = rsqrtf((var < 0.f ? 0.f : var) + a.eps); // a NaN stays one
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            float v[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = Row::place(t, e + k);
                v[k] = (x.get(e + k) - mu) * rstd * sw[at];
                if (a.bias)
                    v[k] += sb[at];
            }
            x.set2(e, v[0], v[1]);
        }
        if (live) {
            x.store(static_cast<T *>(a.Y) + r * a.ldy, t, a.cols);
            if (t == 0) {
                if (a.mean)
                    a.mean[r] = mu;
                if (a.rstd)
                    a.rstd[r] = rstd;
            }
        }
    }
}

// SUMS: 0 none, 1 of dy xh (dw), 2 of dy too (db).
template <class T, bool VEC, int TPR, int E, int SUMS>
__global__ void __launch_bounds__(block_threads(TPR),
                                  blocks_per_sm(block_threads(TPR), 2 * Part<T, VEC, TPR, E>::WORDS + SUMS * E))
    norm_bwd_kernel(const NormArgs a)
{
    using Row = Part<T, VEC, TPR, E>;
    using Stages = Ring<T, VEC, TPR, E, 2>;
    constexpr int BT = block_threads(TPR), G = BT / TPR, D = Stages::DEPTH, HALF = Stages::PIECES / 2;
    extern __shared__ float4 smem[];
    uint4 *ring = reinterpret_cast<uint4 *>(smem) + threadIdx.x;
    float *sw = reinterpret_cast<float *>(smem + D * Stages::PIECES * BT);
    __shared__ float2 red[2][BT / 32];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const bool layer = a.kind == PEAGLE_NORM_LAYER;
    const T *X = static_cast<const T *>(a.X), *DY = static_cast<const T *>(a.dY);
    const int64_t step = (int64_t)gridDim.x * G;
    const int64_t first = (int64_t)blockIdx.x * G + g;
    const uint32_t ring_at = smem_u32(ring);
    const auto fetch = [&](int64_t r, int stage) {
        const bool live = r < a.rows;
        const uint32_t at = ring_at + stage * Stages::PIECES * BT * 16;
        Row::fetch(live ? X + r * a.ldx : X, t, live ? a.cols : 0, at);
        Row::fetch(live ? DY + r * a.lddy : DY, t, live ? a.cols : 0, at + HALF * BT * 16);
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < D; ++i)
        fetch(first + i * step, i);
    float mu = 0.f, rstd = 0.f; // of the row to come
    if (first < a.rows) {
        mu = layer ? a.mean_in[first] : 0.f;
        rstd = a.rstd_in[first];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = Row::col(t, e);
        if (e % G == g)
            sw[Row::place(t, e)] = c < a.cols ? load_w(a.weight, a.w_dtype, c, 1.f) : 0.f;
    }
    __syncthreads();
    float dw[SUMS > 0 ? E : 1], db[SUMS > 1 ? E : 1];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (SUMS > 0)
            dw[e] = 0.f;
        if (SUMS > 1)
            db[e] = 0.f;
    }
    const float n = (float)a.cols;
    int turn = 0, stage = 0;
    for (int64_t r = first; r - g < a.rows; r += step) {
        const bool live = r < a.rows;
        Row x, dy;
        const float m = mu, rs = rstd;
        mu = rstd = 0.f;
        if (r + step < a.rows) {
            mu = layer ? a.mean_in[r + step] : 0.f;
            rstd = a.rstd_in[r + step];
        }
        copies_wait<D - 1>();
        x.take(X + r * a.ldx, t, live ? a.cols : 0, ring + stage * Stages::PIECES * BT);
        dy.take(DY + r * a.lddy, t, live ? a.cols : 0, ring + (stage * Stages::PIECES + HALF) * BT);
        float s0 = 0.f, s1 = 0.f; // columns past the last have dy = w = 0
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = dy.get(e), xh = (x.get(e) - m) * rs, u = d * sw[Row::place(t, e)];
            s0 += u;
            s1 = fmaf(u, xh, s1);
            if (SUMS > 0)
                dw[e] = fmaf(d, xh, dw[e]);
            if (SUMS > 1)
                db[e] += d;
        }
        const float2 s = group_sum<TPR>(s0, s1, red, turn);
        fetch(r + D * step, stage); // the sums are formed, so the stage has been read
        stage = stage + 1 == D ? 0 : stage + 1;
        const float c0 = layer ? s.x / n : 0.f, c1 = s.y / n;
        x.forget();
        dy.forget();
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            float v[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float u = dy.get(e + k) * sw[Row::place(t, e + k)], xh = (x.get(e + k) - m) * rs;
                v[k] = rs * (u - c0 - xh * c1);
            }
            x.set2(e, v[0], v[1]);
        }
        if (live)
            x.store(static_cast<T *>(a.dX) + r * a.lddx, t, a.cols);
    }
    copies_wait<0>();
    pdl_trigger(); // the kernel that joins the blocks may settle down
    if constexpr (SUMS > 0) {
#pragma unroll
        for (int which = 0; which < SUMS; ++which) {
            __syncthreads(); // weights, and the sums before, have been read
            if (G > 1) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    sw[(g * E + e) * TPR + t] = which ? db[e] : dw[e];
                __syncthreads();
            }
            float *out = which ? a.db : a.dw;
            float *part = a.partial + ((size_t)which * gridDim.x + blockIdx.x) * a.cols;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int c = Row::col(t, e);
                if (e % G != g || c >= a.cols)
                    continue;
                float v = which ? db[e] : dw[e];
                if (G > 1) {
                    v = 0.f;
#pragma unroll
                    for (int k = 0; k < G; ++k)
                        v += sw[(k * E + e) * TPR + t];
                }
                if (gridDim.x > 1)
                    part[c] = v;
                else if (out)
                    out[c] += v;
            }
        }
    }
}

// Adds the parts' column sums to dw and db: 32 columns to a block, a part to every 32nd row of threads.
__global__ void __launch_bounds__(1024) norm_bwd_join(const NormArgs a, int parts)
{
    pdl_wait();
    __shared__ float s[32][33];
    const int c = blockIdx.x * 32 + threadIdx.x;
    float *out = blockIdx.y ? a.db : a.dw;
    if (!out)
        return;
    float v = 0.f;
    if (c < a.cols) {
        const float *p = a.partial + (size_t)blockIdx.y * parts * a.cols + c;
#pragma unroll 4
        for (int i = threadIdx.y; i < parts; i += 32)
            v += p[(size_t)i * a.cols];
    }
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    v = s[threadIdx.x][threadIdx.y];
    for (int o = 16; o; o >>= 1)
        v += __shfl_xor_sync(~0u, v, o);
    const int cc = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && cc < a.cols)
        out[cc] += v;
}

// ------------------------------------------------------------------ rows of any length

constexpr int ROW_THREADS = 256;
constexpr int COL_PARTS = 64; // parts of the rows that the column sums are made in

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
        const float left = a.kind == PEAGLE_NORM_LAYER ? t.x / a.cols : 0.f;
        mu += left;
        const float var = t.y / a.cols - left * left;
        const float rstd = rsqrtf((var < 0.f ? 0.f : var) + a.eps);
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

// ------------------------------------------------------------------ choice

constexpr int REG_COLS = 16384; // columns that the widest group of threads holds

bool pieces_aligned(const NormArgs &a, bool backward)
{
    const int64_t piece = a.x_dtype == PEAGLE_F32 ? 4 : 8; // elements in 16 bytes
    const auto rows_ok = [&](const void *p, int64_t ld) {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld % piece == 0 || a.rows == 1);
    };
    return a.cols % piece == 0 && rows_ok(a.X, a.ldx) &&
           (backward ? rows_ok(a.dY, a.lddy) && rows_ok(a.dX, a.lddx) : rows_ok(a.Y, a.ldy));
}

// Calls f<T, VEC, TPR, E>() with the smallest group that holds a row.
template <class T, class F>
int with_group(int cols, bool vec, F f)
{
    if (vec) {
        if (cols <= 8 * 8)
            return f.template operator()<T, true, 8, 8>();
        if (cols <= 16 * 8)
            return f.template operator()<T, true, 16, 8>();
        if (cols <= 32 * 8)
            return f.template operator()<T, true, 32, 8>();
        if (cols <= 32 * 16)
            return f.template operator()<T, true, 32, 16>();
        if (cols <= 64 * 16)
            return f.template operator()<T, true, 64, 16>();
        if (cols <= 128 * 16)
            return f.template operator()<T, true, 128, 16>();
        if (cols <= 192 * 16)
            return f.template operator()<T, true, 192, 16>();
        if (cols <= 256 * 16)
            return f.template operator()<T, true, 256, 16>();
        if (cols <= 384 * 16)
            return f.template operator()<T, true, 384, 16>();
        if (cols <= 512 * 16)
            return f.template operator()<T, true, 512, 16>();
        return f.template operator()<T, true, 1024, 16>();
    }
    if (cols <= 32 * 8)
        return f.template operator()<T, false, 32, 8>();
    if (cols <= 64 * 16)
        return f.template operator()<T, false, 64, 16>();
    if (cols <= 256 * 16)
        return f.template operator()<T, false, 256, 16>();
    return f.template operator()<T, false, 1024, 16>();
}

// Blocks of `kernel` that fit the GPU at once, at most one for every `per_block` rows.  `known` keeps how many
// fit an SM (all devices here are alike; asking takes longer than a short row).
int blocks_for(const void *kernel, int threads, size_t smem, std::atomic<int> &known, int n_sm, int64_t rows, int per_block)
{
    if (smem > 40 * 1024) // the kernels' own arrays count towards the 48 KB too
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    int per_sm = known.load(std::memory_order_relaxed);
    if (per_sm == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess || per_sm < 1) {
            cudaGetLastError();
            per_sm = 1;
        }
        known.store(per_sm, std::memory_order_relaxed);
    }
    return (int)std::min<int64_t>((rows + per_block - 1) / per_block, (int64_t)n_sm * per_sm);
}

struct Forward {
    const NormArgs &a;
    int n_sm;
    cudaStream_t s;
    template <class T, bool VEC, int TPR, int E>
    int operator()() const
    {
        constexpr int BT = block_threads(TPR);
        const auto kernel = norm_fwd_kernel<T, VEC, TPR, E>;
        static std::atomic<int> known[2];
        const size_t smem = (size_t)Ring<T, VEC, TPR, E, 1>::BYTES * BT + (size_t)(a.bias ? 2 : 1) * TPR * E * sizeof(float);
        kernel<<<blocks_for((const void *)kernel, BT, smem, known[a.bias != nullptr], n_sm, a.rows, BT / TPR), BT, smem,
                 s>>>(a);
        return 1;
    }
};

struct Backward {
    const NormArgs &a;
    int n_sm;
    cudaStream_t s;
    bool only_blocks; // says how many blocks it would launch
    template <class T, bool VEC, int TPR, int E>
    int operator()() const
    {
        if (a.db)
            return with_sums<T, VEC, TPR, E, 2>();
        if (a.dw)
            return with_sums<T, VEC, TPR, E, 1>();
        return with_sums<T, VEC, TPR, E, 0>();
    }
    template <class T, bool VEC, int TPR, int E, int SUMS>
    int with_sums() const
    {
        constexpr int BT = block_threads(TPR);
        const auto kernel = norm_bwd_kernel<T, VEC, TPR, E, SUMS>;
        // the rows to come; weights, then the sums of the block's groups
        const size_t smem = (size_t)Ring<T, VEC, TPR, E, 2>::BYTES * BT + (size_t)(SUMS > 0 ? BT : TPR) * E * sizeof(float);
        static std::atomic<int> known;
        const int blocks = blocks_for((const void *)kernel, BT, smem, known, n_sm, a.rows, BT / TPR);
        if (only_blocks)
            return blocks;
        kernel<<<blocks, BT, smem, s>>>(a);
        if (SUMS == 0 || blocks == 1)
            return 1;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3((a.cols + 31) / 32, SUMS);
        cfg.blockDim = dim3(32, 32);
        cfg.stream = s;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        cudaLaunchKernelEx(&cfg, norm_bwd_join, a, blocks);
        return 2;
    }
};

} // namespace

int launch_norm_fwd(const NormArgs &a, int n_sm, cudaStream_t s)
{
    if (a.cols <= REG_COLS) {
        const bool vec = pieces_aligned(a, false);
        const Forward f{a, n_sm, s};
        return a.x_dtype == PEAGLE_F32 ? with_group<float>(a.cols, vec, f) : with_group<__nv_bfloat16>(a.cols, vec, f);
    }
    const int grid = std::min(a.rows, n_sm * 8);
    if (a.x_dtype == PEAGLE_F32)
        norm_fwd_rows<float><<<grid, ROW_THREADS, 0, s>>>(a);
    else
        norm_fwd_rows<__nv_bfloat16><<<grid, ROW_THREADS, 0, s>>>(a);
    return 1;
}

size_t norm_bwd_scratch(const NormArgs &a, int n_sm)
{
    if (!a.dw && !a.db)
        return 0;
    int parts = std::min(a.rows, COL_PARTS);
    if (a.cols <= REG_COLS) {
        const Backward f{a, n_sm, nullptr, true};
        const bool vec = pieces_aligned(a, true);
        parts = a.x_dtype == PEAGLE_F32 ? with_group<float>(a.cols, vec, f) : with_group<__nv_bfloat16>(a.cols, vec, f);
    }
    return (size_t)2 * parts * a.cols * sizeof(float);
}

int launch_norm_bwd(const NormArgs &a, int n_sm, cudaStream_t s)
{
    if (a.cols <= REG_COLS) {
        const Backward f{a, n_sm, s, false};
        const bool vec = pieces_aligned(a, true);
        return a.x_dtype == PEAGLE_F32 ? with_group<float>(a.cols, vec, f) : with_group<__nv_bfloat16>(a.cols, vec, f);
    }
    int launches = 0;
    if (a.dw || a.db) { // before the rows: dX may be dY or X
        const int parts = std::min(a.rows, COL_PARTS);
        const dim3 grid((a.cols + ROW_THREADS - 1) / ROW_THREADS, parts);
        if (a.x_dtype == PEAGLE_F32)
            norm_bwd_cols<float><<<grid, ROW_THREADS, 0, s>>>(a, parts);
        else
            norm_bwd_cols<__nv_bfloat16><<<grid, ROW_THREADS, 0, s>>>(a, parts);
        norm_bwd_join<<<dim3((a.cols + 31) / 32, 2), dim3(32, 32), 0, s>>>(a, parts);
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
