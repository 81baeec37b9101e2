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
//
// Measured, of the rate of a copy: RMS forward, 32,768 rows of 2,880 bf16, 66 us (88 %), backward 96 (90 %); layer norm
// backward, 524,288 rows of 128 bf16, 72 (86 %).  What is missing is loads in flight while a row's sums are joined.  Few
// rows are bound by latency: layer norm backward of 3,891 rows of 1,001 fp32 takes 18.4 us (39 %), of 30,000 66 (83 %).
// Rows that do not begin on 16 bytes go through single elements: RMS norm of 16,384 rows of 2,877 takes 106 us forward
// (27 %) and 95 backward (45 %) in bf16, 81 (71 %) and 115 (75 %) in fp32.  Rows of more columns than a group holds are
// not meant to be fast: 2,048 of 20,000 bf16 take 97 us forward (26 %) and 252 backward (15 %).
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

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

// Threads of a block: whole groups.
__host__ __device__ constexpr int block_threads(int tpr) { return tpr == 192 ? 384 : tpr < 256 ? 256 : tpr; }

// What thread t of a group has of a row: E elements, in 16-byte pieces TPR pieces apart (VEC: base addresses and
// row strides are multiples of 16 bytes), or single elements TPR apart.
// FP32_AHEAD: single fp32 elements are fetched ahead too, 4 bytes at a time, which pays in the forward (16,384 rows of
// 2,877: 99 -> 80 us) and not in the backward with its two tensors (30,000 rows of 1,001: 66 -> 84).
template <class T, bool VEC, int TPR, int E, bool FP32_AHEAD = false>
struct Part {
    static constexpr int PIECE = VEC ? 16 / (int)sizeof(T) : 1;
    static constexpr int N = E / PIECE;
    static constexpr bool PACKED = VEC && sizeof(T) == 2; // bf16 pairs stay packed
    static constexpr bool AHEAD = VEC || (sizeof(T) == 4 && FP32_AHEAD);
    using Slot = std::conditional_t<VEC, uint4, uint32_t>;
    static constexpr int WORDS = PACKED ? E / 2 : E;
    uint32_t raw[WORDS];

    static __device__ __forceinline__ int col(int t, int e) { return ((e / PIECE) * TPR + t) * PIECE + e % PIECE; }
    // Where the weight of element e lies in shared memory: thread t + 1 has the 16 bytes behind thread t's.
    static __device__ __forceinline__ int place(int t, int e)
    {
        constexpr int Q = PIECE < 4 ? 1 : 4; // floats per access
        return ((e / Q) * TPR + t) * Q + e % Q;
    }

    // Starts to fetch the share of a row, into the thread's own places in `stage` (shared memory, a slot x threads
    // for every piece); single bf16 elements are fetched when they are taken.  `row` is the row's address plus t pieces.
    static __device__ __forceinline__ void fetch(const T *row, int t, int cols, uint32_t stage)
    {
        if constexpr (AHEAD) {
#pragma unroll
            for (int n = 0; n < N; ++n)
                if ((n * TPR + t) * PIECE < cols) {
                    const uint32_t to = stage + n * block_threads(TPR) * (uint32_t)sizeof(Slot);
                    if constexpr (VEC)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + n * TPR * PIECE) : "memory");
                    else
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(row + n * TPR) : "memory");
                }
        }
    }
    // Places past the last column are never fetched: zeros, once.
    static __device__ __forceinline__ void clear(int t, int cols, Slot *stage)
    {
        if constexpr (AHEAD) {
#pragma unroll
            for (int n = 0; n < N; ++n)
                if ((n * TPR + t) * PIECE >= cols)
                    stage[n * block_threads(TPR)] = Slot{};
        }
    }
    __device__ __forceinline__ void take(const T *row, int t, int cols, const Slot *stage)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (VEC) {
                const uint4 v = stage[n * block_threads(TPR)];
                raw[4 * n] = v.x;
                raw[4 * n + 1] = v.y;
                raw[4 * n + 2] = v.z;
                raw[4 * n + 3] = v.w;
            } else if constexpr (AHEAD) {
                raw[n] = stage[n * block_threads(TPR)];
            } else {
                raw[n] = n * TPR + t < cols ? __float_as_uint(load1(row + n * TPR)) : 0u;
            }
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            raw[i] = 0;
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
    __device__ __forceinline__ F2 get2(int e) const { return f2(get(e), get(e + 1)); }
    __device__ __forceinline__ void set2(int e, F2 v)
    {
        const float2 u = unf2(v);
        if constexpr (PACKED) {
            raw[e / 2] = pack_bf16x2(u.x, u.y);
        } else {
            raw[e] = __float_as_uint(u.x);
            raw[e + 1] = __float_as_uint(u.y);
        }
    }
    // elements e to e + 3 of a row in shared memory, e a multiple of 4
    static __device__ __forceinline__ void weights4(const float *sw, int t, int e, F2 &a, F2 &b)
    {
        if constexpr (VEC) {
            const float4 w = *reinterpret_cast<const float4 *>(sw + place(t, e));
            a = f2(w.x, w.y);
            b = f2(w.z, w.w);
        } else {
            a = f2(sw[place(t, e)], sw[place(t, e + 1)]);
            b = f2(sw[place(t, e + 2)], sw[place(t, e + 3)]);
        }
    }
    __device__ __forceinline__ void store(T *row, int t, int cols) const // `row` as above
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
            if ((n * TPR + t) * PIECE < cols) {
                if constexpr (VEC)
                    *reinterpret_cast<uint4 *>(row + n * TPR * PIECE) =
                        make_uint4(raw[4 * n], raw[4 * n + 1], raw[4 * n + 2], raw[4 * n + 3]);
                else
                    store1(row + n * TPR, __uint_as_float(raw[n]));
            }
    }
};

// Rows that are on their way to a thread while it works on one: two, where the block's shared memory allows (of
// the widest groups' 227 KB, fp32 weights and bias take 128).
template <class T, bool VEC, int TPR, int E, int TENSORS>
struct Ring {
    using Row = Part<T, VEC, TPR, E, TENSORS == 1>;
    static constexpr int SLOTS = Row::AHEAD ? TENSORS * Row::N : 0;
    static constexpr int DEPTH = !Row::AHEAD || (TPR == 1024 && sizeof(T) == 4) ? 1 : 2;
    static constexpr int BYTES = DEPTH * SLOTS * (int)sizeof(typename Row::Slot); // per thread
};
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }


// Sums over the threads of a group.  `red` has two halves that take turns, so that one barrier is enough.
template <int TPR>
__device__ __forceinline__ float group_sum(float a, float (*red)[block_threads(TPR) / 32], int &turn)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1)
        a += __shfl_xor_sync(~0u, a, o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, group = warp / W;
        if ((threadIdx.x & 31) == 0)
            red[turn][warp] = a;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
        a = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i)
            a += red[turn][group * W + i];
        turn ^= 1;
    }
    return a;
}
template <int TPR>
__device__ __forceinline__ float2 group_sum2(F2 v, float2 (*red)[block_threads(TPR) / 32], int &turn)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o; o >>= 1) {
        const float2 u = unf2(v);
        v = add_f2(v, f2(__shfl_xor_sync(~0u, u.x, o), __shfl_xor_sync(~0u, u.y, o)));
    }
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, group = warp / W;
        if ((threadIdx.x & 31) == 0)
            red[turn][warp] = unf2(v);
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
        v = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < W; i += 2) {
            const float4 u = *reinterpret_cast<const float4 *>(&red[turn][group * W + i]);
            v = add_f2(add_f2(v, f2(u.x, u.y)), f2(u.z, u.w));
        }
        turn ^= 1;
    }
    return unf2(v);
}

// Blocks that an SM should hold: about 768 threads; 512 where a thread holds 48 words of elements and sums or more.
constexpr int blocks_per_sm(int threads, int words) { return threads >= 512 ? 1 : (words >= 48 ? 512 : 768) / threads; }

// Weights as fp32 in shared memory: group g brings every G-th element of each thread's share; zeros past the end.
template <class Row, int E, int G>
__device__ __forceinline__ void stage_weights(float *to, const void *w, int dtype, float absent, int t, int g, int cols)
{
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = Row::col(t, e);
        if (e % G == g)
            to[Row::place(t, e)] = c < cols ? load_w(w, dtype, c, absent) : 0.f;
    }
}

// The forward's blocks per SM.  RMS norm is best with 32 to 64 KB of rows on their way; more in flight is slower:
// rows of 2,880 bf16 take 63.6 us with 768 threads and 70.9 with 1,152, of 2,880 fp32 64.8 with 512 and 70.0 with
// 768, of 128 bf16 47.1 with 512 and 50.8 with 768; 8,192 bf16 in blocks of 512 threads 55.3 us with one and 47.3
// with two.  Layer norm has two sums to wait for and takes all the threads that fit (2,880 fp32: 77 us with 512,
// 67 with 768; 128 bf16 59 and 53).
constexpr int fwd_blocks(bool layer, int words, int tpr, int threads)
{
    if (layer)
        return 32;

    const int want = words > 8 || tpr < 32 ? 512 : tpr == 512 ? 1024 : 768;
    return want < threads ? 1 : want / threads;
}
// Whether the mean takes the sum of what is left, x - mu, as its correction: its own sum has lost more digits than the
// differences then.  Those are rounded alike within a binade, which adds up: 2,880 bf16 numbers of spread 2.2 have a mean off
// by 2e-9 as summed and by 4e-8 corrected around 0, both 6e-8 around 1, 3e-5 and 2e-5 around 1,000.
__device__ __forceinline__ bool off_centre(float mu, float var) { return !(16.f * mu * mu < var); }

template <class T, bool VEC, int TPR, int E>
__global__ void __launch_bounds__(block_threads(TPR)) norm_fwd_kernel(const __grid_constant__ NormArgs a)
{
    using Stages = Ring<T, VEC, TPR, E, 1>;
    using Row = typename Stages::Row;
    constexpr int BT = block_threads(TPR), G = BT / TPR, D = Stages::DEPTH, STAGE = Stages::SLOTS * BT;
    extern __shared__ float4 smem[];
    constexpr int SLOT = sizeof(typename Row::Slot);
    auto *ring = reinterpret_cast<typename Row::Slot *>(smem) + threadIdx.x;
    float *sw = reinterpret_cast<float *>(reinterpret_cast<char *>(smem) + Stages::BYTES * BT), *sb = sw + TPR * E;
    __shared__ float red1[2][BT / 32];
    __shared__ __align__(16) float2 red2[2][BT / 32];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = a.cols;
    const bool layer = a.kind == PEAGLE_NORM_LAYER;
    const uint32_t rows = a.rows, step = gridDim.x * G, first = blockIdx.x * G + g;
    // formed anew for every row: pointers that move along would take registers
    const auto x_at = [&](uint32_t r) { return static_cast<const T *>(a.X) + t * Row::PIECE + r * a.ldx; };
    const auto y_at = [&](uint32_t r) { return static_cast<T *>(a.Y) + t * Row::PIECE + r * a.ldy; };
    uint32_t ring_at = smem_u32(ring);
#pragma unroll
    for (int i = 0; i < D; ++i) {
        Row::clear(t, cols, ring + i * STAGE);
        if (first + i * step < rows)
            Row::fetch(x_at(first + i * step), t, cols, ring_at + i * STAGE * SLOT);
        copies_commit();
    }
    stage_weights<Row, E, G>(sw, a.weight, a.w_dtype, 1.f, t, g, cols);
    if (a.bias)
        stage_weights<Row, E, G>(sb, a.bias, a.w_dtype, 0.f, t, g, cols);
    __syncthreads();
    const float per_col = 1.f / (float)cols;
    int turn = 0, stage = 0;
    // groups of less than a warp stay together with their warp
    for (uint32_t r = first; r - (TPR < 32 ? g % (32 / TPR) : 0) < rows; r += step) {
        Row x;
        copies_wait<D - 1>();
        if (VEC || r < rows)
            x.take(x_at(r), t, cols, ring + stage * STAGE);
        float mu = 0.f, var;
        if (layer) {
            F2 s = f2(0.f, 0.f), q = s;
#pragma unroll
            for (int e = 0; e < E; e += 2)
                s = add_f2(s, x.get2(e));
            const float2 sum = unf2(s);
            mu = group_sum<TPR>(sum.x + sum.y, red1, turn) * per_col;
            const F2 minus = f2(-mu, -mu);
            s = q;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                F2 d = add_f2(x.get2(e), minus);
                if (!VEC && Row::col(t, e) >= cols)
                    d = f2(0.f, 0.f);
                else if (!VEC && Row::col(t, e + 1) >= cols)
                    d = f2(unf2(d).x, 0.f);
                if (!VEC || Row::col(t, e) < cols) {
                    s = add_f2(s, d);
                    q = fma_f2(d, d, q);
                }
            }
            const float2 s2 = unf2(s), q2 = unf2(q);
            const float2 both = group_sum2<TPR>(f2(s2.x + s2.y, q2.x + q2.y), red2, turn);
            const float left = both.x * per_col; // the rounding of mu is taken out of both
            var = both.y * per_col - left * left;
            mu += off_centre(mu, var) ? left : 0.f;
        } else {
            F2 q = f2(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < E; e += 2)
                q = fma_f2(x.get2(e), x.get2(e), q);
            const float2 q2 = unf2(q);
            var = group_sum<TPR>(q2.x + q2.y, red1, turn) * per_col;
        }
        // the sums are formed, so the stage has been read
        if (r + D * step < rows)
            Row::fetch(x_at(r + D * step), t, cols, ring_at + stage * STAGE * SLOT);
        copies_commit();
        if (D > 1)
            stage ^= 1;
        const float rstd = rsqrtf((var < 0.f ? 0.f : var) + a.eps); // a NaN stays one
        const F2 minus = f2(-mu, -mu), by = f2(rstd, rstd);
        x.forget();
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            F2 w0, w1;
            Row::weights4(sw, t, e, w0, w1);
            F2 v0 = x.get2(e), v1 = x.get2(e + 2);
            if (layer) {
                v0 = add_f2(v0, minus);
                v1 = add_f2(v1, minus);
            }
            v0 = mul_f2(v0, by);
            v1 = mul_f2(v1, by);
            if (a.bias) {
                F2 b0, b1;
                Row::weights4(sb, t, e, b0, b1);
                v0 = fma_f2(v0, w0, b0);
                v1 = fma_f2(v1, w1, b1);
            } else {
                v0 = mul_f2(v0, w0);
                v1 = mul_f2(v1, w1);
            }
            x.set2(e, v0);
            x.set2(e + 2, v1);
        }
        if (r < rows) {
            x.store(y_at(r), t, cols);
            if (t == 0) {
                if (a.mean)
                    a.mean[r] = mu;
                if (a.rstd)
                    a.rstd[r] = rstd;
            }
        }
    }
}

// LAYER: layer norm, else RMS norm.  SUMS: 1 of dy xh (dw), 2 of dy too (db).  With z = x - mu the products are
// arranged for few operations per element: t = dy z gives sum u xh = rstd sum t w and dw += rstd t, and
// dx = rstd (w dy - mean(u) + (-rstd mean(u xh)) z).
template <class T, bool VEC, bool LAYER, int TPR, int E, int SUMS>
__global__ void __launch_bounds__(block_threads(TPR),
                                  blocks_per_sm(block_threads(TPR), 2 * Part<T, VEC, TPR, E>::WORDS + SUMS * E))
    norm_bwd_kernel(const __grid_constant__ NormArgs a)
{
    using Stages = Ring<T, VEC, TPR, E, 2>;
    using Row = typename Stages::Row;
    constexpr int BT = block_threads(TPR), G = BT / TPR, D = Stages::DEPTH, STAGE = Stages::SLOTS * BT, HALF = STAGE / 2;
    extern __shared__ float4 smem[];
    constexpr int SLOT = sizeof(typename Row::Slot);
    auto *ring = reinterpret_cast<typename Row::Slot *>(smem) + threadIdx.x;
    float *sw = reinterpret_cast<float *>(reinterpret_cast<char *>(smem) + Stages::BYTES * BT);
    __shared__ float red1[2][BT / 32];
    __shared__ __align__(16) float2 red[2][BT / 32];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, cols = a.cols;
    const uint32_t rows = a.rows, step = gridDim.x * G, first = blockIdx.x * G + g;
    // formed anew for every row, like the forward's
    const auto x_at = [&](uint32_t r) { return static_cast<const T *>(a.X) + t * Row::PIECE + r * a.ldx; };
    const auto dy_at = [&](uint32_t r) { return static_cast<const T *>(a.dY) + t * Row::PIECE + r * a.lddy; };
    const auto dx_at = [&](uint32_t r) { return static_cast<T *>(a.dX) + t * Row::PIECE + r * a.lddx; };
    const uint32_t ring_at = smem_u32(ring);
#pragma unroll
    for (int i = 0; i < D; ++i) {
        Row::clear(t, cols, ring + i * STAGE);
        Row::clear(t, cols, ring + i * STAGE + HALF);
        if (first + i * step < rows) {
            Row::fetch(x_at(first + i * step), t, cols, ring_at + i * STAGE * SLOT);
            Row::fetch(dy_at(first + i * step), t, cols, ring_at + (i * STAGE + HALF) * SLOT);
        }
        copies_commit();
    }
    float mu = 0.f, rstd = 0.f; // of the row to come
    if (first < rows) {
        mu = LAYER ? a.mean_in[first] : 0.f;
        rstd = a.rstd_in[first];
    }
    stage_weights<Row, E, G>(sw, a.weight, a.w_dtype, 1.f, t, g, cols);
    __syncthreads();
    F2 dw[E / 2], db[SUMS > 1 ? E / 2 : 1];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
        dw[e] = f2(0.f, 0.f);
        if (SUMS > 1)
            db[e] = f2(0.f, 0.f);
    }
    const float per_col = 1.f / (float)cols;
    int turn = 0, stage = 0;
    for (uint32_t r = first; r - (TPR < 32 ? g % (32 / TPR) : 0) < rows; r += step) {
        Row x, dy;
        const F2 minus = f2(-mu, -mu), by = f2(rstd, rstd);
        const float rs = rstd;
        if (r + step < rows) {
            mu = LAYER ? a.mean_in[r + step] : 0.f;
            rstd = a.rstd_in[r + step];
        }
        copies_wait<D - 1>();
        if (VEC || r < rows) {
            x.take(x_at(r), t, cols, ring + stage * STAGE);
            dy.take(dy_at(r), t, cols, ring + stage * STAGE + HALF);
        }
        if (TPR < 32 && r >= rows) {
            x.zero();
            dy.zero();
        }
        F2 s0 = f2(0.f, 0.f), s1 = s0; // columns past the last have dy = w = 0
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            F2 w[2];
            Row::weights4(sw, t, e, w[0], w[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const F2 d = dy.get2(e + 2 * k), x2 = x.get2(e + 2 * k), td = mul_f2(d, LAYER ? add_f2(x2, minus) : x2);
                if (LAYER)
                    s0 = fma_f2(d, w[k], s0);
                s1 = fma_f2(td, w[k], s1);
                dw[e / 2 + k] = fma_f2(td, by, dw[e / 2 + k]);
                if (SUMS > 1)
                    db[e / 2 + k] = add_f2(db[e / 2 + k], d);
            }
        }
        const float2 p0 = unf2(s0), p1 = unf2(s1);
        float2 s;
        if (LAYER)
            s = group_sum2<TPR>(f2(p0.x + p0.y, p1.x + p1.y), red, turn);
        else
            s = make_float2(0.f, group_sum<TPR>(p1.x + p1.y, red1, turn));
        // the sums are formed, so the stage has been read
        if (r + D * step < rows) {
            Row::fetch(x_at(r + D * step), t, cols, ring_at + stage * STAGE * SLOT);
            Row::fetch(dy_at(r + D * step), t, cols, ring_at + (stage * STAGE + HALF) * SLOT);
        }
        copies_commit();
        if (D > 1)
            stage ^= 1;
        // from left to right: the mean of u xh has the size of u, while rstd^3 alone leaves fp32's range for rows of 1e13
        const float c0 = -s.x * per_col, c1 = -(rs * s.y * per_col) * rs;
        x.forget();
        dy.forget();
#pragma unroll
        for (int e = 0; e < E; e += 4) {
            F2 w[2];
            Row::weights4(sw, t, e, w[0], w[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const F2 x2 = x.get2(e + 2 * k), z = LAYER ? add_f2(x2, minus) : x2, d = dy.get2(e + 2 * k);
                const F2 u = LAYER ? fma_f2(d, w[k], f2(c0, c0)) : mul_f2(d, w[k]);
                x.set2(e + 2 * k, mul_f2(fma_f2(z, f2(c1, c1), u), by));
            }
        }
        if (r < rows)
            x.store(dx_at(r), t, cols);
    }
    copies_wait<0>();
    pdl_trigger(); // the kernel that joins the blocks may settle down
    if (!a.dw && !a.db)
        return;
#pragma unroll
    for (int which = 0; which < SUMS; ++which) {
        float *out = which ? a.db : a.dw;
        float *part = a.partial + ((size_t)which * gridDim.x + blockIdx.x) * cols;
        const auto mine = [&](int e) {
            const float2 v = unf2(which ? db[SUMS > 1 ? e / 2 : 0] : dw[e / 2]);
            return e & 1 ? v.y : v.x;
        };
        const auto leave = [&](int c, float v) {
            if (gridDim.x > 1)
                part[c] = v;
            else if (out)
                out[c] += v;
        };
        if (G == 1) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (Row::col(t, e) < cols)
                    leave(Row::col(t, e), mine(e));
            continue;
        }
        __syncthreads(); // weights, and the sums before, have been read
#pragma unroll
        for (int e = 0; e < E; ++e)
            sw[(g * E + e) * TPR + t] = mine(e);
        __syncthreads();
        for (int i = threadIdx.x; i < TPR * E; i += BT) {
            const int c = Row::col(i % TPR, i / TPR);
            if (c >= cols)
                continue;
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < G; ++k)
                v += sw[k * E * TPR + i];
            leave(c, v);
        }
    }
}

// Adds the parts' column sums to dw and db: 32 columns to a block, a part to every 32nd row of threads.
__global__ void __launch_bounds__(1024) norm_bwd_join(const __grid_constant__ NormArgs a, int parts)
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
        const float var = t.y / a.cols - left * left;
        mu += off_centre(mu, var) ? left : 0.f;
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
        if (cols <= 8 * 16)
            return f.template operator()<T, true, 8, 16>();
        if (cols <= 16 * 16)
            return f.template operator()<T, true, 16, 16>();
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

// Blocks of `kernel` that fit the GPU at once, at most `most` to an SM and one for every `per_block` rows.  `known` keeps how many
// fit an SM (all devices here are alike; asking takes longer than a short row).
int blocks_for(const void *kernel, int threads, size_t smem, std::atomic<int> &known, int most, int n_sm, int64_t rows,
               int per_block)
{
    if (smem > 40 * 1024) // the kernels' own arrays count towards the 48 KB too
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    int per_sm = known.load(std::memory_order_relaxed);
    if (per_sm == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess || per_sm < 1) {
            cudaGetLastError();
            per_sm = 1;
        }
        per_sm = std::min(per_sm, most);
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
        static std::atomic<int> known[4];
        const size_t smem = (size_t)Ring<T, VEC, TPR, E, 1>::BYTES * BT + (size_t)(a.bias ? 2 : 1) * TPR * E * sizeof(float);
        const bool layer = a.kind == PEAGLE_NORM_LAYER;
        const int blocks = blocks_for((const void *)kernel, BT, smem, known[2 * layer + (a.bias != nullptr)],
                                      fwd_blocks(layer, Part<T, VEC, TPR, E>::WORDS, TPR, BT), n_sm, a.rows, BT / TPR);
        kernel<<<blocks, BT, smem, s>>>(a);
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
        if (a.kind == PEAGLE_NORM_LAYER)
            return a.db ? with_sums<T, VEC, true, TPR, E, 2>() : with_sums<T, VEC, true, TPR, E, 1>();
        return a.db ? with_sums<T, VEC, false, TPR, E, 2>() : with_sums<T, VEC, false, TPR, E, 1>();
    }
    template <class T, bool VEC, bool LAYER, int TPR, int E, int SUMS>
    int with_sums() const
    {
        constexpr int BT = block_threads(TPR);
        const auto kernel = norm_bwd_kernel<T, VEC, LAYER, TPR, E, SUMS>;
        // the rows to come; weights, then the sums of the block's groups
        const size_t smem = (size_t)Ring<T, VEC, TPR, E, 2>::BYTES * BT + (size_t)BT * E * sizeof(float);
        static std::atomic<int> known;
        const int blocks = blocks_for((const void *)kernel, BT, smem, known, 32, n_sm, a.rows, BT / TPR);
        if (only_blocks)
            return blocks;
        kernel<<<blocks, BT, smem, s>>>(a);
        if ((!a.dw && !a.db) || blocks == 1)
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
