// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and the gradient.
//
// Forward: one read of the logits.  In powers of two, with l = scale log2(e), m the maximum and c = m l rounded up:
//     t_j = x_j l - c,  S = sum 2^t_j,  E = sum 2^t_j t_j,  log S = ln 2 (log2 S - (m l - c))
//     lse = scale m + log S,  logprob = scale (x_token - m) - log S,  entropy = ln 2 (log2 S - E / S)
// where x l - c and m l - c are fused operations: logprob and entropy do not lose the digits that a large m would
// take.  A thread keeps (m, S, E) and rescales them when its maximum grows; threads, then blocks, join theirs.
// Backward, with log p = scale x - lse:
//     dx_j = scale ( g ([j = token] - p_j) - h p_j (log p_j + entropy) ).
//
// The floor is one read.  A block takes a row in chunks of 16 bytes per thread and load, the next chunk on its way.  Few
// rows are cut into parts for a cluster of up to 16 blocks, which join through distributed shared memory.  4,096 rows of
// 128,000 bf16 take 176 us without alternatives (91 % of the copy rate), 227 with 8 (71 %), 268 with 20 (60 %); 2,048 rows
// of fp32, the same bytes, 200 with 8 (80 %).  (In a loop over one input; over changing ones with 8 it is 233 to 254.)
// Nothing is full (1,184 rows: issue slots 61 % without alternatives, 69 with, 8 and 11 instructions per entry, exp2 unit
// 50 %): a chunk's steps depend on each other, and the 32 warps of an SM do not cover that.  The next chunk but one is
// sent for as soon as a chunk's pieces are in registers and what of them reaches the list is there, which is 3 % faster
// than after the sums.  More alternatives are slow: 304 us with 32, 402 with 48, 554 with 64 (29 %), where the first bound
// is loose, the list overflows between two looks at it and rows are begun again.
//
// Top alternatives, in the same pass: from the first chunk on there is a bound that at least k entries reach (the
// k-th largest of the maxima of 64 groups of threads, then the k-th best entry so far).  A chunk's maximum, which the
// sums need anyway, says whether a thread has anything to add; what reaches the bound goes to a list in shared memory,
// which is cut to its k best when it has grown by half.  The block's warps meet for that only once in four chunks.  A row
// that brings more than the list holds in that time (in ascending order, or of equal entries) is begun again, with a
// meeting for every chunk; a chunk that does not fit even so is gone through again with the bound that the list gives.
// Entries are compared by value, then by id, so the result does not depend on the order in which they came.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "peagle_internal.h"
#include "sm100_ptx.cuh"

namespace peagle {
using namespace sm100;

namespace {

// Blocks of 128 threads: 4,096 rows of 128,000 bf16 with 8 alternatives take 8 % longer with blocks of 256 (the same
// threads per SM, but more of them at a barrier); 8 blocks to an SM, with 10 the registers do not suffice.
constexpr int LP_THREADS = 128, LP_WARPS = LP_THREADS / 32;
constexpr int FWD_PIECES = 4; // 16-byte pieces per thread and chunk
constexpr int GROUPS = 64;     // of threads, whose maxima give the first bound
constexpr int STAGES = 2;     // chunks on their way or at hand
constexpr int LIST = 1024;    // entries of the list of candidates
constexpr int MEET_EVERY = 4; // chunks between two looks at the list
constexpr int COUNTED = 512; // entries that are ranked by counting, at most
constexpr int LEAST_PART = 4096; // entries of a row's part
static_assert(GROUPS >= PEAGLE_MAX_TOP_K && LP_THREADS % GROUPS == 0, "a first bound for every k");
static_assert(8 * PEAGLE_MAX_TOP_K <= COUNTED && COUNTED <= LIST, "the lists of a cluster fit one");
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float T_FLOOR = -300.f; // below this, in powers of two, a probability is zero in fp32
constexpr float REFERENCE_LARGE = 65536.f; // from here on, in powers of two, x l - c has lost digits
constexpr float LSE_LARGE = 8192.f; // from here on fp32 keeps less than 2^-10 of a log-sum-exp
constexpr float INF = __builtin_huge_valf();

__device__ __forceinline__ float nan_f32() { return __int_as_float(0x7fffffff); }
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

// Larger value first, then the lower id.  0: no entry.
__device__ __forceinline__ uint64_t rank_key(float x, int id) { return (uint64_t)order_key(x) << 32 | (uint32_t)~id; }

template <class V, class F>
__device__ __forceinline__ V block_join(V v, F f)
{
    __shared__ V part[LP_WARPS];
    for (int o = 16; o; o >>= 1)
        v = f(v, __shfl_xor_sync(~0u, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[0];
    for (int i = 1; i < LP_WARPS; ++i)
        v = f(v, part[i]);
    return v;
}

// ------------------------------------------------------------------ sums

struct Sums {
    float m, S, E; // E in powers of two
};

// What S and E refer to: m l rounded up, so that no t is above zero, however coarse the numbers near m l are (entries
// masked with -1e30: a thread that has seen nothing else would have a sum of 2^huge, and then infinity times zero).
// Without a maximum S is 0 (or NaN), whatever it refers to.
__device__ __forceinline__ float reference(float m, float l)
{
    return m == -INF ? 0.f : fminf(fmaxf(__fmul_ru(m, l), -3.4028235e38f), 3.4028235e38f);
}

__device__ __forceinline__ void rescale(Sums &s, float m, float l)
{
    if (s.m != -INF && s.m != m) {
        const float d = reference(s.m, l) - reference(m, l), f = fast_exp2(d);
        s.E = f * fmaf(s.S, fmaxf(d, T_FLOOR), s.E);
        s.S *= f;
    }
    s.m = m;
}

__device__ __forceinline__ Sums join(Sums a, Sums b, float l)
{
    const float m = fmaxf(a.m, b.m);
    rescale(a, m, l);
    rescale(b, m, l);
    return {m, a.S + b.S, a.E + b.E};
}

// What a row's log probabilities are formed with: scale (x - m) - logS.
struct RowStats {
    float m, logS, H;
    bool none, empty; // NaN or +inf in the row; nothing but -inf
};

// `c`: what S and E refer to, m l but for the rounding.
__device__ __forceinline__ RowStats row_stats(Sums s, float c, float scale)
{
    RowStats w;
    const float log2S = log2f(s.S);
    w.m = s.m;
    w.logS = (log2S - (c == 0.f ? 0.f : fmaf(s.m, scale * LOG2E, -c))) * LN2;
    w.H = (log2S - s.E / s.S) * LN2;
    w.empty = s.S == 0.f || s.m * scale == -INF; // S of a row with a maximum is about 1 or more
    w.none = s.S != s.S || s.m * scale == INF;
    return w;
}

__device__ __forceinline__ float logprob_of(const RowStats &w, float x, float scale)
{
    return w.none ? nan_f32() : w.empty ? -INF : fmaf(x - w.m, scale, -w.logS);
}

__device__ __forceinline__ void write_row(const LogprobArgs &a, int r, const RowStats &w, float x_token, int token)
{
    float lp = logprob_of(w, x_token, a.scale);
    if (token == -1)
        lp = 0.f;
    else if (token < 0 || token >= a.vocab) {
        lp = nan_f32();
        atomicCAS(a.status, 0, PEAGLE_ERR_BAD_META);
    }
    if (a.logprob)
        a.logprob[r] = lp;
    if (a.lse)
        a.lse[r] = w.none ? nan_f32() : w.empty ? -INF : fmaf(w.m, a.scale, w.logS);
    if (a.entropy)
        a.entropy[r] = w.none ? nan_f32() : w.empty ? 0.f : w.H;
}

// ------------------------------------------------------------------ lists of the best entries

// The k-th best of n >= k entries, bit by bit.  The whole block; a barrier after.
__device__ __noinline__ uint64_t kth_best(const uint64_t *list, int n, int k)
{
    uint64_t bound = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t trial = bound | 1ull << bit;
        int c = 0;
        for (int i = threadIdx.x; i < n; i += LP_THREADS)
            c += list[i] >= trial;
        if (block_join(c, [](int p, int q) { return p + q; }) >= k)
            bound = trial;
    }
    __syncthreads();
    return bound;
}

// An entry's place is the number of better ones: EACH entries to a thread.
template <int EACH>
__device__ __forceinline__ void rank_list(uint64_t *list, int n, int k)
{
    uint64_t mine[EACH];
    int place[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int i = threadIdx.x + j * LP_THREADS;
        mine[j] = i < n ? list[i] : 0;
        place[j] = 0;
    }
    const ulonglong2 *pairs = reinterpret_cast<const ulonglong2 *>(list);
#pragma unroll 8
    for (int o = 0; o < n / 2; ++o) {
        const ulonglong2 other = pairs[o];
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            place[j] += (other.x > mine[j]) + (other.y > mine[j]);
    }
    if (n & 1) {
        const uint64_t other = list[n - 1];
#pragma unroll
        for (int j = 0; j < EACH; ++j)
            place[j] += other > mine[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < EACH; ++j)
        if (mine[j] && place[j] < k)
            list[place[j]] = mine[j];
    __syncthreads();
}

// Sorts a list and cuts it to its k best; an entry of 0 is none.  The whole block; a barrier before and after.
__device__ __noinline__ void cut_list(uint64_t *list, int n, int k)
{
    __shared__ uint64_t kept[PEAGLE_MAX_TOP_K];
    __shared__ int kept_n;
    if (n > COUNTED) {
        const uint64_t bound = kth_best(list, n, k);
        if (threadIdx.x == 0)
            kept_n = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += LP_THREADS)
            if (list[i] >= bound)
                kept[atomicAdd(&kept_n, 1)] = list[i];
        __syncthreads();
        n = k;
        if (threadIdx.x < k)
            list[threadIdx.x] = kept[threadIdx.x];
        __syncthreads();
    }
    if (n <= LP_THREADS)
        rank_list<1>(list, n, k);
    else if (n <= 2 * LP_THREADS)
        rank_list<2>(list, n, k);
    else
        rank_list<COUNTED / LP_THREADS>(list, n, k);
}

__device__ __forceinline__ uint64_t load_remote(const uint64_t *p, uint32_t rank)
{
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_map(smem_u32(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ float load_remote(const float *p, uint32_t rank)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_map(smem_u32(p), rank)) : "memory");
    return v;
}

// ------------------------------------------------------------------ forward

// 16 bytes of a row: logits in order.
template <class T>
struct Piece {
    static constexpr int N = 16 / sizeof(T);
    uint4 v;
    __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(word(e));
        else
            return __uint_as_float(e & 1 ? word(e / 2) & 0xffff0000u : word(e / 2) << 16);
    }
    // Entries outside [lo, hi) become -inf.
    __device__ __forceinline__ void mask(int lo, int hi)
    {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < lo || e >= hi) {
                if constexpr (sizeof(T) == 4)
                    w[e] = 0xff800000u;
                else
                    w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | 0xff800000u : (w[e / 2] & 0xffff0000u) | 0xff80u;
            }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
// The largest entries of a piece, as one word: a number, or one of the even and one of the odd entries.
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t piece_max(const Piece<float> &p)
{
    return __float_as_uint(fmaxf(max3(p.get(0), p.get(1), p.get(2)), p.get(3)));
}
__device__ __forceinline__ uint32_t piece_max(const Piece<__nv_bfloat16> &p)
{
    return max_bf16x2(max_bf16x2(p.v.x, p.v.y), max_bf16x2(p.v.z, p.v.w));
}
template <class T>
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b)
{
    if constexpr (sizeof(T) == 4)
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    else
        return max_bf16x2(a, b);
}
template <class T>
__device__ __forceinline__ float of_max_word(uint32_t w)
{
    if constexpr (sizeof(T) == 4)
        return fmaxf(__uint_as_float(w), -INF); // a piece of nothing but NaN has no maximum
    else
        return max3(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u), -INF);
}

// Two bf16 entries that are no less than `low`, a NaN as it is.
__device__ __forceinline__ uint32_t raised(uint32_t w, uint32_t low)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(low));
    return r;
}

// A block per part of a row; `parts` blocks, a cluster, have a row.  part_len is a multiple of 8.
template <class T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, 8)
    logprobs_fwd_kernel(const __grid_constant__ LogprobArgs a, int parts, int part_len)
{
    constexpr int N = Piece<T>::N, U = FWD_PIECES, STEP = U * LP_THREADS;
    // a thread's pieces wait in its own places: no barrier between their arrival and their use
    extern __shared__ uint4 ring[]; // [STAGES][U][LP_THREADS]
    __shared__ __align__(16) uint64_t list[TOP ? LIST : 2];
    __shared__ int count; // entries that came to the list; those past its end have been dropped
    __shared__ float4 first_max[TOP ? GROUPS / 4 : 1];
    __shared__ float first_bound;
    __shared__ uint64_t share_bound;
    __shared__ Sums warp_sums[LP_WARPS], sums;
    __shared__ RowStats stats;
    const int r = blockIdx.x / parts, part = blockIdx.x - r * parts;
    const int begin = part * part_len, n = max(0, min(a.vocab - begin, part_len));
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
    // whole 16-byte pieces that hold an entry of this part; `before` entries of the first belong elsewhere
    const int before = (int)(reinterpret_cast<uintptr_t>(row + begin) % 16 / sizeof(T));
    const int pieces = n ? (before + n + N - 1) / N : 0;
    const float l = a.scale * LOG2E;
    const uint32_t ring_at = smem_u32(ring + threadIdx.x);

    const T *x = row; // this thread's first piece of the next chunk to be fetched
    const auto fetch = [&](int first, int stage) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + u * LP_THREADS + (int)threadIdx.x < pieces)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring_at + (stage * U + u) * LP_THREADS * 16),
                             "l"(x + u * LP_THREADS * N)
                             : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
        x += STEP * N;
    };
    Sums s;
    // A list that has grown by half is cut.  (4,096 rows of 128,000, k = 20: 4 % longer when it is cut where it has
    // tripled.)  A short part ends before that pays.
    const int long_list = pieces <= 4 * STEP ? max(LP_THREADS - 8, a.top_k + a.top_k / 2) : a.top_k + a.top_k / 2 + 6;
    // Looking at the list means that all warps wait for the slowest.  (4,096 rows of 128,000 bf16, k = 8: 5 % longer with
    // a look at every chunk than at every fourth; 2,048 rows of fp32 the same.)  A row that overflows the list unseen
    // is begun again.
    for (int every = MEET_EVERY;; every = 1) {
        x = row + begin - before + threadIdx.x * N;
#pragma unroll
        for (int i = 0; i < STAGES; ++i)
            fetch(i * STEP, i);
        if (TOP && threadIdx.x == 0)
            count = 0;
        s = {-INF, 0.f, 0.f};
        float bound = -INF; // an entry at or above it may be among the k best
        int end = 0;        // how far this thread has filled the list since the warps met
        bool overflow = false;
        int stage = 0;
        for (int first = 0; first < pieces; first += STEP) {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            const uint4 *at = ring + stage * STEP + threadIdx.x;
            Piece<T> now[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                now[u].v = at[u * LP_THREADS];
            if (first == 0 || first + STEP >= pieces) { // with the first piece, the last, or none
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = first + u * LP_THREADS + threadIdx.x;
                    if (i == 0 || i >= pieces - 1)
                        now[u].mask(i < pieces ? before - i * N : N, before + n - i * N);
                }
            }
            uint32_t most[U], all = piece_max(now[0]);
            most[0] = all;
#pragma unroll
            for (int u = 1; u < U; ++u) {
                most[u] = piece_max(now[u]);
                all = max_words<T>(all, most[u]);
            }
            const float top = of_max_word<T>(all);
            const auto offer = [&](float v, int id, uint64_t least) {
                const uint64_t key = rank_key(v, begin + id);
                if (id >= 0 && id < n && key >= least) {
                    const int place = atomicAdd(&count, 1);
                    if (place < LIST)
                        list[place] = key;
                    end = place + 1;
                }
            };
            if constexpr (TOP) {
                const int k = a.top_k;
                if (first == 0) { // the k-th largest of the maxima of 64 groups of threads
                    constexpr int LANES = LP_THREADS / GROUPS;
                    float most = top;
#pragma unroll
                    for (int o = 1; o < LANES; o *= 2)
                        most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
                    if (threadIdx.x % LANES == 0)
                        reinterpret_cast<float *>(first_max)[threadIdx.x / LANES] = most;
                    __syncthreads();
                    if (threadIdx.x < GROUPS) {
                        most = reinterpret_cast<float *>(first_max)[threadIdx.x];
                        int above = 0, equal = 0;
#pragma unroll
                        for (int i = 0; i < GROUPS / 4; ++i) {
                            const float4 o = first_max[i];
                            above += (o.x > most) + (o.y > most) + (o.z > most) + (o.w > most);
                            equal += (o.x == most) + (o.y == most) + (o.z == most) + (o.w == most);
                        }
                        if (above < k && above + equal >= k)
                            first_bound = most;
                    }
                    __syncthreads();
                    bound = first_bound;
                }
                if (top >= bound) {
                    // which of the entries reach the bound, without a branch among a piece's: a thread on this path
                    // keeps its whole block waiting
                    uint32_t reach = 0;
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (of_max_word<T>(most[u]) >= bound) {
#pragma unroll
                            for (int e = 0; e < N; ++e)
                                reach |= (uint32_t)(now[u].get(e) >= bound) << (u * N + e);
                        }
                    for (; reach; reach &= reach - 1) {
                        const int i = __ffs(reach) - 1, u = i / N, e = i % N;
                        offer(to_f32(reinterpret_cast<const T *>(at + u * LP_THREADS)[e]),
                              (first + u * LP_THREADS + (int)threadIdx.x) * N + e - before, 0);
                    }
                }
            }
            fetch(first + STAGES * STEP, stage); // into the places of this chunk, which the thread has in registers
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            if (top > s.m)
                rescale(s, top, l);
            const float c = reference(s.m, l);
            // Entries whose probability is zero in any case are raised to where 0 times their t is 0: as pairs of bf16
            // here, else one by one.  The second term is more than the rounding to bf16 takes off.  (Beside a maximum
            // near the end of the type's range there is no room for that: see below.)
            const float from = s.m == -INF ? 0.f : s.m;
            const float low = fabsf(from) < 1e37f ? fmaf(fabsf(from), -0x1p-6f, from + T_FLOOR / l) : -INF;
            const uint32_t low2 = pack_bf16x2(low, low);
            const F2 l2 = f2(l, l), minus = f2(-c, -c);
            F2 S2 = f2(s.S, 0.f), E2 = f2(s.E, 0.f);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    F2 v;
                    if constexpr (ENTROPY && N == 8) {
                        const uint32_t w = raised(now[u].word(e / 2), low2);
                        v = f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
                    } else {
                        v = f2(now[u].get(e), now[u].get(e + 1));
                    }
                    F2 t = fma_f2(v, l2, minus);
                    const float2 tv = unf2(t);
                    const F2 p = f2(fast_exp2(tv.x), fast_exp2(tv.y));
                    S2 = add_f2(S2, p);
                    if (ENTROPY && N == 4)
                        t = f2(fmaxf(tv.x, T_FLOOR), fmaxf(tv.y, T_FLOOR));
                    if (ENTROPY)
                        E2 = fma_f2(p, t, E2);
                }
            const float2 Sv = unf2(S2), Ev = unf2(E2);
            s.S = Sv.x + Sv.y;
            if constexpr (ENTROPY && N == 8) {
                const float E = Ev.x + Ev.y;
                if (E != E && s.S == s.S) {
#pragma unroll 1
                    for (int i = 0; i < U * N; ++i) {
                        const int id = (first + i / N * LP_THREADS + (int)threadIdx.x) * N + i % N - before;
                        if (id < 0 || id >= n)
                            continue;
                        const float t = fmaf(to_f32(row[begin + id]), l, -c);
                        s.E = fmaf(fast_exp2(t), fmaxf(t, T_FLOOR), s.E);
                    }
                } else {
                    s.E = E;
                }
            } else {
                s.E = Ev.x + Ev.y;
            }
            if constexpr (TOP) {
                const int k = a.top_k;
                while (true) {
                    const bool meet = first / STEP % every == every - 1;
                    if (!meet || !__syncthreads_or(end > long_list)) {
                        if (meet)
                            end = 0;
                        if (first == 0)
                            bound = from_key(order_key(bound) + 1); // k entries of this chunk, with lower ids, reach it
                        break;
                    }
                    end = 0;
                    if (count <= LIST) {
                        cut_list(list, count, k);
                        if (threadIdx.x == 0)
                            count = k;
                        bound = from_key((uint32_t)(list[k - 1] >> 32) + 1); // the k best have lower ids than what follows
                        __syncthreads();
                        break;
                    }
                    if (every > 1) {
                        overflow = true;
                        break;
                    }
                    // once more, for what reaches the k-th best of those that found a place
                    const uint64_t least = kth_best(list, LIST, k);
                    uint64_t mine[LIST / LP_THREADS];
#pragma unroll
                    for (int j = 0; j < LIST / LP_THREADS; ++j)
                        mine[j] = list[threadIdx.x + j * LP_THREADS];
                    __syncthreads();
                    if (threadIdx.x == 0)
                        count = 0;
                    __syncthreads();
                    const int chunk_id = begin + first * N - before;
#pragma unroll
                    for (int j = 0; j < LIST / LP_THREADS; ++j)
                        if (mine[j] >= least && (int)~(uint32_t)mine[j] < chunk_id) // from the chunks before
                            list[atomicAdd(&count, 1)] = mine[j];
                    __syncthreads(); // these, k at most, have their places before the chunk's entries take theirs
                    bound = from_key((uint32_t)(least >> 32));
#pragma unroll 1
                    for (int i = 0; i < U * N; ++i) {
                        const int id = (first + i / N * LP_THREADS + (int)threadIdx.x) * N + i % N - before;
                        if (id >= 0 && id < n) {
                            const float v = to_f32(row[begin + id]);
                            if (v >= bound)
                                offer(v, id, least);
                        }
                    }
                }
            }
            if (TOP && overflow)
                break;
        }
        if (!TOP)
            break;
        __syncthreads();
        if (count <= LIST)
            break;
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads(); // everybody has seen the count
    }

    // join the threads' sums, then the blocks'
    for (int o = 16; o; o >>= 1) {
        const Sums other = {__shfl_xor_sync(~0u, s.m, o), __shfl_xor_sync(~0u, s.S, o), __shfl_xor_sync(~0u, s.E, o)};
        s = join(s, other, l);
    }
    if ((threadIdx.x & 31) == 0)
        warp_sums[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x < 32) {
        s = warp_sums[threadIdx.x % LP_WARPS];
        for (int o = LP_WARPS / 2; o; o >>= 1) {
            const Sums other = {__shfl_xor_sync(~0u, s.m, o), __shfl_xor_sync(~0u, s.S, o), __shfl_xor_sync(~0u, s.E, o)};
            s = join(s, other, l);
        }
        if (threadIdx.x == 0)
            sums = s;
    }
    if (TOP) {
        const int held = count;
        cut_list(list, held, a.top_k);
        if ((int)threadIdx.x >= held && threadIdx.x < a.top_k)
            list[threadIdx.x] = 0;
    }
    if (parts > 1) {
        cluster_sync_all();
        if (part == 0) {
            if (threadIdx.x < 32) {
                const int p = threadIdx.x % parts; // a power of two
                s = {load_remote(&sums.m, p), load_remote(&sums.S, p), load_remote(&sums.E, p)};
                for (int o = 1; o < parts; o *= 2) {
                    const Sums other = {__shfl_xor_sync(~0u, s.m, o), __shfl_xor_sync(~0u, s.S, o), __shfl_xor_sync(~0u, s.E, o)};
                    s = join(s, other, l);
                }
            }
            if (TOP) {
                const int k = a.top_k;
                uint64_t theirs[COUNTED / LP_THREADS];
#pragma unroll
                for (int j = 0; j < COUNTED / LP_THREADS; ++j) {
                    const int i = threadIdx.x + j * LP_THREADS;
                    theirs[j] = i < parts * k ? load_remote(&list[i % k], i / k) : 0;
                }
                // what is below the part's share of k in every part is not among the k best
                const int share = (k - 1) / parts;
                uint64_t least = threadIdx.x < parts ? load_remote(&list[share], threadIdx.x) : ~0ull;
                for (int o = 8; o; o >>= 1) {
                    const uint64_t other = __shfl_xor_sync(~0u, least, o);
                    least = other < least ? other : least;
                }
                __syncthreads(); // the first part's own list has been read
                if (threadIdx.x == 0) {
                    share_bound = least;
                    count = 0;
                }
                __syncthreads();
                least = share_bound;
#pragma unroll
                for (int j = 0; j < COUNTED / LP_THREADS; ++j)
                    if (theirs[j] && theirs[j] >= least)
                        list[atomicAdd(&count, 1)] = theirs[j];
                __syncthreads();
                cut_list(list, count, k);
            }
        }
        cluster_sync_all(); // nobody leaves while its lists are read
        if (part != 0)
            return;
    }
    const int token = a.tokens ? a.tokens[r] : -1;
    const float x_token = token >= 0 && token < a.vocab ? to_f32(row[token]) : 0.f;
    if (threadIdx.x == 0) {
        sums = s;
        stats = row_stats(s, reference(s.m, l), a.scale);
        write_row(a, r, stats, x_token, token);
    }
    __syncthreads();
    s = sums;
    if (fabsf(s.m) < INF && fabsf(s.m * l) >= REFERENCE_LARGE) {
        // a row of numbers far from zero, masked throughout for one: again, with x - m in the place of x
        const float m = s.m;
        double S = 0.0, E = 0.0; // long sums of single entries
        for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS) {
            const float t = (to_f32(row[j]) - m) * l, p = fast_exp2(t);
            S += p;
            E += p * fmaxf(t, T_FLOOR);
        }
        S = block_join(S, [](double p, double q) { return p + q; });
        E = block_join(E, [](double p, double q) { return p + q; });
        if (threadIdx.x == 0) {
            stats = row_stats({m, (float)S, (float)E}, 0.f, a.scale);
            write_row(a, r, stats, x_token, token);
        }
        __syncthreads();
    }
    if (TOP && threadIdx.x < a.top_k) {
        const RowStats w = stats;
        const uint64_t key = list[threadIdx.x];
        const size_t at = (size_t)r * a.top_k + threadIdx.x;
        a.top[at] = logprob_of(w, from_key((uint32_t)(key >> 32)), a.scale);
        a.ids[at] = w.none ? -1 : (int)~(uint32_t)key;
    }
}

// ------------------------------------------------------------------ backward

// 16-byte pieces per thread.  They are read and written as data that is not used again: 4,096 rows of 128,000 bf16 took
// 330 us, through ordinary accesses 366.  With the arithmetic on pairs of fp32 they take 301, the rate of a copy (element
// by element it issued in 80 % of the cycles).
constexpr int BWD_PIECES = 4;

// A block per BWD_PIECES * LP_THREADS pieces of a row.
template <class T, bool ENTROPY>
__global__ void __launch_bounds__(LP_THREADS) logprobs_bwd_kernel(const __grid_constant__ LogprobArgs a, int parts)
{
    constexpr int N = Piece<T>::N;
    const int r = blockIdx.x / parts, part = blockIdx.x - r * parts;
    const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
    T *out = static_cast<T *>(a.dlogits) + (size_t)r * a.ldd;
    const int token = a.g_lp ? a.tokens[r] : -1;
    const bool given = token >= 0 && token < a.vocab;
    const float g = given ? a.g_lp[r] : 0.f, h = ENTROPY ? a.g_h[r] : 0.f, lse = a.lse_in[r];
    const float H = ENTROPY ? a.entropy_in[r] : 0.f;
    const bool zero = (g == 0.f && h == 0.f) || lse == -INF;
    // the token's own entry, of t = log p: 1 - p without the digits that p near 1 would take
    const auto of_token = [&](float t) {
        const float p = fast_exp2(t * LOG2E);
        return a.scale * (-g * expm1f(t) - (ENTROPY ? p * h * (fmaxf(t, T_FLOOR) + H) : 0.f));
    };
    if (!zero && fabsf(lse) >= LSE_LARGE) {
        // from the row itself: one block, so that dlogits may be logits
        if (part != 0)
            return;
        float m = -INF;
        for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS)
            m = fmaxf(m, to_f32(row[j]));
        m = block_join(m, [](float p, float q) { return fmaxf(p, q); });
        double S = 0.0; // a long sum of single entries
        for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS)
            S += fast_exp2((to_f32(row[j]) - m) * a.scale * LOG2E);
        const float logS = logf((float)block_join(S, [](double p, double q) { return p + q; }));
        for (int j = threadIdx.x; j < a.vocab; j += LP_THREADS) {
            const float t = (to_f32(row[j]) - m) * a.scale - logS, p = fast_exp2(t * LOG2E);
            from_f32(out + j, j == token ? of_token(t) : a.scale * p * (-g - h * (fmaxf(t, T_FLOOR) + H)));
        }
        return;
    }
    const int before = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
    const bool alike = reinterpret_cast<uintptr_t>(out) % 16 / sizeof(T) == before;
    const int pieces = (before + a.vocab + N - 1) / N;
    const int first = part * BWD_PIECES * LP_THREADS + threadIdx.x;
    Piece<T> p[BWD_PIECES];
    if (!zero) {
#pragma unroll
        for (int u = 0; u < BWD_PIECES; ++u)
            if (first + u * LP_THREADS < pieces)
                p[u].v = __ldcs(reinterpret_cast<const uint4 *>(row - before + (size_t)(first + u * LP_THREADS) * N));
    }
    // v = p (c0 + c1 t)
    const float c1 = -h * a.scale, c0 = fmaf(c1, H, -g * a.scale);
    const F2 scale2 = f2(a.scale, a.scale), minus = f2(-lse, -lse), log2e = f2(LOG2E, LOG2E);
#pragma unroll
    for (int u = 0; u < BWD_PIECES; ++u) {
        const int i = first + u * LP_THREADS, id = i * N - before;
        if (i >= pieces)
            break;
        float v[N];
        if (zero) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                v[e] = 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const F2 t = fma_f2(f2(p[u].get(e), p[u].get(e + 1)), scale2, minus);
                const float2 t2 = unf2(mul_f2(t, log2e)), tv = unf2(t);
                const F2 prob = f2(fast_exp2(t2.x), fast_exp2(t2.y));
                F2 w = f2(c0, c0);
                if (ENTROPY)
                    w = fma_f2(f2(c1, c1), f2(fmaxf(tv.x, T_FLOOR), fmaxf(tv.y, T_FLOOR)), w);
                const float2 d = unf2(mul_f2(prob, w));
                v[e] = d.x;
                v[e + 1] = d.y;
            }
            if ((unsigned)(token - id) < (unsigned)N && given) {
                const float own = of_token(fmaf(to_f32(row[token]), a.scale, -lse));
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (id + e == token)
                        v[e] = own;
            }
        }
        if (alike && id >= 0 && id + N <= a.vocab) {
            uint4 w;
            if constexpr (sizeof(T) == 4)
                w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            else
                w = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                               pack_bf16x2(v[6], v[7]));
            __stcs(reinterpret_cast<uint4 *>(out + id), w);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (id + e >= 0 && id + e < a.vocab)
                    from_f32(out + id + e, v[e]);
        }
    }
}

constexpr int FWD_SMEM = STAGES * FWD_PIECES * LP_THREADS * 16;

// Whether the GPU places clusters of 16 blocks of a kernel, more than every GPU has to.  Asked once per kernel (all
// devices here are alike), which is the template's argument: the instances share a type, not registers and shared memory.
template <auto KERNEL>
bool takes_16()
{
    static std::atomic<int> known; // 0 not asked, 1 no, 2 yes
    if (cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    if (known.load(std::memory_order_relaxed) == 0) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 16;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3(16);
        cfg.blockDim = dim3(LP_THREADS);
        cfg.dynamicSmemBytes = FWD_SMEM;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        int n = 0;
        const bool yes = cudaOccupancyMaxActiveClusters(&n, KERNEL, &cfg) == cudaSuccess && n > 0;
        if (!yes)
            cudaGetLastError();
        known.store(yes ? 2 : 1, std::memory_order_relaxed);
    }
    return known.load(std::memory_order_relaxed) == 2;
}

template <class T, bool ENTROPY, bool TOP>
void forward(const LogprobArgs &a, int n_sm, cudaStream_t s)
{
    constexpr auto kernel = logprobs_fwd_kernel<T, ENTROPY, TOP>;
    // few rows are cut as long as the GPU has places left
    int parts = 1;
    while (parts < 8 && (int64_t)a.rows * parts * 2 <= 8 * n_sm && a.vocab / (parts * 2) >= LEAST_PART)
        parts *= 2;
    // clusters of 16 are harder to place: 16 rows of 128,000 take 20.7 us with them and 14.4 without, one 13.3 and 13.4
    if (parts == 8 && a.rows <= 4 && a.vocab / 16 >= LEAST_PART && 16 * a.top_k <= COUNTED && takes_16<kernel>())
        parts = 16;
    const int part_len = ((a.vocab + parts - 1) / parts + 7) / 8 * 8;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)a.rows * parts);
    cfg.blockDim = dim3(LP_THREADS);
    cfg.dynamicSmemBytes = FWD_SMEM;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    cudaLaunchKernelEx(&cfg, kernel, a, parts, part_len);
}

template <class T>
void forward_of(const LogprobArgs &a, int n_sm, cudaStream_t s)
{
    if (a.top_k)
        a.entropy ? forward<T, true, true>(a, n_sm, s) : forward<T, false, true>(a, n_sm, s);
    else
        a.entropy ? forward<T, true, false>(a, n_sm, s) : forward<T, false, false>(a, n_sm, s);
}

template <class T>
int backward_of(const LogprobArgs &a, cudaStream_t s)
{
    // a row that begins inside a piece may take one more
    const int64_t pieces = ((int64_t)a.vocab + 2 * Piece<T>::N - 2) / Piece<T>::N;
    const int parts = (int)((pieces + BWD_PIECES * LP_THREADS - 1) / (BWD_PIECES * LP_THREADS));
    if ((int64_t)a.rows * parts > INT32_MAX)
        return PEAGLE_ERR_TOO_LARGE;
    if (a.g_h)
        logprobs_bwd_kernel<T, true><<<(unsigned)a.rows * parts, LP_THREADS, 0, s>>>(a, parts);
    else
        logprobs_bwd_kernel<T, false><<<(unsigned)a.rows * parts, LP_THREADS, 0, s>>>(a, parts);
    return 1;
}

} // namespace

int launch_logprobs_fwd(const LogprobArgs &a, int n_sm, cudaStream_t s)
{
    a.dtype == PEAGLE_F32 ? forward_of<float>(a, n_sm, s) : forward_of<__nv_bfloat16>(a, n_sm, s);
    return 1;
}

int launch_logprobs_bwd(const LogprobArgs &a, cudaStream_t s)
{
    return a.dtype == PEAGLE_F32 ? backward_of<float>(a, s) : backward_of<__nv_bfloat16>(a, s);
}

} // namespace peagle
