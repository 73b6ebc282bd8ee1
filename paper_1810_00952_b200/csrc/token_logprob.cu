// Log-probabilities of given tokens, entropies and the most probable tokens of rows of scores, and the gradient group.
// HBM-bound: the forward call reads every score once, the gradient reads and writes it once.
#include <algorithm>

#include "common.h"
#include "ewise_kernels.cuh"
#include "tc_common.cuh"

namespace relay {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float load_score(const T *p)
{
    if (!relay_in_bounds(p, sizeof(T))) return 0.0f;
    if constexpr (sizeof(T) == 2) return __bfloat162float(*p);
    else return *p;
}
// the class a row's token names, -1 if none
__device__ __forceinline__ int token_of(const void *tokens, int is_i64, long long row, int V)
{
    const long long t = is_i64 ? ((const long long *)tokens)[row] : ((const int *)tokens)[row];
    return t >= 0 && t < V ? (int)t : -1;
}

// ---- temperature ---------------------------------------------------------------------------------------------------
// 1 / temperature as a sum of two floats, and log2(e) / temperature
struct Scale { float inv, inv_lo, log2e; };
inline Scale scale_of(float temperature)
{
    const double inv = 1.0 / (double)temperature;
    Scale k;
    k.inv = (float)inv;
    k.inv_lo = (float)(inv - (double)k.inv);
    k.log2e = (float)(1.4426950408889634 * inv);
    return k;
}
// z / temperature - lse with one rounding of the result's own size: the product stays exact inside the multiply-add, so a
// probability is as good where the scores are far from zero.  A score of -inf gives -inf.
__device__ __forceinline__ float log_prob(float z, float lse, const Scale &k)
{
    return fmaf(fmaxf(z, -3.0e38f), k.inv_lo, fmaf(z, k.inv, -lse));
}

// ---- sums of one row, joinable in any order of parts, d = z - m ----------------------------------------------------------
//   m = max z,  s = sum exp(d / temperature),  w = sum exp(d / temperature) d
//   lse = m / temperature + log s;   logp = d / temperature - log s;   entropy = log s - w / (s temperature)
// Everything but lse itself is free of m's size.  A part without a score above -inf has m = -inf, s = w = 0; a NaN stays in m.
struct Sums { float m, s, w; };

__device__ __forceinline__ Sums empty_sums() { return Sums{-INFINITY, 0.0f, 0.0f}; }
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float exp2_(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// a finite difference even where a score or the maximum is infinite: its exponential is 0 and its product with that too
__device__ __forceinline__ float below(float z, float m) { return fmaxf(z - m, -1.0e30f); }

__device__ __forceinline__ Sums join(const Sums &a, const Sums &b, const Scale &k)
{
    Sums r;
    r.m = max_nan(a.m, b.m);
    const float da = below(a.m, r.m), db = below(b.m, r.m);
    const float ea = exp2_(da * k.log2e), eb = exp2_(db * k.log2e);
    // written out, so that every kernel rounds alike
    r.s = fmaf(a.s, ea, __fmul_rn(b.s, eb));
    r.w = fmaf(ea, fmaf(da, a.s, a.w), __fmul_rn(eb, fmaf(db, b.s, b.w)));
    return r;
}
__device__ __forceinline__ Sums shfl_xor(const Sums &a, int d)
{
    return Sums{__shfl_xor_sync(0xffffffffu, a.m, d), __shfl_xor_sync(0xffffffffu, a.s, d), __shfl_xor_sync(0xffffffffu, a.w, d)};
}

// what a row's sums say
struct Row {
    float m, log_s, entropy, lse;
    __device__ __forceinline__ Row(const Sums &a, const Scale &k)
    {
        m = a.m;
        log_s = logf(a.s);
        lse = fmaf(a.m, k.inv, log_s);
        entropy = log_s - __fdiv_rn(__fmul_rn(a.w, k.inv), a.s);
        if (a.m == -INFINITY) { lse = -INFINITY; entropy = 0.0f; }
        else if (!(a.m < INFINITY)) lse = entropy = log_s = __int_as_float(0x7fc00000);
    }
    __device__ __forceinline__ float logp(float z, const Scale &k) const
    {
        return m == -INFINITY ? -INFINITY : fmaf(z - m, k.inv, -log_s);
    }
};

struct Args {
    const void *z;
    const void *tokens;            // null: no logp
    int tokens_i64;
    Scale k;
    float *logp, *entropy, *lse, *top_logp;
    int *top_ids;
    int top;
    long long rows;
    int V;
};

struct GradArgs {
    const void *z;
    const void *tokens;
    int tokens_i64;
    Scale k;
    const float *lse, *entropy, *dlogp, *dentropy;
    void *dz;
    long long rows;
    int V;
};

// ---- order of the scores: larger first, equal ones by the lower id, NaN before everything ------------------------------
// One 64-bit key, different for every class: the score's bits as an ordered unsigned number, then the complement of the id.
__device__ __forceinline__ unsigned long long key_of(float z, int id)
{
    uint32_t b = __float_as_uint(z + 0.0f);               // -0 counts as +0
    b = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    if (z != z) b = 0xfffffffeu;                          // above +inf, and below the largest key, which names nothing
    return ((unsigned long long)b << 32) | (uint32_t)~(uint32_t)id;
}
__device__ __forceinline__ int id_of(unsigned long long key) { return (int)~(uint32_t)key; }

// ---- rows as 16-byte vectors --------------------------------------------------------------------------------------
template <typename T> struct Vec { static constexpr int E = 16 / (int)sizeof(T); };

__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// largest element of a vector (a NaN wins)
__device__ __forceinline__ float largest(const uint4 &q, const __nv_bfloat16 *)
{
    const uint32_t m = max2_nan(max2_nan(q.x, q.y), max2_nan(q.z, q.w));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}
__device__ __forceinline__ float largest(const uint4 &q, const float *)
{
    return max_nan(max_nan(__uint_as_float(q.x), __uint_as_float(q.y)), max_nan(__uint_as_float(q.z), __uint_as_float(q.w)));
}
// the elements with -inf raised to a finite value, so that 0 times its distance is 0
__device__ __forceinline__ void finite_elements(const uint4 &q, float (&x)[8])
{
    const uint32_t low = 0xff7fff7fu;                      // the lowest finite value, twice
    unpack(make_uint4(max2_nan(q.x, low), max2_nan(q.y, low), max2_nan(q.z, low), max2_nan(q.w, low)), x);
}
__device__ __forceinline__ void finite_elements(const uint4 &q, float (&x)[4])
{
    unpack(q, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = max_nan(x[i], __uint_as_float(0xff7fffffu));
}
__device__ __forceinline__ unsigned long long pair(float lo, float hi)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(unsigned long long r, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(r)); }
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// One thread's running sums, in pairs; m is raised (and the sums scaled down) only when a vector holds something larger, some
// ln(vectors) times a row.
// Differences from -inf: the scores are raised to the lowest finite value first, so that 0 times the distance is 0; only where the
// maximum itself is that low (masks of the lowest value and nothing else) are the elements looked at one by one.
struct Running {
    float m = -INFINITY;
    unsigned long long s = 0, w = 0;                       // two partial sums each
    float best = -INFINITY;                                // largest element so far, and the first vector that holds it
    int best_at = -1;
    template <typename T>
    __device__ __forceinline__ void take(const uint4 &q, int j, const Scale &k, const T *type)
    {
        constexpr int E = Vec<T>::E;
        const float top = largest(q, type);
        if (!(top <= m)) {                                 // larger, or NaN
            const float d = below(m, top), f = exp2_(d * k.log2e);
            float s0, s1, w0, w1;
            unpair(s, s0, s1); unpair(w, w0, w1);
            w = pair(f * fmaf(d, s0, w0), f * fmaf(d, s1, w1));
            s = pair(f * s0, f * s1);
            m = max_nan(m, top);
        }
        if (top > best || best_at < 0) { best = top; best_at = j; }
        float x[E];
        if (m < -1.0e36f) {
            if (m == -INFINITY) return;                    // nothing but -inf so far
            unpack(q, x);
            float s0, s1, w0, w1;
            unpair(s, s0, s1); unpair(w, w0, w1);
            for (int i = 0; i < E; ++i)
                if (x[i] != -INFINITY) {
                    const float d = x[i] - m, e = exp2_(d * k.log2e);
                    s0 += e;
                    w0 = fmaf(e, d, w0);
                }
            s = pair(s0, s1); w = pair(w0, w1);
            return;
        }
        finite_elements(q, x);
        const unsigned long long nm = pair(-m, -m), c = pair(k.log2e, k.log2e);
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const unsigned long long d = add2(pair(x[i], x[i + 1]), nm);
            float t0, t1;
            unpair(mul2(d, c), t0, t1);
            const unsigned long long e = pair(exp2_(t0), exp2_(t1));
            s = add2(s, e);
            w = fma2(e, d, w);
        }
    }
    __device__ __forceinline__ Sums sums() const
    {
        float s0, s1, w0, w1;
        unpair(s, s0, s1); unpair(w, w0, w1);
        return Sums{m, s0 + s1, w0 + w1};
    }
};
// Vector j of a row: its elements j E .. j E + E - 1 (-inf behind the row's end), wherever the row starts in memory, so that a
// row's result does not depend on its place.  `skew`: how many elements before the row's first the nearest 16-byte boundary lies;
// then two aligned pieces are read and shifted (the second is the next thread's first, and in L1).
template <typename T>
struct RowVectors {
    const T *aligned;                  // the row's start, rounded down
    int skew, V, safe;                 // vectors below `safe` can be read as whole pieces
    __device__ __forceinline__ RowVectors(const T *z, long long rows, long long row, int V_) : V(V_)
    {
        constexpr int E = Vec<T>::E;
        const long long at = row * V, left = rows * V - at;        // elements from the row's start to the tensor's end
        skew = (int)(at % E);
        aligned = z + (at - skew);
        // piece j + 1 ends (j + 2) E - skew elements behind the row's start
        const long long inside = skew == 0 ? V / E : (left + skew) / E - 1;
        safe = (int)min((long long)(V / E), max(inside, 0ll));
    }
    __device__ __forceinline__ int count() const { return (int)(((long long)V + Vec<T>::E - 1) / Vec<T>::E); }
    __device__ __forceinline__ uint4 operator[](int j) const
    {
        constexpr int E = Vec<T>::E;
        const T *at = aligned + (long long)j * E;
        if (j < safe) {
            if (skew == 0) return ld_stream(at);
            uint4 lo{}, hi{};
            if (relay_in_bounds(at, 32)) { lo = __ldg((const uint4 *)at); hi = __ldg((const uint4 *)at + 1); }
            uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            const int bytes = skew * (int)sizeof(T);
            if (bytes & 8) {
#pragma unroll
                for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
            }
            if (bytes & 4) {
#pragma unroll
                for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
            }
            if (bytes & 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
            }
            return make_uint4(w[0], w[1], w[2], w[3]);
        }
        float x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = (long long)j * E + i < V ? load_score(at + skew + i) : -INFINITY;
        return pack(x);
    }
};

// ---- forward: a cluster of S blocks per row ------------------------------------------------------------------------------
// Each block sums a contiguous part of the row's vectors; the blocks' sums meet in block 0's shared memory.
// Alternatives: a thread remembers its largest element; of the largest of G groups of threads the K-th is a bound that the row's
// K-th largest element cannot be below, so only the groups whose largest reaches it are looked through again (their vectors come
// from L2) and what reaches it is listed; the position of a listed element is the number of larger ones.
constexpr int kList = 512;             // listed elements: K of them by the bound, and as many as happen to share their groups
constexpr int kWarpsPerBlock = kThreads / 32;

struct Lists {
    unsigned long long group[kThreads];
    unsigned long long list[kList];
    unsigned long long chosen[RELAY_MAX_TOP];
    unsigned long long merged[8 * RELAY_MAX_TOP];          // block 0: the chosen of all blocks
    int count;
};

// the K largest of n <= kList different keys in `from`, largest first (0 where there are fewer)
__device__ __forceinline__ void rank_keys(const unsigned long long *from, int n, int K, unsigned long long *to)
{
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const unsigned long long mine = from[i];
        int larger = 0;
        for (int o = 0; o < n; ++o) larger += from[o] > mine;
        if (larger < K) to[larger] = mine;
    }
}

// the K largest keys of vectors [v0, v1) of a row into l.chosen; `best_at` etc. of this thread; block-wide
template <typename T>
__device__ __forceinline__ void choose(Lists &l, const RowVectors<T> &r, int v0, int v1, int K, float best, int best_at, bool has_nan)
{
    constexpr int E = Vec<T>::E;
    const int tid = threadIdx.x;
    for (int i = tid; i < K; i += kThreads) l.chosen[i] = 0;
    if (tid == 0) l.count = 0;
    const int per = K <= 16 ? 4 : K <= 32 ? 2 : 1;         // threads per group: enough groups for K, few enough to compare
    unsigned long long mine = 0;
    if (best_at >= 0) {
        float x[E];
        unpack(r[best_at], x);
#pragma unroll
        for (int i = E - 1; i >= 0; --i) {
            const int id = best_at * E + i;
            if (x[i] == best && id < r.V) mine = key_of(x[i], id);
        }
    }
    if (per > 1) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
    if (per > 2) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, 2));
    if (tid % per == 0) l.group[tid / per] = mine;
    __syncthreads();
    bool searched = !has_nan;
    if (searched) {
        const int groups = kThreads / per;
        bool is_bound = false;
        if (tid < groups) {
            const unsigned long long g = l.group[tid];
            int larger = 0;
            for (int o = 0; o < groups; ++o) larger += l.group[o] > g;
            is_bound = larger == K - 1 && g != 0;
            if (is_bound) l.list[0] = g;
        }
        // groups without elements share the key 0: the bound is then 0, everything is listed (fewer than K groups hold fewer
        // than kList elements)
        const unsigned long long bound = __syncthreads_or(is_bound) ? l.list[0] : 0;
        __syncthreads();
        if (mine != 0 && mine >= bound) {                  // one of the K groups: look through its vectors
            for (int j = v0 + tid; j < v1; j += kThreads) {
                float x[E];
                unpack(r[j], x);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int id = j * E + i;
                    if (id >= r.V) continue;
                    const unsigned long long key = key_of(x[i], id);
                    if (key >= bound) {
                        const int at = atomicAdd(&l.count, 1);
                        if (at < kList) l.list[at] = key;
                    }
                }
            }
        }
        __syncthreads();
        searched = l.count <= kList;
        if (searched) rank_keys(l.list, l.count, K, l.chosen);
    }
    if (!searched) {                                       // a NaN in the row, or a list that overflowed: one pass per alternative
        unsigned long long last = ~0ull;
        for (int k = 0; k < K; ++k) {
            unsigned long long b = 0;
            for (int j = v0 + tid; j < v1; j += kThreads) {
                float x[E];
                unpack(r[j], x);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int id = j * E + i;
                    if (id >= r.V) continue;
                    const unsigned long long key = key_of(x[i], id);
                    if (key < last && key > b) b = key;
                }
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, d));
            __syncthreads();
            if ((tid & 31) == 0) l.group[tid >> 5] = b;
            __syncthreads();
            last = 0;
            for (int i = 0; i < kWarpsPerBlock; ++i) last = max(last, l.group[i]);
            if (tid == 0) l.chosen[k] = last;
        }
    }
    __syncthreads();
}
__device__ __forceinline__ float score_of(unsigned long long key)
{
    const uint32_t b = (uint32_t)(key >> 32);
    if (b == 0xfffffffeu) return __int_as_float(0x7fc00000);
    return __uint_as_float((b & 0x80000000u) ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ void store_remote(uint32_t at, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }

template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) token_logprob_kernel(const Args p, int S)
{
    __shared__ Sums part[kWarpsPerBlock], blocks[8];
    __shared__ Lists l;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x % S;
    const T *z = (const T *)p.z;
    if (S > 1) tc::cluster_sync();                         // block 0 runs before anything is written to it
    pdl_wait();
    for (long long row = blockIdx.x / S; row < p.rows; row += gridDim.x / S) {
        const RowVectors<T> r(z, p.rows, row, p.V);
        const int count = r.count(), each = (count + S - 1) / S, v0 = min(rank * each, count), v1 = min(v0 + each, count);
        Running run;
        int j = v0 + tid;
        // four vectors in flight
        for (; j + 3 * kThreads < v1; j += 4 * kThreads) {
            uint4 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = r[j + i * kThreads];
#pragma unroll
            for (int i = 0; i < 4; ++i) run.take(q[i], j + i * kThreads, p.k, z);
        }
        for (; j < v1; j += kThreads) run.take(r[j], j, p.k, z);
        Sums a = run.sums();
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) a = join(a, shfl_xor(a, d), p.k);
        if (lane == 0) part[warp] = a;
        __syncthreads();
        a = part[0];
#pragma unroll
        for (int i = 1; i < kWarpsPerBlock; ++i) a = join(a, part[i], p.k);
        if (TOP) choose(l, r, v0, v1, p.top, run.best, run.best_at, a.m != a.m);
        if (S > 1) {
            if (tid == 0) {
                const uint32_t to = tc::mapa(tc::smem_u32(&blocks[rank]), 0);
                store_remote(to, __float_as_uint(a.m)); store_remote(to + 4, __float_as_uint(a.s)); store_remote(to + 8, __float_as_uint(a.w));
            }
            if (TOP) {
                const uint32_t to = tc::mapa(tc::smem_u32(&l.merged[rank * p.top]), 0);
                for (int i = tid; i < p.top; i += kThreads) {
                    store_remote(to + 8 * i, (uint32_t)l.chosen[i]); store_remote(to + 8 * i + 4, (uint32_t)(l.chosen[i] >> 32));
                }
            }
            tc::cluster_sync();
            if (rank == 0) {
                a = blocks[0];
                for (int i = 1; i < S; ++i) a = join(a, blocks[i], p.k);
                if (TOP) {
                    __syncthreads();
                    rank_keys(l.merged, S * p.top, p.top, l.chosen);
                    __syncthreads();
                }
            }
        }
        if (rank == 0) {
            const Row sum(a, p.k);
            if (tid == 0) {
                if (p.lse) p.lse[row] = sum.lse;
                if (p.entropy) p.entropy[row] = sum.entropy;
                if (p.logp) {
                    const int t = token_of(p.tokens, p.tokens_i64, row, p.V);
                    p.logp[row] = t < 0 ? 0.0f : sum.logp(load_score(z + row * p.V + t), p.k);
                }
            }
            if (TOP)
                for (int i = tid; i < p.top; i += kThreads) {
                    p.top_ids[row * p.top + i] = id_of(l.chosen[i]);
                    p.top_logp[row * p.top + i] = sum.logp(score_of(l.chosen[i]), p.k);
                }
        }
        if (S > 1) tc::cluster_sync();                     // block 0 has read what the next row overwrites
        else __syncthreads();
    }
}

// ---- gradient: one pass ---------------------------------------------------------------------------------------------------
constexpr int kGradVectors = 4;        // per thread

// A row's pieces are the aligned 16-byte ones that it touches (no sums here whose order would depend on them): piece j holds its
// elements j E - skew .. j E - skew + E - 1; the first and the last are taken element by element where they are not whole.
template <typename T>
struct RowPieces {
    long long first;                   // element of the tensor at which piece 0 starts
    int skew, count, V;
    __device__ __forceinline__ RowPieces(long long row, int V_) : V(V_)
    {
        constexpr int E = Vec<T>::E;
        const long long at = row * V;
        skew = (int)(at % E);
        first = at - skew;
        count = (int)(((long long)skew + V + E - 1) / E);
    }
    __device__ __forceinline__ bool whole(int j) const { return j * Vec<T>::E >= skew && (long long)(j + 1) * Vec<T>::E - skew <= V; }
    __device__ __forceinline__ uint4 load(const T *z, int j) const
    {
        constexpr int E = Vec<T>::E;
        if (whole(j)) return ld_stream(z + first + (long long)j * E);
        float x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int id = j * E - skew + i;
            x[i] = id >= 0 && id < V ? load_score(z + first + (long long)j * E + i) : 0.0f;
        }
        return pack(x);
    }
};

// With q = exp(lp):  dscores = -(d + e (lp + h)) q / temperature,  d = dlogp, e = dentropy; at the token d (1 - q) in place of -d q
template <typename T>
__global__ void __launch_bounds__(kThreads) token_logprob_grad_kernel(const GradArgs p, int parts)
{
    constexpr int E = Vec<T>::E;
    constexpr bool FINE = sizeof(T) == 4;
    pdl_wait();
    const T *z = (const T *)p.z;
    T *dz = (T *)p.dz;
    const long long row = blockIdx.x / parts;
    const int from = (int)(blockIdx.x - row * parts) * (kThreads * kGradVectors) + threadIdx.x;
    const RowPieces<T> r(row, p.V);
    uint4 q[kGradVectors];
#pragma unroll
    for (int i = 0; i < kGradVectors; ++i)
        if (from + i * kThreads < r.count) q[i] = r.load(z, from + i * kThreads);
    const float lse = p.lse[row];
    const int t = token_of(p.tokens, p.tokens_i64, row, p.V);
    const float d = t < 0 ? 0.0f : p.dlogp[row];
    const float e = p.dentropy ? p.dentropy[row] : 0.0f, h = p.dentropy ? p.entropy[row] : 0.0f;
    const bool nothing = lse == -INFINITY;
    const float off = -(d + e * h) * p.k.inv, slope = -e * p.k.inv;
#pragma unroll
    for (int i = 0; i < kGradVectors; ++i) {
        const int j = from + i * kThreads;
        if (j >= r.count) break;
        float x[E], y[E], g[E];
        unpack(q[i], x);
        finite_elements(q[i], y);
#pragma unroll
        for (int c = 0; c < E; c += 2) {
            float l0, l1, t0, t1;
            const unsigned long long v = pair(x[c], x[c + 1]);
            unpair(fma2(pair(y[c], y[c + 1]), pair(p.k.inv_lo, p.k.inv_lo), fma2(v, pair(p.k.inv, p.k.inv), pair(-lse, -lse))), l0, l1);
            l0 = max_nan(l0, -1.0e30f); l1 = max_nan(l1, -1.0e30f);
            const unsigned long long lp = pair(l0, l1);
            unpair(mul2(lp, pair(1.44269504f, 1.44269504f)), t0, t1);
            if (FINE) { t0 = __expf(l0); t1 = __expf(l1); }
            else { t0 = exp2_(t0); t1 = exp2_(t1); }
            unpair(mul2(fma2(lp, pair(slope, slope), pair(off, off)), pair(t0, t1)), g[c], g[c + 1]);
        }
        const int at = t - (j * E - r.skew);
        if (t >= 0 && at >= 0 && at < E) {
#pragma unroll
            for (int c = 0; c < E; ++c)
                if (c == at) {                             // 1 - p of a class that is nearly certain keeps its precision
                    const float lp = log_prob(x[c], lse, p.k), u = __expf(lp);
                    g[c] = (-d * expm1f(lp) - (u != 0.0f ? e * u * (lp + h) : 0.0f)) * p.k.inv;
                }
        }
        if (nothing) {
#pragma unroll
            for (int c = 0; c < E; ++c) g[c] = 0.0f;
        }
        if (r.whole(j)) {
            st_stream(dz + r.first + (long long)j * E, pack(g));
        } else {
#pragma unroll
            for (int c = 0; c < E; ++c) {
                const int id = j * E - r.skew + c;
                T *to = dz + r.first + (long long)j * E + c;
                if (id >= 0 && id < p.V && relay_in_bounds(to, sizeof(T))) {
                    if constexpr (sizeof(T) == 2) *to = __float2bfloat16_rn(g[c]);
                    else *to = g[c];
                }
            }
        }
    }
}

// ---- boundary ------------------------------------------------------------------------------------------------------
struct Sizes { int64_t rows; int64_t V; int rank; };   // rank of the row vectors

relay_status_t check_scores(const relay_tensor_t *z, Sizes *s)
{
    RELAY_TRY(check_type(z, "scores"));
    if (z->rank < 1) return fail(RELAY_ERR_RANK, "scores: rank 0, a row of classes is needed");
    if (!is_float(z->dtype)) return fail(RELAY_ERR_DTYPE, "scores: base type %s, needs f32 or bf16", dtype_name(z->dtype));
    RELAY_TRY(check_layout(z, RELAY_ROWMAJOR, RELAY_ROWMAJOR, "scores"));
    s->rank = z->rank - 1;
    s->V = z->shape[s->rank];
    s->rows = 1;
    for (int d = 0; d < s->rank; ++d) s->rows *= z->shape[d];
    if (s->V == 0) return fail(RELAY_ERR_SHAPE, "scores: a row without classes has no softmax");
    if (s->V > INT32_MAX - 64) return fail(RELAY_ERR_SHAPE, "scores: %lld classes do not fit an i32", (long long)s->V);
    return RELAY_OK;
}
// a vector with one entry per row (rank and extents of scores without its last axis)
relay_status_t check_rows(const relay_tensor_t *t, const relay_tensor_t *z, const Sizes &s, int32_t d0, int32_t d1, const char *name)
{
    if (!t) return RELAY_OK;
    RELAY_TRY(check_type(t, name));
    RELAY_TRY(check_rank(t, s.rank, name));
    if (t->dtype != d0 && t->dtype != d1) return fail(RELAY_ERR_DTYPE, "%s: base type %s", name, dtype_name(t->dtype));
    RELAY_TRY(check_layout(t, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
    return check_shape_n(t, z->shape, s.rank, name);
}
// (..,K) beside scores (..,V)
relay_status_t check_top(const relay_tensor_t *t, const relay_tensor_t *z, const Sizes &s, int32_t dtype, int64_t K, const char *name)
{
    RELAY_TRY(check_type(t, name));
    RELAY_TRY(check_rank(t, s.rank + 1, name));
    RELAY_TRY(check_dtype(t, dtype, name));
    RELAY_TRY(check_layout(t, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
    int64_t want[RELAY_MAX_RANK];
    for (int d = 0; d < s.rank; ++d) want[d] = z->shape[d];
    want[s.rank] = K;
    return check_shape_n(t, want, s.rank + 1, name);
}
relay_status_t check_temperature(float t)
{
    if (!(t > 0.0f) || t > 3.0e38f) return fail(RELAY_ERR_ATTR, "temperature = %g, needs a positive finite number", (double)t);
    return RELAY_OK;
}

template <typename T>
relay_status_t launch_forward(const Args &p, cudaStream_t st)
{
    int dev = 0, sms = 148;
    RELAY_CUDA(cudaGetDevice(&dev));
    RELAY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // few rows: several blocks each, as long as a block keeps a vector per thread
    const long long vectors = (p.V + Vec<T>::E - 1) / Vec<T>::E;
    int S = 1;
    while (S < 8 && p.rows * S < sms && vectors > (long long)S * 2 * kThreads) S *= 2;
    const dim3 grid((unsigned)std::min<long long>(p.rows * S, 1 << 20)), block(kThreads), cluster((unsigned)S);
    if (p.top) RELAY_CUDA(launch_pdl_cluster(token_logprob_kernel<T, true>, grid, block, cluster, 0, st, p, S));
    else RELAY_CUDA(launch_pdl_cluster(token_logprob_kernel<T, false>, grid, block, cluster, 0, st, p, S));
    return check_launch("token_logprob");
}
template <typename T>
relay_status_t launch_gradient(const GradArgs &p, cudaStream_t st)
{
    const long long vectors = ((long long)p.V + 2 * (Vec<T>::E - 1)) / Vec<T>::E;      // whatever the skew
    const long long parts = (vectors + kThreads * kGradVectors - 1) / (kThreads * kGradVectors);
    if (p.rows * parts > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "token_logprob_grad: %lld rows of %d classes", p.rows, p.V);
    RELAY_CUDA(launch_pdl(token_logprob_grad_kernel<T>, dim3((unsigned)(p.rows * parts)), dim3(kThreads), 0, st, p, (int)parts));
    return check_launch("token_logprob_grad");
}

}  // namespace
}  // namespace relay

using namespace relay;

extern "C" relay_status_t relay_token_logprob(const relay_tensor_t *scores, const relay_tensor_t *tokens, float temperature,
                                              const relay_tensor_t *logp, const relay_tensor_t *entropy, const relay_tensor_t *lse,
                                              const relay_tensor_t *top_logp, const relay_tensor_t *top_ids, void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(scores, "scores"));
    if (tokens || logp) { RELAY_TRY(check_not_null(tokens, "tokens")); RELAY_TRY(check_not_null(logp, "logp")); }
    if (top_logp || top_ids) { RELAY_TRY(check_not_null(top_logp, "top_logp")); RELAY_TRY(check_not_null(top_ids, "top_ids")); }
    if (!logp && !entropy && !lse && !top_ids) return fail(RELAY_ERR_NULL, "no output is wanted");
    Sizes s;
    RELAY_TRY(check_scores(scores, &s));
    RELAY_TRY(check_rows(tokens, scores, s, RELAY_I32, RELAY_I64, "tokens"));
    RELAY_TRY(check_rows(logp, scores, s, RELAY_F32, RELAY_F32, "logp"));
    RELAY_TRY(check_rows(entropy, scores, s, RELAY_F32, RELAY_F32, "entropy"));
    RELAY_TRY(check_rows(lse, scores, s, RELAY_F32, RELAY_F32, "lse"));
    int64_t K = 0;
    if (top_ids) {
        RELAY_TRY(check_type(top_ids, "top_ids"));
        RELAY_TRY(check_rank(top_ids, s.rank + 1, "top_ids"));
        K = top_ids->shape[s.rank];
        RELAY_TRY(check_top(top_ids, scores, s, RELAY_I32, K, "top_ids"));
        RELAY_TRY(check_top(top_logp, scores, s, RELAY_F32, K, "top_logp"));
        if (K < 1 || K > s.V || K > RELAY_MAX_TOP)
            return fail(RELAY_ERR_SHAPE, "top_ids: %lld alternatives, needs 1..%lld", (long long)K, (long long)std::min<int64_t>(s.V, RELAY_MAX_TOP));
    }
    RELAY_TRY(check_temperature(temperature));
    const relay_tensor_t *ins[2] = {scores, tokens}, *outs[5] = {logp, entropy, lse, top_logp, top_ids};
    for (const relay_tensor_t *t : ins) if (t) RELAY_TRY(check_data(t, "input"));
    for (const relay_tensor_t *t : outs) if (t) RELAY_TRY(check_data(t, "output"));
    RELAY_TRY(check_no_overlap(outs, 5, ins, 2));
    if (s.rows == 0) return RELAY_OK;
    Args p{};
    p.z = scores->data; p.rows = s.rows; p.V = (int)s.V; p.k = scale_of(temperature); p.top = (int)K;
    p.tokens = tokens ? tokens->data : nullptr;
    p.tokens_i64 = tokens && tokens->dtype == RELAY_I64;
    p.logp = logp ? (float *)logp->data : nullptr;
    p.entropy = entropy ? (float *)entropy->data : nullptr;
    p.lse = lse ? (float *)lse->data : nullptr;
    p.top_logp = top_logp ? (float *)top_logp->data : nullptr;
    p.top_ids = top_ids ? (int *)top_ids->data : nullptr;
    BoundsReg reg;
    for (const relay_tensor_t *t : ins) reg.add(t);
    for (const relay_tensor_t *t : outs) reg.add(t);
    cudaStream_t st = (cudaStream_t)stream;
    RELAY_TRY(reg.commit(st));
    return scores->dtype == RELAY_F32 ? launch_forward<float>(p, st) : launch_forward<__nv_bfloat16>(p, st);
}

extern "C" relay_status_t relay_token_logprob_grad(const relay_tensor_t *scores, const relay_tensor_t *tokens, float temperature,
                                                   const relay_tensor_t *lse, const relay_tensor_t *entropy, const relay_tensor_t *dlogp,
                                                   const relay_tensor_t *dentropy, const relay_tensor_t *dscores, void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(scores, "scores"));
    RELAY_TRY(check_not_null(tokens, "tokens"));
    RELAY_TRY(check_not_null(lse, "lse"));
    RELAY_TRY(check_not_null(dlogp, "dlogp"));
    RELAY_TRY(check_not_null(dscores, "dscores"));
    if (dentropy) RELAY_TRY(check_not_null(entropy, "entropy"));
    Sizes s;
    RELAY_TRY(check_scores(scores, &s));
    RELAY_TRY(check_rows(tokens, scores, s, RELAY_I32, RELAY_I64, "tokens"));
    RELAY_TRY(check_rows(lse, scores, s, RELAY_F32, RELAY_F32, "lse"));
    RELAY_TRY(check_rows(entropy, scores, s, RELAY_F32, RELAY_F32, "entropy"));
    RELAY_TRY(check_rows(dlogp, scores, s, RELAY_F32, RELAY_F32, "dlogp"));
    RELAY_TRY(check_rows(dentropy, scores, s, RELAY_F32, RELAY_F32, "dentropy"));
    RELAY_TRY(check_top(dscores, scores, s, scores->dtype, s.V, "dscores"));
    RELAY_TRY(check_temperature(temperature));
    const relay_tensor_t *ins[6] = {scores, tokens, lse, entropy, dlogp, dentropy}, *outs[1] = {dscores};
    for (const relay_tensor_t *t : ins) if (t) RELAY_TRY(check_data(t, "input"));
    RELAY_TRY(check_data(dscores, "dscores"));
    RELAY_TRY(check_no_overlap(outs, 1, ins, 6));
    if (s.rows == 0) return RELAY_OK;
    GradArgs p{};
    p.z = scores->data; p.rows = s.rows; p.V = (int)s.V; p.k = scale_of(temperature);
    p.tokens = tokens->data; p.tokens_i64 = tokens->dtype == RELAY_I64;
    p.lse = (const float *)lse->data; p.dlogp = (const float *)dlogp->data;
    p.dentropy = dentropy ? (const float *)dentropy->data : nullptr;
    p.entropy = dentropy ? (const float *)entropy->data : nullptr;
    p.dz = dscores->data;
    BoundsReg reg;
    for (const relay_tensor_t *t : ins) reg.add(t);
    reg.add(dscores);
    cudaStream_t st = (cudaStream_t)stream;
    RELAY_TRY(reg.commit(st));
    return scores->dtype == RELAY_F32 ? launch_gradient<float>(p, st) : launch_gradient<__nv_bfloat16>(p, st);
}
