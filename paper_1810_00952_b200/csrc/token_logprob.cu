// Log-probabilities of given tokens, entropies and the most probable tokens of rows of scores, and the gradient group.
// The forward call reads every score once, the gradient reads and writes it once.  Measured against a copy at 6.53 TB/s:
//   4096 x 32768 bf16, K = 8    68 us, 4.0 TB/s: no pipe is full (of the active cycles the exponentials' is busy 50 % and 60 % issue, with 44 %
//                               of the warps there are: a row ends in barriers); without alternatives 55 us, 4.9 TB/s; two register buffers, a
//                               bulk-copy ring and several blocks a row were no faster
//   4096 x 32768 f32            93 us, 5.8 TB/s: HBM
//   8 x 131072 bf16, K = 20     10.4 us, 0.2 TB/s: the launch, the exchange between a row's blocks and the choice of the largest
//   gradient, 4096 x 32768 bf16 with the entropy's term  94 us, 5.7 TB/s;  509 x 50021 f32  34 us, 6.0 TB/s: HBM
#include <algorithm>
#include <cfloat>

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
// 1 / temperature as a sum of two floats.  Distances d of two scores are kept in units of 1 / unit: one, but 2^64 where the temperature is
// so high that classes far apart share the probability; then a sum of distances stays finite, and `limit` sends every row to the
// path that looks at its elements one by one (elsewhere a distance of 1e30 is as good as an infinite one).
struct Scale {
    float inv, inv_lo;
    float unit, inv_d, inv_2d, log2e_d;                    // 1, 2 and log2(e) over the temperature, per unit of d
    float limit;                                           // of the largest score's size on the short path
};
inline Scale scale_of(float temperature)
{
    const bool high = temperature > 1.0e20f;
    const double inv = 1.0 / std::max((double)temperature, (double)FLT_MIN), unit = high ? 0x1p-64 : 1.0;
    Scale k;
    k.inv = (float)inv;
    k.inv_lo = (float)(inv - (double)k.inv);
    k.unit = (float)unit;
    k.inv_d = (float)(inv / unit);
    k.inv_2d = 2.0f * k.inv_d;
    k.log2e_d = (float)(1.4426950408889634 * inv / unit);
    k.limit = high ? 0.0f : 1.0e30f;
    return k;
}
// z / temperature - lse with one rounding of the result's own size: the product stays exact inside the multiply-add, so a
// probability is as good where the scores are far from zero.  A score of -inf gives -inf.
__device__ __forceinline__ float log_prob(float z, float lse, const Scale &k)
{
    return fmaf(fmaxf(z, -3.0e38f), k.inv_lo, fmaf(z, k.inv, -lse));
}

// ---- sums of one row, joinable in any order of parts, d = z - m (times `unit`) ----------------------------------------------
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
// a finite distance even where a score or the maximum is infinite: its exponential is 0 and its product with that too
__device__ __forceinline__ float below(float z, float m, const Scale &k) { return fmaxf(fmaf(z, k.unit, -(m * k.unit)), -1.0e30f); }

// the sums of a warp's lanes together, in every lane; written out with intrinsics, so that every kernel rounds alike
__device__ __forceinline__ Sums join_lanes(Sums a, const Scale &k)
{
    float m = a.m;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
    const float d = below(a.m, m, k), f = exp2_(d * k.log2e_d);
    float s = __fmul_rn(f, a.s), w = __fmul_rn(f, fmaf(d, a.s, a.w));
#pragma unroll
    for (int d2 = 16; d2 > 0; d2 >>= 1) {
        s = __fadd_rn(s, __shfl_xor_sync(0xffffffffu, s, d2));
        w = __fadd_rn(w, __shfl_xor_sync(0xffffffffu, w, d2));
    }
    return Sums{m, s, w};
}

// what a row's sums say
struct Row {
    float m, log_s, entropy, lse;
    __device__ __forceinline__ Row(const Sums &a, const Scale &k)
    {
        m = a.m;
        log_s = logf(a.s);
        lse = fmaf(a.m, k.inv, log_s);
        entropy = log_s - __fdiv_rn(__fmul_rn(a.w, k.inv_d), a.s);
        if (a.m == -INFINITY) { lse = -INFINITY; entropy = 0.0f; }
        else if (!(a.m < INFINITY)) lse = entropy = log_s = __int_as_float(0x7fc00000);
    }
    __device__ __forceinline__ float logp(float z, const Scale &k) const
    {
        return m == -INFINITY ? -INFINITY : fmaf((0.5f * z - 0.5f * m) * k.unit, k.inv_2d, -log_s);   // half the distance: finite
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

// One thread's running sums, in pairs, N vectors at a time: the maximum over all of them is looked at first, and only where it is
// larger than the one so far are the sums scaled down (some ln(row / N) times a row).
// Differences from -inf: the scores are raised to the lowest finite value first, so that 0 times the distance is 0.  That holds as
// long as the distance is finite: where the maximum is so low (masks of the lowest value and nothing else) or so high that it may
// not be, the elements are looked at one by one.
struct Running {
    float m = -INFINITY;
    unsigned long long s = 0, w = 0;                       // two partial sums each
    int best_at = -1;                                      // the first vector that holds the largest element, m unless NaN are about
    template <typename T, int N>
    __device__ __forceinline__ float take(const uint4 (&q)[N], int j, int stride, const Scale &k, const T *type)      // their largest
    {
        constexpr int E = Vec<T>::E;
        float top[N], most;
#pragma unroll
        for (int n = 0; n < N; ++n) top[n] = largest(q[n], type);
        most = top[0];
#pragma unroll
        for (int n = 1; n < N; ++n) most = max_nan(most, top[n]);
        if (best_at < 0) best_at = j;
        if (!(most <= m)) {                                // larger, or NaN
            const float d = below(m, most, k), f = exp2_(d * k.log2e_d);
            float s0, s1, w0, w1;
            unpair(s, s0, s1); unpair(w, w0, w1);
            w = pair(f * fmaf(d, s0, w0), f * fmaf(d, s1, w1));
            s = pair(f * s0, f * s1);
            m = max_nan(m, most);
#pragma unroll
            for (int n = N - 1; n >= 0; --n)
                if (top[n] == most) best_at = j + n * stride;
        }
        if (!(fabsf(m) < k.limit)) {                       // also NaN: what the sums are then does not matter
            if (m == -INFINITY) return most;               // nothing but -inf so far
            for (int n = 0; n < N; ++n) {
                float x[E], s0, s1, w0, w1;
                unpack(q[n], x);
                unpair(s, s0, s1); unpair(w, w0, w1);
                for (int i = 0; i < E; ++i)
                    if (x[i] != -INFINITY) {
                        const float d = below(x[i], m, k), e = exp2_(d * k.log2e_d);
                        s0 += e;
                        w0 = fmaf(e, d, w0);
                    }
                s = pair(s0, s1); w = pair(w0, w1);
            }
            return most;
        }
        const unsigned long long nm = pair(-m, -m), c = pair(k.log2e_d, k.log2e_d);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float x[E];
            finite_elements(q[n], x);
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
        return most;
    }
    __device__ __forceinline__ Sums sums() const
    {
        float s0, s1, w0, w1;
        unpair(s, s0, s1); unpair(w, w0, w1);
        return Sums{m, s0 + s1, w0 + w1};
    }
};
// Vector j of a row: its elements j E .. j E + E - 1 (-inf behind the row's end), wherever the row starts in memory, so that a
// row's result does not depend on its place.  EVEN: V is a multiple of E, every vector of every row is one aligned piece.
// Otherwise `skew` is how many elements before the row's first the nearest 16-byte boundary lies, and two aligned pieces are read
// and shifted (the second is the next thread's first, and in L1).
template <typename T, bool EVEN>
struct RowVectors {
    const T *aligned;                  // the row's start, rounded down
    int skew, V, safe;                 // vectors below `safe` can be read as whole pieces
    __device__ __forceinline__ RowVectors(const T *z, long long rows, long long row, int V_) : V(V_)
    {
        constexpr int E = Vec<T>::E;
        const long long at = row * V;
        if (EVEN) {
            aligned = z + at;
            skew = 0;
            safe = V / E;
            return;
        }
        const long long left = rows * V - at;              // elements from the row's start to the tensor's end
        skew = (int)(at % E);
        aligned = z + (at - skew);
        // piece j + 1 ends (j + 2) E - skew elements behind the row's start
        const long long inside = skew == 0 ? V / E : (left + skew) / E - 1;
        safe = (int)min((long long)(V / E), max(inside, 0ll));
    }
    __device__ __forceinline__ int count() const { return (int)(((long long)V + Vec<T>::E - 1) / Vec<T>::E); }
    // N vectors j, j + stride, .. as far as they lie below `last`, which is at most `safe`; -inf from there on.  All loads come before
    // the first use.
    template <int N>
    __device__ __forceinline__ void whole(int j, int stride, int last, uint4 (&q)[N]) const
    {
        const uint4 *at = (const uint4 *)aligned;
        constexpr uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
        if (EVEN) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                q[n] = make_uint4(none, none, none, none);
                if (j + n * stride < last) q[n] = ld_stream(at + j + n * stride);
            }
            return;
        }
        uint4 hi[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            q[n] = hi[n] = make_uint4(none, none, none, none);
            const uint4 *a = at + j + n * stride;
            if (j + n * stride < last && relay_in_bounds(a, skew ? 32 : 16)) { q[n] = __ldg(a); hi[n] = __ldg(a + (skew != 0)); }
        }
        const int bytes = skew * (int)sizeof(T);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t w[8] = {q[n].x, q[n].y, q[n].z, q[n].w, hi[n].x, hi[n].y, hi[n].z, hi[n].w};
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = bytes & 8 ? w[i + 2] : w[i];
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = bytes & 4 ? w[i + 1] : w[i];
            if (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (bytes & 2) * 8);
            }
            q[n] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    __device__ __forceinline__ uint4 operator[](int j) const
    {
        constexpr int E = Vec<T>::E;
        uint4 q[1];
        if (EVEN || j < safe) {
            whole(j, 0, j + 1, q);
            return q[0];
        }
        float x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = (long long)j * E + i < V ? load_score(aligned + (long long)j * E + skew + i) : -INFINITY;
        return pack(x);
    }
};

// the score that a key was made of; 0 (the key of nothing) gives NaN, which nothing is below
__device__ __forceinline__ float score_of(unsigned long long key)
{
    const uint32_t b = (uint32_t)(key >> 32);
    if (b == 0xfffffffeu) return __int_as_float(0x7fc00000);
    return __uint_as_float((b & 0x80000000u) ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ void store_remote(uint32_t at, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }

// ---- forward: a cluster of S blocks of NT threads per row --------------------------------------------------------------------
// Each block sums a contiguous part of the row's vectors; the blocks' sums meet in block 0's shared memory.
// Alternatives: a thread remembers the vector of its largest element.  With the threads in G groups, the K-th largest of the
// groups' largest is a bound that the part's K-th largest element is not below.  Each thread also keeps the largest of every
// eighth of its vectors; only the eighths that reach the bound (K and a few) can hold elements that do: they are looked through
// again, shared out over the block (they come from L2), and what reaches the bound is listed; the position of a listed element is
// the number of larger ones.
constexpr int kList = 512;             // listed elements; expected -G ln(1 - K / G): 31 for K = 20, G = 32, 89 for K = 64, G = 128

// Up to how many alternatives 32 groups bound them, in blocks of 128 and of 512 threads.  More groups list fewer elements, but finding
// their K-th largest takes longer.  32 groups against 128: 8192 x 4000 bf16 (128 threads) K = 20 52 and 62 us, 24 60 and 63, 28 67 and
// 65, 31 87 and 67; 4096 x 32768 74 and 77, 78 and 78, 84 and 80, 98 and 82; 8 x 131072 (512 threads) K = 20 10.5 and 19.3, 28 11.9 and
// 20.2, 31 14 and 20.5.  32 groups cannot bound more than 31.
constexpr int kFewGroups128 = 24, kFewGroups512 = 31;
template <int NT>
struct Lists {
    unsigned long long largest[NT];    // per thread: a key not above its largest element's
    unsigned long long list[kList];
    unsigned long long chosen[RELAY_MAX_TOP];
    unsigned long long merged[8 * RELAY_MAX_TOP];          // block 0: the chosen of all blocks
    unsigned long long bound;
    float eighth[8][NT];
    short reached[8 * NT];             // thread * 8 + eighth
    int count, eighths;
};

// the K largest of n <= kList different keys in `from`, largest first; calls put(position, key)
template <int NT, typename Put>
__device__ __forceinline__ void rank_keys(const unsigned long long *from, int n, int K, Put put)
{
    for (int i = threadIdx.x; i < n; i += NT) {
        const unsigned long long mine = from[i];
        int larger = 0;
#pragma unroll 4
        for (int o = 0; o < n; ++o) larger += from[o] > mine;
        if (larger < K && mine != 0) put(larger, mine);
    }
}
// Lists what can be among the K largest of vectors [v0, v1) of a row; l.largest is set, and a barrier has passed.  False: more
// than fit the list.  `meanwhile` is run by the last warp while the others find the bound.
template <int NT, typename T, bool EVEN, typename Meanwhile>
__device__ __forceinline__ bool list_largest(Lists<NT> &l, const RowVectors<T, EVEN> &r, int v0, int v1, int K, unsigned long long mine, int per, int used, Meanwhile meanwhile)
{
    constexpr int E = Vec<T>::E;
    const int tid = threadIdx.x, groups = K <= (NT == 128 ? kFewGroups128 : kFewGroups512) ? 32 : 128;     // group: the threads of equal tid mod groups
    if (tid == 0) l.count = l.eighths = 0;
    bool is_bound = false;
    if (tid < groups) {
        unsigned long long g = l.largest[tid];
        for (int i = groups; i < NT; i += groups) g = max(g, l.largest[tid + i]);
        int larger = 0;
        if (groups == 32) {
#pragma unroll
            for (int o = 0; o < 32; ++o) larger += __shfl_sync(0xffffffffu, g, o) > g;
        } else {
            for (int o = 0; o < NT; o += 4) {              // by groups, four at a time
                if (o >= groups) break;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    unsigned long long other = l.largest[o + c];
                    for (int i = groups; i < NT; i += groups) other = max(other, l.largest[o + c + i]);
                    larger += other > g;
                }
            }
        }
        is_bound = larger == K - 1 && g != 0;
        if (is_bound) l.bound = g;
    }
    if (tid >= NT - 32) meanwhile();
    // groups without elements share the key 0: the bound is then 0 and everything is listed (fewer than K groups have fewer than K
    // vectors among them)
    const unsigned long long bound = __syncthreads_or(is_bound) ? l.bound : 0;
    const float least = score_of(bound);
    if (mine != 0 && mine >= bound)
        for (int c = 0; c < used; ++c)
            if (!(l.eighth[c][tid] < least)) l.reached[atomicAdd(&l.eighths, 1)] = (short)(tid * 8 + c);
    __syncthreads();
    const int items = l.eighths * per;
    for (int it = tid; it < items; it += 4 * NT) {         // four vectors in flight
        uint4 q[4];
        int at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int which = (it + u * NT) / per, i = it + u * NT - which * per;
            at[u] = v1;
            if (it + u * NT < items) at[u] = v0 + ((l.reached[which] & 7) * per + i) * NT + (l.reached[which] >> 3);
            if (at[u] < v1) q[u] = r[at[u]];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (at[u] >= v1 || largest(q[u], r.aligned) < least) continue;
            float x[E];
            unpack(q[u], x);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int id = at[u] * E + i;
                const unsigned long long key = key_of(x[i], id);
                if (key >= bound && id < r.V) {
                    const int n = atomicAdd(&l.count, 1);
                    if (n < kList) l.list[n] = key;
                }
            }
        }
    }
    __syncthreads();
    return l.count <= kList;
}
// The same without a bound, one pass per alternative, into l.list in order: for a row with a NaN, or one whose list overflowed.
template <int NT, typename T, bool EVEN>
__device__ __forceinline__ void list_by_passes(Lists<NT> &l, const RowVectors<T, EVEN> &r, int v0, int v1, int K)
{
    constexpr int E = Vec<T>::E;
    unsigned long long last = ~0ull;
    for (int k = 0; k < K; ++k) {
        unsigned long long b = 0;
        for (int j = v0 + threadIdx.x; j < v1; j += NT) {
            float x[E];
            unpack(r[j], x);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int id = j * E + i;
                const unsigned long long key = key_of(x[i], id);
                if (id < r.V && key < last && key > b) b = key;
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, d));
        __syncthreads();
        if ((threadIdx.x & 31) == 0) l.largest[threadIdx.x >> 5] = b;
        __syncthreads();
        last = 0;
        for (int i = 0; i < NT / 32; ++i) last = max(last, l.largest[i]);
        if (threadIdx.x == 0) l.list[k] = last;
    }
    if (threadIdx.x == 0) l.count = K;
    __syncthreads();
}

template <typename T, int NT, bool TOP, bool EVEN>
__global__ void __launch_bounds__(NT, 1024 / NT) token_logprob_kernel(const Args p, int S)
{
    constexpr int E = Vec<T>::E, NW = NT / 32;
    __shared__ Sums part[NW], blocks[8], total;
    __shared__ Lists<TOP ? NT : 32> l;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x % S;
    const T *z = (const T *)p.z;
    if (S > 1) tc::cluster_sync();                         // block 0 runs before anything is written to it
    pdl_wait();
    for (long long row = blockIdx.x / S; row < p.rows; row += gridDim.x / S) {
        const RowVectors<T, EVEN> r(z, p.rows, row, p.V);
        const int count = r.count(), each = (count + S - 1) / S, v0 = min(rank * each, count), v1 = min(v0 + each, count);
        int token = -1;                                    // fetched now, used when the sums are there
        float token_score = 0.0f;
        if (tid == NT - 1 && rank == 0 && p.logp) {
            token = token_of(p.tokens, p.tokens_i64, row, p.V);
            if (token >= 0) token_score = load_score(z + row * p.V + token);
        }
        Running run;
        const int rounds = (v1 - v0 + NT - 1) / NT, per = max(4, (rounds + 31) / 32 * 4);      // vectors of an eighth: whole fours
        float eighth = -INFINITY;
        int used = 0, in = 0;
        auto mark = [&](float most, int n) {
            if constexpr (TOP) {
                eighth = max_nan(eighth, most);
                if ((in += n) == per) { l.eighth[used++][tid] = eighth; eighth = -INFINITY; in = 0; }
            }
        };
        const int last = min(v1, r.safe);
        int j = v0 + tid;
        for (; j < last; j += 4 * NT) {                    // four vectors in flight
            uint4 q[4];
            r.whole(j, NT, last, q);
            mark(run.take(q, j, NT, p.k, z), min(4, (last - j + NT - 1) / NT));
        }
        for (j = v0 + tid + (max(last - v0 - tid, 0) + NT - 1) / NT * NT; j < v1; j += NT) {       // one or two that are not whole
            const uint4 q[1] = {r[j]};
            mark(run.take(q, j, NT, p.k, z), 1);
        }
        if constexpr (TOP)
            if (in > 0) l.eighth[used++][tid] = eighth;
        const Sums mine = join_lanes(run.sums(), p.k);
        if (lane == 0) part[warp] = mine;
        // the vector's last id, not the element's: not above the largest element's key, and no second look at the vector
        const unsigned long long key = run.best_at < 0 ? 0 : key_of(run.m, run.best_at * E + E - 1);
        bool fits = false;
        if constexpr (TOP) l.largest[tid] = key;
        const bool has_nan = __syncthreads_or(run.m != run.m);
        auto sum_up = [&] {                                // the last warp
            const Sums a = join_lanes(lane < NW ? part[lane] : empty_sums(), p.k);
            if (lane == 31) total = a;
        };
        if constexpr (TOP) {
            if (!has_nan) fits = list_largest<NT>(l, r, v0, v1, p.top, key, per, used, sum_up);
            if (!fits) {
                if (has_nan && warp == NW - 1) sum_up();
                list_by_passes<NT>(l, r, v0, v1, p.top);
            }
        } else {
            if (warp == NW - 1) sum_up();
            __syncwarp();
        }
        if (S > 1) {
            if (tid == NT - 1) {
                const uint32_t to = tc::mapa(tc::smem_u32(&blocks[rank]), 0);
                store_remote(to, __float_as_uint(total.m)); store_remote(to + 4, __float_as_uint(total.s)); store_remote(to + 8, __float_as_uint(total.w));
            }
            if constexpr (TOP) {
                for (int i = tid; i < p.top; i += NT) l.chosen[i] = 0;
                __syncthreads();
                rank_keys<NT>(l.list, l.count, p.top, [&](int at, unsigned long long k) { l.chosen[at] = k; });
                __syncthreads();
                const uint32_t to = tc::mapa(tc::smem_u32(&l.merged[rank * p.top]), 0);
                for (int i = tid; i < p.top; i += NT) {
                    store_remote(to + 8 * i, (uint32_t)l.chosen[i]); store_remote(to + 8 * i + 4, (uint32_t)(l.chosen[i] >> 32));
                }
            }
            tc::cluster_sync();
            if (rank == 0) {
                if (warp == NW - 1) {
                    const Sums a = join_lanes(lane < S ? blocks[lane] : empty_sums(), p.k);
                    if (lane == 31) total = a;
                }
                __syncthreads();
            }
        }
        if (rank == 0) {
            if (tid == NT - 1) {
                const Row sum(total, p.k);
                if (p.lse) p.lse[row] = sum.lse;
                if (p.entropy) p.entropy[row] = sum.entropy;
                if (p.logp) p.logp[row] = token < 0 ? 0.0f : sum.logp(token_score, p.k);
            }
            if constexpr (TOP) {
                auto put = [&](int at, unsigned long long k) {
                    const Row sum(total, p.k);
                    p.top_ids[row * p.top + at] = id_of(k);
                    p.top_logp[row * p.top + at] = sum.logp(score_of(k), p.k);
                };
                if (S > 1) rank_keys<NT>(l.merged, S * p.top, p.top, put);
                else rank_keys<NT>(l.list, l.count, p.top, put);
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

// Log-probabilities are held at kNothing, where exp is zero: its product with a slope is zero unless that is above 1e35.
constexpr float kNothing = -1.0e3f;

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
            l0 = max_nan(l0, kNothing); l1 = max_nan(l1, kNothing);
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

template <typename T, int NT>
relay_status_t launch_blocks(const Args &p, int S, cudaStream_t st)
{
    const dim3 grid((unsigned)std::min<long long>(p.rows * S, 1 << 20)), block(NT), cluster((unsigned)S);
    if (p.V % Vec<T>::E == 0) {
        if (p.top) RELAY_CUDA(launch_pdl_cluster(token_logprob_kernel<T, NT, true, true>, grid, block, cluster, 0, st, p, S));
        else RELAY_CUDA(launch_pdl_cluster(token_logprob_kernel<T, NT, false, true>, grid, block, cluster, 0, st, p, S));
    } else {
        if (p.top) RELAY_CUDA(launch_pdl_cluster(token_logprob_kernel<T, NT, true, false>, grid, block, cluster, 0, st, p, S));
        else RELAY_CUDA(launch_pdl_cluster(token_logprob_kernel<T, NT, false, false>, grid, block, cluster, 0, st, p, S));
    }
    return check_launch("token_logprob");
}
template <typename T>
relay_status_t launch_forward(const Args &p, cudaStream_t st)
{
    int dev = 0, sms = 148;
    RELAY_CUDA(cudaGetDevice(&dev));
    RELAY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    // Rows enough for every SM: small blocks, eight to an SM, each with a row (at 8192 x 4000 a block spends most of its time on
    // what follows the sums, and what counts is how many are at it).  Fewer rows: large blocks, and several per row as long as a
    // thread keeps four vectors.
    const long long vectors = ((long long)p.V + Vec<T>::E - 1) / Vec<T>::E;
    if (p.rows >= 2 * sms) return launch_blocks<T, 128>(p, 1, st);
    int S = 1;
    while (S < 8 && p.rows * S < sms && vectors > (long long)S * 512) S *= 2;
    return launch_blocks<T, 512>(p, S, st);
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
