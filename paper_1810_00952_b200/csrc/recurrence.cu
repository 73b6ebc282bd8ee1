// Gated linear recurrence over a sequence, h_t = a_t h_{t-1} + b_t per channel, and its gradient group (Section 4.2 of the
// paper: reverse mode through the recursion over time).  Elementwise steps: HBM-bound where the channels fill the GPU.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "ewise_kernels.cuh"

namespace relay {
namespace {

constexpr int kThreads = 128;

struct Args {
    const void *f, *u;             // row of step t, batch element b: f + t * ld + b * bs, D entries (u alike)
    long long ld, bs;
    const float *h0;               // [C] or null
    const int *lengths;            // [C / D] or null
    void *h;                       // [T][C]: written by the forward kernels, read by the gradient's
    float *h_final;                // [C] or null
    const void *dh;                // [T][C]
    const float *dh_final;         // [C] or null
    void *df, *du;                 // addressed like f and u
    float *dh0;                    // [C] or null
    long long T, C, D;             // C = batch * D channels
};

// ---- vectors of V consecutive channels -----------------------------------------------------------------
template <typename T, int V> struct RawOf { using type = T; };
template <> struct RawOf<__nv_bfloat16, 2> { using type = uint32_t; };
template <> struct RawOf<float, 2> { using type = uint2; };
template <typename T, int V> using Raw = typename RawOf<T, V>::type;

// Each value is touched once: past L1.
template <typename R>
__device__ __forceinline__ R load_raw(const void *p)
{
    if (!relay_in_bounds(p, sizeof(R))) return R{};
    return __ldcs((const R *)p);
}
template <>
__device__ __forceinline__ __nv_bfloat16 load_raw<__nv_bfloat16>(const void *p)
{
    if (!relay_in_bounds(p, 2)) return __nv_bfloat16{};
    return __ushort_as_bfloat16(__ldcs((const unsigned short *)p));
}
template <typename R>
__device__ __forceinline__ void store_raw(void *p, const R &r)
{
    if (relay_in_bounds(p, sizeof(R))) __stcs((R *)p, r);
}
template <>
__device__ __forceinline__ void store_raw<__nv_bfloat16>(void *p, const __nv_bfloat16 &r)
{
    if (relay_in_bounds(p, 2)) __stcs((unsigned short *)p, __bfloat16_as_ushort(r));
}
__device__ __forceinline__ void to_f32(uint32_t r, float (&x)[2]) { x[0] = __uint_as_float(r << 16); x[1] = __uint_as_float(r & 0xffff0000u); }
__device__ __forceinline__ void to_f32(uint2 r, float (&x)[2]) { x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); }
__device__ __forceinline__ void to_f32(__nv_bfloat16 r, float (&x)[1]) { x[0] = __bfloat162float(r); }
__device__ __forceinline__ void to_f32(float r, float (&x)[1]) { x[0] = r; }
__device__ __forceinline__ void from_f32(const float (&x)[2], uint32_t &r) { r = pack2(x[0], x[1]); }
__device__ __forceinline__ void from_f32(const float (&x)[2], uint2 &r) { r = make_uint2(__float_as_uint(x[0]), __float_as_uint(x[1])); }
__device__ __forceinline__ void from_f32(const float (&x)[1], __nv_bfloat16 &r) { r = __float2bfloat16_rn(x[0]); }
__device__ __forceinline__ void from_f32(const float (&x)[1], float &r) { r = x[0]; }

template <typename T, int V>
__device__ __forceinline__ void load(const void *base, long long at, float (&x)[V])
{
    to_f32(load_raw<Raw<T, V>>((const T *)base + at), x);
}
template <typename T, int V>
__device__ __forceinline__ void store(void *base, long long at, const float (&x)[V])
{
    Raw<T, V> r;
    from_f32(x, r);
    store_raw((T *)base + at, r);
}
// V values of an optional f32 vector (absent: zero)
template <int V>
__device__ __forceinline__ void load_state(const float *p, long long c, float (&x)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.0f;
    if (p != nullptr) load<float, V>(p, c, x);
}
template <int V>
__device__ __forceinline__ void store_state(float *p, long long c, const float (&x)[V])
{
    if (p != nullptr) store<float, V>(p, c, x);
}

// ---- coefficients ------------------------------------------------------------------------------------
// a = sigmoid(f) and 1 - a.  Of the two the smaller is e / (1 + e) with e = exp(-|f|), so it keeps its relative precision
// however far the gate is open or shut; the larger is one minus it, rounded once.  A long sum weighs its terms by powers of
// a: a relative error of 1 - a would move the whole sum by that much, which rules out the one-instruction tanh form.
// With fp32 gates e and the quotient are within about one unit in the last place (FINE): the state's own rounding is no larger.
// With bf16 gates the hardware's exponential and reciprocal serve, a few units off.
// exp of x <= 0: x = n log 2 + z with log 2 in two parts, Taylor's polynomial of degree 7 on |z| <= log(2) / 2 (remainder
// 0.347^8 / 8! = 5e-9), times 2^n.
__device__ __forceinline__ float exp_fine(float x)
{
    const float n = rintf(x * 1.44269504f);
    const float z = fmaf(n, -1.42860677e-6f, fmaf(n, -0.693145752f, x));      // 0.693145752 has 15 bits: its product with n is exact
    float p = 1.0f / 5040.0f;
    p = fmaf(p, z, 1.0f / 720.0f);
    p = fmaf(p, z, 1.0f / 120.0f);
    p = fmaf(p, z, 1.0f / 24.0f);
    p = fmaf(p, z, 1.0f / 6.0f);
    p = fmaf(p, z, 0.5f);
    p = fmaf(p, z, 1.0f);
    p = fmaf(p, z, 1.0f);
    return x < -87.0f ? 0.0f : __int_as_float(__float_as_int(p) + ((int)n << 23));
}
template <bool FINE>
__device__ __forceinline__ void sigmoid_pair(float f, float &a, float &one_less)
{
    float small;
    if (FINE) {
        const float e = exp_fine(-fabsf(f)), d = 1.0f + e, r = __fdividef(1.0f, d);
        small = e * fmaf(r, fmaf(-d, r, 1.0f), r);         // one Newton step on the reciprocal
    } else {
        const float e = __expf(-fabsf(f));
        small = __fdividef(e, 1.0f + e);
    }
    const float large = 1.0f - small;
    a = f >= 0.0f ? large : small;
    one_less = f >= 0.0f ? small : large;
    if (f != f) a = one_less = f;
}
// A step's coefficient and the type F that states are carried in: fp32; beside fp32 gates fp64, rounded where a state is stored,
// so that a result which is the difference of two states' terms is as good as its inputs (the arithmetic is far from being the
// bound).  There an open gate (f >= 0) is held as -(1 - a), its sign saying so: a in fp32, near one, has no bits left for 1 - a,
// and over a long span of like gates that error would add up.
template <typename T, int GATE> struct Coefficient {
    static constexpr bool FINE = sizeof(T) == 4, SIGNED = FINE && GATE != RELAY_GATE_GIVEN;
    using F = std::conditional_t<FINE, double, float>;
    static __device__ __forceinline__ float keep() { return SIGNED ? -0.0f : 1.0f; }                     // a = 1
    static __device__ __forceinline__ F value(float k) { return SIGNED && __float_as_int(k) < 0 ? F(1) + F(k) : F(k); }
    static __device__ __forceinline__ void of(float f, float u, float &k, float &b)
    {
        if (GATE == RELAY_GATE_GIVEN) {
            k = f;
            b = u;
        } else {
            float a, s;
            sigmoid_pair<FINE>(f, a, s);
            b = GATE == RELAY_GATE_MIX ? s * u : u;
            k = SIGNED && f >= 0.0f ? -s : a;
        }
    }
};
// partials of one step: g = dh_t + G_{t+1}
template <int GATE, bool FINE>
__device__ __forceinline__ void partials(float f, float u, float before, float g, float &df, float &du)
{
    if (GATE == RELAY_GATE_GIVEN) {
        df = g * before;
        du = g;
    } else {
        float a, s;
        sigmoid_pair<FINE>(f, a, s);
        df = (GATE == RELAY_GATE_MIX ? g * (before - u) : g * before) * (a * s);
        du = GATE == RELAY_GATE_MIX ? g * s : g;
    }
}

__device__ __forceinline__ long long end_of(const Args &p, long long b)
{
    if (p.lengths == nullptr) return p.T;
    if (!relay_in_bounds(p.lengths + b, 4)) return 0;
    const long long n = p.lengths[b];
    return n < 0 ? 0 : n > p.T ? p.T : n;
}

template <typename F, int V>
__device__ __forceinline__ void load_initial(const float *p, long long c, bool live, F (&state)[V])
{
    float x[V];
    load_state(live ? p : nullptr, c, x);
#pragma unroll
    for (int i = 0; i < V; ++i) state[i] = (F)x[i];
}
template <typename F, int V>
__device__ __forceinline__ void store_final(float *p, long long c, const F (&state)[V])
{
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)state[i];
    store_state(p, c, x);
}

// ---- one thread per V channels, step by step ------------------------------------------------------------
template <typename T, typename TH, int GATE, int V>
__global__ void __launch_bounds__(kThreads) recurrence_steps_kernel(const Args p)
{
    using K = Coefficient<T, GATE>;
    using F = typename K::F;
    const long long c = ((long long)blockIdx.x * kThreads + threadIdx.x) * V;
    pdl_wait();
    if (c >= p.C) return;
    const long long b = c / p.D, at = b * p.bs + (c - b * p.D), end = end_of(p, b);
    F h[V];
    load_initial(p.h0, c, true, h);
#pragma unroll 8
    for (long long t = 0; t < p.T; ++t) {
        float f[V], u[V], out[V];
        load<T, V>(p.f, t * p.ld + at, f);
        load<T, V>(p.u, t * p.ld + at, u);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float k, x;
            K::of(f[i], u[i], k, x);
            const F next = K::value(k) * h[i] + F(x);
            if (t < end) h[i] = next;
            out[i] = t < end ? (float)next : 0.0f;
        }
        store<TH, V>(p.h, t * p.C + c, out);
    }
    store_final(p.h_final, c, h);
}

template <typename T, typename TH, int GATE, int V>
__global__ void __launch_bounds__(kThreads) recurrence_grad_steps_kernel(const Args p)
{
    using K = Coefficient<T, GATE>;
    using F = typename K::F;
    const long long c = ((long long)blockIdx.x * kThreads + threadIdx.x) * V;
    pdl_wait();
    if (c >= p.C) return;
    const long long b = c / p.D, at = b * p.bs + (c - b * p.D), end = end_of(p, b);
    F G[V];
    load_initial(p.dh_final, c, true, G);
#pragma unroll 4
    for (long long t = p.T - 1; t >= 0; --t) {
        float f[V], u[V], dh[V], before[V], df[V], du[V];
        load<T, V>(p.f, t * p.ld + at, f);
        load<T, V>(p.u, t * p.ld + at, u);
        load<TH, V>(p.dh, t * p.C + c, dh);
        if (t > 0) load<TH, V>(p.h, (t - 1) * p.C + c, before);
        else load_state(p.h0, c, before);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const F g = F(dh[i]) + G[i];
            float k, x;
            K::of(f[i], u[i], k, x);
            partials<GATE, K::FINE>(f[i], u[i], before[i], (float)g, df[i], du[i]);
            if (t < end) G[i] = K::value(k) * g;
            else df[i] = du[i] = 0.0f;
        }
        store<T, V>(p.df, t * p.ld + at, df);
        store<T, V>(p.du, t * p.ld + at, du);
    }
    store_final(p.dh0, c, G);
}

// ---- the time axis cut over warps, blocks and a cluster --------------------------------------------------
// A step maps the state h to a h + b, and maps compose: (A2, H2) after (A1, H1) is (A2 A1, A2 H1 + H2).  A lane owns V channels, a
// warp TS consecutive steps of them, a block kWarps such spans one after the other, a cluster of S blocks S such blocks; a
// cluster walks the sequence in slabs of S * kWarps * TS steps.  Per slab every thread reads its steps once into registers,
// composes them, the block's spans are joined through shared memory, the blocks' through their neighbours' shared memory (each
// block writes its map to all of the cluster, one cluster barrier), and the steps are then run again from registers with the
// right state.  Every value is read from memory once.  The next slab's values are requested before the barriers.
// The gradient is the same recursion backwards in time: G_t = a_t G_{t+1} + a_t dh_t.
constexpr int kWarps = 8;

template <typename F, int V> struct Map { F a[V], h[V]; };
template <typename F, int V>
__device__ __forceinline__ Map<F, V> then(const Map<F, V> &first, const Map<F, V> &second)
{
    Map<F, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        r.a[i] = first.a[i] * second.a[i];
        r.h[i] = second.a[i] * first.h[i] + second.h[i];
    }
    return r;
}
template <typename F, int V>
__device__ __forceinline__ Map<F, V> identity()
{
    Map<F, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) { r.a[i] = F(1); r.h[i] = F(0); }
    return r;
}
// the state behind a map: an overflowed product must not turn a zero state into NaN
template <typename F, int V>
__device__ __forceinline__ void apply(const Map<F, V> &m, F (&h)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = h[i] == F(0) ? m.h[i] : m.a[i] * h[i] + m.h[i];
}

template <typename F, int V>
struct Joints {
    Map<F, V> span[kWarps][32];        // this block's spans
    Map<F, V> block[2][8][32];         // the cluster's blocks, alternating between slabs
};
__device__ __forceinline__ uint32_t cluster_address(const void *p, uint32_t rank)
{
    uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
template <typename F, int V>
__device__ __forceinline__ void store_cluster(uint32_t at, const Map<F, V> &m)
{
    static_assert(sizeof(m) % 8 == 0, "pairs of words");
    const uint2 *w = reinterpret_cast<const uint2 *>(&m);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(m) / 8); ++i)
        asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(at + 8 * i), "r"(w[i].x), "r"(w[i].y) : "memory");
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Joins the maps of all threads of a lane's channels over the slab.  `state` is the state before the slab on entry, the state
// behind it on return; the result is the state before this thread's own span.
template <typename F, int V>
__device__ __forceinline__ void join_slab(Joints<F, V> &j, const Map<F, V> &mine, int warp, int lane, uint32_t rank, int S, int slab,
                                          F (&state)[V], F (&before)[V])
{
    j.span[warp][lane] = mine;
    __syncthreads();
    Map<F, V> ahead = identity<F, V>(), all = identity<F, V>();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) ahead = all;
        all = then(all, j.span[w][lane]);
    }
    // warp r tells block r of the cluster
    if (warp < S) store_cluster(cluster_address(&j.block[slab & 1][rank][lane], (uint32_t)warp), all);
    cluster_barrier();
#pragma unroll 1
    for (int r = 0; r < S; ++r) {
        if (r == (int)rank) {
#pragma unroll
            for (int i = 0; i < V; ++i) before[i] = state[i];
        }
        apply(j.block[slab & 1][r][lane], state);
    }
    apply(ahead, before);
}
template <typename T, typename TH, int GATE, int V, int TS>
__global__ void __launch_bounds__(32 * kWarps, 2) recurrence_spans_kernel(const Args p, int S)
{
    using K = Coefficient<T, GATE>;
    using F = typename K::F;
    __shared__ __align__(16) Joints<F, V> joints;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x % S;
    const long long c = ((long long)(blockIdx.x / S) * 32 + lane) * V;
    const bool live = c < p.C;
    cluster_barrier();                 // every block of the cluster runs before its shared memory is written
    pdl_wait();
    const long long b = live ? c / p.D : 0, at = b * p.bs + (c - b * p.D), end = live ? end_of(p, b) : 0;
    F state[V];
    load_initial(p.h0, c, live, state);
    const long long slab_steps = (long long)S * kWarps * TS;
    const int slabs = (int)((p.T + slab_steps - 1) / slab_steps);
    long long t0 = ((long long)rank * kWarps + warp) * TS;

    Raw<T, V> rf[TS], ru[TS];
    auto request = [&](long long first) {
        const T *f = (const T *)p.f + first * p.ld + at, *u = (const T *)p.u + first * p.ld + at;
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            rf[s] = Raw<T, V>{}; ru[s] = Raw<T, V>{};
            if (live && first + s < p.T) { rf[s] = load_raw<Raw<T, V>>(f + s * p.ld); ru[s] = load_raw<Raw<T, V>>(u + s * p.ld); }
        }
    };
    request(t0);
    for (int slab = 0; slab < slabs; ++slab, t0 += slab_steps) {
        float a[TS][V], x[TS][V];
        Map<F, V> mine = identity<F, V>();
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            float f[V], u[V];
            to_f32(rf[s], f); to_f32(ru[s], u);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                K::of(f[i], u[i], a[s][i], x[s][i]);
                if (t0 + s >= end) { a[s][i] = K::keep(); x[s][i] = 0.0f; }
                const F v = K::value(a[s][i]);
                mine.a[i] *= v;
                mine.h[i] = v * mine.h[i] + F(x[s][i]);
            }
        }
        if (slab + 1 < slabs) request(t0 + slab_steps);
        F h[V];
        join_slab(joints, mine, warp, lane, rank, S, slab, state, h);
        TH *out = (TH *)p.h + t0 * p.C + c;
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                h[i] = K::value(a[s][i]) * h[i] + F(x[s][i]);
                o[i] = t0 + s < end ? (float)h[i] : 0.0f;
            }
            if (live && t0 + s < p.T) store<TH, V>(out, (long long)s * p.C, o);
        }
    }
    if (live && rank == 0 && warp == 0) store_final(p.h_final, c, state);
    cluster_barrier();                 // no block leaves while another may still write to its shared memory
}

template <typename T, typename TH, int GATE, int V, int TS>
__global__ void __launch_bounds__(32 * kWarps, 2) recurrence_grad_spans_kernel(const Args p, int S)
{
    using K = Coefficient<T, GATE>;
    using F = typename K::F;
    __shared__ __align__(16) Joints<F, V> joints;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x % S;
    const long long c = ((long long)(blockIdx.x / S) * 32 + lane) * V;
    const bool live = c < p.C;
    cluster_barrier();                 // every block of the cluster runs before its shared memory is written
    pdl_wait();
    const long long b = live ? c / p.D : 0, at = b * p.bs + (c - b * p.D), end = live ? end_of(p, b) : 0;
    F state[V];
    load_initial(p.dh_final, c, live, state);
    const long long slab_steps = (long long)S * kWarps * TS;
    const int slabs = (int)((p.T + slab_steps - 1) / slab_steps);
    long long t0 = p.T - 1 - ((long long)rank * kWarps + warp) * TS;      // this thread's steps are t0, t0 - 1, ..

    Raw<T, V> nf[TS], nu[TS];
    Raw<TH, V> nd[TS], nh[TS];
    auto request = [&](long long first) {
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            const long long t = first - s;
            nf[s] = Raw<T, V>{}; nu[s] = Raw<T, V>{}; nd[s] = Raw<TH, V>{}; nh[s] = Raw<TH, V>{};
            if (live && t >= 0) {
                nf[s] = load_raw<Raw<T, V>>((const T *)p.f + t * p.ld + at);
                nu[s] = load_raw<Raw<T, V>>((const T *)p.u + t * p.ld + at);
                nd[s] = load_raw<Raw<TH, V>>((const TH *)p.dh + t * p.C + c);
                if (t > 0) nh[s] = load_raw<Raw<TH, V>>((const TH *)p.h + (t - 1) * p.C + c);
            }
        }
    };
    request(t0);
    for (int slab = 0; slab < slabs; ++slab, t0 -= slab_steps) {
        Raw<T, V> rf[TS], ru[TS];
        Raw<TH, V> rd[TS], rh[TS];
        Map<F, V> mine = identity<F, V>();
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            rf[s] = nf[s]; ru[s] = nu[s]; rd[s] = nd[s]; rh[s] = nh[s];
            float f[V], dh[V];
            to_f32(rf[s], f); to_f32(rd[s], dh);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float k, unused;
                K::of(f[i], 0.0f, k, unused);
                if (t0 - s < end && t0 - s >= 0) {
                    const F v = K::value(k);
                    mine.a[i] *= v;
                    mine.h[i] = v * (mine.h[i] + F(dh[i]));
                }
            }
        }
        if (slab + 1 < slabs) request(t0 - slab_steps);
        F G[V];
        join_slab(joints, mine, warp, lane, rank, S, slab, state, G);
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            const long long t = t0 - s;
            float f[V], u[V], dh[V], before[V], df[V], du[V];
            to_f32(rf[s], f); to_f32(ru[s], u); to_f32(rd[s], dh); to_f32(rh[s], before);
            if (live && t == 0) load_state(p.h0, c, before);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const F g = F(dh[i]) + G[i];
                float k, unused;
                K::of(f[i], u[i], k, unused);
                partials<GATE, K::FINE>(f[i], u[i], before[i], (float)g, df[i], du[i]);
                if (t < end) G[i] = K::value(k) * g;
                else df[i] = du[i] = 0.0f;
            }
            if (live && t >= 0) {
                store<T, V>(p.df, t * p.ld + at, df);
                store<T, V>(p.du, t * p.ld + at, du);
            }
        }
    }
    if (live && rank == 0 && warp == 0) store_final(p.dh0, c, state);
    cluster_barrier();
}

// Sequences of up to kSteps steps run step by step.  Longer ones: the smallest cluster that gives every SM a block.
constexpr long long kSteps = 32;

template <typename T, typename TH, int GATE, int V>
relay_status_t launch(const Args &p, bool grad, cudaStream_t st)
{
    if (p.T > kSteps) {
        constexpr int TS = sizeof(T) == 2 ? 16 : 8, TSG = sizeof(T) + sizeof(TH) == 4 ? 8 : 4;
        int dev = 0, sms = 148;
        RELAY_CUDA(cudaGetDevice(&dev));
        RELAY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        const long long tiles = (p.C + 32 * V - 1) / (32 * V), steps = kWarps * (grad ? TSG : TS);
        int S = 1;
        while (S < 8 && tiles * S < sms && p.T > S * steps) S *= 2;
        if (tiles * S > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "gated_recurrence: %lld channels", p.C);
        const dim3 grid((unsigned)(tiles * S)), block(32 * kWarps), cluster((unsigned)S);
        if (grad) RELAY_CUDA(launch_pdl_cluster(recurrence_grad_spans_kernel<T, TH, GATE, V, TSG>, grid, block, cluster, 0, st, p, S));
        else RELAY_CUDA(launch_pdl_cluster(recurrence_spans_kernel<T, TH, GATE, V, TS>, grid, block, cluster, 0, st, p, S));
        return check_launch("gated_recurrence");
    }
    const dim3 grid((unsigned)((p.C / V + kThreads - 1) / kThreads));
    if (grad) RELAY_CUDA(launch_pdl(recurrence_grad_steps_kernel<T, TH, GATE, V>, grid, dim3(kThreads), 0, st, p));
    else RELAY_CUDA(launch_pdl(recurrence_steps_kernel<T, TH, GATE, V>, grid, dim3(kThreads), 0, st, p));
    return check_launch("gated_recurrence");
}
template <typename T, typename TH>
relay_status_t launch_typed(const Args &p, int32_t gate, bool grad, cudaStream_t st)
{
    // two channels a thread where every row starts at an even element, so that the pair is one aligned access
    const bool pair = p.D % 2 == 0 && p.ld % 2 == 0 && p.bs % 2 == 0;
    switch (gate) {
    case RELAY_GATE_GIVEN: return pair ? launch<T, TH, RELAY_GATE_GIVEN, 2>(p, grad, st) : launch<T, TH, RELAY_GATE_GIVEN, 1>(p, grad, st);
    case RELAY_GATE_SIGMOID: return pair ? launch<T, TH, RELAY_GATE_SIGMOID, 2>(p, grad, st) : launch<T, TH, RELAY_GATE_SIGMOID, 1>(p, grad, st);
    default: return pair ? launch<T, TH, RELAY_GATE_MIX, 2>(p, grad, st) : launch<T, TH, RELAY_GATE_MIX, 1>(p, grad, st);
    }
}
relay_status_t launch_any(const Args &p, int32_t t, int32_t th, int32_t gate, bool grad, cudaStream_t st)
{
    if (t == RELAY_F32) return launch_typed<float, float>(p, gate, grad, st);
    if (th == RELAY_BF16) return launch_typed<__nv_bfloat16, __nv_bfloat16>(p, gate, grad, st);
    return launch_typed<__nv_bfloat16, float>(p, gate, grad, st);
}

// ---- boundary ------------------------------------------------------------------------------------------
struct Sizes { int64_t T, B, D; bool packed; };

// gates and values: types, ranks and shapes; fills the sizes of the result
relay_status_t check_inputs(const relay_tensor_t *f, const relay_tensor_t *u, Sizes *s)
{
    RELAY_TRY(check_type(f, "f"));
    if (u) RELAY_TRY(check_type(u, "u"));
    RELAY_TRY(check_rank(f, 3, "f"));
    if (u) RELAY_TRY(check_rank(u, 3, "u"));
    if (!is_float(f->dtype)) return fail(RELAY_ERR_DTYPE, "f: base type %s, needs f32 or bf16", dtype_name(f->dtype));
    if (u) RELAY_TRY(check_dtype(u, f->dtype, "u"));
    RELAY_TRY(check_layout(f, RELAY_ROWMAJOR, RELAY_ROWMAJOR, "f"));
    if (u) RELAY_TRY(check_layout(u, RELAY_ROWMAJOR, RELAY_ROWMAJOR, "u"));
    s->T = f->shape[0]; s->B = f->shape[1]; s->packed = u == nullptr;
    if (s->packed && f->shape[2] % 2)
        return fail(RELAY_ERR_SHAPE, "f: last axis has %lld entries, the two blocks [ f | u ] need an even number", (long long)f->shape[2]);
    s->D = s->packed ? f->shape[2] / 2 : f->shape[2];
    if (u) RELAY_TRY(check_shape(u, {s->T, s->B, s->D}, "u"));
    return RELAY_OK;
}
relay_status_t check_state(const relay_tensor_t *t, const Sizes &s, const char *name)
{
    if (!t) return RELAY_OK;
    RELAY_TRY(check_type(t, name));
    RELAY_TRY(check_rank(t, 2, name));
    RELAY_TRY(check_dtype(t, RELAY_F32, name));
    RELAY_TRY(check_layout(t, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
    return check_shape(t, {s.B, s.D}, name);
}
relay_status_t check_lengths(const relay_tensor_t *t, const Sizes &s)
{
    if (!t) return RELAY_OK;
    RELAY_TRY(check_type(t, "lengths"));
    RELAY_TRY(check_rank(t, 1, "lengths"));
    RELAY_TRY(check_dtype(t, RELAY_I32, "lengths"));
    return check_shape(t, {s.B}, "lengths");
}
relay_status_t check_sequence(const relay_tensor_t *t, int32_t t0, int32_t t1, const Sizes &s, int64_t last, const char *name)
{
    RELAY_TRY(check_type(t, name));
    RELAY_TRY(check_rank(t, 3, name));
    if (t->dtype != t0 && t->dtype != t1)
        return fail(RELAY_ERR_DTYPE, "%s: base type %s, needs %s%s%s", name, dtype_name(t->dtype), dtype_name(t0), t0 == t1 ? "" : " or ",
                    t0 == t1 ? "" : dtype_name(t1));
    RELAY_TRY(check_layout(t, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
    return check_shape(t, {s.T, s.B, last}, name);
}
relay_status_t check_gate(int32_t gate)
{
    if (gate < RELAY_GATE_GIVEN || gate > RELAY_GATE_MIX) return fail(RELAY_ERR_ATTR, "gate = %d", gate);
    return RELAY_OK;
}

Args make_args(const relay_tensor_t *f, const relay_tensor_t *u, const relay_tensor_t *h0, const relay_tensor_t *lengths, const Sizes &s)
{
    Args p{};
    p.f = f->data;
    p.u = s.packed ? (const char *)f->data + s.D * dtype_size(f->dtype) : u->data;
    p.T = s.T; p.C = s.B * s.D; p.D = s.D;
    p.bs = s.packed ? 2 * s.D : s.D;
    p.ld = s.B * p.bs;
    p.h0 = h0 ? (const float *)h0->data : nullptr;
    p.lengths = lengths ? (const int *)lengths->data : nullptr;
    if (!s.packed && !lengths) p.D = p.C;          // nothing depends on the batch element: one row of channels
    return p;
}

}  // namespace
}  // namespace relay

using namespace relay;

extern "C" relay_status_t relay_infer_gated_recurrence(const relay_tensor_t *f, const relay_tensor_t *u, relay_tensor_t *h_all,
                                                       relay_tensor_t *h_final)
{
    clear_error();
    RELAY_TRY(check_not_null(f, "f"));
    RELAY_TRY(check_not_null(h_all, "h_all"));
    RELAY_TRY(check_not_null(h_final, "h_final"));
    Sizes s;
    RELAY_TRY(check_inputs(f, u, &s));
    *h_all = relay_tensor_t{};
    h_all->dtype = f->dtype; h_all->rank = 3; h_all->layout = RELAY_ROWMAJOR;
    h_all->shape[0] = s.T; h_all->shape[1] = s.B; h_all->shape[2] = s.D;
    *h_final = relay_tensor_t{};
    h_final->dtype = RELAY_F32; h_final->rank = 2; h_final->layout = RELAY_ROWMAJOR;
    h_final->shape[0] = s.B; h_final->shape[1] = s.D;
    return RELAY_OK;
}

extern "C" relay_status_t relay_gated_recurrence(const relay_tensor_t *f, const relay_tensor_t *u, const relay_tensor_t *h0,
                                                 const relay_tensor_t *lengths, int32_t gate, const relay_tensor_t *h_all,
                                                 const relay_tensor_t *h_final, void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(f, "f"));
    RELAY_TRY(check_not_null(h_all, "h_all"));
    Sizes s;
    RELAY_TRY(check_inputs(f, u, &s));
    RELAY_TRY(check_state(h0, s, "h0"));
    RELAY_TRY(check_lengths(lengths, s));
    RELAY_TRY(check_sequence(h_all, f->dtype, RELAY_F32, s, s.D, "h_all"));
    RELAY_TRY(check_state(h_final, s, "h_final"));
    RELAY_TRY(check_gate(gate));
    const relay_tensor_t *ins[4] = {f, u, h0, lengths}, *outs[2] = {h_all, h_final};
    for (const relay_tensor_t *t : ins) if (t) RELAY_TRY(check_data(t, "input"));
    for (const relay_tensor_t *t : outs) if (t) RELAY_TRY(check_data(t, "output"));
    RELAY_TRY(check_no_overlap(outs, 2, ins, 4));
    if (s.B == 0 || s.D == 0) return RELAY_OK;
    Args p = make_args(f, u, h0, lengths, s);
    p.h = h_all->data;
    p.h_final = h_final ? (float *)h_final->data : nullptr;
    BoundsReg reg;
    for (const relay_tensor_t *t : ins) reg.add(t);
    for (const relay_tensor_t *t : outs) reg.add(t);
    RELAY_TRY(reg.commit((cudaStream_t)stream));
    return launch_any(p, f->dtype, h_all->dtype, gate, false, (cudaStream_t)stream);
}

extern "C" relay_status_t relay_gated_recurrence_grad(const relay_tensor_t *f, const relay_tensor_t *u, const relay_tensor_t *h0,
                                                      const relay_tensor_t *lengths, int32_t gate, const relay_tensor_t *h_all,
                                                      const relay_tensor_t *dh_all, const relay_tensor_t *dh_final,
                                                      const relay_tensor_t *df, const relay_tensor_t *du, const relay_tensor_t *dh0,
                                                      void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(f, "f"));
    RELAY_TRY(check_not_null(h_all, "h_all"));
    RELAY_TRY(check_not_null(dh_all, "dh_all"));
    RELAY_TRY(check_not_null(df, "df"));
    if (u) RELAY_TRY(check_not_null(du, "du"));
    Sizes s;
    RELAY_TRY(check_inputs(f, u, &s));
    RELAY_TRY(check_state(h0, s, "h0"));
    RELAY_TRY(check_lengths(lengths, s));
    RELAY_TRY(check_sequence(h_all, f->dtype, RELAY_F32, s, s.D, "h_all"));
    RELAY_TRY(check_sequence(dh_all, h_all->dtype, h_all->dtype, s, s.D, "dh_all"));
    RELAY_TRY(check_state(dh_final, s, "dh_final"));
    RELAY_TRY(check_sequence(df, f->dtype, f->dtype, s, f->shape[2], "df"));
    if (u) RELAY_TRY(check_sequence(du, f->dtype, f->dtype, s, s.D, "du"));
    RELAY_TRY(check_state(dh0, s, "dh0"));
    RELAY_TRY(check_gate(gate));
    if (!u && du) return fail(RELAY_ERR_ATTR, "du is given, but u is part of f: its partial is part of df");
    const relay_tensor_t *ins[7] = {f, u, h0, lengths, h_all, dh_all, dh_final}, *outs[3] = {df, du, dh0};
    for (const relay_tensor_t *t : ins) if (t) RELAY_TRY(check_data(t, "input"));
    for (const relay_tensor_t *t : outs) if (t) RELAY_TRY(check_data(t, "output"));
    RELAY_TRY(check_no_overlap(outs, 3, ins, 7));
    if (s.B == 0 || s.D == 0) return RELAY_OK;
    Args p = make_args(f, u, h0, lengths, s);
    p.h = h_all->data;
    p.dh = dh_all->data;
    p.dh_final = dh_final ? (const float *)dh_final->data : nullptr;
    p.df = df->data;
    p.du = s.packed ? (char *)df->data + s.D * dtype_size(f->dtype) : du->data;
    p.dh0 = dh0 ? (float *)dh0->data : nullptr;
    BoundsReg reg;
    for (const relay_tensor_t *t : ins) reg.add(t);
    for (const relay_tensor_t *t : outs) reg.add(t);
    RELAY_TRY(reg.commit((cudaStream_t)stream));
    return launch_any(p, f->dtype, h_all->dtype, gate, true, (cudaStream_t)stream);
}
