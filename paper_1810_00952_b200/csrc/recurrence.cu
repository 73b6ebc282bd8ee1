// Gated linear recurrence over a sequence, h_t = a_t h_{t-1} + b_t per channel, and its gradient group (Section 4.2 of the
// paper: reverse mode through the recursion over time).  Elementwise steps: HBM-bound where the channels fill the GPU.
//
// Bytes: the forward group reads f and u and writes h once, the gradient reads f, u, h, dh and writes df, du once.  Measured against
// a copy at 6.53 TB/s: 16384 x 1 x 4096 in bf16 85 us (4.7 TB/s), gradient of 4096 x 8 x 1024 in bf16 87 us (4.6 TB/s); the same
// in fp32, with fp64 states, 108 us forward (3.7 TB/s) and 233 the gradient (3.5 TB/s, one block an SM).  Short of that the length of the
// chain counts: 128 x 64 x 1024 in bf16 15.4 us (3.3 TB/s), 16384 steps of 64 channels 38 us forward (eight blocks at most work on them), one
// step of 64 x 1024 7.4 us, nearly all of it the call and the launch.
//
// Three forms: step by step, a thread per one or two channels (few steps); the time axis cut into spans that stay in registers (rows that
// are not whole 16-byte pieces); the same with tiles fetched ahead by TMA and a warp that only joins (all others).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "common.h"
#include "ewise_kernels.cuh"
#include "tc_common.cuh"

namespace relay {

relay_status_t make_tmap_2d(CUtensorMap *m, bool f32, const void *base, uint64_t inner, uint64_t outer, uint64_t row_stride,
                            uint32_t box_inner, uint32_t box_outer, bool swizzle128);

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
    int *err;
};

// ---- vectors of V consecutive channels -----------------------------------------------------------------
template <typename T, int V> struct RawOf { using type = T; };
template <> struct RawOf<__nv_bfloat16, 2> { using type = uint32_t; };
template <> struct RawOf<__nv_bfloat16, 4> { using type = uint2; };
template <> struct RawOf<float, 2> { using type = uint2; };
template <> struct RawOf<float, 4> { using type = uint4; };
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
__device__ __forceinline__ void to_f32(uint2 r, float (&x)[4])
{
    x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xffff0000u);
    x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xffff0000u);
}
__device__ __forceinline__ void to_f32(uint4 r, float (&x)[4]) { unpack(r, x); }
__device__ __forceinline__ void to_f32(uint2 r, float (&x)[2]) { x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); }
__device__ __forceinline__ void to_f32(__nv_bfloat16 r, float (&x)[1]) { x[0] = __bfloat162float(r); }
__device__ __forceinline__ void to_f32(float r, float (&x)[1]) { x[0] = r; }
__device__ __forceinline__ void from_f32(const float (&x)[2], uint32_t &r) { r = pack2(x[0], x[1]); }
__device__ __forceinline__ void from_f32(const float (&x)[2], uint2 &r) { r = make_uint2(__float_as_uint(x[0]), __float_as_uint(x[1])); }
__device__ __forceinline__ void from_f32(const float (&x)[4], uint2 &r) { r = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3])); }
__device__ __forceinline__ void from_f32(const float (&x)[4], uint4 &r) { r = pack(x); }
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

// ---- arithmetic on V channels: fp32 in pairs (one instruction for two), fp64 one by one ------------------------------------
__device__ __forceinline__ unsigned long long pair(float lo, float hi)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(unsigned long long r, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(r)); }
template <int V>
__device__ __forceinline__ void mul(const float (&a)[V], const float (&b)[V], float (&r)[V])
{
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            unsigned long long q;
            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(q) : "l"(pair(a[i], a[i + 1])), "l"(pair(b[i], b[i + 1])));
            unpair(q, r[i], r[i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = a[i] * b[i];
    }
}
template <int V>
__device__ __forceinline__ void add(const float (&a)[V], const float (&b)[V], float (&r)[V])
{
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            unsigned long long q;
            asm("add.rn.f32x2 %0, %1, %2;" : "=l"(q) : "l"(pair(a[i], a[i + 1])), "l"(pair(b[i], b[i + 1])));
            unpair(q, r[i], r[i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = a[i] + b[i];
    }
}
// a b + c
template <int V>
__device__ __forceinline__ void muladd(const float (&a)[V], const float (&b)[V], const float (&c)[V], float (&r)[V])
{
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            unsigned long long q;
            asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(q) : "l"(pair(a[i], a[i + 1])), "l"(pair(b[i], b[i + 1])), "l"(pair(c[i], c[i + 1])));
            unpair(q, r[i], r[i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = fmaf(a[i], b[i], c[i]);
    }
}
template <int V>
__device__ __forceinline__ void mul(const double (&a)[V], const double (&b)[V], double (&r)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = a[i] * b[i];
}
template <int V>
__device__ __forceinline__ void add(const double (&a)[V], const double (&b)[V], double (&r)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = a[i] + b[i];
}
template <int V>
__device__ __forceinline__ void muladd(const double (&a)[V], const double (&b)[V], const double (&c)[V], double (&r)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = a[i] * b[i] + c[i];
}
template <int V>
__device__ __forceinline__ void fill(float x, float (&r)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = x;
}

// ---- coefficients ------------------------------------------------------------------------------------
// a = sigmoid(f) and 1 - a.  Of the two the smaller is e / (1 + e) with e = exp(-|f|), so it keeps its relative precision
// however far the gate is open or shut; the larger is one minus it, rounded once.  A long sum weighs its terms by powers of
// a: a relative error of 1 - a would move the whole sum by that much, which rules out the one-instruction tanh form.
// With fp32 gates e and the quotient are within about one unit in the last place (FINE): the state's own rounding is no larger.
// With bf16 gates the hardware's exponential and reciprocal serve, a few units off.
// exp of x <= 0: x = n log 2 + z with log 2 in two parts, Taylor's polynomial of degree 7 on |z| <= log(2) / 2 (remainder
// 0.347^8 / 8! = 5e-9), times 2^n.  n comes as the low bits of a sum with 1.5 * 2^23.
// x is held at -88, where n = -127 and the power's bits are those of zero.
template <int V>
__device__ __forceinline__ void exp_fine(float (&x)[V])
{
    float c[V], t[V], n[V], p[V];
#pragma unroll
    for (int i = 0; i < V; ++i) asm("max.NaN.f32 %0, %0, 0fC2B00000;" : "+f"(x[i]));       // -88
    fill(1.44269504f, c);
    fill(12582912.0f, p);
    muladd(x, c, p, t);
    fill(-12582912.0f, c);
    add(t, c, n);
    fill(-0.693115234375f, c);                             // 2839 / 4096: its product with n is exact
    muladd(n, c, x, x);
    fill(-3.19461849e-5f, c);                              // what log 2 has beyond it
    muladd(n, c, x, x);
    const float of[7] = {1.0f / 720.0f, 1.0f / 120.0f, 1.0f / 24.0f, 1.0f / 6.0f, 0.5f, 1.0f, 1.0f};
    fill(1.0f / 5040.0f, p);
#pragma unroll
    for (int k = 0; k < 7; ++k) {
        fill(of[k], c);
        muladd(p, x, c, p);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = __int_as_float(0x3f800000 + (__float_as_int(t[i]) << 23));
    mul(p, t, x);                                          // a product, for NaN to stay NaN
}
// the smaller of sigmoid(f) and 1 - sigmoid(f): e / (1 + e), the reciprocal with one Newton step
template <int V>
__device__ __forceinline__ void sigmoid_small(const float (&f)[V], float (&small)[V])
{
    float e[V], d[V], r[V], c[V], t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = -fabsf(f[i]);
    exp_fine(e);
    fill(-1.0f, c);
    fill(-1.0f, t);
    muladd(e, c, t, d);                                    // -(1 + e)
#pragma unroll
    for (int i = 0; i < V; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r[i]) : "f"(-d[i]));
    fill(1.0f, c);
    muladd(d, r, c, t);
    muladd(r, t, r, r);
    mul(e, r, small);
}
template <bool FINE, int V>
__device__ __forceinline__ void sigmoid_pair(const float (&f)[V], float (&a)[V], float (&one_less)[V])
{
    if constexpr (FINE) {
        float small[V], large[V];
        sigmoid_small(f, small);
        float c[V], m[V];
        fill(1.0f, c);
        fill(-1.0f, m);
        muladd(small, m, c, large);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = f[i] >= 0.0f ? large[i] : small[i];
            one_less[i] = f[i] >= 0.0f ? small[i] : large[i];
        }
    } else {
        // 1 - a = 1 / (1 + exp(f)).  Where the gate is shut a is the smaller one and is exp(f) times that; where it is open a is one
        // minus that, also where the exponential is infinite.  (One minus it everywhere: 81 us against 85 at 16384 x 1 x 4096, but a has
        // an absolute error of 6e-8 then: nothing is left of it, or of the gate's partial, at f = -17.)
        float y[V], c[V], shut[V];
        fill(1.44269504f, c);
        mul(f, c, y);
#pragma unroll
        for (int i = 0; i < V; ++i) asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(y[i]));
        float d[V];
        fill(1.0f, c);
        add(y, c, d);
#pragma unroll
        for (int i = 0; i < V; ++i) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(one_less[i]) : "f"(d[i]));
        float m[V];
        fill(-1.0f, m);
        muladd(one_less, m, c, a);
        mul(y, one_less, shut);
#pragma unroll
        for (int i = 0; i < V; ++i) {                      // by f's sign; a compare and a select were slower
            const int k = __float_as_int(f[i]) >> 31;
            a[i] = __int_as_float((__float_as_int(a[i]) & ~k) | (__float_as_int(shut[i]) & k));
        }
    }
}
// A step's coefficient and the type F that states are carried in: fp32; beside fp32 gates fp64, rounded where a state is stored,
// so that a result which is the difference of two states' terms is as good as its inputs (the arithmetic is far from being the
// bound).  There an open gate (f >= 0) is held as -(1 - a), its sign saying so: a in fp32, near one, has no bits left for 1 - a,
// and over a long span of like gates that error would add up.
template <typename T, int GATE, int V> struct Coefficient {
    static constexpr bool FINE = sizeof(T) == 4, SIGNED = FINE && GATE != RELAY_GATE_GIVEN;
    using F = std::conditional_t<FINE, double, float>;
    static __device__ __forceinline__ float keep() { return SIGNED ? -0.0f : 1.0f; }                     // a = 1
    static __device__ __forceinline__ void value(const float (&k)[V], F (&a)[V])
    {
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = SIGNED && __float_as_int(k[i]) < 0 ? F(1) + F(k[i]) : F(k[i]);
    }
    static __device__ __forceinline__ void of(const float (&f)[V], float (&k)[V])
    {
        float s[V];
        if constexpr (GATE == RELAY_GATE_GIVEN) {
#pragma unroll
            for (int i = 0; i < V; ++i) k[i] = f[i];
        } else {
            if constexpr (SIGNED) {
                sigmoid_small(f, s);
                signed_by(f, s, k);
            } else {
                sigmoid_pair<FINE>(f, k, s);
            }
        }
    }
    // -(1 - a) of an open gate, a of one that is not: the smaller of the two either way, with the opposite of f's sign bit
    static __device__ __forceinline__ void signed_by(const float (&f)[V], const float (&small)[V], float (&k)[V])
    {
#pragma unroll
        for (int i = 0; i < V; ++i) k[i] = __int_as_float(__float_as_int(small[i]) | (~__float_as_int(f[i]) & 0x80000000));
    }
    static __device__ __forceinline__ void of(const float (&f)[V], const float (&u)[V], float (&k)[V], float (&b)[V])
    {
        if constexpr (GATE == RELAY_GATE_MIX) {
            float s[V];
            if constexpr (SIGNED) {
                float less[V];
                sigmoid_small(f, s);
                signed_by(f, s, k);
#pragma unroll
                for (int i = 0; i < V; ++i) less[i] = f[i] >= 0.0f ? s[i] : 1.0f - s[i];
                mul(less, u, b);
            } else {
                sigmoid_pair<FINE>(f, k, s);
                mul(s, u, b);
            }
        } else {
            of(f, k);
#pragma unroll
            for (int i = 0; i < V; ++i) b[i] = u[i];
        }
    }
    // h <- a h + b
    static __device__ __forceinline__ void step(const float (&k)[V], const float (&b)[V], F (&h)[V])
    {
        F a[V], x[V];
        value(k, a);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = F(b[i]);
        muladd(a, h, x, h);
    }
};
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

// One step backwards: with g = dh + G, partials of f and u, and G <- a g; a step behind the end has none and leaves G.
template <typename K, int GATE, int V>
__device__ __forceinline__ void backward_step(const float (&f)[V], const float (&u)[V], const float (&dh)[V], const float (&before)[V], bool on,
                                              typename K::F (&G)[V], float (&df)[V], float (&du)[V])
{
    using F = typename K::F;
    F g[V], a[V];
    float g32[V];
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = F(dh[i]);
    add(g, G, g);
#pragma unroll
    for (int i = 0; i < V; ++i) g32[i] = (float)g[i];
    if constexpr (GATE == RELAY_GATE_GIVEN) {
        mul(g32, before, df);
#pragma unroll
        for (int i = 0; i < V; ++i) { du[i] = g32[i]; a[i] = F(f[i]); }
    } else {
        float open[V], s[V], gs[V];
        sigmoid_pair<K::FINE>(f, open, s);
        mul(g32, s, gs);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            du[i] = GATE == RELAY_GATE_MIX ? gs[i] : g32[i];
            a[i] = K::FINE && f[i] >= 0.0f ? F(1) - F(s[i]) : F(open[i]);
        }
        mul(gs, open, gs);
        if constexpr (GATE == RELAY_GATE_MIX) {
            float d[V], m[V];
            fill(-1.0f, m);
            muladd(u, m, before, d);
            mul(gs, d, df);
        } else {
            mul(gs, before, df);
        }
    }
    if (on) {
        mul(a, g, G);
    } else {
        fill(0.0f, df);
        fill(0.0f, du);
    }
}

// ---- one thread per V channels, step by step ------------------------------------------------------------
template <typename T, typename TH, int GATE, int V>
__global__ void __launch_bounds__(kThreads) recurrence_steps_kernel(const Args p)
{
    using K = Coefficient<T, GATE, V>;
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
        float k[V], x[V];
        K::of(f, u, k, x);
        if (t < end) K::step(k, x, h);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = t < end ? (float)h[i] : 0.0f;
        store<TH, V>(p.h, t * p.C + c, out);
    }
    store_final(p.h_final, c, h);
}

template <typename T, typename TH, int GATE, int V>
__global__ void __launch_bounds__(kThreads) recurrence_grad_steps_kernel(const Args p)
{
    using K = Coefficient<T, GATE, V>;
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
        backward_step<K, GATE, V>(f, u, dh, before, t < end, G, df, du);
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
// block sends its map to all of the cluster), and the steps are then run again from registers with the
// right state.  Every value is read from memory once.  The next slab's values are requested before the barriers.
// The gradient is the same recursion backwards in time: G_t = a_t G_{t+1} + a_t dh_t.
constexpr int kWarps = 8;

template <typename F, int V> struct Map { F a[V], h[V]; };
template <typename F, int V>
__device__ __forceinline__ Map<F, V> then(const Map<F, V> &first, const Map<F, V> &second)
{
    Map<F, V> r;
    mul(first.a, second.a, r.a);
    muladd(second.a, first.h, second.h, r.h);
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
// The state behind a map.  SAFE, for coefficients that may exceed one: an overflowed product must not turn a zero state into NaN.
template <bool SAFE, typename F, int V>
__device__ __forceinline__ void apply(const Map<F, V> &m, F (&h)[V])
{
    F r[V];
    muladd(m.a, h, m.h, r);
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = SAFE && h[i] == F(0) ? m.h[i] : r[i];
}

template <typename F, int V>
struct Joints {
    Map<F, V> span[kWarps][32];        // this block's spans, then what lies ahead of each
    struct { F h[V]; } state[32];      // before this block
    Map<F, V> block[2][8][32];         // the cluster's blocks, sent by each; alternating between slabs
    uint64_t arrived[2];               // all of block[.] is here
    int gave_up;
    __device__ __forceinline__ void init()
    {
        if (threadIdx.x == 0) {
            tc::mbar_init(&arrived[0], 1);
            tc::mbar_init(&arrived[1], 1);
            gave_up = 0;
            tc::fence_barrier_init();
        }
        tc::cluster_sync();            // every block of the cluster runs, its barriers set up, before anything is sent to it
    }
};
// one-way: the data and the byte count that completes the receiver's barrier travel together.  (A cluster barrier per slab
// would make every block wait for its own stores to global memory.)
template <typename F, int V>
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, const Map<F, V> &m)
{
    const uint2 *w = reinterpret_cast<const uint2 *>(&m);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(m) / 8); ++i)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.u32 [%0], {%1, %2}, [%3];" ::"r"(to + 8 * i), "r"(w[i].x), "r"(w[i].y), "r"(bar) : "memory");
}
// Joins the maps of all threads of a lane's channels over the slab.  Warp 0 does it for the block (eight warps doing it each for
// themselves would execute more instructions than the steps do); its `state` is the state before the slab on entry, behind it on
// return.  The result is the state before this thread's own span.
template <bool SAFE, typename F, int V>
__device__ __forceinline__ void join_slab(Joints<F, V> &j, const Map<F, V> &mine, int warp, int lane, uint32_t rank, int S, int slab, int *err,
                                          F (&state)[V], F (&before)[V])
{
    j.span[warp][lane] = mine;
    __syncthreads();
    if (warp == 0) {
        Map<F, V> m[kWarps], all = mine;                  // all loads in flight together
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m[w] = j.span[w][lane];
        j.span[0][lane] = identity<F, V>();
#pragma unroll
        for (int w = 1; w < kWarps; ++w) {
            j.span[w][lane] = all;
            all = then(all, m[w]);
        }
        if (S == 1) {
#pragma unroll
            for (int i = 0; i < V; ++i) j.state[lane].h[i] = state[i];
            apply<SAFE>(all, state);
        } else {
            const int buf = slab & 1;
            // arming may come after a neighbour's first bytes: the phase ends when both are complete
            if (lane == 0) tc::mbar_expect_tx(&j.arrived[buf], (uint32_t)(S * 32 * sizeof(mine)));
            const uint32_t to = tc::smem_u32(&j.block[buf][rank][lane]), bar = tc::smem_u32(&j.arrived[buf]);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < S) send(tc::mapa(to, (uint32_t)r), tc::mapa(bar, (uint32_t)r), all);
            // A neighbour sends for slab i + 2 only when it has this block's message for slab i + 1, which this warp sends after it
            // has read slab i's: two buffers are enough.
            tc::wait_arrived(&j.arrived[buf], (slab >> 1) & 1, &j.gave_up, err);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < S) m[r] = j.block[buf][r][lane];
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < S) {
                    if (r == (int)rank) {
#pragma unroll
                        for (int i = 0; i < V; ++i) j.state[lane].h[i] = state[i];
                    }
                    apply<SAFE>(m[r], state);
                }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) before[i] = j.state[lane].h[i];
    apply<SAFE>(j.span[warp][lane], before);
}

// The place of a thread: warp-uniform rows, and 32-bit byte offsets of its channels within a row, so that an access needs no
// 64-bit arithmetic of its own.  Lanes behind the last channel repeat it and store nothing.
template <typename T, typename TH, int V>
struct Place {
    int warp, lane;
    uint32_t rank;
    bool live;
    long long c, end;
    uint32_t at_f, at_h;               // in rows of f / u and of h / dh
    __device__ __forceinline__ Place(const Args &p, int S)
    {
        warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0); lane = threadIdx.x & 31;
        rank = blockIdx.x % S;
        const long long wanted = ((long long)(blockIdx.x / S) * 32 + lane) * V;
        live = wanted < p.C;
        c = live ? wanted : p.C - V;
        const long long b = c / p.D;
        at_f = (uint32_t)((b * p.bs + (c - b * p.D)) * sizeof(T));
        at_h = (uint32_t)(c * sizeof(TH));
        end = end_of(p, b);
    }
};
template <typename R>
__device__ __forceinline__ R load_at(const char *row, uint32_t off) { return load_raw<R>(row + off); }
// how many of the TS steps from t0 on lie before `end`
template <int TS> __device__ __forceinline__ int steps_before(long long t0, long long end)
{
    return t0 >= end ? 0 : end - t0 < TS ? (int)(end - t0) : TS;
}

template <typename T, typename TH, int GATE, int V, int TS>
__global__ void __launch_bounds__(32 * kWarps, 2) recurrence_spans_kernel(const Args p, int S)
{
    using K = Coefficient<T, GATE, V>;
    using F = typename K::F;
    using R = Raw<T, V>;
    __shared__ __align__(16) Joints<F, V> joints;
    joints.init();
    pdl_wait();
    const Place<T, TH, V> me(p, S);
    F state[V];
    load_initial(p.h0, me.c, true, state);
    const long long slab_steps = (long long)S * kWarps * TS;
    const int slabs = (int)((p.T + slab_steps - 1) / slab_steps);
    const long long ldf = p.ld * (long long)sizeof(T), ldh = p.C * (long long)sizeof(TH);
    long long t0 = ((long long)me.rank * kWarps + me.warp) * TS;

    R rf[TS], ru[TS];
    auto request = [&](long long first) {
        const char *f = (const char *)p.f + first * ldf, *u = (const char *)p.u + first * ldf;
        if (first + TS <= p.T) {
#pragma unroll
            for (int s = 0; s < TS; ++s) { rf[s] = load_at<R>(f + s * ldf, me.at_f); ru[s] = load_at<R>(u + s * ldf, me.at_f); }
        } else {
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                rf[s] = R{}; ru[s] = R{};
                if (first + s < p.T) { rf[s] = load_at<R>(f + s * ldf, me.at_f); ru[s] = load_at<R>(u + s * ldf, me.at_f); }
            }
        }
    };
    request(t0);
    for (int slab = 0; slab < slabs; ++slab, t0 += slab_steps) {
        const int n = steps_before<TS>(t0, me.end);
        const bool full = __all_sync(0xffffffffu, n == TS);
        float a[TS][V], x[TS][V];
        Map<F, V> mine = identity<F, V>();
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            float f[V], u[V];
            to_f32(rf[s], f); to_f32(ru[s], u);
            K::of(f, u, a[s], x[s]);
        }
        if (!full) {
#pragma unroll
            for (int s = 0; s < TS; ++s)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (s >= n) { a[s][i] = K::keep(); x[s][i] = 0.0f; }
        }
        if (slab + 1 < slabs) request(t0 + slab_steps);
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            F v[V], b[V];
            K::value(a[s], v);
#pragma unroll
            for (int i = 0; i < V; ++i) b[i] = F(x[s][i]);
            mul(mine.a, v, mine.a);
            muladd(v, mine.h, b, mine.h);
        }
        F h[V];
        join_slab<GATE == RELAY_GATE_GIVEN>(joints, mine, me.warp, me.lane, me.rank, S, slab, p.err, state, h);
        char *out = (char *)p.h + t0 * ldh;
        if (full) {
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                float o[V];
                K::step(a[s], x[s], h);
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = (float)h[i];
                if (me.live) store<TH, V>(out + s * ldh + me.at_h, 0, o);
            }
        } else {
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                float o[V];
                K::step(a[s], x[s], h);
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = s < n ? (float)h[i] : 0.0f;
                if (me.live && t0 + s < p.T) store<TH, V>(out + s * ldh + me.at_h, 0, o);
            }
        }
    }
    if (me.live && me.rank == 0 && me.warp == 0) store_final(p.h_final, me.c, state);
    tc::cluster_sync();                // no block leaves while another may still write to its shared memory
}

template <typename T, typename TH, int GATE, int V, int TS>
__global__ void __launch_bounds__(32 * kWarps, 2) recurrence_grad_spans_kernel(const Args p, int S)
{
    using K = Coefficient<T, GATE, V>;
    using F = typename K::F;
    using R = Raw<T, V>;
    using RH = Raw<TH, V>;
    __shared__ __align__(16) Joints<F, V> joints;
    joints.init();
    pdl_wait();
    const Place<T, TH, V> me(p, S);
    F state[V];
    load_initial(p.dh_final, me.c, true, state);
    const long long slab_steps = (long long)S * kWarps * TS;
    const int slabs = (int)((p.T + slab_steps - 1) / slab_steps);
    const long long ldf = p.ld * (long long)sizeof(T), ldh = p.C * (long long)sizeof(TH);
    long long t0 = p.T - 1 - ((long long)me.rank * kWarps + me.warp) * TS;      // this thread's steps are t0, t0 - 1, ..

    R nf[TS], nu[TS];
    RH nd[TS], nh[TS];
    auto request = [&](long long first) {
        const char *f = (const char *)p.f + first * ldf, *u = (const char *)p.u + first * ldf;
        const char *d = (const char *)p.dh + first * ldh, *h = (const char *)p.h + (first - 1) * ldh;
        if (first >= TS) {             // h is wanted for the step before each
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                nf[s] = load_at<R>(f - s * ldf, me.at_f); nu[s] = load_at<R>(u - s * ldf, me.at_f);
                nd[s] = load_at<RH>(d - s * ldh, me.at_h); nh[s] = load_at<RH>(h - s * ldh, me.at_h);
            }
        } else {
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                nf[s] = R{}; nu[s] = R{}; nd[s] = RH{}; nh[s] = RH{};
                if (first - s >= 0) {
                    nf[s] = load_at<R>(f - s * ldf, me.at_f); nu[s] = load_at<R>(u - s * ldf, me.at_f);
                    nd[s] = load_at<RH>(d - s * ldh, me.at_h);
                    if (first - s > 0) nh[s] = load_at<RH>(h - s * ldh, me.at_h);
                }
            }
        }
    };
    request(t0);
    for (int slab = 0; slab < slabs; ++slab, t0 -= slab_steps) {
        R rf[TS], ru[TS];
        RH rd[TS], rh[TS];
#pragma unroll
        for (int s = 0; s < TS; ++s) { rf[s] = nf[s]; ru[s] = nu[s]; rd[s] = nd[s]; rh[s] = nh[s]; }
        const bool full = __all_sync(0xffffffffu, t0 < me.end && t0 >= TS);     // every step exists, and none is the first
        Map<F, V> mine = identity<F, V>();
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            float f[V], dh[V];
            to_f32(rf[s], f); to_f32(rd[s], dh);
            float k[V];
            F v[V], d[V];
            K::of(f, k);
            K::value(k, v);
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] = F(dh[i]);
            if (full || (t0 - s < me.end && t0 - s >= 0)) {
                mul(mine.a, v, mine.a);
                add(mine.h, d, mine.h);
                mul(mine.h, v, mine.h);
            }
        }
        if (slab + 1 < slabs) request(t0 - slab_steps);
        F G[V];
        join_slab<GATE == RELAY_GATE_GIVEN>(joints, mine, me.warp, me.lane, me.rank, S, slab, p.err, state, G);
        char *df_row = (char *)p.df + t0 * ldf, *du_row = (char *)p.du + t0 * ldf;
#pragma unroll
        for (int s = 0; s < TS; ++s) {
            const long long t = t0 - s;
            float f[V], u[V], dh[V], before[V], df[V], du[V];
            to_f32(rf[s], f); to_f32(ru[s], u); to_f32(rd[s], dh); to_f32(rh[s], before);
            if (!full && t == 0) load_state(p.h0, me.c, before);
            backward_step<K, GATE, V>(f, u, dh, before, full || t < me.end, G, df, du);
            if (me.live && (full || t >= 0)) {
                store<T, V>(df_row - s * ldf + me.at_f, 0, df);
                store<T, V>(du_row - s * ldf + me.at_f, 0, du);
            }
        }
    }
    if (me.live && me.rank == 0 && me.warp == 0) store_final(p.dh0, me.c, state);
    tc::cluster_sync();
}

// ---- the same with tiles fetched ahead and the joining left to a warp of its own --------------------------------
// The cluster's blocks run in step, so per slab each waits for the slowest of its loads and for an exchange of about a
// microsecond.  Where rows are whole 16-byte pieces these waits are taken off the path:
//   - a block's part of a slab (kWarps * TS steps x 64 channels of each operand) is a 2-D tile, asked for by TMA up to a ring's
//     length ahead;
//   - a ninth warp joins: it takes the spans' maps, tells the cluster, collects its blocks' maps and hands the state back, while
//     the other warps already compose the next slab and only then run the current one;
//   - a cluster stays for several tiles of channels, whose slabs follow each other without a gap.
// 16384 x 1 x 4096 in bf16: spans in registers 122 us, tiles with all warps joining 140 (8 steps a thread) and 100 (16), with the
// joining warp and one slab composed ahead 85.  4096 x 13 x D, forward and gradient in bf16: D = 336 in tiles 32 and 60 us, in spans 34 and
// 61; 4096 x 8 x 1024 43 and 86 against 57 and 109.  In fp32 tiles are ahead at few steps (128 x 64 x 1024: 30 and 59 against 39 and 62),
// spans at many (4096 x 8 x 1024: 108 and 232 against 99 and 202); with rows of whole pieces fp32 takes tiles throughout.
constexpr int kTile = 64;              // channels
constexpr int kStages = 3;
constexpr int kTileThreads = 32 * (kWarps + 1);

struct TilePlan {
    int S;                             // blocks per cluster
    int per_row;                       // tiles per batch element
    long long tiles;
    int slabs;                         // of a sequence
};

// Walks a cluster's slabs, tile after tile.  A tile: batch element b, channels d0 .. of its D.
template <typename T>
struct Cursor {
    long long tile;
    int slab;
    bool live;                         // this lane's channels exist
    int x_f, x_h;                      // first column of the tile in rows of f / u and of h / dh
    long long c, end;
    uint32_t at_f;                     // this lane's byte offset in a row of df / du
    __device__ __forceinline__ void place(const Args &p, const TilePlan &q, int lane)
    {
        const long long b = tile / q.per_row, d0 = (tile - b * q.per_row) * kTile, d = d0 + 2 * lane;
        live = d < p.D;
        x_f = (int)(b * p.bs + d0); x_h = (int)(b * p.D + d0);
        c = b * p.D + (live ? d : p.D - 2);
        at_f = (uint32_t)((b * p.bs + d) * sizeof(T));
        end = end_of(p, b);
    }
    __device__ __forceinline__ void start(const Args &p, const TilePlan &q, int lane)
    {
        tile = blockIdx.x / q.S;
        slab = 0;
        if (tile < q.tiles) place(p, q, lane);
    }
    __device__ __forceinline__ bool more(const TilePlan &q) const { return tile < q.tiles; }
    __device__ __forceinline__ void next(const Args &p, const TilePlan &q, int lane)
    {
        if (++slab == q.slabs) {
            slab = 0;
            tile += gridDim.x / q.S;
            if (tile < q.tiles) place(p, q, lane);
        }
    }
};
// counts through a ring of N barriers
template <int N> struct Turn {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() { if (++at == N) { at = 0; phase ^= 1; } }
};

template <typename F, int V>
struct Exchange {                      // everything but the ring twice, alternating between slabs
    Map<F, V> span[2][kWarps][32];     // this block's spans, then what lies ahead of each
    struct { F h[V]; } state[2][32];   // before this block
    Map<F, V> block[2][8][32];         // the cluster's blocks, sent by each
    uint64_t full[kStages];            // a tile is here
    uint64_t handed[2], arrived[2], ready[2];      // all spans are here; all of block[.]; state and span are what a warp needs
    int gave_up;
    __device__ __forceinline__ void init()
    {
        if (threadIdx.x == 0) {
            for (int s = 0; s < kStages; ++s) tc::mbar_init(&full[s], 1);
            for (int b = 0; b < 2; ++b) { tc::mbar_init(&handed[b], kWarps); tc::mbar_init(&arrived[b], 1); tc::mbar_init(&ready[b], 1); }
            gave_up = 0;
            tc::fence_barrier_init();
        }
        tc::cluster_sync();            // every block of the cluster runs, its barriers set up, before anything is sent to it
    }
    __device__ __forceinline__ void wait(uint64_t *bar, uint32_t parity, int *err, int code) { (void)tc::mbar_wait(bar, parity, &gave_up, err, code); }
    // a working warp's side
    __device__ __forceinline__ void hand(Turn<2> &turn, int warp, int lane, const Map<F, V> &m)
    {
        span[turn.at][warp][lane] = m;
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&handed[turn.at]);
        turn.next();
    }
    template <bool SAFE>
    __device__ __forceinline__ void take(Turn<2> &turn, int warp, int lane, int *err, F (&h)[V])
    {
        wait(&ready[turn.at], turn.phase, err, tc::ERR_WAIT_STEP);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = state[turn.at][lane].h[i];
        apply<SAFE>(span[turn.at][warp][lane], h);
        turn.next();
    }
};

// The joining warp over all slabs.  `initial` and `final` are the states before a sequence's first slab and behind its last
// (null: zero, not wanted).  request(cursor, stage) asks for a slab's tiles; a tile may be overwritten once its slab has been
// composed (LAG 0) or run (LAG 2: the map of the slab two later has been handed in).
template <bool SAFE, int LAG, typename T, typename F, int V, typename Request>
__device__ __forceinline__ void join_slabs(Exchange<F, V> &x, const Args &p, const TilePlan &q, int lane, const float *initial, float *final, Request request)
{
    constexpr int HELD = sizeof(F) == 8 ? 2 : 8;           // maps in registers
    const uint32_t rank = blockIdx.x % q.S;
    Cursor<T> ahead, here;
    ahead.start(p, q, lane);
    here = ahead;
    Turn<kStages> ring;
    int asked = 0, done = 0;
    auto ask = [&] {
        if (!ahead.more(q)) return;
        if (lane == 0) request(ahead, ring.at);
        ring.next();
        ahead.next(p, q, lane);
        ++asked;
    };
    for (int s = 0; s < kStages; ++s) ask();
    F state[V];
    Turn<2> turn;
    for (; here.more(q); here.next(p, q, lane), turn.next(), ++done) {
        const int buf = turn.at;
        if (here.slab == 0) load_initial(initial, here.c, true, state);
        // arming may come after a neighbour's first bytes: the phase ends when both are complete
        if (q.S > 1 && lane == 0) tc::mbar_expect_tx(&x.arrived[buf], (uint32_t)(q.S * 32 * sizeof(Map<F, V>)));
        x.wait(&x.handed[buf], turn.phase, p.err, tc::ERR_WAIT_STEP);
        if (done >= LAG) ask();
        Map<F, V> m[HELD], all = identity<F, V>();                    // loads in flight together
#pragma unroll
        for (int w0 = 0; w0 < kWarps; w0 += HELD) {
#pragma unroll
            for (int w = 0; w < HELD; ++w) m[w] = x.span[buf][w0 + w][lane];
#pragma unroll
            for (int w = 0; w < HELD; ++w) all = then(all, m[w]);
        }
        if (q.S > 1) {
            const uint32_t to = tc::smem_u32(&x.block[buf][rank][lane]), bar = tc::smem_u32(&x.arrived[buf]);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < q.S) send(tc::mapa(to, (uint32_t)r), tc::mapa(bar, (uint32_t)r), all);
        }
        Map<F, V> before = identity<F, V>();                          // while the exchange is under way
#pragma unroll
        for (int w0 = 0; w0 < kWarps; w0 += HELD) {
#pragma unroll
            for (int w = 0; w < HELD; ++w) m[w] = x.span[buf][w0 + w][lane];
#pragma unroll
            for (int w = 0; w < HELD; ++w) {
                x.span[buf][w0 + w][lane] = before;
                before = then(before, m[w]);
            }
        }
        if (q.S > 1) {
            // A neighbour sends for slab i + 2 only when it has this block's message for slab i + 1, which this warp sends after
            // it has read slab i's: two buffers are enough.
            tc::wait_arrived(&x.arrived[buf], turn.phase, &x.gave_up, p.err);
#pragma unroll
            for (int r0 = 0; r0 < 8; r0 += HELD) {
#pragma unroll
                for (int r = 0; r < HELD; ++r)
                    if (r0 + r < q.S) m[r] = x.block[buf][r0 + r][lane];
#pragma unroll
                for (int r = 0; r < HELD; ++r)
                    if (r0 + r < q.S) {
                        if (r0 + r == (int)rank) {
#pragma unroll
                            for (int i = 0; i < V; ++i) x.state[buf][lane].h[i] = state[i];
                        }
                        apply<SAFE>(m[r], state);
                    }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x.state[buf][lane].h[i] = state[i];
            apply<SAFE>(all, state);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&x.ready[buf]);
        if (here.slab + 1 == q.slabs && here.live && rank == 0) store_final(final, here.c, state);
    }
    // a block that gave up still lets the tiles land that it asked for
    if (*(volatile int *)&x.gave_up && lane == 0)
        for (int s = max(0, asked - kStages); s < asked; ++s)
            for (int i = 0; i < 1000000 && !tc::mbar_try_wait(&x.full[s % kStages], (s / kStages) & 1); ++i) {}
    __syncwarp();
}

// Steps a thread takes of a slab, a block's ring of tiles in bytes, and how many blocks an SM's 228 KB hold (1 KB of each is the
// system's): 96 KB and 17 KB of maps in bf16, 48 and 34 in fp32, two of them; 96 and 34 for the fp32 gradient, one.
template <typename T, typename TH, bool GRAD> struct TileShape {
    using F = std::conditional_t<sizeof(T) == 4, double, float>;
    static constexpr int TS = (GRAD ? sizeof(T) + sizeof(TH) == 4 : sizeof(T) == 2) ? 8 : 4;
    static constexpr int ROWS = kWarps * TS;
    static constexpr size_t RING = (size_t)kStages * ROWS * kTile * 2 * (sizeof(T) + (GRAD ? sizeof(TH) : 0));
    static constexpr size_t BYTES = RING + sizeof(Exchange<F, 2>) + 128 + 1024;
    static constexpr int BLOCKS = 2 * BYTES <= 228 * 1024 ? 2 : 1;
};

template <typename T, typename TH, int GATE>
__global__ void __launch_bounds__(kTileThreads, (TileShape<T, TH, false>::BLOCKS))
recurrence_tiles_kernel(const __grid_constant__ CUtensorMap tm_f, const __grid_constant__ CUtensorMap tm_u, const Args p, const TilePlan q)
{
    using Shape = TileShape<T, TH, false>;
    constexpr int V = 2, TS = Shape::TS, ROWS = Shape::ROWS, TILE = ROWS * kTile * (int)sizeof(T);
    constexpr bool SAFE = GATE == RELAY_GATE_GIVEN;
    using K = Coefficient<T, GATE, V>;
    using F = typename K::F;
    using R = Raw<T, V>;
    extern __shared__ __align__(128) uint8_t tiles[];                // [kStages][f, u][ROWS][kTile]
    __shared__ __align__(16) Exchange<F, V> ex;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x % q.S;
    const long long slab_steps = (long long)q.S * ROWS;
    ex.init();
    pdl_wait();
    if (warp == kWarps) {
        join_slabs<SAFE, 0, T>(ex, p, q, lane, p.h0, p.h_final, [&](const Cursor<T> &at, int stage) {
            const int row = (int)(at.slab * slab_steps) + rank * ROWS;
            uint8_t *to = tiles + stage * 2 * TILE;
            tc::mbar_expect_tx(&ex.full[stage], 2 * TILE);
            tc::tma_load_2d(to, &tm_f, &ex.full[stage], at.x_f, row);
            tc::tma_load_2d(to + TILE, &tm_u, &ex.full[stage], at.x_f, row);
        });
    } else {
        const long long ldh = p.C * (long long)sizeof(TH);
        const int first = (rank * kWarps + warp) * TS;
        Cursor<T> composing, running;
        composing.start(p, q, lane);
        running = composing;
        Turn<kStages> ring;
        Turn<2> handing, taking;
        auto compose = [&](float (&a)[TS][V], float (&x)[TS][V]) {
            if (!composing.more(q)) return;
            ex.wait(&ex.full[ring.at], ring.phase, p.err, tc::ERR_WAIT_FULL);
            const R *f = reinterpret_cast<const R *>(tiles + ring.at * 2 * TILE) + warp * TS * (kTile / V) + lane;
            const R *u = f + TILE / (int)sizeof(R);
            ring.next();
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                float fv[V], uv[V];
                to_f32(f[s * (kTile / V)], fv); to_f32(u[s * (kTile / V)], uv);
                K::of(fv, uv, a[s], x[s]);
            }
            const int n = steps_before<TS>(first + composing.slab * slab_steps, composing.end);
            if (!__all_sync(0xffffffffu, n == TS)) {
#pragma unroll
                for (int s = 0; s < TS; ++s)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (s >= n) { a[s][i] = K::keep(); x[s][i] = 0.0f; }
            }
            Map<F, V> mine = identity<F, V>();
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                F v[V], b[V];
                K::value(a[s], v);
#pragma unroll
                for (int i = 0; i < V; ++i) b[i] = F(x[s][i]);
                mul(mine.a, v, mine.a);
                muladd(v, mine.h, b, mine.h);
            }
            ex.hand(handing, warp, lane, mine);
            composing.next(p, q, lane);
        };
        auto run = [&](const float (&a)[TS][V], const float (&x)[TS][V]) {
            if (!running.more(q)) return;
            F h[V];
            ex.template take<SAFE>(taking, warp, lane, p.err, h);
            const long long t0 = first + running.slab * slab_steps;
            const int n = steps_before<TS>(t0, running.end);
            char *out = (char *)p.h + t0 * ldh + running.c * (long long)sizeof(TH);
            if (__all_sync(0xffffffffu, n == TS)) {
#pragma unroll
                for (int s = 0; s < TS; ++s) {
                    float o[V];
                    K::step(a[s], x[s], h);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] = (float)h[i];
                    if (running.live) store<TH, V>(out, 0, o);
                    out += ldh;
                }
            } else {
#pragma unroll
                for (int s = 0; s < TS; ++s) {
                    float o[V];
                    K::step(a[s], x[s], h);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] = s < n ? (float)h[i] : 0.0f;
                    if (running.live && t0 + s < p.T) store<TH, V>(out, 0, o);
                    out += ldh;
                }
            }
            running.next(p, q, lane);
        };
        float a0[TS][V], x0[TS][V], a1[TS][V], x1[TS][V];
        compose(a0, x0);
        while (running.more(q)) {
            compose(a1, x1);
            run(a0, x0);
            compose(a0, x0);
            run(a1, x1);
        }
    }
    tc::cluster_sync();                // no block leaves while another may still send to it
}

template <typename T, typename TH, int GATE>
__global__ void __launch_bounds__(kTileThreads, (TileShape<T, TH, true>::BLOCKS))
recurrence_grad_tiles_kernel(const __grid_constant__ CUtensorMap tm_f, const __grid_constant__ CUtensorMap tm_u, const __grid_constant__ CUtensorMap tm_d,
                             const __grid_constant__ CUtensorMap tm_h, const Args p, const TilePlan q)
{
    using Shape = TileShape<T, TH, true>;
    constexpr int V = 2, TS = Shape::TS, ROWS = Shape::ROWS, TILE = ROWS * kTile * (int)sizeof(T), TILE_H = ROWS * kTile * (int)sizeof(TH), STAGE = 2 * (TILE + TILE_H);
    constexpr bool SAFE = GATE == RELAY_GATE_GIVEN;
    using K = Coefficient<T, GATE, V>;
    using F = typename K::F;
    using R = Raw<T, V>;
    using RH = Raw<TH, V>;
    extern __shared__ __align__(128) uint8_t tiles[];                // [kStages][f, u, dh, h one step earlier][ROWS][kTile]
    __shared__ __align__(16) Exchange<F, V> ex;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x % q.S;
    const long long slab_steps = (long long)q.S * ROWS;
    ex.init();
    pdl_wait();
    if (warp == kWarps) {
        join_slabs<SAFE, 2, T>(ex, p, q, lane, p.dh_final, p.dh0, [&](const Cursor<T> &at, int stage) {
            uint8_t *to = tiles + stage * STAGE;
            const int row = (int)(p.T - (at.slab * slab_steps + (long long)(rank + 1) * ROWS));     // rows in front of the first read as zero
            tc::mbar_expect_tx(&ex.full[stage], STAGE);
            tc::tma_load_2d(to, &tm_f, &ex.full[stage], at.x_f, row);
            tc::tma_load_2d(to + TILE, &tm_u, &ex.full[stage], at.x_f, row);
            tc::tma_load_2d(to + 2 * TILE, &tm_d, &ex.full[stage], at.x_h, row);
            tc::tma_load_2d(to + 2 * TILE + TILE_H, &tm_h, &ex.full[stage], at.x_h, row - 1);
        });
    } else {
        const long long ldf = p.ld * (long long)sizeof(T);
        const long long first = p.T - 1 - (long long)(rank * kWarps + warp) * TS;             // the steps of slab i are this - i slab_steps and before
        const int last = (ROWS - 1 - warp * TS) * (kTile / V) + lane;                         // the first of them in the tile
        Cursor<T> composing, running;
        composing.start(p, q, lane);
        running = composing;
        Turn<kStages> ring, ring_run;
        Turn<2> handing, taking;
        auto compose = [&] {
            if (!composing.more(q)) return;
            ex.wait(&ex.full[ring.at], ring.phase, p.err, tc::ERR_WAIT_FULL);
            const long long t0 = first - composing.slab * slab_steps;
            const bool all_on = __all_sync(0xffffffffu, t0 < composing.end && t0 >= TS);
            const R *f = reinterpret_cast<const R *>(tiles + ring.at * STAGE) + last;
            const RH *d = reinterpret_cast<const RH *>(tiles + ring.at * STAGE + 2 * TILE) + last;
            ring.next();
            Map<F, V> mine = identity<F, V>();
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                float fv[V], dh[V], k[V];
                F v[V], dv[V];
                to_f32(f[-s * (kTile / V)], fv); to_f32(d[-s * (kTile / V)], dh);
                K::of(fv, k);
                K::value(k, v);
#pragma unroll
                for (int i = 0; i < V; ++i) dv[i] = F(dh[i]);
                if (all_on || (t0 - s < composing.end && t0 - s >= 0)) {
                    mul(mine.a, v, mine.a);
                    add(mine.h, dv, mine.h);
                    mul(mine.h, v, mine.h);
                }
            }
            ex.hand(handing, warp, lane, mine);
            composing.next(p, q, lane);
        };
        compose();
        while (running.more(q)) {
            compose();
            F G[V];
            ex.template take<SAFE>(taking, warp, lane, p.err, G);
            const long long t0 = first - running.slab * slab_steps;
            const bool all_on = __all_sync(0xffffffffu, t0 < running.end && t0 >= TS);        // and none is the first step
            const uint8_t *at = tiles + ring_run.at * STAGE;
            ring_run.next();
            const R *f = reinterpret_cast<const R *>(at) + last, *u = reinterpret_cast<const R *>(at + TILE) + last;
            const RH *d = reinterpret_cast<const RH *>(at + 2 * TILE) + last, *hb = reinterpret_cast<const RH *>(at + 2 * TILE + TILE_H) + last;
            char *df_at = (char *)p.df + t0 * ldf + running.at_f, *du_at = (char *)p.du + t0 * ldf + running.at_f;
#pragma unroll
            for (int s = 0; s < TS; ++s) {
                const long long t = t0 - s;
                float fv[V], uv[V], dh[V], before[V], df[V], du[V];
                to_f32(f[-s * (kTile / V)], fv); to_f32(u[-s * (kTile / V)], uv);
                to_f32(d[-s * (kTile / V)], dh); to_f32(hb[-s * (kTile / V)], before);
                if (!all_on && t == 0) load_state(p.h0, running.c, before);
                backward_step<K, GATE, V>(fv, uv, dh, before, all_on || t < running.end, G, df, du);
                if (running.live && (all_on || t >= 0)) {
                    store<T, V>(df_at, 0, df);
                    store<T, V>(du_at, 0, du);
                }
                df_at -= ldf; du_at -= ldf;
            }
            running.next(p, q, lane);
        }
    }
    tc::cluster_sync();
}

// Clusters of S blocks of a kernel that are resident at once on the present device; asked for once per size.
template <typename Kernel>
int resident_clusters(Kernel kernel, std::atomic<int> (&known)[64][9], int dev, int S, size_t smem)
{
    if (dev < 0 || dev >= 64) return 1;
    int n = known[dev][S].load(std::memory_order_relaxed);
    if (n > 0) return n;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)S); cfg.blockDim = dim3(kTileThreads); cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)S; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
    n = std::max(n, 1);
    known[dev][S].store(n, std::memory_order_relaxed);
    return n;
}

template <typename T, typename TH, int GATE>
relay_status_t launch_tiles(const Args &p, bool grad, cudaStream_t st)
{
    using Forward = TileShape<T, TH, false>;
    using Gradient = TileShape<T, TH, true>;
    int dev = 0;
    RELAY_CUDA(cudaGetDevice(&dev));
    const int rows = grad ? Gradient::ROWS : Forward::ROWS;
    TilePlan q;
    q.per_row = (int)((p.D + kTile - 1) / kTile);
    q.tiles = (p.C / p.D) * q.per_row;
    const size_t smem = grad ? Gradient::RING : Forward::RING;
    static std::atomic<int> known[2][64][9];
    if (grad) RELAY_CUDA(cudaFuncSetAttribute(recurrence_grad_tiles_kernel<T, TH, GATE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    else RELAY_CUDA(cudaFuncSetAttribute(recurrence_tiles_kernel<T, TH, GATE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    // Blocks per tile: the fewest rounds over the clusters that are resident at once, each of a tile's slabs and one more for its first,
    // which nothing hides; from three blocks on the exchange costs 2 % a block.  Two blocks also where they are 2 % behind one: at 128
    // tiles on 148 SMs they keep all of them busy in the first of two rounds (fp32 gradient of 4096 x 8 x 1024: 232 us against 247; 128 x
    // 64 x 1024 in bf16, 14 % behind: 16.4 against 15.4).
    long long clusters = 1;
    double best = 0;
    q.S = 1;
    for (int S = 1; S <= 8 && (S == 1 || (long long)(S - 1) * rows < p.T); ++S) {
        const long long room = grad ? resident_clusters(recurrence_grad_tiles_kernel<T, TH, GATE>, known[1], dev, S, smem)
                                    : resident_clusters(recurrence_tiles_kernel<T, TH, GATE>, known[0], dev, S, smem);
        const long long rounds = (q.tiles + room - 1) / room, slabs = (p.T + (long long)S * rows - 1) / ((long long)S * rows);
        const double cost = (double)rounds * (double)(slabs + 1) * (S > 2 ? 1.0 + 0.02 * S : 1.0);
        if (S == 1 || cost < best * (S == 2 ? 1.02 : 1.0)) { best = cost; q.S = S; clusters = std::min(room, q.tiles); }
    }
    q.slabs = (int)((p.T + (long long)q.S * rows - 1) / ((long long)q.S * rows));
    const dim3 grid((unsigned)(clusters * q.S)), block(kTileThreads), cluster((unsigned)q.S);
    const bool t32 = sizeof(T) == 4, h32 = sizeof(TH) == 4;
    CUtensorMap f, u, d, h;
    const uint64_t ld = (uint64_t)p.ld;
    // packed: the map of u starts D columns into the rows, the last D columns of f's belong to nobody's u
    RELAY_TRY(make_tmap_2d(&f, t32, p.f, ld, p.T, ld, kTile, rows, false));
    RELAY_TRY(make_tmap_2d(&u, t32, p.u, ld - (p.bs == 2 * p.D ? p.D : 0), p.T, ld, kTile, rows, false));
    if (!grad) {
        RELAY_CUDA(launch_pdl_cluster(recurrence_tiles_kernel<T, TH, GATE>, grid, block, cluster, smem, st, f, u, p, q));
    } else {
        RELAY_TRY(make_tmap_2d(&d, h32, p.dh, p.C, p.T, p.C, kTile, rows, false));
        RELAY_TRY(make_tmap_2d(&h, h32, p.h, p.C, p.T, p.C, kTile, rows, false));
        RELAY_CUDA(launch_pdl_cluster(recurrence_grad_tiles_kernel<T, TH, GATE>, grid, block, cluster, smem, st, f, u, d, h, p, q));
    }
    return check_launch("gated_recurrence");
}

// Which form takes a call.  Sequences of up to kSteps steps run step by step, in the spans kernels' place; of up to kTileSteps, in the
// tile kernels' place.
// 64 x 1024 channels in bf16, forward: 12 steps 13.3 us and in tiles 14.3, 16 steps 15.4 and 14.3, 32 steps 23.6 and 14.3; gradient in
// fp32: 16 steps 21.5 and 24.6, 24 steps 27.7 and 26.6; 8 x 256 channels, forward: 8 steps 9.3 and 8.2, 32 steps 21.5 and 8.2.
// Longer sequences in spans: the smallest cluster that gives every SM a block.
// Tiles and spans keep byte offsets within a step's row of f and u in 32 bits (spans those of h too): wider rows, of which only few
// steps fit the GPU's memory, run step by step.
constexpr long long kSteps = 32, kTileSteps = 12;
enum Form { STEPS, SPANS, TILES };
Form form_of(const Args &p, long long of_t, long long of_h)
{
    const long long piece = 16 / of_t;
    if (p.ld * of_t >= (1ll << 32)) return STEPS;
    if (p.T > kTileSteps && p.D % piece == 0 && p.bs % piece == 0 && p.C < (1ll << 31) && p.T < (1ll << 30)) return TILES;
    return p.T > kSteps && p.C * of_h < (1ll << 32) ? SPANS : STEPS;
}

// V channels a lane.  Two, where rows allow it: bf16, and the fp32 forward call where all steps of a lane's channels are one slab or two;
// not where there are too few channels to give every SM a block then.  The steps a lane keeps in registers are as many as fit without
// spilling to memory (a few words in the fp32 instances).  4096 steps of 13 x 334 channels, one and two a lane: bf16 forward 39.7 and 34.0
// us, gradient 79.6 and 62.0; fp32 60.8 and 89, gradient 116 and 157.  64 steps of 64 x 1022: bf16 27.9 and 17.3, fp32 29.5 and 24.9, its
// gradient 40.4 and 36.8.  16384 x 1 x 66 in bf16: 32 and 59.
constexpr long long kShortSpans = 64;
template <typename T, typename TH, int GATE, int V>
relay_status_t launch_spans(const Args &p, bool grad, int sms, cudaStream_t st)
{
    constexpr int TS = (sizeof(T) == 2 ? 16 : 8) / V, TSG = sizeof(T) + sizeof(TH) == 4 ? 8 / V : 4;
    const long long tiles = (p.C + 32 * V - 1) / (32 * V), steps = kWarps * (grad ? TSG : TS);
    int S = 1;
    while (S < 8 && tiles * S < sms && p.T > S * steps) S *= 2;
    if (tiles * S > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "gated_recurrence: %lld channels", p.C);
    const dim3 grid((unsigned)(tiles * S)), block(32 * kWarps), cluster((unsigned)S);
    if constexpr (sizeof(T) == 2 || V == 1) {
        if (grad) {
            RELAY_CUDA(launch_pdl_cluster(recurrence_grad_spans_kernel<T, TH, GATE, V, TSG>, grid, block, cluster, 0, st, p, S));
            return check_launch("gated_recurrence");
        }
    }
    RELAY_CUDA(launch_pdl_cluster(recurrence_spans_kernel<T, TH, GATE, V, TS>, grid, block, cluster, 0, st, p, S));
    return check_launch("gated_recurrence");
}
template <typename T, typename TH, int GATE, int V>
relay_status_t launch_steps(const Args &p, bool grad, cudaStream_t st)
{
    const long long blocks = (p.C / V + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "gated_recurrence: %lld channels", p.C);
    const dim3 grid((unsigned)blocks);
    if (grad) RELAY_CUDA(launch_pdl(recurrence_grad_steps_kernel<T, TH, GATE, V>, grid, dim3(kThreads), 0, st, p));
    else RELAY_CUDA(launch_pdl(recurrence_steps_kernel<T, TH, GATE, V>, grid, dim3(kThreads), 0, st, p));
    return check_launch("gated_recurrence");
}
template <typename T, typename TH, int GATE>
relay_status_t launch_gate(const Args &p, bool grad, cudaStream_t st)
{
    if (!p.err) return fail(RELAY_ERR_CUDA, "no device error word");
    const Form form = form_of(p, sizeof(T), sizeof(TH));
    if (form == TILES) return launch_tiles<T, TH, GATE>(p, grad, st);
    // two channels a thread where every row starts at a multiple of them, so that they are one aligned access
    const bool even = (p.D | p.ld | p.bs) % 2 == 0;
    if (form == STEPS) return even ? launch_steps<T, TH, GATE, 2>(p, grad, st) : launch_steps<T, TH, GATE, 1>(p, grad, st);
    int dev = 0, sms = 148;
    RELAY_CUDA(cudaGetDevice(&dev));
    RELAY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    const bool two = even && (p.C + 63) / 64 * 8 >= sms && (sizeof(T) == 2 || (!grad && p.T <= kShortSpans));
    return two ? launch_spans<T, TH, GATE, 2>(p, grad, sms, st) : launch_spans<T, TH, GATE, 1>(p, grad, sms, st);
}
template <typename T, typename TH>
relay_status_t launch_typed(const Args &p, int32_t gate, bool grad, cudaStream_t st)
{
    switch (gate) {
    case RELAY_GATE_GIVEN: return launch_gate<T, TH, RELAY_GATE_GIVEN>(p, grad, st);
    case RELAY_GATE_SIGMOID: return launch_gate<T, TH, RELAY_GATE_SIGMOID>(p, grad, st);
    default: return launch_gate<T, TH, RELAY_GATE_MIX>(p, grad, st);
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

Args sizes_of(const Sizes &s, bool ragged)
{
    Args p{};
    p.T = s.T; p.C = s.B * s.D; p.D = s.D;
    p.bs = s.packed ? 2 * s.D : s.D;
    p.ld = s.B * p.bs;
    if (!s.packed && !ragged) p.D = p.bs = p.C;    // nothing depends on the batch element: one row of channels
    return p;
}
Args make_args(const relay_tensor_t *f, const relay_tensor_t *u, const relay_tensor_t *h0, const relay_tensor_t *lengths, const Sizes &s)
{
    Args p = sizes_of(s, lengths != nullptr);
    p.f = f->data;
    p.u = s.packed ? (const char *)f->data + s.D * dtype_size(f->dtype) : u->data;
    p.h0 = h0 ? (const float *)h0->data : nullptr;
    p.lengths = lengths ? (const int *)lengths->data : nullptr;
    p.err = device_error_word();
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

// Which form the call takes: 0 step by step, 1 spans in registers, 2 tiles; -1 where the types or shapes are refused.  Host only.
extern "C" int32_t relay_debug_recurrence_form(const relay_tensor_t *f, const relay_tensor_t *u, const relay_tensor_t *h_all, int32_t ragged)
{
    clear_error();
    Sizes s;
    if (!f || !h_all || check_inputs(f, u, &s) != RELAY_OK || check_sequence(h_all, f->dtype, RELAY_F32, s, s.D, "h_all") != RELAY_OK) return -1;
    if (s.B == 0 || s.D == 0) return STEPS;
    return form_of(sizes_of(s, ragged != 0), (long long)dtype_size(f->dtype), (long long)dtype_size(h_all->dtype));
}
