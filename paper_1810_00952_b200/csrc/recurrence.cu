// Gated linear recurrence over a sequence, h_t = a_t h_{t-1} + b_t per channel, and its gradient group (Section 4.2 of the
// paper: reverse mode through the recursion over time).  Elementwise steps: HBM-bound where the channels fill the GPU.
#include <algorithm>

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
__device__ __forceinline__ void sigmoid_pair(float f, float &a, float &one_less)
{
    const float e = __expf(-fabsf(f));
    const float small = __fdividef(e, 1.0f + e), large = 1.0f - small;
    a = f >= 0.0f ? large : small;
    one_less = f >= 0.0f ? small : large;
    if (f != f) a = one_less = f;
}
template <int GATE>
__device__ __forceinline__ void coefficients(float f, float u, float &a, float &b)
{
    if (GATE == RELAY_GATE_GIVEN) {
        a = f;
        b = u;
    } else {
        float s;
        sigmoid_pair(f, a, s);
        b = GATE == RELAY_GATE_MIX ? s * u : u;
    }
}
// partials of one step: g = dh_t + G_{t+1}
template <int GATE>
__device__ __forceinline__ void partials(float f, float u, float before, float g, float &df, float &du)
{
    if (GATE == RELAY_GATE_GIVEN) {
        df = g * before;
        du = g;
    } else {
        float a, s;
        sigmoid_pair(f, a, s);
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

// ---- one thread per V channels, step by step ------------------------------------------------------------
template <typename T, typename TH, int GATE, int V>
__global__ void __launch_bounds__(kThreads) recurrence_steps_kernel(const Args p)
{
    const long long c = ((long long)blockIdx.x * kThreads + threadIdx.x) * V;
    pdl_wait();
    if (c >= p.C) return;
    const long long b = c / p.D, at = b * p.bs + (c - b * p.D), end = end_of(p, b);
    float h[V];
    load_state(p.h0, c, h);
#pragma unroll 8
    for (long long t = 0; t < p.T; ++t) {
        float f[V], u[V], out[V];
        load<T, V>(p.f, t * p.ld + at, f);
        load<T, V>(p.u, t * p.ld + at, u);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float a, x;
            coefficients<GATE>(f[i], u[i], a, x);
            const float next = fmaf(a, h[i], x);
            if (t < end) h[i] = next;
            out[i] = t < end ? next : 0.0f;
        }
        store<TH, V>(p.h, t * p.C + c, out);
    }
    store_state(p.h_final, c, h);
}

template <typename T, typename TH, int GATE, int V>
__global__ void __launch_bounds__(kThreads) recurrence_grad_steps_kernel(const Args p)
{
    const long long c = ((long long)blockIdx.x * kThreads + threadIdx.x) * V;
    pdl_wait();
    if (c >= p.C) return;
    const long long b = c / p.D, at = b * p.bs + (c - b * p.D), end = end_of(p, b);
    float G[V];
    load_state(p.dh_final, c, G);
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
            const float g = dh[i] + G[i];
            float a, x;
            coefficients<GATE>(f[i], u[i], a, x);
            partials<GATE>(f[i], u[i], before[i], g, df[i], du[i]);
            if (t < end) G[i] = a * g;
            else df[i] = du[i] = 0.0f;
        }
        store<T, V>(p.df, t * p.ld + at, df);
        store<T, V>(p.du, t * p.ld + at, du);
    }
    store_state(p.dh0, c, G);
}

template <typename T, typename TH, int GATE, int V>
relay_status_t launch(const Args &p, bool grad, cudaStream_t st)
{
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
