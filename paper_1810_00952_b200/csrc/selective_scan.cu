// Selective scan: h = exp(delta a) h + delta u b per channel and state, y = sum_n c h + d u, with an optional gate silu(z).
#include <algorithm>

#include "selective_scan.cuh"

namespace relay {
namespace {

using namespace scan;

// ---- few steps: four lanes a channel, the states in registers from step to step ----------------------------------------
constexpr int kStepThreads = 128;

template <typename T, int NB>
__global__ void __launch_bounds__(kStepThreads) selective_scan_steps_kernel(const Args p)
{
    pdl_wait();
    const long long at = ((long long)blockIdx.x * kStepThreads + threadIdx.x) >> 2;      // b * D + d
    const int nl = threadIdx.x & 3;
    const bool live = at < p.B * p.D;                                                    // the lanes of a warp stay together
    const long long i = live ? at / p.D : 0, d = live ? at - i * p.D : 0;
    const long long end = live ? end_of(p, i) : 0;
    float h[NB][4], a[NB][4];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        load_states(p, live ? p.h0 : nullptr, at * p.N, k * 16 + nl * 4, h[k]);
        load_states(p, live ? p.a : nullptr, d * p.N, k * 16 + nl * 4, a[k]);
    }
    const float skip = p.d && live && relay_in_bounds(p.d + d, 4) ? p.d[d] : 0.0f;
    const float bias = p.delta_bias && live && relay_in_bounds(p.delta_bias + d, 4) ? p.delta_bias[d] : 0.0f;
    for (long long t = 0; t < p.T; ++t) {
        const long long row = (t * p.B + i) * p.D;
        float y = 0.0f, u = 0.0f;
        if (live && p.states && t % kSpan == 0) {
#pragma unroll
            for (int k = 0; k < NB; ++k) store_states(p, p.states, ((t / kSpan) * p.B * p.D + at) * p.N, k * 16 + nl * 4, h[k]);
        }
        if (t < end) {
            u = load_weight<T>(p.u, row + d);
            float step = load_weight<T>(p.delta, row + d) + bias, slope;
            if (p.softplus) step = softplus_(step, slope);
            const long long bc = (t * p.B + i) * p.ld_bc;
#pragma unroll
            for (int k = 0; k < NB; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = k * 16 + nl * 4 + j;
                    if (n >= p.N) continue;
                    h[k][j] = fmaf(exp2_(step * a[k][j] * kLog2e), h[k][j], step * u * load_weight<T>(p.b, bc + n));
                    y = fmaf(load_weight<T>(p.c, bc + n), h[k][j], y);
                }
        }
        y += __shfl_xor_sync(0xffffffffu, y, 1);
        y += __shfl_xor_sync(0xffffffffu, y, 2);
        if (live && nl == 0) {
            float out[1] = {0.0f};
            if (t < end) {
                out[0] = fmaf(skip, u, y);
                if (p.z) {
                    const float z = load_weight<T>(p.z, row + d);
                    out[0] *= z * logistic<sizeof(T) == 4>(z);
                }
            }
            store<T, 1>(p.y, row + d, out);
        }
    }
    if (!live) return;
#pragma unroll
    for (int k = 0; k < NB; ++k) store_states(p, p.h_final, at * p.N, k * 16 + nl * 4, h[k]);
}

// ---- chunks -----------------------------------------------------------------------------------------------------------
// A block: WC warps of eight channels side by side, WT rows of them, each with a run of RUN steps of the chunk.
constexpr int RUN = 8;

template <int WT, int WC, int NB>
struct Tile {
    static constexpr int THREADS = 32 * WT * WC, CHANNELS = 8 * WC, STEPS = RUN * WT, NP = 16 * NB;
    float2 step[STEPS][CHANNELS];          // delta, delta u
    float b[STEPS][NP], c[STEPS][NP];
    float y[STEPS][CHANNELS];
    float4 decay[2][WT][WC][32], sum[2][WT][WC][32];
};

template <typename T, int WT, int WC, int NB>
__global__ void __launch_bounds__(32 * WT * WC, NB == 1 ? 2 : 1) selective_scan_kernel(const Args p)
{
    using S = Tile<WT, WC, NB>;
    constexpr bool FINE = sizeof(T) == 4;
    constexpr int WEIGHTS = S::STEPS * S::NP / S::THREADS;                 // values of b (and of c) that a thread fetches per chunk
    extern __shared__ uint4 shared_raw[];
    S &s = *reinterpret_cast<S *>(shared_raw);
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wt = warp / WC, wc = warp % WC, nl = lane & 3, cl = lane >> 2;
    const long long i = blockIdx.x / p.groups;
    const long long c0 = (blockIdx.x - i * p.groups) * S::CHANNELS;
    const long long end = end_of(p, i);
    // this thread's states: of channel mine
    const int ch = wc * 8 + cl;
    const long long mine = c0 + ch;
    const bool live = mine < p.D;
    f32x2 a[NB][2], h[NB][2];                                              // a log2(e); the state at the chunk's start
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        float x[4];
        load_states(p, live ? p.a : nullptr, mine * p.N, k * 16 + nl * 4, x);
        a[k][0] = pair(x[0] * kLog2e, x[1] * kLog2e);
        a[k][1] = pair(x[2] * kLog2e, x[3] * kLog2e);
        load_states(p, live ? p.h0 : nullptr, (i * p.D + mine) * p.N, k * 16 + nl * 4, x);
        h[k][0] = pair(x[0], x[1]);
        h[k][1] = pair(x[2], x[3]);
    }
    // this thread's pair of channels and step of the chunk in what surrounds the scan
    const int pt = tid / (S::CHANNELS / 2), pc = 2 * (tid % (S::CHANNELS / 2));
    const long long two = c0 + pc;
    float skip[2] = {0.0f, 0.0f}, bias[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 2; ++j)
        if (two + j < p.D) {
            if (p.d && relay_in_bounds(p.d + two + j, 4)) skip[j] = p.d[two + j];
            if (p.delta_bias && relay_in_bounds(p.delta_bias + two + j, 4)) bias[j] = p.delta_bias[two + j];
        }
    float u[2], raw[2], z[2], wb[WEIGHTS], wc_[WEIGHTS];
    auto fetch = [&](long long t0) {
        const long long t = t0 + pt;
#pragma unroll
        for (int j = 0; j < 2; ++j) u[j] = raw[j] = z[j] = 0.0f;
        if (t < end && two < p.D) {
            const long long row = (t * p.B + i) * p.D;
            load_channels<T>(p, p.u, row, two, u);
            load_channels<T>(p, p.delta, row, two, raw);
            if (p.z) load_channels<T>(p, p.z, row, two, z);
        }
#pragma unroll
        for (int k = 0; k < WEIGHTS; ++k) {
            const int e = tid + k * S::THREADS, tt = e / S::NP, n = e % S::NP;
            wb[k] = wc_[k] = 0.0f;
            if (t0 + tt < end && n < p.N) {
                const long long at = ((t0 + tt) * p.B + i) * p.ld_bc + n;
                wb[k] = load_weight<T>(p.b, at);
                wc_[k] = load_weight<T>(p.c, at);
            }
        }
    };
    fetch(0);
    for (long long t0 = 0; t0 < p.T; t0 += S::STEPS) {
        const bool inside = t0 + pt < end;
        float un[2], zn[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float step = raw[j] + bias[j], slope;
            if (p.softplus) step = softplus_(step, slope);
            if (!inside || two + j >= p.D) step = 0.0f;                    // nothing decays and nothing is added
            s.step[pt][pc + j] = make_float2(step, step * u[j]);
            un[j] = u[j];
            zn[j] = z[j];
        }
#pragma unroll
        for (int k = 0; k < WEIGHTS; ++k) {
            const int e = tid + k * S::THREADS;
            (&s.b[0][0])[e] = wb[k];
            (&s.c[0][0])[e] = wc_[k];
        }
        __syncthreads();
        if (t0 + S::STEPS < p.T) fetch(t0 + S::STEPS);
        float y[RUN];
#pragma unroll
        for (int r = 0; r < RUN; ++r) y[r] = 0.0f;
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            f32x2 da[RUN][2], x[RUN][2], P[2], H[2];                       // decays; what is added, then the states
            P[0] = P[1] = pair(1.0f, 1.0f);
            H[0] = H[1] = pair(0.0f, 0.0f);
#pragma unroll
            for (int r = 0; r < RUN; ++r) {
                const float2 st = s.step[wt * RUN + r][ch];
                const float4 b = *reinterpret_cast<const float4 *>(&s.b[wt * RUN + r][k * 16 + nl * 4]);
                const f32x2 dd = pair(st.x, st.x), du = pair(st.y, st.y);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float lo, hi;
                    unpair(mul2(dd, a[k][q]), lo, hi);
                    da[r][q] = pair(exp2_(lo), exp2_(hi));
                    x[r][q] = mul2(du, q ? pair(b.z, b.w) : pair(b.x, b.y));
                    H[q] = fma2(da[r][q], H[q], x[r][q]);
                    P[q] = mul2(da[r][q], P[q]);
                }
            }
            const int slot = k & 1;
            float4 v;
            unpair(P[0], v.x, v.y); unpair(P[1], v.z, v.w);
            s.decay[slot][wt][wc][lane] = v;
            unpair(H[0], v.x, v.y); unpair(H[1], v.z, v.w);
            s.sum[slot][wt][wc][lane] = v;
            __syncthreads();
            f32x2 from[2] = {h[k][0], h[k][1]};                            // the state at the start of this run
#pragma unroll
            for (int w = 0; w < WT; ++w) {
                const float4 pw = s.decay[slot][w][wc][lane], hw = s.sum[slot][w][wc][lane];
                if (w == wt) { from[0] = h[k][0]; from[1] = h[k][1]; }
                h[k][0] = fma2(pair(pw.x, pw.y), h[k][0], pair(hw.x, hw.y));
                h[k][1] = fma2(pair(pw.z, pw.w), h[k][1], pair(hw.z, hw.w));
            }
            if (p.states && live && t0 + wt * RUN < p.T && (t0 + wt * RUN) % kSpan == 0) {
                float g[4];
                unpair(from[0], g[0], g[1]); unpair(from[1], g[2], g[3]);
                store_states(p, p.states, (((t0 + wt * RUN) / kSpan * p.B + i) * p.D + mine) * p.N, k * 16 + nl * 4, g);
            }
#pragma unroll
            for (int r = 0; r < RUN; ++r) {
                const float4 c = *reinterpret_cast<const float4 *>(&s.c[wt * RUN + r][k * 16 + nl * 4]);
                f32x2 sum;
                from[0] = fma2(da[r][0], from[0], x[r][0]);
                from[1] = fma2(da[r][1], from[1], x[r][1]);
                sum = fma2(pair(c.z, c.w), from[1], mul2(pair(c.x, c.y), from[0]));
                y[r] += sum2(sum);
            }
        }
        float yr[RUN / 4];
        reduce_lanes<RUN, 1, 4>(y, lane, yr);
#pragma unroll
        for (int j = 0; j < RUN / 4; ++j) s.y[wt * RUN + 4 * j + nl][ch] = yr[j];
        __syncthreads();
        if (t0 + pt < p.T && two < p.D) {
            float out[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                out[j] = inside ? fmaf(skip[j], un[j], s.y[pt][pc + j]) : 0.0f;
                if (p.z) out[j] *= zn[j] * logistic<FINE>(zn[j]);
            }
            store_channels<T>(p, p.y, ((t0 + pt) * p.B + i) * p.D, two, out);
        }
    }
    if (wt == 0 && live) {
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            float x[4];
            unpair(h[k][0], x[0], x[1]); unpair(h[k][1], x[2], x[3]);
            store_states(p, p.h_final, (i * p.D + mine) * p.N, k * 16 + nl * 4, x);
        }
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------
constexpr long long kFewSteps = 4;

template <typename T, int NB>
relay_status_t launch_steps(const Args &p, cudaStream_t st)
{
    const long long blocks = (p.B * p.D * 4 + kStepThreads - 1) / kStepThreads;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "selective_scan: %lld x %lld channels", p.B, p.D);
    RELAY_CUDA(launch_pdl(selective_scan_steps_kernel<T, NB>, dim3((unsigned)blocks), dim3(kStepThreads), 0, st, p));
    return check_launch("selective_scan");
}
template <typename T, int WT, int WC, int NB>
relay_status_t launch_chunks(Args p, cudaStream_t st)
{
    using S = Tile<WT, WC, NB>;
    p.groups = (int)((p.D + S::CHANNELS - 1) / S::CHANNELS);
    const long long blocks = p.B * p.groups;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "selective_scan: %lld x %lld channels", p.B, p.D);
    RELAY_CUDA(cudaFuncSetAttribute(selective_scan_kernel<T, WT, WC, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(S)));
    RELAY_CUDA(launch_pdl(selective_scan_kernel<T, WT, WC, NB>, dim3((unsigned)blocks), dim3(S::THREADS), sizeof(S), st, p));
    return check_launch("selective_scan");
}
template <typename T, int NB>
relay_status_t launch_form(const Args &p, cudaStream_t st)
{
    if (p.T <= kFewSteps) return launch_steps<T, NB>(p, st);
    return launch_chunks<T, 4, 2, NB>(p, st);
}
template <typename T>
relay_status_t launch_states(const Args &p, cudaStream_t st)
{
    if (p.N <= 16) return launch_form<T, 1>(p, st);
    return p.N <= 32 ? launch_form<T, 2>(p, st) : launch_form<T, 4>(p, st);
}

}  // namespace

namespace scan {

relay_status_t check_inputs(const Inputs &in, Sizes *s, int64_t *N)
{
    RELAY_TRY(check_not_null(in.u, "u"));
    RELAY_TRY(check_not_null(in.delta, "delta"));
    RELAY_TRY(check_not_null(in.a, "a"));
    RELAY_TRY(check_not_null(in.b, "b"));
    RELAY_TRY(check_sizes(in.u, in.a, s, N));
    const int32_t t = in.u->dtype;
    RELAY_TRY(check_tensor(in.delta, t, t, {s->T, s->B, s->D}, "delta"));
    RELAY_TRY(check_tensor(in.b, t, t, {s->T, s->B, in.c ? *N : 2 * *N}, "b"));
    RELAY_TRY(check_tensor(in.c, t, t, {s->T, s->B, *N}, "c"));
    RELAY_TRY(check_tensor(in.d, RELAY_F32, RELAY_F32, {s->D}, "d"));
    RELAY_TRY(check_tensor(in.z, t, t, {s->T, s->B, s->D}, "z"));
    RELAY_TRY(check_tensor(in.delta_bias, RELAY_F32, RELAY_F32, {s->D}, "delta_bias"));
    return check_tensor(in.lengths, RELAY_I32, RELAY_I32, {s->B}, "lengths");
}
relay_status_t check_sizes(const relay_tensor_t *u, const relay_tensor_t *a, Sizes *s, int64_t *N)
{
    RELAY_TRY(check_sequence(u, s, "u"));
    RELAY_TRY(check_type(a, "a"));
    RELAY_TRY(check_rank(a, 2, "a"));
    *N = a->shape[1];
    RELAY_TRY(check_tensor(a, RELAY_F32, RELAY_F32, {s->D, *N}, "a"));
    if (*N < 1 || *N > RELAY_MAX_SCAN_STATES)
        return fail(RELAY_ERR_SHAPE, "a: %lld states, needs 1..%d", (long long)*N, RELAY_MAX_SCAN_STATES);
    return RELAY_OK;
}
relay_status_t check_softplus(int32_t softplus)
{
    if (softplus != 0 && softplus != 1) return fail(RELAY_ERR_ATTR, "softplus = %d, needs 0 or 1", softplus);
    return RELAY_OK;
}
Args make_args(const Inputs &in, int32_t softplus, const Sizes &s, int64_t N)
{
    Args p{};
    p.u = in.u->data; p.delta = in.delta->data; p.a = (const float *)in.a->data;
    p.b = in.b->data;
    p.c = in.c ? in.c->data : (const char *)in.b->data + N * dtype_size(in.b->dtype);
    p.d = in.d ? (const float *)in.d->data : nullptr;
    p.z = in.z ? in.z->data : nullptr;
    p.delta_bias = in.delta_bias ? (const float *)in.delta_bias->data : nullptr;
    p.lengths = in.lengths ? (const int *)in.lengths->data : nullptr;
    p.T = s.T; p.B = s.B; p.D = s.D; p.N = (int)N;
    p.ld_bc = (int)(in.c ? N : 2 * N);
    p.softplus = softplus;
    p.pairs = s.D % 2 == 0;
    p.quads = N % 4 == 0;
    return p;
}

}  // namespace scan
}  // namespace relay

using namespace relay;

extern "C" relay_status_t relay_infer_selective_scan(const relay_tensor_t *u, const relay_tensor_t *a, relay_tensor_t *y,
                                                     relay_tensor_t *h_final, relay_tensor_t *states)
{
    clear_error();
    RELAY_TRY(check_not_null(u, "u"));
    RELAY_TRY(check_not_null(a, "a"));
    RELAY_TRY(check_not_null(y, "y"));
    RELAY_TRY(check_not_null(h_final, "h_final"));
    RELAY_TRY(check_not_null(states, "states"));
    seq::Sizes s;
    int64_t N;
    RELAY_TRY(scan::check_sizes(u, a, &s, &N));
    *y = *u;
    y->data = nullptr;
    *h_final = relay_tensor_t{};
    h_final->dtype = RELAY_F32; h_final->rank = 3; h_final->layout = RELAY_ROWMAJOR;
    h_final->shape[0] = s.B; h_final->shape[1] = s.D; h_final->shape[2] = N;
    *states = relay_tensor_t{};
    states->dtype = RELAY_F32; states->rank = 4; states->layout = RELAY_ROWMAJOR;
    states->shape[0] = (s.T + RELAY_SCAN_SPAN - 1) / RELAY_SCAN_SPAN;
    states->shape[1] = s.B; states->shape[2] = s.D; states->shape[3] = N;
    return RELAY_OK;
}

extern "C" relay_status_t relay_selective_scan(const relay_tensor_t *u, const relay_tensor_t *delta, const relay_tensor_t *a,
                                               const relay_tensor_t *b, const relay_tensor_t *c, const relay_tensor_t *d,
                                               const relay_tensor_t *z, const relay_tensor_t *delta_bias, const relay_tensor_t *h0,
                                               const relay_tensor_t *lengths, int32_t softplus, const relay_tensor_t *y,
                                               const relay_tensor_t *h_final, const relay_tensor_t *states, void *stream)
{
    clear_error();
    const scan::Inputs in{u, delta, a, b, c, d, z, delta_bias, lengths};
    seq::Sizes s;
    int64_t N;
    RELAY_TRY(check_not_null(y, "y"));
    RELAY_TRY(scan::check_inputs(in, &s, &N));
    RELAY_TRY(seq::check_tensor(h0, RELAY_F32, RELAY_F32, {s.B, s.D, N}, "h0"));
    RELAY_TRY(seq::check_tensor(y, u->dtype, u->dtype, {s.T, s.B, s.D}, "y"));
    RELAY_TRY(seq::check_tensor(h_final, RELAY_F32, RELAY_F32, {s.B, s.D, N}, "h_final"));
    RELAY_TRY(seq::check_tensor(states, RELAY_F32, RELAY_F32, {(s.T + RELAY_SCAN_SPAN - 1) / RELAY_SCAN_SPAN, s.B, s.D, N}, "states"));
    RELAY_TRY(scan::check_softplus(softplus));
    const relay_tensor_t *ins[10] = {u, delta, a, b, c, d, z, delta_bias, h0, lengths}, *outs[3] = {y, h_final, states};
    RELAY_TRY(seq::check_buffers(ins, outs));
    if (s.B == 0 || s.D == 0) return RELAY_OK;
    scan::Args p = scan::make_args(in, softplus, s, N);
    p.h0 = h0 ? (const float *)h0->data : nullptr;
    p.y = y->data;
    p.h_final = h_final ? (float *)h_final->data : nullptr;
    p.states = states ? (float *)states->data : nullptr;
    cudaStream_t st = (cudaStream_t)stream;
    RELAY_TRY(seq::register_buffers(ins, outs, nullptr, 0, st));
    return u->dtype == RELAY_F32 ? launch_states<float>(p, st) : launch_states<__nv_bfloat16>(p, st);
}
