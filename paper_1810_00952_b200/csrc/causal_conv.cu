// Short causal convolution of a sequence, one filter of K taps per channel, and its gradient group:
//   s_t = b + sum_k w[k] x_{t-K+1+k},  y_t = act(s_t)
// The forward group reads x and writes y once, the gradient reads x and dy and writes dx once; K multiply-adds an element, and two
// instructions of the special-function pipe an element for the activation.  Measured, K = 4, silu: 8192 x 2 x 4096 54 us in bf16 (5.0 TB/s of 6.56
// copied) and 107 in fp32, gradient of 2048 x 8 x 2048 with its column sums 72 us (2.8 TB/s) and 97.  Counters before the rows inside a span had code
// without conditions (57, 169, 73, 106 us): 57 and 62 % of issue slots, 48 and 25 % of the special-function pipe, 31 and 23 % of the warps there are:
// registers hold the window, the filter, the slopes and the rows on their way.
// A thread owns V consecutive channels and a span of steps; the K - 1 inputs before the current one stay in its registers, and at the
// start of a span they are read again (K - 1 rows in S).  The gradient walks a span forwards and K - 1 steps beyond it: the partial of an
// input needs those of the K sums that it entered.
#include <algorithm>
#include <type_traits>

#include "sequence.cuh"

namespace relay {
namespace {

using namespace seq;

constexpr int kMaxTaps = 8;
constexpr int kThreads = 256;
constexpr int kRows = 8;           // spans of a gradient block: their partial sums of dw and db are joined on the chip
constexpr int kGradV = 2;          // most channels of a gradient thread: filter, window, slopes and sums of each stay in registers

struct Args {
    const void *x;                 // [T][C]
    const void *w, *b;             // [K][D], [D] or null
    const void *before;            // [K-1][C] or null
    const int *lengths;            // [C / D] or null
    void *y, *after;               // [T][C], [K-1][C] or null
    const void *dy, *dafter;       // [T][C], [K-1][C] or null
    void *dx, *dbefore;            // [T][C], [K-1][C] or null
    float *part;                   // [parts][C / D][K + 1][D]
    long long T, C, D;
    int K, S, w_bf16, b_bf16, silu;
    long long blocks_c;            // blocks along the channels
};

__device__ __forceinline__ long long end_of(const Args &p, long long c)
{
    if (p.lengths == nullptr) return p.T;
    const int *at = p.lengths + c / p.D;
    const long long n = relay_in_bounds(at, 4) ? *at : 0;
    return n < 0 ? 0 : n > p.T ? p.T : n;
}
// Input of step t, which may lie ahead of the first one; zero behind the sequence's end.  As stored: a load that is widened under its
// condition is waited for there, and what bounds these kernels is how many loads are on their way.
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> fetch_input(const Args &p, long long t, long long c, long long end)
{
    const bool ahead = t < 0;
    const T *from = ahead ? (const T *)p.before : (const T *)p.x;
    const long long at = (ahead ? t + p.K - 1 : t) * p.C + c;
    Raw<T, V> r{};
    if (ahead ? from != nullptr && t >= 1 - p.K : t < end) r = load_raw<T, V>(from, at);
    return r;
}
// rows of a span, by 32-bit offsets from its first one (the spans are cut so that these fit)
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> load_row(const T *first, unsigned off) { return load_raw<T, V>((const char *)first + off, 0); }
template <typename T, int V>
__device__ __forceinline__ void store_row(T *first, unsigned off, const float (&x)[V]) { store<T, V>((char *)first + off, 0, x); }
template <typename T, int V>
__device__ __forceinline__ void load_input(const Args &p, long long t, long long c, long long end, float (&x)[V])
{
    widen(fetch_input<T, V>(p, t, c, end), x, T());
}
// the filter, right-aligned to KP taps (the first KP - K do not exist), and the bias
template <int V, int KP>
__device__ __forceinline__ void load_filter(const Args &p, long long d, float (&w)[KP][V], float (&b)[V])
{
#pragma unroll
    for (int k = 0; k < KP; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) w[k][i] = 0.0f;
        const int first = KP < kMaxTaps ? 0 : KP - p.K;
        if (k >= first) load_operand<V>(p.w, p.w_bf16, (k - first) * p.D + d, w[k]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = 0.0f;
    if (p.b != nullptr) load_operand<V>(p.b, p.b_bf16, d, b);
}

template <typename T, int V, int KP>
__global__ void __launch_bounds__(kThreads) causal_conv_kernel(const Args p)
{
    constexpr bool FINE = sizeof(T) == 4;
    constexpr int U = 8;                                   // rows on their way (four: 62 us against 57 at 8192 x 2 x 4096)
    pdl_wait();
    const long long span = blockIdx.x / p.blocks_c;
    const long long c = ((blockIdx.x - span * p.blocks_c) * kThreads + threadIdx.x) * V;
    if (c >= p.C) return;
    const long long end = end_of(p, c), t0 = span * p.S, t1 = min(t0 + p.S, p.T);
    const int first = KP < kMaxTaps ? 0 : KP - p.K;        // the taps before it do not exist
    float w[KP][V], b[V], x[KP - 1 + U][V];
    load_filter<V, KP>(p, c % p.D, w, b);
    // the state for the next call: the last K - 1 inputs of the sequence
    if (span == 0 && p.after != nullptr) {
        for (int j = 0; j < p.K - 1; ++j) {
            float q[V];
            load_input<T, V>(p, end - (p.K - 1) + j, c, end, q);
            store<T, V>(p.after, j * p.C + c, q);
        }
    }
#pragma unroll
    for (int j = 0; j < KP - 1; ++j) load_input<T, V>(p, t0 - (KP - 1) + j, c, end, x[j]);
    const T *row = (const T *)p.x + t0 * p.C + c;
    T *to = (T *)p.y + t0 * p.C + c;
    const int steps = (int)(t1 - t0), inside = (int)min(max(end - t0, 0ll), (long long)steps);
    const unsigned bytes = (unsigned)(p.C * sizeof(T));    // of a row
    Raw<T, V> raw[U];
    auto fetch = [&](int n, auto whole) {                  // rows n .. n + U - 1 of the span; whole: all inside the sequence
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (!whole) raw[u] = Raw<T, V>{};
            if (whole || n + u < inside) raw[u] = load_row<T, V>(row, (unsigned)(n + u) * bytes);
        }
    };
    auto results = [&](int n, auto whole) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = b[i];
#pragma unroll
            for (int k = 0; k < KP; ++k)
                if (k >= first) muladd(w[k], x[u + k], y, y);
            if (p.silu) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] *= logistic<FINE>(y[i]);
            }
            if (!whole && n + u >= inside) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = 0.0f;
            }
            if (whole || n + u < steps) store_row<T, V>(to, (unsigned)(n + u) * bytes, y);
        }
    };
    using Yes = std::true_type;
    using No = std::false_type;
    fetch(0, No());
    for (int n = 0; n < steps; n += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) widen(raw[u], x[KP - 1 + u], T());
        if (n + 2 * U <= inside) fetch(n + U, Yes());
        else fetch(n + U, No());
        if (n + U <= inside) results(n, Yes());
        else results(n, No());
#pragma unroll
        for (int j = 0; j < KP - 1; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) x[j][i] = x[U + j][i];
    }
}

// One span: dx of its steps (and of the inputs ahead of the first step), its share of dw and db.  Blocks an SM: as many as
// the registers of the form's window, slopes and sums leave room for (eight taps of two channels on one block 147 us against 103 on two, 2048 x 8 x 2048).
template <typename T, int V, int KP>
__global__ void __launch_bounds__(32 * kRows, KP * V > 4 ? 2 : 3) causal_conv_grad_kernel(const Args p)
{
    constexpr bool FINE = sizeof(T) == 4;
    __shared__ float joint[kRows][32 * V];
    pdl_wait();
    const long long part = blockIdx.x / p.blocks_c;
    const long long c = ((blockIdx.x - part * p.blocks_c) * 32 + threadIdx.x) * V;
    const bool live = c < p.C;
    const long long end = live ? end_of(p, c) : 0, t0 = (part * kRows + threadIdx.y) * p.S, t1 = min(t0 + p.S, p.T);
    const int first = KP < kMaxTaps ? 0 : KP - p.K;        // the taps before it do not exist
    float w[KP][V], b[V], x[KP][V], g[KP][V], dw[KP][V], db[V];   // x[k]: the input under tap k;  g[k]: the slope k steps back
#pragma unroll
    for (int k = 0; k < KP; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) x[k][i] = g[k][i] = dw[k][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) db[i] = 0.0f;
    if (live && (t0 < p.T || t0 == 0)) {
        load_filter<V, KP>(p, c % p.D, w, b);
#pragma unroll
        for (int j = 1; j < KP; ++j) load_input<T, V>(p, t0 - KP + j, c, end, x[j]);
        // U rows of x and dy on their way while U are worked on
        constexpr int U = 4;
        const T *px = (const T *)p.x + t0 * p.C + c, *pg = (const T *)p.dy + t0 * p.C + c;
        T *to = (T *)p.dx + t0 * p.C + c;
        const unsigned bytes = (unsigned)(p.C * sizeof(T));                  // of a row
        const int steps = (int)(t1 - t0), inside = (int)min(max(end - t0, 0ll), (long long)(steps + KP - 1));
        const int summed = min(inside, steps);             // steps that this span's dw and db are made of
        const int after = p.dafter != nullptr ? (int)min(end - (p.K - 1) - t0, 1ll << 20) : 1 << 20;     // dafter's first step
        const int from = t0 == 0 ? 1 - p.K : 0;            // the first step whose partial this span gives
        Raw<T, V> rx[U], rg[U];
        auto fetch = [&](int n, auto whole) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if constexpr (!whole) rx[u] = rg[u] = Raw<T, V>{};
                if (whole || n + u < inside) rx[u] = load_row<T, V>(px, (unsigned)(n + u) * bytes);
                if (whole || n + u < inside) rg[u] = load_row<T, V>(pg, (unsigned)(n + u) * bytes);
            }
        };
        float nx[U][V], ng[U][V];
        auto work = [&](int n, auto whole) {               // whole: no step here is at an end of the span or of the sequence
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int k = 0; k + 1 < KP; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) { x[k][i] = x[k + 1][i]; g[KP - 1 - k][i] = g[KP - 2 - k][i]; }
#pragma unroll
                for (int i = 0; i < V; ++i) { x[KP - 1][i] = nx[u][i]; g[0][i] = ng[u][i]; }
                if (p.silu) {
                    float s[V], q[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) s[i] = b[i];
#pragma unroll
                    for (int k = 0; k < KP; ++k) if (k >= first) muladd(w[k], x[k], s, s);
#pragma unroll
                    for (int i = 0; i < V; ++i) { q[i] = logistic<FINE>(s[i]); s[i] *= 1.0f - q[i]; }
                    muladd(s, q, q, s);                    // the slope, q (1 + s (1 - q))
                    mul(g[0], s, g[0]);
                }
                if (!whole && n + u >= inside) {
#pragma unroll
                    for (int i = 0; i < V; ++i) g[0][i] = 0.0f;
                }
                if (whole || n + u < summed) {             // not behind the end: a zero slope times an infinite input is NaN
#pragma unroll
                    for (int i = 0; i < V; ++i) db[i] += g[0][i];
#pragma unroll
                    for (int k = 0; k < KP; ++k)
                        if (k >= first) muladd(g[0], x[k], dw[k], dw[k]);
                }
                const int at = n + u - (KP - 1);           // the step whose K sums are complete
                if (!whole && (at < from || at >= steps)) continue;
                float dx[V];
#pragma unroll
                for (int i = 0; i < V; ++i) dx[i] = 0.0f;
                if (whole || at < inside) {
#pragma unroll
                    for (int k = 0; k < KP; ++k)
                        if (k >= first) muladd(w[k], g[k], dx, dx);
                    if (!whole && at >= after) {
                        float q[V];
                        load<T, V>(p.dafter, (at - after) * p.C + c, q);
#pragma unroll
                        for (int i = 0; i < V; ++i) dx[i] += q[i];
                    }
                }
                if (whole || at >= 0) store_row<T, V>(to, (unsigned)at * bytes, dx);
                else if (p.dbefore != nullptr) store<T, V>(p.dbefore, (at + p.K - 1) * p.C + c, dx);
            }
        };
        using Yes = std::true_type;
        using No = std::false_type;
        const int whole_to = min(summed, after + KP - 1);        // steps from KP - 1 up to here
        fetch(0, No());
        for (int n = 0; n < steps + KP - 1; n += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) { widen(rx[u], nx[u], T()); widen(rg[u], ng[u], T()); }
            if (n + 2 * U <= inside) fetch(n + U, Yes());
            else fetch(n + U, No());
            if (n >= KP - 1 && n + U <= whole_to) work(n, Yes());
            else work(n, No());
        }
    }
    if (p.part == nullptr) return;
    const long long bd = live ? c / p.D : 0;
    float *out = p.part + ((part * (p.C / p.D) + bd) * (p.K + 1)) * p.D + (c - bd * p.D);
#pragma unroll
    for (int k = 0; k <= KP; ++k) {
        if (k < first) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) joint[threadIdx.y][threadIdx.x * V + i] = k < KP ? dw[k < KP ? k : 0][i] : db[i];
        __syncthreads();
        if (threadIdx.y == 0 && live) {
            float s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[i] = joint[0][threadIdx.x * V + i];
#pragma unroll
                for (int r = 1; r < kRows; ++r) s[i] += joint[r][threadIdx.x * V + i];
            }
            store<float, V>(out, (k - first) * p.D, s);
        }
        __syncthreads();
    }
}

// ---- launches ------------------------------------------------------------------------------------------------
constexpr long long kSms = 148;

// Steps of a span: the longest that still give every SM its threads, so that as few rows as possible are read twice; and no longer than
// 32-bit offsets reach (S + 8 rows of 4 bytes a channel at most).
int span_of(long long C, long long enough, long long per_span, long long T, int rows)
{
    int S = 64;
    while (S > 8 && per_span * ((T + (long long)S * rows - 1) / ((long long)S * rows)) < enough) S /= 2;
    while (S > 1 && (S + 8) * C >= 1ll << 30) S /= 2;
    return S;
}
int forward_span(long long T, long long C, int V) { return span_of(C, kSms * 1024, C / V, T, 1); }
int gradient_span(long long T, long long C, int V) { return span_of(C, kSms * 4, (C / V + 31) / 32, T, kRows); }
relay_status_t check_offsets(const Args &p)
{
    if ((p.S + 8) * p.C >= 1ll << 30) return fail(RELAY_ERR_UNSUPPORTED, "causal_conv: rows of %lld channels", p.C);
    return RELAY_OK;
}
int channels_of_gradient(long long D) { return D % kGradV == 0 ? kGradV : 1; }
long long gradient_parts(long long T, long long C, long long D)
{
    const long long steps = (long long)gradient_span(T, C, channels_of_gradient(D)) * kRows;
    return std::max<long long>(1, (T + steps - 1) / steps);
}

template <typename T, int V, int KP>
relay_status_t launch_forward(Args p, cudaStream_t st)
{
    p.S = forward_span(p.T, p.C, V);
    RELAY_TRY(check_offsets(p));
    p.blocks_c = (p.C / V + kThreads - 1) / kThreads;
    const long long blocks = p.blocks_c * std::max<long long>(1, (p.T + p.S - 1) / p.S);
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "causal_conv: %lld steps of %lld channels", p.T, p.C);
    RELAY_CUDA(launch_pdl(causal_conv_kernel<T, V, KP>, dim3((unsigned)blocks), dim3(kThreads), 0, st, p));
    return check_launch("causal_conv");
}
template <typename T, int V, int KP>
relay_status_t launch_gradient(Args p, cudaStream_t st)
{
    p.S = gradient_span(p.T, p.C, V);
    RELAY_TRY(check_offsets(p));
    p.blocks_c = (p.C / V + 31) / 32;
    const long long blocks = p.blocks_c * gradient_parts(p.T, p.C, p.D);
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "causal_conv_grad: %lld steps of %lld channels", p.T, p.C);
    RELAY_CUDA(launch_pdl(causal_conv_grad_kernel<T, V, KP>, dim3((unsigned)blocks), dim3(32, kRows), 0, st, p));
    return check_launch("causal_conv_grad");
}
// taps: kernels for 2, 3 and 4; all others are right-aligned in one for 8.  Channels of a thread: as many as divide the rows into
// whole aligned accesses of 8 bytes (16 take so many registers that an SM has half the warps).
template <typename T, int V>
relay_status_t forward_taps(const Args &p, cudaStream_t st)
{
    switch (p.K) {
    case 2: return launch_forward<T, V, 2>(p, st);
    case 3: return launch_forward<T, V, 3>(p, st);
    case 4: return launch_forward<T, V, 4>(p, st);
    default: return launch_forward<T, V, kMaxTaps>(p, st);
    }
}
template <typename T, int V>
relay_status_t gradient_taps(const Args &p, cudaStream_t st)
{
    switch (p.K) {
    case 2: return launch_gradient<T, V, 2>(p, st);
    case 3: return launch_gradient<T, V, 3>(p, st);
    case 4: return launch_gradient<T, V, 4>(p, st);
    default: return launch_gradient<T, V, kMaxTaps>(p, st);
    }
}
template <typename T>
relay_status_t forward_channels(const Args &p, cudaStream_t st)
{
    if (p.D % 4 == 0) return forward_taps<T, 4>(p, st);
    return p.D % 2 == 0 ? forward_taps<T, 2>(p, st) : forward_taps<T, 1>(p, st);
}
template <typename T>
relay_status_t gradient_channels(const Args &p, cudaStream_t st)
{
    return channels_of_gradient(p.D) == kGradV ? gradient_taps<T, kGradV>(p, st) : gradient_taps<T, 1>(p, st);
}

// ---- boundary ---------------------------------------------------------------------------------------------------
relay_status_t check_filter(const relay_tensor_t *x, const relay_tensor_t *w, Sizes *s, int64_t *K)
{
    RELAY_TRY(check_sequence(x, s, "x"));
    RELAY_TRY(check_type(w, "w"));
    RELAY_TRY(check_rank(w, 2, "w"));
    *K = w->shape[0];
    RELAY_TRY(check_tensor(w, x->dtype, RELAY_F32, {*K, s->D}, "w"));
    if (*K < 1 || *K > kMaxTaps) return fail(RELAY_ERR_SHAPE, "w: %lld taps, needs 1..%d", (long long)*K, kMaxTaps);
    return RELAY_OK;
}
relay_status_t check_act(int32_t act)
{
    if (act != RELAY_ACT_NONE && act != RELAY_ACT_SILU) return fail(RELAY_ERR_ATTR, "activation %d, needs none or silu", act);
    return RELAY_OK;
}
Args make_args(const relay_tensor_t *x, const relay_tensor_t *w, const relay_tensor_t *b, const relay_tensor_t *before,
               const relay_tensor_t *lengths, int32_t act, const Sizes &s, int64_t K)
{
    Args p{};
    p.x = x->data; p.w = w->data; p.b = b ? b->data : nullptr;
    p.before = before ? before->data : nullptr;
    p.lengths = lengths ? (const int *)lengths->data : nullptr;
    p.T = s.T; p.C = s.B * s.D; p.D = s.D; p.K = (int)K;
    p.w_bf16 = w->dtype == RELAY_BF16; p.b_bf16 = b && b->dtype == RELAY_BF16;
    p.silu = act == RELAY_ACT_SILU;
    return p;
}
size_t gradient_bytes(const Sizes &s, int64_t K)
{
    if (s.B == 0 || s.D == 0) return 0;
    return (size_t)gradient_parts(s.T, s.B * s.D, s.D) * s.B * (K + 1) * s.D * sizeof(float);
}

}  // namespace
}  // namespace relay

using namespace relay;

extern "C" relay_status_t relay_infer_causal_conv(const relay_tensor_t *x, const relay_tensor_t *w, relay_tensor_t *y, relay_tensor_t *after)
{
    clear_error();
    RELAY_TRY(check_not_null(x, "x"));
    RELAY_TRY(check_not_null(w, "w"));
    RELAY_TRY(check_not_null(y, "y"));
    RELAY_TRY(check_not_null(after, "after"));
    seq::Sizes s;
    int64_t K;
    RELAY_TRY(check_filter(x, w, &s, &K));
    *y = *x;
    y->data = nullptr;
    *after = *y;
    after->shape[0] = K - 1;
    return RELAY_OK;
}

extern "C" relay_status_t relay_causal_conv(const relay_tensor_t *x, const relay_tensor_t *w, const relay_tensor_t *b,
                                            const relay_tensor_t *before, const relay_tensor_t *lengths, int32_t act,
                                            const relay_tensor_t *y, const relay_tensor_t *after, void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(x, "x"));
    RELAY_TRY(check_not_null(w, "w"));
    RELAY_TRY(check_not_null(y, "y"));
    seq::Sizes s;
    int64_t K;
    RELAY_TRY(check_filter(x, w, &s, &K));
    RELAY_TRY(seq::check_tensor(b, x->dtype, RELAY_F32, {s.D}, "b"));
    RELAY_TRY(seq::check_tensor(before, x->dtype, x->dtype, {K - 1, s.B, s.D}, "before"));
    RELAY_TRY(seq::check_tensor(lengths, RELAY_I32, RELAY_I32, {s.B}, "lengths"));
    RELAY_TRY(seq::check_tensor(y, x->dtype, x->dtype, {s.T, s.B, s.D}, "y"));
    RELAY_TRY(seq::check_tensor(after, x->dtype, x->dtype, {K - 1, s.B, s.D}, "after"));
    RELAY_TRY(check_act(act));
    const relay_tensor_t *ins[5] = {x, w, b, before, lengths}, *outs[2] = {y, after};
    RELAY_TRY(seq::check_buffers(ins, outs));
    if (s.B == 0 || s.D == 0 || (s.T == 0 && (!after || K == 1))) return RELAY_OK;
    Args p = make_args(x, w, b, before, lengths, act, s, K);
    p.y = y->data;
    p.after = after ? after->data : nullptr;
    cudaStream_t st = (cudaStream_t)stream;
    RELAY_TRY(seq::register_buffers(ins, outs, nullptr, 0, st));
    return x->dtype == RELAY_F32 ? forward_channels<float>(p, st) : forward_channels<__nv_bfloat16>(p, st);
}

extern "C" size_t relay_workspace_bytes_causal_conv_grad(const relay_tensor_t *x, const relay_tensor_t *w)
{
    clear_error();
    seq::Sizes s;
    int64_t K;
    if (!x || !w || check_filter(x, w, &s, &K) != RELAY_OK) return 0;
    return gradient_bytes(s, K);
}

extern "C" relay_status_t relay_causal_conv_grad(const relay_tensor_t *x, const relay_tensor_t *w, const relay_tensor_t *b,
                                                 const relay_tensor_t *before, const relay_tensor_t *lengths, int32_t act,
                                                 const relay_tensor_t *dy, const relay_tensor_t *dafter, const relay_tensor_t *dx,
                                                 const relay_tensor_t *dw, const relay_tensor_t *db, const relay_tensor_t *dbefore, void *ws,
                                                 size_t ws_bytes, void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(x, "x"));
    RELAY_TRY(check_not_null(w, "w"));
    RELAY_TRY(check_not_null(dy, "dy"));
    RELAY_TRY(check_not_null(dx, "dx"));
    seq::Sizes s;
    int64_t K;
    RELAY_TRY(check_filter(x, w, &s, &K));
    RELAY_TRY(seq::check_tensor(b, x->dtype, RELAY_F32, {s.D}, "b"));
    RELAY_TRY(seq::check_tensor(before, x->dtype, x->dtype, {K - 1, s.B, s.D}, "before"));
    RELAY_TRY(seq::check_tensor(lengths, RELAY_I32, RELAY_I32, {s.B}, "lengths"));
    RELAY_TRY(seq::check_tensor(dy, x->dtype, x->dtype, {s.T, s.B, s.D}, "dy"));
    RELAY_TRY(seq::check_tensor(dafter, x->dtype, x->dtype, {K - 1, s.B, s.D}, "dafter"));
    RELAY_TRY(seq::check_tensor(dx, x->dtype, x->dtype, {s.T, s.B, s.D}, "dx"));
    RELAY_TRY(seq::check_tensor(dw, RELAY_F32, RELAY_F32, {K, s.D}, "dw"));
    RELAY_TRY(seq::check_tensor(db, RELAY_F32, RELAY_F32, {s.D}, "db"));
    RELAY_TRY(seq::check_tensor(dbefore, x->dtype, x->dtype, {K - 1, s.B, s.D}, "dbefore"));
    RELAY_TRY(check_act(act));
    const relay_tensor_t *ins[7] = {x, w, b, before, lengths, dy, dafter}, *outs[4] = {dx, dw, db, dbefore};
    RELAY_TRY(seq::check_buffers(ins, outs));
    const size_t need = dw || db ? gradient_bytes(s, K) : 0;
    RELAY_TRY(check_workspace(ws, ws_bytes, need));
    cudaStream_t st = (cudaStream_t)stream;
    if (s.D == 0) return RELAY_OK;
    Args p = make_args(x, w, b, before, lengths, act, s, K);
    p.dy = dy->data;
    p.dafter = dafter ? dafter->data : nullptr;
    p.dx = dx->data;
    p.dbefore = dbefore ? dbefore->data : nullptr;
    p.part = dw || db ? (float *)ws : nullptr;
    RELAY_TRY(seq::register_buffers(ins, outs, ws, need, st));
    if (s.B > 0)
        RELAY_TRY(x->dtype == RELAY_F32 ? gradient_channels<float>(p, st) : gradient_channels<__nv_bfloat16>(p, st));
    const long long rows = s.B > 0 ? gradient_parts(s.T, p.C, p.D) * s.B : 0;
    return seq::launch_column_sums((const float *)ws, rows, {{dw ? (float *)dw->data : nullptr, db ? (float *)db->data : nullptr, nullptr}, {K * s.D, s.D, 0}},
                                   st);
}
