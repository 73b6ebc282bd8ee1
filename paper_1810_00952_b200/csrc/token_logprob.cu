// Log-probabilities of given tokens, entropies and the most probable tokens of rows of scores, and the gradient group.
// HBM-bound: the forward call reads every score once, the gradient reads and writes it once.
#include <algorithm>

#include "common.h"
#include "ewise_kernels.cuh"

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
    r.s = a.s * ea + b.s * eb;
    r.w = ea * fmaf(da, a.s, a.w) + eb * fmaf(db, b.s, b.w);
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
        entropy = log_s - a.w * k.inv / a.s;
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

// ---- one block per row ----------------------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kThreads) token_logprob_rows_kernel(const Args p)
{
    __shared__ Sums part[kThreads / 32];
    __shared__ unsigned long long best[kThreads / 32];
    __shared__ unsigned long long chosen;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *z = (const T *)p.z + row * p.V;
        Sums a = empty_sums();
        for (int j = tid; j < p.V; j += kThreads) {
            const float x = load_score(z + j);
            a = join(a, Sums{x, x == -INFINITY ? 0.0f : 1.0f, 0.0f}, p.k);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) a = join(a, shfl_xor(a, d), p.k);
        if (lane == 0) part[warp] = a;
        __syncthreads();
        a = part[0];
        for (int k = 1; k < kThreads / 32; ++k) a = join(a, part[k], p.k);
        const Row r(a, p.k);
        if (tid == 0) {
            if (p.lse) p.lse[row] = r.lse;
            if (p.entropy) p.entropy[row] = r.entropy;
            if (p.logp) {
                const int t = token_of(p.tokens, p.tokens_i64, row, p.V);
                p.logp[row] = t < 0 ? 0.0f : r.logp(load_score(z + t), p.k);
            }
        }
        unsigned long long last = ~0ull;
        for (int k = 0; k < p.top; ++k) {                  // the largest key below the last one
            unsigned long long b = 0;
            for (int j = tid; j < p.V; j += kThreads) {
                const unsigned long long key = key_of(load_score(z + j), j);
                if (key < last && key > b) b = key;
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, d));
            if (lane == 0) best[warp] = b;
            __syncthreads();
            if (tid == 0) {
                for (int i = 1; i < kThreads / 32; ++i) b = max(b, best[i]);
                chosen = b;
                const int id = id_of(b);
                p.top_ids[row * p.top + k] = id;
                p.top_logp[row * p.top + k] = r.logp(load_score(z + id), p.k);
            }
            __syncthreads();
            last = chosen;
        }
        __syncthreads();
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) token_logprob_grad_rows_kernel(const GradArgs p)
{
    pdl_wait();
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *z = (const T *)p.z + row * p.V;
        T *dz = (T *)p.dz + row * p.V;
        const float lse = p.lse[row];
        const int t = token_of(p.tokens, p.tokens_i64, row, p.V);
        const float d = t < 0 ? 0.0f : p.dlogp[row];
        const float e = p.dentropy ? p.dentropy[row] : 0.0f, h = p.dentropy ? p.entropy[row] : 0.0f;
        for (int j = threadIdx.x; j < p.V; j += kThreads) {
            float g = 0.0f;
            if (lse != -INFINITY) {
                const float lp = log_prob(load_score(z + j), lse, p.k), q = __expf(lp);
                g = j == t ? -d * expm1f(lp) : -d * q;     // 1 - p of a class that is nearly certain keeps its precision
                if (p.dentropy && q != 0.0f) g -= e * q * (lp + h);
                g *= p.k.inv;
            }
            if (relay_in_bounds(dz + j, sizeof(T))) {
                if constexpr (sizeof(T) == 2) dz[j] = __float2bfloat16_rn(g);
                else dz[j] = g;
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
    if (s->V > INT32_MAX) return fail(RELAY_ERR_SHAPE, "scores: %lld classes do not fit an i32", (long long)s->V);
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

template <typename A, typename K>
relay_status_t launch_rows(K kernel, const A &p, cudaStream_t st, const char *name)
{
    const dim3 grid((unsigned)std::min<long long>(p.rows, 1 << 20));
    RELAY_CUDA(launch_pdl(kernel, grid, dim3(kThreads), 0, st, p));
    return check_launch(name);
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
    if (scores->dtype == RELAY_F32) return launch_rows(token_logprob_rows_kernel<float>, p, st, "token_logprob");
    return launch_rows(token_logprob_rows_kernel<__nv_bfloat16>, p, st, "token_logprob");
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
    if (scores->dtype == RELAY_F32) return launch_rows(token_logprob_grad_rows_kernel<float>, p, st, "token_logprob_grad");
    return launch_rows(token_logprob_grad_rows_kernel<__nv_bfloat16>, p, st, "token_logprob_grad");
}
