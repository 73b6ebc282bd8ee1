// Orthogonalised update of weight matrices by Newton-Schulz products.
//
//   X <- x / (|x|_F + eps);   `steps` times:  G = X X^T,  P = b G + c G G,  X <- a X + P X        (M <= N; m = M, n = N)
//                                             G = X^T X,  P = b G + c G G,  X <- a X + X P        (M >  N; m = N, n = M)
//   y = scale X
//
// Three products a step on the tensor cores (tcgen05, kind::f16).  G and P are symmetric: only the tiles on and above the
// diagonal are computed, each stored to both places, so a step costs m m n + m m m + 2 m m n operations.  The operands lie in
// the workspace as fp16: at the tensor rate of bf16 it keeps 10 fraction bits instead of 7, and with them an update that is 1e-3
// instead of 1e-2 off (where singular values fall off, 0.3 to 5 % instead of 3 to 38: see the entry point).  Their range: with the usual coefficients singular values never leave [0, 1.3]; X is kept times a power of two,
// S = 2^round(log2(sqrt(M N) / 8)), which puts its elements around 1/8 at the start and below 0.16 sqrt(M N) ever after; other
// coefficients may let X grow or shrink, and further powers of two per step follow that (steps_of).  What is too small for fp16 in G
// and P is small against the diagonal.  The diagonals of G and P, whose entries grow to 1 and -2.7
// and whose rounding would move whole rows, are kept apart in fp32: with G = D + O,
//   P = b O + c (D O + O D + O O) off the diagonal,  e = a + b d + c (d d + diag(O O)) on it,   X <- e X + offdiag(P) X
// (one multiplier per row of X, per column where M > N), all of it in the products' epilogues.
//
// Three forms, all steps in one launch each:
//   up to 512 elements          one block in shared memory in fp32 (16-bit operands' errors do not average out over so few); 32 x 32
//                               would take 23 us against 17 on the tensor cores, 64 x 64 71 against 18
//   up to 128 x 2048            a cluster that keeps the matrix on the chip (orthogonalize_resident.cu): 128 x 256 32 us against 86
//   all others                  pairs of SMs over the products' units (orthogonalize_tc.cu), after two passes for norm and copy
// Measured: 4096 x 4096 1.33 ms = 1.04 PFLOP/s of the operations above (cuBLAS on a plain product: 1.63 burst, 1.38 sustained);
// 8 x 1024 x 4096 0.84 ms = 0.66 PFLOP/s; 3 x 500 x 333 114 us, a step 19 to 21: three phases of 6 to 7 us each, whatever their size.
#include <algorithm>
#include <cmath>
#include <cuda_fp16.h>

#include "common.h"
#include "ewise_kernels.cuh"
#include "orthogonalize.h"

namespace relay {

namespace {

using namespace orth;

// ---- norm and the 16-bit copy ----------------------------------------------------------------------------
constexpr int kNormThreads = 256;
constexpr int kNormMost = 256;                         // partial sums per matrix, at most

// The sum of squares in fp64: a square of any finite element fits, and the sum does not depend on the elements' scale.
template <typename T>
__global__ void __launch_bounds__(kNormThreads) orth_norm_kernel(const T *__restrict__ x, long long size, int even, double *__restrict__ partial)
{
    __shared__ double warp_sum[kNormThreads / 32];
    pdl_wait();
    x += (long long)blockIdx.y * size;
    double s = 0.0;
    const long long groups = (size + 7) / 8, stride = (long long)gridDim.x * kNormThreads;
    for (long long i = (long long)blockIdx.x * kNormThreads + threadIdx.x; i < groups; i += 4 * stride) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long at = (i + u * stride) * 8, n = size - at;
            eight(x + at, even && n >= 8, n < 0 ? 0 : n < 8 ? (int)n : 8, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int c = 0; c < 8; ++c) { const double d = v[u][c]; s = fma(d, d, s); }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kNormThreads / 32; ++i) s += warp_sum[i];
        partial[(long long)blockIdx.y * gridDim.x + blockIdx.x] = s;
    }
}

// out = fp16(x s / (|x| + eps)), rows padded to ld, and the matrix's counter set to zero; a thread takes eight columns of a row at a time
template <typename T>
__global__ void __launch_bounds__(kNormThreads) orth_convert_kernel(const T *__restrict__ x, int rows, int cols, int even, const double *__restrict__ partial, int partials,
                                                                   float eps, float s, __half *__restrict__ out, long long ld, unsigned int *__restrict__ done)
{
    __shared__ double warp_sum[kNormThreads / 32];
    pdl_wait();
    const long long b = blockIdx.y;
    if (blockIdx.x == 0 && threadIdx.x == 0) done[b] = 0;  // what the products count in
    double sum = threadIdx.x < partials ? partial[b * partials + threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < kNormThreads / 32; ++i) sum += warp_sum[i];
    float f1, f2;
    normalizer(sum, eps, s, f1, f2);
    const int per_row = (cols + 7) / 8;
    const long long items = (long long)rows * per_row;
    x += b * rows * cols;
    out += b * rows * ld;
    for (long long i = (long long)blockIdx.x * kNormThreads + threadIdx.x; i < items; i += (long long)gridDim.x * kNormThreads) {
        const long long r = i / per_row;
        const int c = (int)(i - r * per_row) * 8;
        float v[8];
        eight(x + r * cols + c, even, min(8, cols - c), v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] * f1 * f2;
        *reinterpret_cast<uint4 *>(out + r * ld + c) = make_uint4(pack_half2(v[0], v[1]), pack_half2(v[2], v[3]), pack_half2(v[4], v[5]), pack_half2(v[6], v[7]));
    }
}

// ---- small matrices: one block each -----------------------------------------------------------------------------
constexpr int kSmallThreads = 256;
constexpr int64_t kSmallSize = 512;
// rows of shared memory: whole float4, an odd number of them, so that rows next to each other start on other banks
__host__ __device__ inline int small_ld(int n) { return ((n + 3) / 4 | 1) * 4; }
inline bool small_fits(int64_t m, int64_t n) { return m * n <= kSmallSize; }
inline size_t small_smem(int m, int n)
{
    const int rm = (m + 3) / 4 * 4;
    return (size_t)(2 * rm * small_ld(n) + 2 * rm * small_ld(m)) * 4 + 64;
}

// 4 x 4 results C(i,j) = sum_k a[i][k] b[j][k] (rows of K padded to float4 with zeros)
__device__ __forceinline__ void dot_rows(const float *a, const float *b, int ld, int k4, float (&c)[4][4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = 0.0f;
    for (int k = 0; k < k4; ++k) {
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = *reinterpret_cast<const float4 *>(a + i * ld + 4 * k); y[i] = *reinterpret_cast<const float4 *>(b + i * ld + 4 * k); }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c[i][j] = fmaf(x[i].w, y[j].w, fmaf(x[i].z, y[j].z, fmaf(x[i].y, y[j].y, fmaf(x[i].x, y[j].x, c[i][j]))));
    }
}

template <typename T>
__global__ void __launch_bounds__(kSmallThreads) orth_small_kernel(const T *__restrict__ x, int M, int N, const Steps step, float eps, __nv_bfloat16 *__restrict__ y)
{
    extern __shared__ float4 smem4[];
    __shared__ double warp_sum[kSmallThreads / 32];
    const bool tall = M > N;
    const int m = tall ? N : M, n = tall ? M : N, tid = threadIdx.x;
    const int ldx = small_ld(n), ldg = small_ld(m), rm = (m + 3) / 4 * 4, mt = rm / 4, nt = (n + 3) / 4;
    float *X = reinterpret_cast<float *>(smem4), *X2 = X + rm * ldx, *G = X2 + rm * ldx, *P = G + rm * ldg;
    for (int i = tid; i < 2 * rm * (ldx + ldg); i += kSmallThreads) X[i] = 0.0f;     // the padding stays zero
    pdl_wait();
    __syncthreads();
    x += (long long)blockIdx.x * M * N;
    y += (long long)blockIdx.x * M * N;
    double s = 0.0;
    for (int i = tid; i < M * N; i += kSmallThreads) {
        const double v = element(x + i);
        s = fma(v, v, s);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if ((tid & 31) == 0) warp_sum[tid >> 5] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < kSmallThreads / 32; ++i) s += warp_sum[i];
    const double f = 1.0 / (sqrt(s) + (double)eps);
    for (int i = tid; i < M * N; i += kSmallThreads) {
        const int r = i / N, q = i - r * N;
        X[tall ? q * ldx + r : r * ldx + q] = (float)(f * (double)element(x + i));
    }
    __syncthreads();
    for (int k = 0; k < step.n; ++k) {
        const float a = step.a[k], b = step.b[k], c = step.c[k];
        float t[4][4];
        for (int u = tid; u < mt * mt; u += kSmallThreads) {                          // G = X X^T
            const int i0 = u / mt * 4, j0 = u % mt * 4;
            dot_rows(X + i0 * ldx, X + j0 * ldx, ldx, nt, t);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) G[(i0 + i) * ldg + j0 + j] = t[i][j];
        }
        __syncthreads();
        for (int u = tid; u < mt * mt; u += kSmallThreads) {                          // P = a I + b G + c G G
            const int i0 = u / mt * 4, j0 = u % mt * 4;
            dot_rows(G + i0 * ldg, G + j0 * ldg, ldg, mt, t);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    P[(i0 + i) * ldg + j0 + j] = fmaf(c, t[i][j], b * G[(i0 + i) * ldg + j0 + j]) + (i0 + i == j0 + j ? a : 0.0f);
        }
        __syncthreads();
        for (int u = tid; u < mt * nt; u += kSmallThreads) {                          // X2 = P X
            const int i0 = u / nt * 4, j0 = u % nt * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) t[i][j] = 0.0f;
            for (int q = 0; q < m; ++q) {
                const float4 v = *reinterpret_cast<const float4 *>(X + q * ldx + j0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = P[(i0 + i) * ldg + q];
                    t[i][0] = fmaf(w, v.x, t[i][0]); t[i][1] = fmaf(w, v.y, t[i][1]);
                    t[i][2] = fmaf(w, v.z, t[i][2]); t[i][3] = fmaf(w, v.w, t[i][3]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i0 + i < m) *reinterpret_cast<float4 *>(X2 + (i0 + i) * ldx + j0) = make_float4(t[i][0], t[i][1], t[i][2], t[i][3]);
        }
        __syncthreads();
        float *w = X; X = X2; X2 = w;
    }
    for (int i = tid; i < M * N; i += kSmallThreads) {
        const int r = i / N, q = i - r * N;
        if (relay_in_bounds(y + i, 2)) y[i] = __float2bfloat16_rn(step.scale * X[tall ? q * ldx + r : r * ldx + q]);
    }
}

template <typename T>
relay_status_t launch_small(const relay_tensor_t *x, const Steps &steps, float eps, const relay_tensor_t *y, int64_t L, int M, int N, cudaStream_t st)
{
    const size_t smem = small_smem(std::min(M, N), std::max(M, N));
    RELAY_CUDA(cudaFuncSetAttribute(orth_small_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024));
    RELAY_CUDA(launch_pdl(orth_small_kernel<T>, dim3((unsigned)L), dim3(kSmallThreads), smem, st, (const T *)x->data, M, N, steps, eps, (__nv_bfloat16 *)y->data));
    return check_launch("orthogonalize_small");
}

}  // namespace

// Singular values start in [0, 1]; a step takes t to t (a + b t^2 + c t^4), so g, the largest absolute value that the steps can have made,
// is known beforehand.  Where 2^-r g leaves [1/4, 16], or 16-bit elements of s X may leave their range, X is kept times 2^-r from
// there on, which is a change of each step's coefficients.  With the usual coefficients g is 1.2 and r stays 0.  A g that single
// values near one may reach, but none near zero (those grow by a a step), is followed for 2^10 only: most elements would be lost.
orth::Steps orth::steps_of(const relay_orthogonalize_attrs_t &at, double s)
{
    Steps p{};
    p.n = at.steps;
    const double a = at.a, b = at.b, c = at.c, most = std::min(16.0, 32768.0 / s);
    double g = 1.0, grown = 0.0;                           // log2 of what values near zero have grown by
    int r = 0;
    for (int k = 0; k < at.steps; ++k) {
        auto value = [&](double t) { const double q = t * t; return std::fabs(t * (a + q * (b + c * q))); };
        double next = value(g);
        const double root = 9.0 * b * b - 20.0 * a * c;    // extrema: a + 3 b t^2 + 5 c t^4 = 0
        for (int sign = -1; sign <= 1 && root >= 0.0; sign += 2) {
            const double q = c != 0.0 ? (-3.0 * b + sign * std::sqrt(root)) / (10.0 * c) : b != 0.0 ? -a / (3.0 * b) : 0.0;
            if (q > 0.0 && q < g * g) next = std::max(next, value(std::sqrt(q)));
        }
        g = std::min(std::max(next, 1e-300), 1e300);
        grown += std::log2(std::max(std::fabs(a), 1e-30));
        int to = 0;
        if (g > most) to = std::min((int)std::ceil(std::log2(g / most)), (int)std::max(0.0, std::floor(grown)) + 10);
        else if (g < 0.25) to = (int)std::ceil(std::log2(g));
        p.a[k] = (float)std::ldexp(a, r - to);
        p.b[k] = (float)std::ldexp(b, 3 * r - to);
        p.c[k] = (float)std::ldexp(c, 5 * r - to);
        r = to;
    }
    p.scale = (float)std::ldexp((double)at.scale, r);
    return p;
}

namespace {

// ---- workspace -------------------------------------------------------------------------------------------------
struct Plan {
    int64_t L, M, N, m, n;             // matrices; m = min(M, N), n = max(M, N)
    int64_t xld, gld;                  // row strides of X (rows M, N columns) and G, P (m x m), in elements
    size_t x_bytes, g_bytes, v_bytes, n_bytes, total;
    bool small, resident;              // one block's fp32 kernel; one cluster's
};
Plan plan_of(const relay_tensor_t *x)
{
    Plan p{};
    p.L = 1;
    for (int d = 0; d + 2 < x->rank; ++d) p.L *= x->shape[d];
    p.M = x->shape[x->rank - 2]; p.N = x->shape[x->rank - 1];
    p.m = std::min(p.M, p.N); p.n = std::max(p.M, p.N);
    p.xld = (int64_t)align_up((size_t)p.N, 64);
    p.gld = (int64_t)align_up((size_t)p.m, 64);
    p.x_bytes = align_up((size_t)(p.L * p.M * p.xld) * 2, 256);
    p.g_bytes = align_up((size_t)(p.L * p.m * p.gld) * 2, 256);
    p.v_bytes = align_up((size_t)(p.L * p.gld) * 4, 256);
    p.n_bytes = align_up((size_t)p.L * kNormMost * sizeof(double), 256);
    p.total = p.n_bytes + 2 * p.x_bytes + 2 * p.g_bytes + 2 * p.v_bytes + align_up((size_t)p.L * 4, 256);
    p.small = small_fits(p.m, p.n);
    p.resident = !p.small && resident_fits(p.m, p.n);
    // No kernel reads or writes the 256 bytes of a matrix that stays on the chip: they are only the documented minimum above kSmallSize.
    if (p.resident) p.total = 256;
    if (p.small) p.total = 0;
    return p;
}

relay_status_t check_matrices(const relay_tensor_t *x)
{
    RELAY_TRY(check_type(x, "x"));
    if (x->rank < 2) return fail(RELAY_ERR_RANK, "x: rank %d, a matrix has rank 2", x->rank);
    if (!is_float(x->dtype)) return fail(RELAY_ERR_DTYPE, "x: base type %s, needs f32 or bf16", dtype_name(x->dtype));
    RELAY_TRY(check_layout(x, RELAY_ROWMAJOR, RELAY_ROWMAJOR, "x"));
    const Plan p = plan_of(x);
    if (p.n > 65536 || p.L > 65535) return fail(RELAY_ERR_SHAPE, "x: %lld matrices of %lld x %lld, at most 65535 of 65536 x 65536", (long long)p.L, (long long)p.M, (long long)p.N);
    return RELAY_OK;
}

template <typename T>
relay_status_t prepare_x(const relay_tensor_t *x, const Plan &pl, double *partial, float eps, float s, int sms, __half *out, unsigned int *done, cudaStream_t st)
{
    const long long size = pl.M * pl.N, each = kNormThreads * 8;
    const int share = (int)std::max<int64_t>(1, 4 * sms / pl.L);             // blocks per matrix that fill the GPU
    const int partials = (int)std::min<long long>({(size + each - 1) / each, share, kNormMost});
    RELAY_CUDA(launch_pdl(orth_norm_kernel<T>, dim3((unsigned)partials, (unsigned)pl.L), dim3(kNormThreads), 0, st, (const T *)x->data, size, (int)(size % 8 == 0), partial));
    RELAY_TRY(check_launch("orthogonalize_norm"));
    const dim3 grid((unsigned)std::min<long long>((pl.M * ((pl.N + 7) / 8) + kNormThreads - 1) / kNormThreads, 2 * share), (unsigned)pl.L);
    RELAY_CUDA(launch_pdl(orth_convert_kernel<T>, grid, dim3(kNormThreads), 0, st, (const T *)x->data, (int)pl.M, (int)pl.N, (int)(pl.N % 8 == 0),
                          (const double *)partial, partials, eps, s, out, (long long)pl.xld, done));
    return check_launch("orthogonalize_convert");
}

}  // namespace
}  // namespace relay

using namespace relay;

extern "C" size_t relay_workspace_bytes_orthogonalize(const relay_tensor_t *x)
{
    clear_error();
    if (check_matrices(x) != RELAY_OK || numel(x) == 0) return 0;
    return plan_of(x).total;
}

extern "C" relay_status_t relay_orthogonalize(const relay_tensor_t *x, const relay_orthogonalize_attrs_t *at, const relay_tensor_t *y, void *ws,
                                              size_t ws_bytes, void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(x, "x"));
    RELAY_TRY(check_not_null(at, "attrs"));
    RELAY_TRY(check_not_null(y, "y"));
    RELAY_TRY(check_matrices(x));
    RELAY_TRY(check_type(y, "y"));
    RELAY_TRY(check_rank(y, x->rank, "y"));
    RELAY_TRY(check_dtype(y, RELAY_BF16, "y"));
    RELAY_TRY(check_layout(y, RELAY_ROWMAJOR, RELAY_ROWMAJOR, "y"));
    RELAY_TRY(check_shape_n(y, x->shape, x->rank, "y"));
    if (at->steps < 1 || at->steps > 16) return fail(RELAY_ERR_ATTR, "steps = %d, needs 1..16", at->steps);
    if (!std::isfinite(at->a) || !std::isfinite(at->b) || !std::isfinite(at->c) || !std::isfinite(at->scale))
        return fail(RELAY_ERR_ATTR, "a coefficient or the scale is not finite");
    if (!(at->eps >= 0.0f) || !std::isfinite(at->eps)) return fail(RELAY_ERR_ATTR, "eps = %g, needs a finite number of at least 0", (double)at->eps);
    RELAY_TRY(check_data(x, "x"));
    RELAY_TRY(check_data(y, "y"));
    const relay_tensor_t *ins[1] = {x}, *outs[1] = {y};
    RELAY_TRY(check_no_overlap(outs, 1, ins, 1));
    if (numel(x) == 0) return RELAY_OK;
    const Plan pl = plan_of(x);
    RELAY_TRY(check_workspace(ws, ws_bytes, pl.total));
    cudaStream_t st = (cudaStream_t)stream;
    if (pl.small) {
        BoundsReg reg;
        reg.add(x); reg.add(y);
        RELAY_TRY(reg.commit(st));
        const Steps steps = steps_of(*at, 1.0);
        if (x->dtype == RELAY_F32) return launch_small<float>(x, steps, at->eps, y, pl.L, (int)pl.M, (int)pl.N, st);
        return launch_small<__nv_bfloat16>(x, steps, at->eps, y, pl.L, (int)pl.M, (int)pl.N, st);
    }
    const float s = exp2f(roundf(log2f(sqrtf((float)pl.M * (float)pl.N) / 8.0f)));
    const Steps steps = steps_of(*at, s);
    if (pl.resident) return launch_resident(x, steps, at->eps, y, pl.L, (int)pl.M, (int)pl.N, s, st);
    int dev = 0, sms = 148;
    RELAY_CUDA(cudaGetDevice(&dev));
    RELAY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    int *err = device_error_word();
    if (!err) return fail(RELAY_ERR_CUDA, "no device error word");

    char *w = (char *)ws;
    auto take = [&](size_t bytes) { char *at = w; w += bytes; return at; };
    double *partial = (double *)take(pl.n_bytes);
    __half *x0 = (__half *)take(pl.x_bytes), *x1 = (__half *)take(pl.x_bytes);
    __half *g = (__half *)take(pl.g_bytes), *q = (__half *)take(pl.g_bytes);
    float *d = (float *)take(pl.v_bytes), *e = (float *)take(pl.v_bytes);

    Launch l;
    l.done = (unsigned int *)w;
    l.tall = pl.M > pl.N; l.step = steps; l.batch = (int)pl.L; l.err = err;
    l.x[0] = x0; l.x[1] = x1;
    // operands: boxes of 128 rows (A) or 64 (B) x 64 contiguous contraction elements, or 64 contraction rows x 64 contiguous columns
    const uint64_t M = pl.M, N = pl.N, m = pl.m, L = pl.L, xld = pl.xld, gld = pl.gld;
    for (int i = 0; i < 2; ++i) {
        RELAY_TRY(make_tmap_3d_f16(&l.map[X_K0 + i], l.x[i], N, M, L, xld, M * xld, 64, 128));
        RELAY_TRY(make_tmap_3d_f16(&l.map[X_K64_0 + i], l.x[i], N, M, L, xld, M * xld, 64, 64));
        RELAY_TRY(make_tmap_3d_f16(&l.map[X_MN0 + i], l.x[i], N, M, L, xld, M * xld, 64, 64));
        const __half *sq = i ? q : g;
        RELAY_TRY(make_tmap_3d_f16(&l.map[i ? P_K : G_K], sq, m, m, L, gld, m * gld, 64, 128));
        RELAY_TRY(make_tmap_3d_f16(&l.map[i ? P_K64 : G_K64], sq, m, m, L, gld, m * gld, 64, 64));
    }

    Product &pg = l.product[0], &pp = l.product[1], &px = l.product[2];
    for (Product &p : l.product) p = Product{};
    for (Product *p : {&pg, &pp}) {
        p->rows = p->cols = (int)m;
        p->symmetric = 1;
        p->out_ld = gld; p->out_bs = (long long)(m * gld);
        p->v_bs = gld;
    }
    pg.k_blocks = (int)((pl.n + 63) / 64);
    pg.a_mn = pg.b_mn = l.tall;
    pg.alpha = 1.0f / (s * s);
    pg.out = g;
    pg.diag = d;
    pp.k_blocks = (int)((m + 63) / 64);
    pp.row_v = pp.col_v = d;
    pp.add = g; pp.add_ld = gld; pp.add_bs = (long long)(m * gld);
    pp.out = q;
    pp.diag = e;                                           // its coefficients are the step's
    px.rows = (int)M; px.cols = (int)N;
    px.k_blocks = pp.k_blocks;
    px.b_mn = !l.tall;
    px.alpha = px.gamma = 1.0f;
    (l.tall ? px.col_v : px.row_v) = e;
    px.v_bs = gld;
    px.add_ld = px.out_ld = xld; px.add_bs = px.out_bs = (long long)(M * xld);
    l.product[3] = px;
    l.product[3].alpha = l.product[3].gamma = steps.scale / s;
    l.product[3].out = y->data; l.product[3].out_ld = N; l.product[3].out_bs = (long long)(M * N); l.product[3].out_bf16 = 1;

    BoundsReg reg;
    reg.add(x); reg.add(y); reg.add(ws, ws_bytes);
    RELAY_TRY(reg.commit(st));
    if (x->dtype == RELAY_F32) RELAY_TRY(prepare_x<float>(x, pl, partial, at->eps, s, sms, x0, l.done, st));
    else RELAY_TRY(prepare_x<__nv_bfloat16>(x, pl, partial, at->eps, s, sms, x0, l.done, st));
    return launch_products(l, sms, st);
}
