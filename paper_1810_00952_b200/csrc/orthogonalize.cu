// Orthogonalised update of weight matrices by Newton-Schulz products.
//
//   X <- x / (|x|_F + eps);   `steps` times:  G = X X^T,  P = b G + c G G,  X <- a X + P X        (M <= N; m = M, n = N)
//                                             G = X^T X,  P = b G + c G G,  X <- a X + X P        (M >  N; m = N, n = M)
//   y = scale X
//
// Three products a step on the tensor cores (tcgen05, kind::f16).  G and P are symmetric: only the tiles on and above the
// diagonal are computed, each stored to both places, so a step costs m m n + m m m + 2 m m n operations.  The operands lie in
// the workspace as fp16: at the tensor rate of bf16 it keeps 10 fraction bits instead of 7, and with them an update that is 1e-3
// instead of 1e-2 off.  Range is no concern: singular values never leave [0, 1.3], X is kept times a power of two,
// S = 2^round(log2(sqrt(M N) / 8)), which puts its elements around 1/8 at the start and below 0.16 sqrt(M N) ever after, and
// what is too small for fp16 in G and P is small against the diagonal.  The diagonals of G and P, whose entries grow to 1 and -2.7
// and whose rounding would move whole rows, are kept apart in fp32: with G = D + O,
//   P = b O + c (D O + O D + O O) off the diagonal,  e = a + b d + c (d d + diag(O O)) on it,   X <- e X + offdiag(P) X
// (one multiplier per row of X, per column where M > N), all of it in the products' epilogues.
//
// A matrix that is small enough is done by one block in shared memory in fp32, all steps in one launch.
#include <algorithm>
#include <cmath>
#include <cuda_fp16.h>

#include "common.h"
#include "ewise_kernels.cuh"
#include "orthogonalize.cuh"

namespace relay {

namespace {

using namespace orth;

constexpr int BM = 128, BN = 128, BK = 64, STAGES = 6;
constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int MN_BOX_BYTES = 64 * BK * 2;              // one TMA box of an operand whose row index is contiguous
constexpr int NUM_THREADS = 192;                       // warp 0 TMA producer, warp 1 MMA issuer, warps 2-5 epilogue
constexpr int TMEM_COLS = 256;                         // two accumulators
constexpr size_t SMEM_BYTES = 1024 + (size_t)STAGES * STAGE_BYTES + 256;

// ---- norm and the 16-bit copy ----------------------------------------------------------------------------
constexpr int kNormThreads = 256;
constexpr int kNormMost = 256;                         // partial sums per matrix, at most

template <typename T>
__device__ __forceinline__ float element(const T *p)
{
    if (!relay_in_bounds(p, sizeof(T))) return 0.0f;
    if constexpr (sizeof(T) == 2) return __bfloat162float(*p);
    else return *p;
}
// eight consecutive elements; whole: they are 16-byte aligned
template <typename T>
__device__ __forceinline__ void eight(const T *p, bool whole, int n, float (&x)[8])
{
    if (whole) {
        if constexpr (sizeof(T) == 2) {
            unpack(ld_stream(p), x);
        } else {
            float lo[4], hi[4];
            unpack(ld_stream(p), lo);
            unpack(ld_stream(p + 4), hi);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = lo[i]; x[4 + i] = hi[i]; }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < n ? element(p + i) : 0.0f;
    }
}

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

// out = fp16(x s / (|x| + eps)), rows padded to ld; a thread takes eight columns of a row at a time
template <typename T>
__global__ void __launch_bounds__(kNormThreads) orth_convert_kernel(const T *__restrict__ x, int rows, int cols, int even, const double *__restrict__ partial, int partials,
                                                                   float eps, float s, __half *__restrict__ out, long long ld)
{
    __shared__ double warp_sum[kNormThreads / 32];
    pdl_wait();
    const long long b = blockIdx.y;
    double sum = threadIdx.x < partials ? partial[b * partials + threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < kNormThreads / 32; ++i) sum += warp_sum[i];
    // in two factors, each of them within fp32's range where the whole may not be
    const double f = (double)s / (sqrt(sum) + (double)eps);
    int e;
    const float lo = (float)frexp(f, &e);
    const float f1 = ldexpf(lo, e / 2), f2 = ldexpf(1.0f, e - e / 2);
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

// ---- products ----------------------------------------------------------------------------------------------
__device__ __forceinline__ Tile tile_of(const Product &p, int unit)
{
    Tile t;
    t.batch = unit / p.units;
    int u = unit - t.batch * p.units;
    if (p.symmetric) {                                 // u = j (j + 1) / 2 + i,  i <= j
        int j = (int)((sqrtf(8.0f * (float)u + 1.0f) - 1.0f) * 0.5f);
        while (j * (j + 1) / 2 > u) --j;
        while ((j + 1) * (j + 2) / 2 <= u) ++j;
        const int i = u - j * (j + 1) / 2;
        t.m0 = i * BM; t.n0 = j * BN; t.mirror = i != j;
    } else {
        t.m0 = (u % p.tiles_m) * BM; t.n0 = (u / p.tiles_m) * BN; t.mirror = false;
    }
    return t;
}

template <bool A_MN, bool B_MN>
__global__ void __launch_bounds__(NUM_THREADS, 1)
orth_product_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const Product p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + (size_t)STAGES * STAGE_BYTES);
    uint64_t *full = bars, *empty = bars + STAGES, *tmem_full = bars + 2 * STAGES, *tmem_empty = bars + 2 * STAGES + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * STAGES + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int n_units = p.units * p.batch;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { tc::mbar_init(&full[s], 1); tc::mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { tc::mbar_init(&tmem_full[b], 1); tc::mbar_init(&tmem_empty[b], 4); }
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tmap(&tm_a);
        tc::prefetch_tmap(&tm_b);
    }
    if (warp == 1) {
        tc::tmem_alloc(tmem_slot, TMEM_COLS);
        tc::tmem_relinquish();
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();

    if (warp == 0) {
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int unit = blockIdx.x; unit < n_units && ok; unit += gridDim.x) {
            const Tile t = tile_of(p, unit);
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(&empty[s], phase ^ 1, abort_flag, p.err, tc::ERR_WAIT_EMPTY));
                if (!ok) break;
                uint8_t *sa = smem + (size_t)s * STAGE_BYTES, *sb = sa + A_BYTES;
                const int k0 = kb * BK;
                if (tc::elect_one()) {
                    tc::mbar_expect_tx(&full[s], STAGE_BYTES);
                    if (A_MN) {
#pragma unroll
                        for (int i = 0; i < BM / 64; ++i) tc::tma_load_3d(sa + i * MN_BOX_BYTES, &tm_a, &full[s], t.m0 + i * 64, k0, t.batch);
                    } else {
                        tc::tma_load_3d(sa, &tm_a, &full[s], k0, t.m0, t.batch);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int i = 0; i < BN / 64; ++i) tc::tma_load_3d(sb + i * MN_BOX_BYTES, &tm_b, &full[s], t.n0 + i * 64, k0, t.batch);
                    } else {
                        tc::tma_load_3d(sb, &tm_b, &full[s], k0, t.n0, t.batch);
                    }
                }
                __syncwarp();
                if (++s == STAGES) { s = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1) {
        constexpr uint32_t idesc = instr_desc_f16(BM, BN, A_MN, B_MN);
        constexpr uint32_t a_lbo = A_MN ? MN_BOX_BYTES : 16, b_lbo = B_MN ? MN_BOX_BYTES : 16;
        constexpr uint32_t a_step = A_MN ? 2048 : 32, b_step = B_MN ? 2048 : 32;
        const uint64_t desc_a0 = tc::smem_desc(tc::smem_u32(smem), a_lbo, 1024);
        const uint64_t desc_b0 = tc::smem_desc(tc::smem_u32(smem) + A_BYTES, b_lbo, 1024);
        uint32_t local = 0, phase = 0, stage_off = 0;
        int s = 0;
        bool ok = true;
        for (int unit = blockIdx.x; unit < n_units && ok; unit += gridDim.x, ++local) {
            const int buf = local & 1;
            if (!__all_sync(0xffffffffu, tc::mbar_wait(&tmem_empty[buf], ((local >> 1) & 1) ^ 1, abort_flag, p.err, tc::ERR_WAIT_TMEM_EMPTY))) break;
            tc::tc_fence_after_sync();
            const uint32_t d_tmem = tmem_base + buf * BN;
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[s], phase, abort_flag, p.err, tc::ERR_WAIT_FULL));
                if (!ok) break;
                tc::tc_fence_after_sync();
                const uint64_t da = desc_a0 + stage_off, db = desc_b0 + stage_off;
#pragma unroll
                for (int kk = 0; kk < BK / 16; ++kk)
                    tc::mma_bf16_elect(d_tmem, da + ((kk * a_step) >> 4), db + ((kk * b_step) >> 4), idesc, (uint32_t)(kb != 0 || kk != 0));
                tc::mma_commit_elect(&empty[s]);
                stage_off += STAGE_BYTES >> 4;
                if (++s == STAGES) { s = 0; phase ^= 1; stage_off = 0; }
            }
            if (ok) tc::mma_commit_elect(&tmem_full[buf]);
        }
    } else {
        const int quarter = warp & 3;
        uint32_t local = 0;
        for (int unit = blockIdx.x; unit < n_units; unit += gridDim.x, ++local) {
            const int buf = local & 1;
            const Tile t = tile_of(p, unit);
            int ok = 1;
            if (lane == 0) ok = tc::mbar_wait(&tmem_full[buf], (local >> 1) & 1, abort_flag, p.err, tc::ERR_WAIT_TMEM_FULL) ? 1 : 0;
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            tc::tc_fence_after_sync();
            const int row = t.m0 + quarter * 32 + lane;
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * BN;
#pragma unroll 1
            for (int g = 0; g < BN / 32; ++g) {
                uint32_t acc[32];
                tc::tmem_ld_32x32(taddr + g * 32, acc);
                tc::tmem_ld_wait();
                finish_columns(p, t, lane, row, t.n0 + g * 32, acc);
            }
            tc::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&tmem_empty[buf]);
        }
    }

    tc::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc::tc_fence_after_sync();
        tc::tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

relay_status_t launch_product(const Product &p, bool a_mn, bool b_mn, const CUtensorMap &ta, const CUtensorMap &tb, int sms, cudaStream_t st)
{
    const dim3 grid((unsigned)std::min<long long>((long long)p.units * p.batch, sms));
#define LAUNCH(AMN, BMN)                                                                                                              \
    do {                                                                                                                              \
        RELAY_CUDA(cudaFuncSetAttribute(orth_product_kernel<AMN, BMN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_BYTES)); \
        RELAY_CUDA(launch_pdl(orth_product_kernel<AMN, BMN>, grid, dim3(NUM_THREADS), SMEM_BYTES, st, ta, tb, p));                     \
    } while (0)
    if (a_mn && b_mn) LAUNCH(true, true);
    else if (b_mn) LAUNCH(false, true);
    else LAUNCH(false, false);
#undef LAUNCH
    return check_launch("orthogonalize_product");
}

// ---- small matrices: one block each -----------------------------------------------------------------------------
constexpr int kSmallThreads = 256;
constexpr int64_t kSmallSide = 64, kSmallSize = 64 * 96;
// rows of shared memory: whole float4, an odd number of them, so that rows next to each other start on other banks
__host__ __device__ inline int small_ld(int n) { return ((n + 3) / 4 | 1) * 4; }
inline bool small_fits(int64_t m, int64_t n) { return m <= kSmallSide && m * n <= kSmallSize; }
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
__global__ void __launch_bounds__(kSmallThreads) orth_small_kernel(const T *__restrict__ x, int M, int N, int steps, float a, float b, float c, float eps, float scale,
                                                                  __nv_bfloat16 *__restrict__ y)
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
    for (int k = 0; k < steps; ++k) {
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
        if (relay_in_bounds(y + i, 2)) y[i] = __float2bfloat16_rn(scale * X[tall ? q * ldx + r : r * ldx + q]);
    }
}

template <typename T>
relay_status_t launch_small(const relay_tensor_t *x, const relay_orthogonalize_attrs_t *at, const relay_tensor_t *y, int64_t L, int M, int N, cudaStream_t st)
{
    const size_t smem = small_smem(std::min(M, N), std::max(M, N));
    RELAY_CUDA(cudaFuncSetAttribute(orth_small_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024));
    RELAY_CUDA(launch_pdl(orth_small_kernel<T>, dim3((unsigned)L), dim3(kSmallThreads), smem, st, (const T *)x->data, M, N, at->steps, at->a, at->b, at->c, at->eps,
                          at->scale, (__nv_bfloat16 *)y->data));
    return check_launch("orthogonalize_small");
}

// Matrices whose shorter side has at least this many entries go to the two-SM kernel.
constexpr int64_t kPairSide = 256;

// ---- workspace -------------------------------------------------------------------------------------------------
struct Plan {
    int64_t L, M, N, m, n;             // matrices; m = min(M, N), n = max(M, N)
    int64_t xld, gld;                  // row strides of X (rows M, N columns) and G, P (m x m), in elements
    size_t x_bytes, g_bytes, v_bytes, total;
    bool small;
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
    p.total = align_up((size_t)p.L * kNormMost * sizeof(double), 256) + 2 * p.x_bytes + 2 * p.g_bytes + 2 * p.v_bytes;
    p.small = small_fits(p.m, p.n);
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
relay_status_t prepare_x(const relay_tensor_t *x, const Plan &pl, double *partial, float eps, float s, int sms, __half *out, cudaStream_t st)
{
    const long long size = pl.M * pl.N, each = kNormThreads * 8;
    const int share = (int)std::max<int64_t>(1, 4 * sms / pl.L);             // blocks per matrix that fill the GPU
    const int partials = (int)std::min<long long>({(size + each - 1) / each, share, kNormMost});
    RELAY_CUDA(launch_pdl(orth_norm_kernel<T>, dim3((unsigned)partials, (unsigned)pl.L), dim3(kNormThreads), 0, st, (const T *)x->data, size, (int)(size % 8 == 0), partial));
    RELAY_TRY(check_launch("orthogonalize_norm"));
    const dim3 grid((unsigned)std::min<long long>((pl.M * ((pl.N + 7) / 8) + kNormThreads - 1) / kNormThreads, 2 * share), (unsigned)pl.L);
    RELAY_CUDA(launch_pdl(orth_convert_kernel<T>, grid, dim3(kNormThreads), 0, st, (const T *)x->data, (int)pl.M, (int)pl.N, (int)(pl.N % 8 == 0),
                          (const double *)partial, partials, eps, s, out, (long long)pl.xld));
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
        if (x->dtype == RELAY_F32) return launch_small<float>(x, at, y, pl.L, (int)pl.M, (int)pl.N, st);
        return launch_small<__nv_bfloat16>(x, at, y, pl.L, (int)pl.M, (int)pl.N, st);
    }
    int dev = 0, sms = 148;
    RELAY_CUDA(cudaGetDevice(&dev));
    RELAY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    int *err = device_error_word();
    if (!err) return fail(RELAY_ERR_CUDA, "no device error word");

    char *w = (char *)ws;
    double *partial = (double *)w;
    w += align_up((size_t)pl.L * kNormMost * sizeof(double), 256);
    __half *xa = (__half *)w, *xb = (__half *)(w + pl.x_bytes);
    __half *g = (__half *)(w + 2 * pl.x_bytes), *q = (__half *)(w + 2 * pl.x_bytes + pl.g_bytes);
    float *d = (float *)(w + 2 * pl.x_bytes + 2 * pl.g_bytes), *e = (float *)(w + 2 * pl.x_bytes + 2 * pl.g_bytes + pl.v_bytes);
    const float s = exp2f(roundf(log2f(sqrtf((float)pl.M * (float)pl.N) / 8.0f)));

    BoundsReg reg;
    reg.add(x); reg.add(y); reg.add(ws, ws_bytes);
    RELAY_TRY(reg.commit(st));
    if (x->dtype == RELAY_F32) RELAY_TRY(prepare_x<float>(x, pl, partial, at->eps, s, sms, xa, st));
    else RELAY_TRY(prepare_x<__nv_bfloat16>(x, pl, partial, at->eps, s, sms, xa, st));

    const bool tall = pl.M > pl.N;
    // boxes: 128 rows x 64 contiguous contraction elements, or 64 contraction rows x 64 contiguous rows/columns
    // the two-SM kernel takes its B operand in boxes of 64 rows
    const bool pair = pl.m >= kPairSide && sms >= 2;
    CUtensorMap x_k[2], x_mn[2], g_k, q_k, x_k64[2], g_k64, q_k64;
    for (int i = 0; i < 2; ++i) {
        const __half *b = i ? xb : xa;
        RELAY_TRY(make_tmap_3d_f16(&x_k[i], b, pl.N, pl.M, pl.L, pl.xld, pl.M * pl.xld, BK, 128));
        RELAY_TRY(make_tmap_3d_f16(&x_mn[i], b, pl.N, pl.M, pl.L, pl.xld, pl.M * pl.xld, 64, BK));
        RELAY_TRY(make_tmap_3d_f16(&x_k64[i], b, pl.N, pl.M, pl.L, pl.xld, pl.M * pl.xld, BK, 64));
    }
    RELAY_TRY(make_tmap_3d_f16(&g_k64, g, pl.m, pl.m, pl.L, pl.gld, pl.m * pl.gld, BK, 64));
    RELAY_TRY(make_tmap_3d_f16(&q_k64, q, pl.m, pl.m, pl.L, pl.gld, pl.m * pl.gld, BK, 64));
    UnitTable plans[3];                                // of the three products of a step
    auto product = [&](const Product &p, int kind, bool first, bool a_mn, bool b_mn, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &b64) {
        if (!pair) return launch_product(p, a_mn, b_mn, a, b, sms, st);
        if (first) plan_units(p, sms, &plans[kind]);
        return launch_product_pair(p, a_mn, b_mn, a, b64, plans[kind], sms, st);
    };
    RELAY_TRY(make_tmap_3d_f16(&g_k, g, pl.m, pl.m, pl.L, pl.gld, pl.m * pl.gld, BK, 128));
    RELAY_TRY(make_tmap_3d_f16(&q_k, q, pl.m, pl.m, pl.L, pl.gld, pl.m * pl.gld, BK, 128));

    const int tm = (int)((pl.m + 127) / 128);
    const long long v_ld = pl.gld;
    Product sym{};                                     // G and P
    sym.rows = sym.cols = (int)pl.m;
    sym.tiles_m = sym.tiles_n = tm;
    sym.units = tm * (tm + 1) / 2;
    sym.batch = (int)pl.L;
    sym.symmetric = 1;
    sym.out_ld = pl.gld; sym.out_bs = pl.m * pl.gld;
    sym.v_bs = v_ld;
    sym.err = err;
    Product up{};                                      // X
    up.rows = (int)pl.M; up.cols = (int)pl.N;
    up.tiles_m = (int)((pl.M + 127) / 128); up.tiles_n = (int)((pl.N + 127) / 128);
    up.units = up.tiles_m * up.tiles_n;
    up.batch = (int)pl.L;
    up.k_blocks = (int)((pl.m + BK - 1) / BK);
    up.v_bs = v_ld;
    (tall ? up.col_v : up.row_v) = e;
    up.err = err;
    for (int k = 0; k < at->steps; ++k) {
        const int cur = k & 1;
        const bool last = k + 1 == at->steps;
        Product p = sym;
        p.k_blocks = (int)((pl.n + BK - 1) / BK);
        p.alpha = 1.0f / (s * s);
        p.out = g;
        p.diag = d;
        if (tall) RELAY_TRY(product(p, 0, k == 0, true, true, x_mn[cur], x_mn[cur], x_mn[cur]));
        else RELAY_TRY(product(p, 0, k == 0, false, false, x_k[cur], x_k[cur], x_k64[cur]));
        p = sym;
        p.k_blocks = (int)((pl.m + BK - 1) / BK);
        p.alpha = at->c; p.beta = at->b; p.gamma = at->c;
        p.row_v = p.col_v = d;
        p.diag = e;
        p.q0 = at->a; p.q1 = at->b; p.q2 = at->c;
        p.add = g; p.add_ld = pl.gld; p.add_bs = pl.m * pl.gld;
        p.out = q;
        RELAY_TRY(product(p, 1, k == 0, false, false, g_k, g_k, g_k64));
        p = up;
        const float f = last ? at->scale / s : 1.0f;
        p.alpha = p.gamma = f;
        p.add = cur ? xb : xa; p.add_ld = pl.xld; p.add_bs = pl.M * pl.xld;
        if (last) { p.out = y->data; p.out_ld = pl.N; p.out_bs = pl.M * pl.N; p.out_bf16 = 1; }
        else { p.out = cur ? xa : xb; p.out_ld = pl.xld; p.out_bs = pl.M * pl.xld; }
        if (tall) RELAY_TRY(product(p, 2, k == 0, false, false, x_k[cur], q_k, q_k64));
        else RELAY_TRY(product(p, 2, k == 0, false, true, q_k, x_mn[cur], x_mn[cur]));
    }
    return RELAY_OK;
}
