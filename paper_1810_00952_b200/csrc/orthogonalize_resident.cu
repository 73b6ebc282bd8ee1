// Orthogonalised updates of matrices that stay on the chip: at most 128 rows (columns, where M > N), all steps in one launch.
//
// One cluster of S = 1..8 blocks per matrix.  Each block keeps a slice of at most 256 of the n columns of X (of X^T where M > N) in
// shared memory as fp16, and copies of G and P: a product's operands never leave the SM.  The slice's layout, groups of 64 columns
// with 128-byte rows swizzled, is K-major for G = X X^T and MN-major for P X at once.  Per step:
//   G      over the slice's columns, accumulated in TMEM; with S > 1 the blocks' parts are sent to the block that owns the row, added
//          there in the order of the blocks, and the sum is sent to all as fp16
//   P      = b G + c G G by every block for itself: 128^3 products are less than an exchange
//   X      <- e X + offdiag(P) X in place
// with the diagonals apart in fp32, as in the products of larger matrices.  Every phase ends in a barrier of the block, so what
// bounds a step is its chain of latencies: three times MMA, TMEM to registers, shared memory (4.8 us at 128 x 256); and the exchange
// of G (3.3 us between two blocks, 5 between eight; by st.async, whose every 16 bytes update a barrier, 5 and 5).
#include <algorithm>

#include "common.h"
#include "orthogonalize.h"
#include "tc_common.cuh"

namespace relay {
namespace orth {
namespace {

constexpr int kThreads = 512, kRows = 128, kWidest = 256, kMostBlocks = 8;
constexpr int kGroup = kRows * 128;                        // bytes of 64 columns

struct Resident {
    int M, N, m, n, tall, S, w;        // w: columns of a slice, a multiple of 32
    float eps, s, scale;
    int steps;
    int *err;
    Steps step;
};
struct Scalars {                       // behind the matrices in shared memory
    float d[kRows], e[kRows];          // the diagonals of G and of a I + P
    float a[kMostSteps], b[kMostSteps], c[kMostSteps];     // the steps' coefficients (indexing the parameters by step instead: 0.1 us a step more)
    double warp_sum[kThreads / 32], norm[kMostBlocks];
    uint64_t bar;
    uint32_t tmem;
    int gave_up;
};
// byte offset of an element (of the 16 bytes that begin with it) in a swizzled matrix of 128 rows
__device__ __forceinline__ uint32_t place(int row, int col)
{
    return (uint32_t)((col >> 6) * kGroup + row * 128 + ((((col >> 3) & 7) ^ (row & 7)) << 4) + (col & 7) * 2);
}
__device__ __forceinline__ void unpack_half(const uint4 &v, float (&x)[8])
{
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&r[i]));
        x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 pack_half(const float (&x)[8])
{
    return make_uint4(pack_half2(x[0], x[1]), pack_half2(x[2], x[3]), pack_half2(x[4], x[5]), pack_half2(x[6], x[7]));
}
__device__ __forceinline__ void st_cluster(uint32_t to, const uint4 &v)
{
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// what was stored to a neighbour's shared memory is to be read by its tensor core
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }

// The slice in registers, as pieces of eight elements that lie together in memory: columns j to j + 7 of row i of X, or, where
// M > N, rows i to i + 7 of column j.  A warp's pieces are next to each other in memory, or four of them by sixteen columns, two
// to a thread: what it stores side by side then shares few banks.
constexpr int kPieces = kRows * kWidest / 8 / kThreads;
struct Pieces {
    int i, j;                          // of the present piece
    int hi, lo, across, by_hi, by_lo, tall;
    __device__ __forceinline__ explicit Pieces(const Resident &q)
    {
        tall = q.tall;
        across = tall ? q.w / 16 : q.w / 8;
        const int first = tall ? (int)(threadIdx.x >> 5) : (int)threadIdx.x, by = tall ? kThreads / 32 : kThreads;
        hi = first / across; lo = first - hi * across;
        by_hi = by / across; by_lo = by - by_hi * across;
        set(0);
    }
    __device__ __forceinline__ void set(int u)
    {
        const int lane = threadIdx.x & 31;
        i = tall ? 8 * (hi * 4 + (lane >> 3)) : hi;
        j = tall ? lo * 16 + (lane & 7) * 2 + (u & 1) : lo * 8;
    }
    __device__ __forceinline__ void next(int u)                       // on from piece u
    {
        if (!tall || (u & 1)) {
            hi += by_hi; lo += by_lo;
            if (lo >= across) { lo -= across; ++hi; }
        }
        set(u + 1);
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 1) orth_resident_kernel(const T *__restrict__ x, __nv_bfloat16 *__restrict__ y, const Resident q)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *X = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int groups = (q.w + 63) / 64;
    uint8_t *G = X + groups * kGroup, *P = G + 2 * kGroup, *parts = P + 2 * kGroup;     // parts: [block][row][128 floats]
    Scalars &sc = *reinterpret_cast<Scalars *>(parts + (q.S > 1 ? kRows * 512 : 0));

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int rank = (int)(blockIdx.x % (unsigned)q.S), mp = (q.m + 31) / 32 * 32;
    const int n0 = rank * q.w, cols = max(0, min(q.w, q.n - n0));
    const long long b = blockIdx.x / (unsigned)q.S;
    const uint32_t tmem_cols = q.w > 128 ? 512 : 256;
    if (tid == 0) {
        tc::mbar_init(&sc.bar, 1);
        sc.gave_up = 0;
        tc::fence_barrier_init();
    }
    if (warp == 0) {
        tc::tmem_alloc(&sc.tmem, tmem_cols);
        tc::tmem_relinquish();
    }
    if (tid < kMostSteps) { sc.a[tid] = q.step.a[tid]; sc.b[tid] = q.step.b[tid]; sc.c[tid] = q.step.c[tid]; }
    for (int i = tid; i < groups * kGroup / 16; i += kThreads) reinterpret_cast<uint4 *>(X)[i] = make_uint4(0, 0, 0, 0);
    tc::tc_fence_before_sync();
    __syncthreads();
    if (q.S > 1) tc::cluster_sync();                       // all blocks of the cluster run from here on
    tc::tc_fence_after_sync();
    const uint32_t tmem = sc.tmem;
    pdl_wait();

    // the slice, its norm, and the slice as fp16
    x += b * q.M * q.N;
    y += b * q.M * q.N;
    float v[kPieces][8];
    const bool whole = q.N % 8 == 0;
    float most = 0.0f;
    Pieces in(q);
#pragma unroll
    for (int u = 0; u < kPieces; ++u, in.next(u - 1)) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u][k] = 0.0f;
        if (in.i >= q.m || in.j >= cols) continue;
        if (q.tall) eight(x + (long long)(n0 + in.j) * q.N + in.i, whole, q.m - in.i, v[u]);
        else eight(x + (long long)in.i * q.N + n0 + in.j, whole, cols - in.j, v[u]);
    }
    // a thread's squares in fp32, of values scaled to the largest one's exponent; their sum goes on in fp64, where any square fits
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(v[u][k]));
    const int exponent = min(__float_as_int(most) >> 23, 253);
    const float unit = __int_as_float((254 - exponent) << 23);
    float squares = 0.0f;
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) { const float t = v[u][k] * unit; squares = fmaf(t, t, squares); }
    double s = (double)squares * __longlong_as_double((long long)(1023 + 2 * (exponent - 127)) << 52);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (lane == 0) sc.warp_sum[warp] = s;
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) s += sc.warp_sum[i];
    if (q.S > 1) {
        if (tid < q.S) asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(tc::mapa(tc::smem_u32(&sc.norm[rank]), (uint32_t)tid)), "d"(s) : "memory");
        tc::cluster_sync();
        s = 0.0;
        for (int i = 0; i < q.S; ++i) s += sc.norm[i];
    }
    float f1, f2;
    normalizer(s, q.eps, q.s, f1, f2);
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u][k] = v[u][k] * f1 * f2;
    Pieces to(q);
#pragma unroll
    for (int u = 0; u < kPieces; ++u, to.next(u - 1)) {
        if (to.i >= q.m || to.j >= cols) continue;
        if (!q.tall) {
            *reinterpret_cast<uint4 *>(X + place(to.i, to.j)) = pack_half(v[u]);
        } else if (u % 2 == 0) {                           // its second column is zero behind the last
#pragma unroll
            for (int k = 0; k < 8; ++k) *reinterpret_cast<uint32_t *>(X + place(to.i + k, to.j)) = pack_half2(v[u][k], v[u + 1][k]);
        }
    }
    tc::fence_proxy_async();
    __syncthreads();

    const int quarter = warp & 3, row = quarter * 32 + lane, c0 = (warp >> 2) * 32;
    const bool mine = quarter * 32 < mp;                   // rows behind mp hold nothing that is read
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t idesc_m = instr_desc_f16(128, mp, 0, 0), idesc_x = instr_desc_f16(128, q.w, 0, 1);
    const uint64_t desc_x = tc::smem_desc(tc::smem_u32(X), 16, 1024), desc_g = tc::smem_desc(tc::smem_u32(G), 16, 1024),
                   desc_p = tc::smem_desc(tc::smem_u32(P), 16, 1024), desc_xn = tc::smem_desc(tc::smem_u32(X), kGroup, 1024);
    auto deep = [](int kk) { return (uint64_t)(((kk >> 2) * kGroup + (kk & 3) * 32) >> 4); };     // 16 contraction indices further, K-major
    uint32_t phase = 0;
    auto wait = [&] {                                      // for the products of this phase, by all
        if (warp == 0) tc::mma_commit_elect(&sc.bar);
        tc::mbar_wait(&sc.bar, phase, &sc.gave_up, q.err, tc::ERR_WAIT_TMEM_FULL);
        phase ^= 1;
        __syncwarp();
        tc::tc_fence_after_sync();
    };
    auto handover = [&] {                                  // of shared memory to the tensor core and of TMEM's columns
        tc::fence_proxy_async();
        tc::tc_fence_before_sync();
        __syncthreads();
        tc::tc_fence_after_sync();
    };
    const float alpha = 1.0f / (q.s * q.s);
    const int k_x = (max(cols, 1) + 15) / 16, k_m = mp / 16, owned = mp / q.S;
    for (int step = 0; step < q.steps; ++step) {
        const bool last = step + 1 == q.steps;
        if (warp == 0)
            for (int kk = 0; kk < k_x; ++kk) tc::mma_bf16_elect(tmem, desc_x + deep(kk), desc_x + deep(kk), idesc_m, kk != 0);
        wait();
        if (mine && c0 < mp) {
            uint32_t acc[32];
            tc::tmem_ld_32x32(tmem + lanes + c0, acc);
            tc::tmem_ld_wait();
            if (q.S == 1) {
#pragma unroll
                for (int j = 0; j < 32; j += 8) {
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        v[k] = alpha * __uint_as_float(acc[j + k]);
                        if (c0 + j + k == row) { sc.d[row] = v[k]; v[k] = 0.0f; }
                    }
                    *reinterpret_cast<uint4 *>(G + place(row, c0 + j)) = pack_half(v);
                }
            } else {
                const int owner = row / owned, at = row - owner * owned;
                const uint32_t to = tc::mapa(tc::smem_u32(parts), (uint32_t)owner) + (uint32_t)(rank * owned + at) * 512;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    st_cluster(to + (uint32_t)(((c0 / 4 + j) ^ (row & 7)) << 4), make_uint4(acc[4 * j], acc[4 * j + 1], acc[4 * j + 2], acc[4 * j + 3]));
            }
        }
        if (q.S > 1) {
            tc::tc_fence_before_sync();
            tc::cluster_sync();
            for (int i = tid; i < owned * (mp / 8); i += kThreads) {
                const int at = i / (mp / 8), c = (i - at * (mp / 8)) * 8, r = rank * owned + at;
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = 0.0f;
                for (int o = 0; o < q.S; ++o) {
                    const uint8_t *from = parts + (o * owned + at) * 512;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 t = *reinterpret_cast<const float4 *>(from + (((c / 4 + h) ^ (r & 7)) << 4));
                        v[4 * h] += t.x; v[4 * h + 1] += t.y; v[4 * h + 2] += t.z; v[4 * h + 3] += t.w;
                    }
                }
                const bool diagonal = r >= c && r < c + 8;
                float d = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] *= alpha;
                    if (c + k == r) { d = v[k]; v[k] = 0.0f; }
                }
                const uint4 g = pack_half(v);
                for (int o = 0; o < q.S; ++o) {
                    st_cluster(tc::mapa(tc::smem_u32(G + place(r, c)), (uint32_t)o), g);
                    if (diagonal) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(tc::mapa(tc::smem_u32(&sc.d[r]), (uint32_t)o)), "f"(d) : "memory");
                }
            }
            // Behind this barrier every block has read its parts: they may be sent again.  G is sent again only behind the next
            // step's first barrier, which follows every block's last look at this one.
            fence_proxy_async_all();
            tc::cluster_sync();
            fence_proxy_async_all();
            tc::tc_fence_after_sync();
        } else {
            handover();
        }

        if (warp == 0)
            for (int kk = 0; kk < k_m; ++kk) tc::mma_bf16_elect(tmem, desc_g + deep(kk), desc_g + deep(kk), idesc_m, kk != 0);
        wait();
        if (mine && c0 < mp) {
            uint32_t acc[32];
            tc::tmem_ld_32x32(tmem + lanes + c0, acc);
            const float d_row = sc.d[row], ka = sc.a[step], kb = sc.b[step], kc = sc.c[step];
            tc::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                float v[8];
                unpack_half(*reinterpret_cast<const uint4 *>(G + place(row, c0 + j)), v);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float gg = __uint_as_float(acc[j + k]);
                    v[k] = fmaf(kc, gg, fmaf(kc, d_row + sc.d[c0 + j + k], kb) * v[k]);
                    if (c0 + j + k == row) {
                        sc.e[row] = ka + d_row * kb + kc * fmaf(d_row, d_row, gg);
                        v[k] = 0.0f;
                    }
                }
                *reinterpret_cast<uint4 *>(P + place(row, c0 + j)) = pack_half(v);
            }
        }
        handover();

        if (warp == 0)
            for (int kk = 0; kk < k_m; ++kk) tc::mma_bf16_elect(tmem + 128, desc_p + deep(kk), desc_xn + (uint64_t)(kk * 2048 >> 4), idesc_x, kk != 0);
        wait();
        if (mine) {
            const float e_row = sc.e[row], out = q.scale / q.s;
            for (int c = c0; c < q.w; c += 128) {
                uint32_t acc[32];
                tc::tmem_ld_32x32(tmem + 128 + lanes + c, acc);
                tc::tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; j += 8) {
                    uint4 *at = reinterpret_cast<uint4 *>(X + place(row, c + j));
                    float v[8];
                    unpack_half(*at, v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = fmaf(e_row, v[k], __uint_as_float(acc[j + k]));
                    if (!last) {
                        *at = pack_half(v);
                        continue;
                    }
                    __nv_bfloat16 h[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) h[k] = __float2bfloat16_rn(out * v[k]);
                    if (q.tall) {                          // a warp's rows lie next to each other in y
                        __nv_bfloat16 *to = y + (long long)(n0 + c + j) * q.N + row;
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (row < q.m && c + j + k < cols && relay_in_bounds(to + (long long)k * q.N, 2)) to[(long long)k * q.N] = h[k];
                    } else {
                        *at = *reinterpret_cast<const uint4 *>(h);
                    }
                }
            }
        }
        handover();
    }
    if (!q.tall) {
        if (q.N % 8 == 0) {
            const int across = cols / 8;
            for (int i = tid; i < q.m * across; i += kThreads) {
                const int r = i / across, c = (i - r * across) * 8;
                __nv_bfloat16 *to = y + (long long)r * q.N + n0 + c;
                if (relay_in_bounds(to, 16)) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(X + place(r, c));
            }
        } else {
            for (int i = tid; i < q.m * cols; i += kThreads) {
                const int r = i / cols, c = i - r * cols;
                __nv_bfloat16 *to = y + (long long)r * q.N + n0 + c;
                if (relay_in_bounds(to, 2)) *to = *reinterpret_cast<const __nv_bfloat16 *>(X + place(r, c));
            }
        }
    }
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, tmem_cols);
}

constexpr size_t smem_bytes(int w, bool parts) { return 1024 + (size_t)((w + 63) / 64 + 4) * kGroup + (parts ? kRows * 512 : 0) + sizeof(Scalars); }

template <typename T>
relay_status_t launch(const relay_tensor_t *x, const relay_tensor_t *y, int64_t L, const Resident &q, size_t smem, cudaStream_t st)
{
    // the most that any shape needs: the attribute is the kernel's, and another thread may be launching a larger matrix
    RELAY_CUDA(cudaFuncSetAttribute(orth_resident_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(kWidest, true)));
    RELAY_CUDA(launch_pdl_cluster(orth_resident_kernel<T>, dim3((unsigned)(L * q.S)), dim3(kThreads), dim3((unsigned)q.S), smem, st, (const T *)x->data,
                                  (__nv_bfloat16 *)y->data, q));
    return check_launch("orthogonalize_resident");
}

}  // namespace

bool resident_fits(int64_t m, int64_t n) { return m <= kRows && n <= (int64_t)kMostBlocks * kWidest; }

relay_status_t launch_resident(const relay_tensor_t *x, const Steps &steps, float eps, const relay_tensor_t *y, int64_t L, int M, int N, float s, cudaStream_t st)
{
    Resident q;
    q.M = M; q.N = N; q.m = std::min(M, N); q.n = std::max(M, N);
    q.tall = M > N;
    q.S = 1;
    while (q.S * kWidest < q.n) q.S *= 2;
    q.w = ((q.n + q.S - 1) / q.S + 31) / 32 * 32;
    q.step = steps; q.steps = steps.n; q.scale = steps.scale; q.eps = eps; q.s = s;
    q.err = device_error_word();
    if (!q.err) return fail(RELAY_ERR_CUDA, "no device error word");
    BoundsReg reg;
    reg.add(x); reg.add(y);
    RELAY_TRY(reg.commit(st));
    if (x->dtype == RELAY_F32) return launch<float>(x, y, L, q, smem_bytes(q.w, q.S > 1), st);
    return launch<__nv_bfloat16>(x, y, L, q, smem_bytes(q.w, q.S > 1), st);
}

}  // namespace orth
}  // namespace relay
