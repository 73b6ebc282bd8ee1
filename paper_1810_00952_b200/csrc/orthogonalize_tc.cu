// All products of an orthogonalisation in one launch on pairs of SMs (tcgen05, cta_group::2): per step G = X X^T, P = b G + c G G
// and X <- e X + offdiag(P) X, 256 rows x up to 512 columns per pair and unit.
//
// What bounds a product here is how fast an SM can fill its shared memory (about 48 bytes a cycle): a k-step of 64 over 256 x 128 c
// columns costs a pair max(256 c cycles of MMA, (16 + 8 c) KB per SM / 48 B).  256 x 512 (c = 4) balances the two, but fills both
// TMEM accumulators, so its epilogue is not overlapped; c <= 2 leaves the other accumulator to the next unit.  The host cuts each
// product into units of 64 columns or c = 1..4 chunks of 128, whichever cut finishes first (see plan below): small matrices into
// units of 64, whose epilogue, the part of a phase that nothing hides, is the shortest.  Symmetric products have
// units on and above the diagonal only.
//
// The pairs run through all units of all phases (three per step) in one order.  A unit of matrix b needs every unit of b's phase
// before: each epilogue warp counts itself into done[b] when its stores have landed, and loaders and epilogue wait for the count.
// Matrices of a batch so run into each other's phases, and between two phases of one matrix lie a few microseconds instead of the
// end of one kernel and the start of the next.  Pairs wait for units of other pairs, so all of them have to run at once: the grid is
// no larger than what fits an empty GPU, and the cooperative launch places it whole or, while other work holds SMs, not yet (3 x
// 500 x 333: 114 us against 112 with a launch that overlaps the copy before it).  Every unit's needs come before it in the order, and
// all waits are bounded.
//
// Measured at 4096 x 4096: 1.33 ms, 1.04 PFLOP/s; per step of 222 us the MMAs take 163 (at the power-limited clock) and the three
// changes of phase 59, in which the last unit's epilogue runs with all SMs storing at once.  One launch per product: 1.39 ms for 8 x 1024
// x 4096 against 0.84, 194 us for 3 x 500 x 333 against 122 (114 since units of 64 columns).  Epilogues with TMA stores, with sixteen warps
// (whose registers spill in every unit), or in line with the roles were slower; this form keeps some 100 bytes of a unit's terms on the stack.
//
// Roles per block: warp 0 loads A, the last warp loads B, warp 1 of the leader issues the MMAs, eight warps are the epilogue.  full[] lives
// in the leader; empty[] and tmem_full[] in each block, by multicast commits; tmem_empty[] in the leader.
#include <algorithm>
#include <atomic>
#include <cuda_fp16.h>

#include "common.h"
#include "ewise_kernels.cuh"
#include "orthogonalize.h"
#include "tc_common.cuh"

namespace relay {
namespace orth {
namespace {

constexpr int BK = 64, BN = 256;                           // BN: columns of one accumulator
constexpr int A_BYTES = 128 * BK * 2;                      // this block's 128 rows of A: 16 KB
constexpr int CHUNK_BYTES = 64 * BK * 2;                   // this block's 64 columns of one 128-column chunk: 8 KB
constexpr int MN_BOX_BYTES = 64 * BK * 2;
constexpr int RING_BYTES = 192 * 1024;
constexpr int EPI_WARPS = 8, NUM_THREADS = 32 * (3 + EPI_WARPS), TMEM_COLS = 512;     // registers for a group and the next one's addend
constexpr int WARP_STAGE = 2 * 2048 + 128;                 // per epilogue warp: two 32 x 32 blocks of 16-bit values, 32 floats
constexpr int STAGING_BYTES = EPI_WARPS * WARP_STAGE;
constexpr size_t SMEM_BYTES = 1024 + (size_t)RING_BYTES + STAGING_BYTES + 512;
constexpr unsigned int kArrivals = 2 * EPI_WARPS;          // per unit

__host__ __device__ constexpr int cls_stages(int c) { return c == 1 ? 8 : c == 2 ? 6 : 4; }
__host__ __device__ constexpr int cls_stage_bytes(int c) { return A_BYTES + c * CHUNK_BYTES; }
__host__ __device__ constexpr int cls_bar_base(int c) { return c == 1 ? 0 : c == 2 ? 16 : c == 3 ? 28 : 36; }   // full[], then empty[]
constexpr int BAR_TMEM = 44;                               // tmem_full[2], tmem_empty[2]

// Each width class has barriers of its own over the same shared memory.  A class that is left and taken up again goes on where it
// stood: its barriers remember how often their stages went round.
struct Rings {
    uint32_t at = 0;                   // per class: stage (at most 7), and its phase in the fourth bit
    __device__ __forceinline__ void leave(int c, int s, uint32_t phase)
    {
        if (c > 0) at = (at & ~(15u << (4 * (c - 1)))) | (((uint32_t)s | phase << 3) << (4 * (c - 1)));
    }
    __device__ __forceinline__ void resume(int c, int &s, uint32_t &phase) const
    {
        const uint32_t v = at >> (4 * (c - 1));
        s = (int)(v & 7u);
        phase = (v >> 3) & 1u;
    }
};

struct Unit { int batch, m0, n0, width; };

// A walk through this pair's units: phase after phase, in each every n_pairs-th unit, going on where the phase before left off.
struct Walk {
    const Launch &l;
    int pair, pairs;
    int phase, kind, cur;              // kind: 0 G, 1 P, 2 X;  cur: X's buffer that is read
    long long unit, units;             // of the phase, all matrices
    unsigned int need;                 // done[b] before a unit of this phase may run
    int first;
    __device__ __forceinline__ Walk(const Launch &l_, int pair_, int pairs_) : l(l_), pair(pair_), pairs(pairs_), phase(-1), kind(2), cur(1), unit(0), units(0), need(0), first(0)
    {
        enter();
    }
    __device__ __forceinline__ const Product &product() const { return l.product[phase == 3 * l.step.n - 1 ? 3 : kind]; }
    __device__ __forceinline__ int per_matrix() const { return l.product[kind].units; }
    __device__ __forceinline__ void enter()
    {
        do {
            if (phase >= 0) {
                need += kArrivals * (unsigned)per_matrix();
                first = (int)((first + units) % pairs);
            }
            ++phase;
            if (++kind == 3) { kind = 0; cur ^= 1; }
            units = (long long)per_matrix() * l.batch;
            unit = pair - first;
            if (unit < 0) unit += pairs;
        } while (unit >= units && phase < 3 * l.step.n);
    }
    __device__ __forceinline__ bool more() const { return phase < 3 * l.step.n; }
    __device__ __forceinline__ void next()
    {
        unit += pairs;
        if (unit >= units) enter();
    }
    __device__ __forceinline__ Unit at() const
    {
        Unit w;
        const UnitTable &t = l.table[kind];
        if (t.n > 0) {
            w.batch = (int)(unit / t.n);                   // matrix by matrix: while the last ones are in this phase, the first have
            const uint32_t e = t.e[unit - (long long)w.batch * t.n];       // long been counted and can enter the next
            w.m0 = (int)(e & 0xffu) * 256;
            w.n0 = (int)((e >> 8) & 0x7ffu) * 64;
            w.width = (int)(e >> 19) * 64;
            return w;
        }
        const Product &p = l.product[kind];
        w.batch = (int)(unit / p.units);
        const int v = (int)(unit - (long long)w.batch * p.units);
        if (p.symmetric) {
            int j = (int)((sqrtf(8.0f * (float)v + 1.0f) - 1.0f) * 0.5f);
            while (j * (j + 1) / 2 > v) --j;
            while ((j + 1) * (j + 2) / 2 <= v) ++j;
            w.m0 = (v - j * (j + 1) / 2) * 256; w.n0 = j * 256;
        } else {
            w.m0 = (v % p.tiles_m) * 256; w.n0 = (v / p.tiles_m) * 256;
        }
        w.width = 256;
        return w;
    }
};
// every lane waits until matrix b's units of the phases before are done (and their stores can be read by TMA too); bounded
template <bool LOADER>
__device__ __forceinline__ bool wait_done(const unsigned int *done, unsigned int need, volatile int *abort_flag, int *err)
{
    if (need == 0) return true;
    if (tc::ld_acquire_u32(done) < need) {
        const long long began = clock64();
        while (tc::ld_acquire_u32(done) < need) {
            if (*abort_flag) return false;
            if (clock64() - began > tc::kWaitLimitCycles) {
                *abort_flag = 1;
                atomicCAS(err, 0, tc::ERR_WAIT_STEP);
                return false;
            }
            if (!LOADER) __nanosleep(100);                 // the epilogue is waiting for its accumulator anyway
        }
    }
    tc::fence_proxy_async_global();
    return true;
}

__device__ __forceinline__ void tma_load_3d_pair(void *dst, const CUtensorMap *m, uint32_t bar_cluster_addr, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar_cluster_addr), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

// ---- epilogue --------------------------------------------------------------------------------------------------------
// A warp finishes 32 rows x 32 columns at a time.  Between the last product of a phase and the first of the next nothing hides
// this, and registers that spill (a prefetched addend then waits for its loads) or instructions that can be saved show at once (8 to 17 us a
// unit): one instance per kind of product, arithmetic in pairs, addend and result through shared memory so that four lanes share a
// row's 64 bytes, the mirrored copy by transposing loads of the staged block.  The blocks lie in 16-byte pieces, piece c of row r
// at c ^ ((r >> 1) & 3): no bank conflicts either way.
enum Kind { IS_G, IS_P, IS_X_ROWS, IS_X_COLUMNS };         // X: one multiplier per row, or per column (M > N)

__device__ __forceinline__ uint8_t *piece(uint8_t *block, int r, int c) { return block + r * 64 + ((c ^ ((r >> 1) & 3)) << 4); }
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f32x2 pair_of(uint32_t lo, uint32_t hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ void unpair(f32x2 r, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(r)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// What the epilogue keeps of a unit's product in registers (the launch's description lies in constant memory and would be
// indexed by the phase at every use): pointers are the matrix's own.
struct Terms {
    float alpha, beta, gamma, q0, q1, q2;
    int rows, cols, add_ld, out_ld;
    const __half *add;
    uint16_t *out;
    const float *row_v, *col_v;
    float *diag;
    __device__ __forceinline__ Terms(const Product &p, int batch, const void *add_, void *out_, const Steps &s, int step)
        : Terms(p, batch, add_, out_)
    {
        q0 = s.a[step]; beta = q1 = s.b[step]; alpha = gamma = q2 = s.c[step];
    }
    __device__ __forceinline__ Terms(const Product &p, int batch, const void *add_, void *out_)
    {
        const long long v_at = batch * p.v_bs;
        alpha = p.alpha; beta = p.beta; gamma = p.gamma;
        q0 = p.q0; q1 = p.q1; q2 = p.q2;
        rows = p.rows; cols = p.cols;
        add_ld = (int)p.add_ld; out_ld = (int)p.out_ld;
        add = (const __half *)add_ + batch * p.add_bs;
        out = (uint16_t *)out_ + batch * p.out_bs;
        row_v = p.row_v + v_at; col_v = p.col_v + v_at; diag = p.diag + v_at;
    }
};
// What a group needs from memory, requested a group ahead (past L1: other SMs write it): the addend, four lanes to a row, and the
// columns' vector, a lane each.  Rows and vectors of the workspace are padded to whole 16-byte pieces.
struct Fetched { uint4 add[4]; float col; };
template <int KIND>
__device__ __forceinline__ void fetch(const Terms &p, int row0, int c0, int lane, Fetched &f)
{
    if (KIND == IS_G) return;
    const int c = c0 + (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = row0 + i * 8 + (lane >> 2);
        f.add[i] = uint4{};
        if (r < p.rows && c < p.cols) f.add[i] = __ldcg(reinterpret_cast<const uint4 *>(p.add + (long long)r * p.add_ld + c));
    }
    f.col = 0.0f;
    if ((KIND == IS_P || KIND == IS_X_COLUMNS) && c0 + lane < p.cols) f.col = __ldcg(p.col_v + c0 + lane);
}
struct Block { int row0, c0; bool mirror; };
template <int KIND, bool LAST>
__device__ __forceinline__ void finish_block(const Terms &p, uint8_t *stage, const Block &t, int lane, float of_row, float d_row,
                                             const Fetched &f, const uint32_t (&acc)[32])
{
    constexpr bool ADD = KIND != IS_G, COLUMN = KIND == IS_P || KIND == IS_X_COLUMNS, SYMMETRIC = KIND == IS_G || KIND == IS_P;
    uint8_t *in = stage, *res = stage + 2048;
    float *col = reinterpret_cast<float *>(stage + 4096);
    const int row = t.row0 + lane, part = lane & 3, sub = lane >> 2;
    f32x2 v[16];
    const f32x2 alpha = pair_of(p.alpha, p.alpha), by_row = pair_of(of_row, of_row);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        v[j] = pair_of(acc[2 * j], acc[2 * j + 1]);
        if (SYMMETRIC || LAST) v[j] = mul2(alpha, v[j]);   // X's alpha is one but in the last step
    }
    __syncwarp();                                          // the last group's blocks have been read
    if (ADD) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(piece(in, i * 8 + sub, part)) = f.add[i];
        if (COLUMN) col[lane] = p.gamma * f.col;
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 a = *reinterpret_cast<const uint4 *>(piece(in, lane, q));
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
            f32x2 beta[4] = {by_row, by_row, by_row, by_row};
            if (COLUMN) {
                const float4 lo = *reinterpret_cast<const float4 *>(col + 8 * q), hi = *reinterpret_cast<const float4 *>(col + 8 * q + 4);
                const f32x2 c[4] = {pair_of(lo.x, lo.y), pair_of(lo.z, lo.w), pair_of(hi.x, hi.y), pair_of(hi.z, hi.w)};
#pragma unroll
                for (int i = 0; i < 4; ++i) beta[i] = KIND == IS_P ? add2(by_row, c[i]) : c[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                v[4 * q + i] = fma2(beta[i], pair_of(x.x, x.y), v[4 * q + i]);
            }
        }
    }
    if (SYMMETRIC && t.row0 == t.c0) {                     // the diagonal's blocks start on it
        float mine = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float lo, hi;
            unpair(v[j], lo, hi);
            if (lane == 2 * j) { mine = lo; lo = 0.0f; }   // `add` has a zero here: v is alpha times the sum
            if (lane == 2 * j + 1) { mine = hi; hi = 0.0f; }
            v[j] = pair_of(lo, hi);
        }
        if (row < p.rows) p.diag[row] = mine + p.q0 + d_row * (p.q1 + p.q2 * d_row);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            unpair(v[4 * q + i], lo, hi);
            h[i] = LAST ? pack2(lo, hi) : pack_half2(lo, hi);
        }
        *reinterpret_cast<uint4 *>(piece(res, lane, q)) = make_uint4(h[0], h[1], h[2], h[3]);
    }
    __syncwarp();
    if (SYMMETRIC && t.mirror) {
        // eight columns at a time: four transposed 8 x 8 blocks, whose lanes hold two neighbouring rows of one column each
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t m[4];
            asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                         : "=r"(m[0]), "=r"(m[1]), "=r"(m[2]), "=r"(m[3]) : "r"(tc::smem_u32(piece(res, lane, q))) : "memory");
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<uint32_t *>(piece(in, q * 8 + sub, j) + part * 4) = m[j];
        }
        __syncwarp();
    }
    if (LAST && p.out_ld % 8 != 0) {                       // the caller's rows of an odd width: element by element
        __nv_bfloat16 *to = (__nv_bfloat16 *)p.out + t.c0 + lane;
        const int rows = min(32, p.rows - t.row0);
        for (int r = 0; r < rows; ++r)
            if (t.c0 + lane < p.cols) to[(long long)(t.row0 + r) * p.out_ld] = *reinterpret_cast<const __nv_bfloat16 *>(piece(res, r, lane >> 3) + (lane & 7) * 2);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + sub;
        const uint4 x = *reinterpret_cast<const uint4 *>(piece(res, r, part));
        if (t.row0 + r < p.rows && t.c0 + part * 8 < p.cols) *reinterpret_cast<uint4 *>(p.out + (long long)(t.row0 + r) * p.out_ld + t.c0 + part * 8) = x;
    }
    if (SYMMETRIC && t.mirror) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = i * 8 + sub;
            const uint4 x = *reinterpret_cast<const uint4 *>(piece(in, c, part));
            if (t.c0 + c < p.cols && t.row0 + part * 8 < p.rows) *reinterpret_cast<uint4 *>(p.out + (long long)(t.c0 + c) * p.out_ld + t.row0 + part * 8) = x;
        }
    }
}

// One unit's epilogue by one warp; false: gave up.  Out of line, so that the six instances do not share one allocation of
// registers; what it gets of the launch comes by value (a reference would turn the constant bank into generic memory).
struct Place { int row0, m0, n0, width, slot, lane; uint32_t taddr; };
template <int KIND, bool LAST>
__device__ __noinline__ bool finish_unit(const Terms p, const Place w, uint8_t *stage, uint64_t *tmem_full, uint64_t *tmem_empty, uint32_t t_local, volatile int *abort_flag,
                                         int *err)
{
    const int row0 = w.row0, lane = w.lane, slot = w.slot;
    const int items = w.width > BN ? 2 : 1;                // accumulators of this unit
    const float d_row = (KIND == IS_P || KIND == IS_X_ROWS) && row0 + lane < p.rows ? __ldcg(p.row_v + row0 + lane) : 0.0f;
    const float of_row = fmaf(p.gamma, d_row, p.beta);
    Fetched now;                                           // the first group's, before the accumulator is awaited
    fetch<KIND>(p, row0, w.n0 + slot * (min(w.width, BN) / 64) * 32, lane, now);
    for (int item = 0; item < items; ++item, ++t_local) {
        const int buf = t_local & 1;
        const int n0 = w.n0 + item * BN, width = item == 0 ? min(w.width, BN) : w.width - BN;
        const int per = width / 64;                        // 32-column groups per warp: 4 for a 256-column accumulator, 2 for 128
        if (!__all_sync(0xffffffffu, tc::mbar_wait(&tmem_full[buf], (t_local >> 1) & 1, abort_flag, err, tc::ERR_WAIT_TMEM_FULL))) return false;
        tc::tc_fence_after_sync();
        const uint32_t taddr = w.taddr + buf * BN;
#pragma unroll 1
        for (int g = slot * per; g < slot * per + per; ++g) {
            uint32_t acc[32];
            tc::tmem_ld_32x32(taddr + g * 32, acc);
            Fetched next;
            const int c0 = n0 + g * 32;
            const int then = g + 1 < slot * per + per ? c0 + 32 : n0 + BN + slot * ((w.width - BN) / 64) * 32;
            if (g + 1 < slot * per + per || item + 1 < items) fetch<KIND>(p, row0, then, lane, next);
            tc::tmem_ld_wait();
            // right of the diagonal's 256 x 256 block the mirrored place is not computed by anyone
            const Block t{row0, c0, c0 >= w.m0 + 256};
            if (row0 < p.rows && c0 < p.cols) finish_block<KIND, LAST>(p, stage, t, lane, of_row, d_row, now, acc);
            now = next;
        }
        tc::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_cluster(tc::mapa(tc::smem_u32(&tmem_empty[buf]), 0));
    }
    return true;
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NUM_THREADS, 1) orth_products_kernel(const __grid_constant__ Launch l)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *staging = smem + RING_BYTES;
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + STAGING_BYTES);
    uint64_t *tmem_full = bars + BAR_TMEM, *tmem_empty = bars + BAR_TMEM + 2;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + BAR_TMEM + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = tc::cluster_ctarank();           // 0 = leader
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int i = 0; i < BAR_TMEM; ++i) tc::mbar_init(&bars[i], 1);
        for (int b = 0; b < 2; ++b) { tc::mbar_init(&tmem_full[b], 1); tc::mbar_init(&tmem_empty[b], 2 * EPI_WARPS); }
        *abort_flag = 0;
        tc::fence_barrier_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x < MAPS) tc::prefetch_tmap(&l.map[threadIdx.x]);
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();
    tc::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();                                            // for the sake of the next kernel: this one starts behind the one before

    if (warp == 0 || warp == 2 + EPI_WARPS) {
        const bool load_a = warp == 0;
        int cur = 0, s = 0, n_st = 0, st_bytes = 0;
        uint32_t phase = 0;
        uint64_t *full = bars, *empty = bars;
        Rings rings;
        bool ok = true;
        for (Walk walk(l, pair, pairs); walk.more() && ok; walk.next()) {
            const Unit w = walk.at();
            const Product &p = walk.product();
            const int c = max(1, w.width >> 7);
            if (c != cur) {
                rings.leave(cur, s, phase);
                // the new class's stages lie over the old one's: every old stage must have been released
                for (int i = 0; i < n_st && ok; ++i) {
                    ok = __all_sync(0xffffffffu, tc::mbar_wait(&empty[s], phase ^ 1, abort_flag, l.err, tc::ERR_WAIT_EMPTY));
                    if (++s == n_st) { s = 0; phase ^= 1; }
                }
                if (!ok) break;
                cur = c; n_st = cls_stages(c); st_bytes = cls_stage_bytes(c);
                full = bars + cls_bar_base(c); empty = full + n_st;
                rings.resume(c, s, phase);
            }
            ok = __all_sync(0xffffffffu, wait_done<true>(l.done + w.batch, walk.need, abort_flag, l.err));
            if (!ok) break;
            const int which = walk.kind == 1 ? (load_a ? G_K : G_K64)
                              : walk.kind == 0 ? (l.tall ? X_MN0 + walk.cur : load_a ? X_K0 + walk.cur : X_K64_0 + walk.cur)
                              : l.tall ? (load_a ? X_K0 + walk.cur : (int)P_K64) : (load_a ? (int)P_K : X_MN0 + walk.cur);
            const CUtensorMap *map = &l.map[which];
            // the first MMA of a 16-deep step covers 2 h0 columns, the second 2 h1; this block holds h0 + h1 of them
            const int h0 = w.width == 64 ? 32 : c == 1 ? 64 : 128, h1 = c == 3 ? 64 : c == 4 ? 128 : 0;
            const int m0 = w.m0 + (int)rank * 128;
            const int na = w.n0 + (int)rank * h0, nb = w.n0 + 2 * h0 + (int)rank * h1;
            const int boxes0 = max(1, h0 >> 6), boxes = boxes0 + (h1 >> 6);         // 64 columns: of one box only the first half is used
            const uint32_t tx = 2u * (uint32_t)st_bytes;                            // bytes of both blocks
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(&empty[s], phase ^ 1, abort_flag, l.err, tc::ERR_WAIT_EMPTY));
                if (!ok) break;
                uint8_t *sa = smem + (size_t)s * st_bytes, *sb = sa + A_BYTES;
                const uint32_t bar = tc::mapa(tc::smem_u32(&full[s]), 0);           // the leader's barrier
                const int k0 = kb * BK;
                if (tc::elect_one()) {
                    if (load_a) {
                        if (rank == 0) tc::mbar_expect_tx_cluster(bar, tx);
                        if (p.a_mn) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) tma_load_3d_pair(sa + i * MN_BOX_BYTES, map, bar, m0 + i * 64, k0, w.batch);
                        } else {
                            tma_load_3d_pair(sa, map, bar, k0, m0, w.batch);
                        }
                    } else {
                        for (int i = 0; i < boxes; ++i) {
                            const int n = i < boxes0 ? na + i * 64 : nb + (i - boxes0) * 64;
                            if (p.b_mn) tma_load_3d_pair(sb + i * MN_BOX_BYTES, map, bar, n, k0, w.batch);
                            else tma_load_3d_pair(sb + i * MN_BOX_BYTES, map, bar, k0, n, w.batch);
                        }
                    }
                }
                __syncwarp();
                if (++s == n_st) { s = 0; phase ^= 1; }
            }
        }
        // Neither block leaves before the copies into both have landed, whoever gave up; bounded, for a stage that lacks a part.
        if (rank == 0 && load_a)
            for (int i = 0; i < n_st; ++i)
                for (int k = 0; k < 100000 && !tc::mbar_try_wait(&full[i], i < s ? phase : phase ^ 1); ++k) {}
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t b1_off = (2 * CHUNK_BYTES) >> 4;   // the second MMA's columns follow the first's 128 in this block
            uint32_t t_local = 0, phase = 0, stage_off = 0;       // t_local counts accumulators handed to the epilogue
            int cur = 0, s = 0, n_st = 0, st_bytes = 0;
            uint64_t *full = bars, *empty = bars;
            Rings rings;
            bool ok = true;
            for (Walk walk(l, pair, pairs); walk.more() && ok; walk.next()) {
                const Unit w = walk.at();
                const Product &p = walk.product();
                const int c = max(1, w.width >> 7);
                if (c != cur) {
                    rings.leave(cur, s, phase);
                    cur = c; n_st = cls_stages(c); st_bytes = cls_stage_bytes(c);
                    full = bars + cls_bar_base(c); empty = full + n_st;
                    rings.resume(c, s, phase);
                    stage_off = (uint32_t)s * ((uint32_t)st_bytes >> 4);
                }
                // K-major: 8-row atoms 1024 B apart, 16 k = 32 bytes along the swizzled row; MN-major: 64-wide groups one box
                // apart, 8-k atoms 1024 B apart, 16 k = 2 atoms
                const uint32_t a_step = p.a_mn ? 2048 : 32, b_step = p.b_mn ? 2048 : 32;
                const uint64_t desc_a0 = tc::smem_desc(tc::smem_u32(smem), p.a_mn ? MN_BOX_BYTES : 16, 1024);
                const uint64_t desc_b0 = tc::smem_desc(tc::smem_u32(smem) + A_BYTES, p.b_mn ? MN_BOX_BYTES : 16, 1024);
                const uint32_t idesc_256 = instr_desc_f16(256, 256, p.a_mn, p.b_mn), idesc_128 = instr_desc_f16(256, 128, p.a_mn, p.b_mn), idesc_64 = instr_desc_f16(256, 64, p.a_mn, p.b_mn);
                const bool both = c >= 3;                  // both accumulators, in the order in which they come free
                const int buf = t_local & 1;
                if (!__all_sync(0xffffffffu, tc::mbar_wait(&tmem_empty[buf], ((t_local >> 1) & 1) ^ 1, abort_flag, l.err, tc::ERR_WAIT_TMEM_EMPTY))) break;
                if (both && !__all_sync(0xffffffffu, tc::mbar_wait(&tmem_empty[buf ^ 1], (((t_local + 1) >> 1) & 1) ^ 1, abort_flag, l.err, tc::ERR_WAIT_TMEM_EMPTY)))
                    break;
                tc::tc_fence_after_sync();
                const uint32_t d0 = tmem_base + buf * BN, d1 = tmem_base + (buf ^ 1) * BN;
                const uint32_t idesc0 = w.width == 64 ? idesc_64 : c == 1 ? idesc_128 : idesc_256, idesc1 = c == 3 ? idesc_128 : idesc_256;
                for (int kb = 0; kb < p.k_blocks; ++kb) {
                    ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[s], phase, abort_flag, l.err, tc::ERR_WAIT_FULL));
                    if (!ok) break;
                    tc::tc_fence_after_sync();
                    const uint64_t da = desc_a0 + stage_off, db = desc_b0 + stage_off;
                    const uint32_t acc = kb != 0;
                    if (both) {
#pragma unroll
                        for (int kk = 0; kk < BK / 16; ++kk) {
                            tc::mma_bf16_pair_elect(d0, da + ((kk * a_step) >> 4), db + ((kk * b_step) >> 4), idesc0, acc | (kk != 0));
                            tc::mma_bf16_pair_elect(d1, da + ((kk * a_step) >> 4), db + b1_off + ((kk * b_step) >> 4), idesc1, acc | (kk != 0));
                        }
                    } else {
#pragma unroll
                        for (int kk = 0; kk < BK / 16; ++kk)
                            tc::mma_bf16_pair_elect(d0, da + ((kk * a_step) >> 4), db + ((kk * b_step) >> 4), idesc0, acc | (kk != 0));
                    }
                    tc::mma_commit_pair_elect(&empty[s]);
                    stage_off += (uint32_t)st_bytes >> 4;
                    if (++s == n_st) { s = 0; phase ^= 1; stage_off = 0; }
                }
                if (!ok) break;
                tc::mma_commit_pair_elect(&tmem_full[buf]);
                if (both) tc::mma_commit_pair_elect(&tmem_full[buf ^ 1]);
                t_local += both ? 2 : 1;
            }
        }
    } else {
        const int quarter = warp & 3;                      // TMEM lanes [32 quarter, 32 quarter + 32)
        const int slot = (warp - 2) >> 2;                  // which half of an accumulator's 32-column groups this warp drains
        uint8_t *my_stage = staging + (size_t)(warp - 2) * WARP_STAGE;
        uint32_t t_local = 0;
        bool ok = true;
        for (Walk walk(l, pair, pairs); walk.more() && ok; walk.next()) {
            const Unit w = walk.at();
            const Product &p = walk.product();
            const int row0 = w.m0 + (int)rank * 128 + quarter * 32;
            const bool last = walk.phase == 3 * l.step.n - 1;
            const void *x = l.x[walk.cur];
            void *x_out = last ? p.out : l.x[walk.cur ^ 1];
            ok = __all_sync(0xffffffffu, wait_done<false>(l.done + w.batch, walk.need, abort_flag, l.err));
            if (!ok) break;
            const Place at{row0, w.m0, w.n0, w.width, slot, lane, tmem_base + ((uint32_t)(quarter * 32) << 16)};
#define FINISH(KIND, LAST, ADD, OUT) finish_unit<KIND, LAST>(Terms(p, w.batch, ADD, OUT), at, my_stage, tmem_full, tmem_empty, t_local, abort_flag, l.err)
            if (walk.kind == 0) ok = FINISH(IS_G, false, nullptr, p.out);
            else if (walk.kind == 1) ok = finish_unit<IS_P, false>(Terms(p, w.batch, p.add, p.out, l.step, walk.phase / 3), at, my_stage, tmem_full, tmem_empty, t_local, abort_flag, l.err);
            else if (l.tall) ok = last ? FINISH(IS_X_COLUMNS, true, x, x_out) : FINISH(IS_X_COLUMNS, false, x, x_out);
            else ok = last ? FINISH(IS_X_ROWS, true, x, x_out) : FINISH(IS_X_ROWS, false, x, x_out);
#undef FINISH
            t_local += w.width > BN ? 2 : 1;
            if (!ok) break;
            if (!last) {                                   // this warp's stores are there, for TMA too: count it in
                tc::fence_proxy_async_global();
                __syncwarp();
                if (lane == 0) tc::red_release_add_u32(l.done + w.batch, 1u);
            }
        }
    }

    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();                                    // neither block leaves while the other may still signal it
    if (warp == 1) {
        tc::tc_fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// ---- plan: widths c in pieces of 64 columns, 1 or an even number up to 8 -----------------------------------------------------
double main_cycles(int c, int k_blocks) { return k_blocks * std::max(128.0 * c, (16.0 + 4.0 * std::max(c, 2)) * 1024.0 / 48.0); }
double epilogue_cycles(int c) { return 1500.0 + 1250.0 * c; }
constexpr int kWidths[] = {1, 2, 4, 6, 8};
int width_of(long long pieces) { return pieces <= 1 ? 1 : (int)((pieces + 1) / 2 * 2); }

// The widths of a cut's rounds: one throughout, or (share) as many pieces as are left of a pair's share, the widest first.
struct Widths {
    int widest;
    bool share;
    long long left;                    // of the share
    int now() const { return share ? std::min(widest, width_of(left)) : widest; }
    void next() { if (share && left > now()) left -= now(); }
};
// Cuts the rows of pieces of one matrix into units, a width for each `quota0` of them, widest first in the table; false if they are
// more than it holds.  Nothing here allocates: a call cannot fail for want of host memory.
bool cut(const Product &p, int quota0, Widths width, UnitTable *units)
{
    UnitTable cut;
    cut.n = 0;
    const int per_row = (p.cols + 63) / 64;
    int quota = quota0;
    for (int m = 0; m < p.tiles_m; ++m) {
        int at = p.symmetric ? 4 * m : 0;
        while (at < per_row) {
            const int c = std::min(width.now(), width_of(per_row - at));
            if (cut.n == UnitTable::kMax) return false;
            cut.e[cut.n++] = (uint32_t)m | ((uint32_t)at << 8) | ((uint32_t)c << 19);
            at += c;
            if (--quota == 0) { quota = quota0; width.next(); }
        }
    }
    units->n = 0;
    for (int k = (int)(sizeof kWidths / sizeof *kWidths) - 1; k >= 0; --k)
        for (int i = 0; i < cut.n; ++i)
            if ((int)(cut.e[i] >> 19) == kWidths[k]) units->e[units->n++] = cut.e[i];
    return true;
}
// The phase's length: each round over the pairs takes as long as its widest unit; a wide unit's epilogue is in the way of the next
// unit, and the last unit's is always in the way of the next phase.  A matrix's units come widest first, so the widest of a round is
// its first or, where another matrix begins in it, the widest of all.  Of very many rounds the first few stand for all.
double finish_time(const UnitTable &units, int batch, int pairs, int k_blocks)
{
    constexpr long long kLook = 256;
    double t = 0, last = 0;
    const long long size = units.n, n = size * batch, rounds = (n + pairs - 1) / pairs;
    for (long long r = 0; r < std::min(rounds, kLook); ++r) {
        const long long at = r * pairs % size;
        const int c = (int)(units.e[at + std::min<long long>(pairs, n - r * pairs) > size ? 0 : at] >> 19);
        if (c >= 6 && last > 0) t += last;
        t += main_cycles(c, k_blocks);
        last = epilogue_cycles(c);
    }
    return (t + last) * std::max(1.0, (double)rounds / (double)kLook);
}
// the cut that finishes first
void plan(Product *p, int batch, int pairs, UnitTable *tb)
{
    p->tiles_m = (p->rows + 255) / 256;
    p->units = p->symmetric ? p->tiles_m * (p->tiles_m + 1) / 2 : p->tiles_m * ((p->cols + 255) / 256);
    tb->n = 0;
    const int per_row = (p->cols + 63) / 64;
    long long total = 0;
    for (int m = 0; m < p->tiles_m; ++m) total += std::max(0, per_row - (p->symmetric ? 4 * m : 0));
    const int quota = std::max(1, pairs / batch);
    UnitTable units;
    double best_time = 0;
    for (int widest : kWidths)
        for (int share = 0; share < 2; ++share) {
            if (!cut(*p, quota, Widths{widest, share != 0, (total + quota - 1) / quota}, &units)) continue;
            const double t = finish_time(units, batch, pairs, p->k_blocks);
            if (tb->n == 0 || t < best_time) { *tb = units; best_time = t; }
        }
    if (tb->n > 0) p->units = tb->n;
}

// pairs that are resident at once on this device
int resident_pairs(int sms)
{
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (known[dev].load(std::memory_order_relaxed) == 0) {
        if (cudaFuncSetAttribute(orth_products_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_BYTES) != cudaSuccess) { cudaGetLastError(); return 0; }
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(sms / 2 * 2)); cfg.blockDim = dim3(NUM_THREADS); cfg.dynamicSmemBytes = SMEM_BYTES;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, orth_products_kernel, &cfg) != cudaSuccess) { cudaGetLastError(); return 0; }
        known[dev].store(n, std::memory_order_relaxed);
    }
    return std::min(known[dev].load(std::memory_order_relaxed), sms / 2);
}

}  // namespace

relay_status_t launch_products(Launch &l, int sms, cudaStream_t st)
{
    const int pairs = resident_pairs(sms);
    if (pairs < 1) return fail(RELAY_ERR_CUDA, "orthogonalize: no pair of SMs takes the product kernel");
    long long most = 0;
    for (int k = 0; k < 3; ++k) {
        plan(&l.product[k], l.batch, pairs, &l.table[k]);
        most = std::max(most, (long long)l.product[k].units * l.batch);
    }
    l.product[3].tiles_m = l.product[2].tiles_m; l.product[3].units = l.product[2].units;
    RELAY_CUDA(launch_cooperative(orth_products_kernel, dim3((unsigned)(2 * std::min<long long>(most, pairs))), dim3(NUM_THREADS), SMEM_BYTES, st, l));
    return check_launch("orthogonalize_products");
}

}  // namespace orth
}  // namespace relay

// Host-only view of the plan of one product (rows x cols results per matrix, contraction steps of 64): units as in UnitTable, widest
// first; -1 where 256 x 256 units in order would run, -2 for bad arguments.
extern "C" int32_t relay_debug_orthogonalize_units(int32_t rows, int32_t cols, int32_t symmetric, int32_t k_blocks, int32_t batch, int32_t pairs, uint32_t *units,
                                                   int32_t max_units)
{
    using namespace relay::orth;
    if (rows < 1 || cols < 1 || rows > 65536 || cols > 65536 || k_blocks < 1 || batch < 1 || pairs < 1 || !units || (symmetric && rows != cols)) return -2;
    Product p{};
    p.rows = rows; p.cols = cols; p.symmetric = symmetric != 0; p.k_blocks = k_blocks;
    UnitTable tb;
    plan(&p, batch, pairs, &tb);
    if (tb.n == 0) return -1;
    if (tb.n > max_units) return -2;
    std::copy(tb.e, tb.e + tb.n, units);
    return tb.n;
}
