// The product of an orthogonalisation step on pairs of SMs (cta_group::2): 256 rows x up to 512 columns per pair.
//
// What bounds a product here is how fast an SM can fill its shared memory (about 48 bytes a cycle): a k-step of 64 over 256 x 128 c
// columns costs a pair max(256 c cycles of MMA, (16 + 8 c) KB per SM / 48 B).  256 x 512 (c = 4) balances the two, but fills both
// TMEM accumulators, so its epilogue is not overlapped; c <= 2 leaves the other accumulator to the next unit.  The host cuts the
// product into units of c = 1..4 chunks of 128 columns, whichever cut finishes first (see plan below), and the pairs take
// them in order, widest first.  Symmetric products have units on and above the diagonal only.
// Roles per block: warp 0 loads A, warp 18 loads B, warp 1 of the leader issues the MMAs, warps 2-17 are the epilogue.  The barrier
// scheme is that of the dense groups' two-SM contraction (gemm_tc2.cu): full[] in the leader, empty[] and tmem_full[] in each block
// by multicast commits, tmem_empty[] in the leader.  All waits are bounded.
#include <algorithm>
#include <vector>

#include "common.h"
#include "orthogonalize.cuh"

namespace relay {
namespace orth {
namespace {

constexpr int BK = 64, BN = 256;                           // BN: columns of one accumulator
constexpr int A_BYTES = 128 * BK * 2;                      // this block's 128 rows of A: 16 KB
constexpr int CHUNK_BYTES = 64 * BK * 2;                   // this block's 64 columns of one 128-column chunk: 8 KB
constexpr int MN_BOX_BYTES = 64 * BK * 2;
constexpr int RING_BYTES = 144 * 1024;
constexpr int NUM_THREADS = 608, EPI_WARPS = 16, TMEM_COLS = 512;
constexpr int STAGING_BYTES = EPI_WARPS * 4096;            // two 32 x 32 blocks of 16-bit results per epilogue warp
constexpr size_t SMEM_BYTES = 1024 + (size_t)RING_BYTES + STAGING_BYTES + 512;

__host__ __device__ constexpr int cls_stages(int c) { return c == 1 ? 6 : c == 2 ? 4 : 3; }
__host__ __device__ constexpr int cls_stage_bytes(int c) { return A_BYTES + c * CHUNK_BYTES; }
__host__ __device__ constexpr int cls_bar_base(int c) { return c == 1 ? 0 : c == 2 ? 12 : c == 3 ? 20 : 26; }   // full[], then empty[]
constexpr int BAR_TMEM = 32;                               // tmem_full[2], tmem_empty[2]

struct Unit { int batch, m0, n0, width; };
__device__ __forceinline__ Unit unit_of(const Product &p, const UnitTable &tb, long long u)
{
    Unit w;
    if (tb.n > 0) {
        const uint32_t e = tb.e[u];
        w.m0 = (int)(e & 0xffu) * 256;
        w.n0 = (int)((e >> 8) & 0x1ffu) * 128;
        w.width = (int)((e >> 17) & 7u) * 128;
        w.batch = (int)(e >> 20);
        return w;
    }
    w.batch = (int)(u / p.units);
    const int v = (int)(u - (long long)w.batch * p.units);
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

__device__ __forceinline__ void tma_load_3d_pair(void *dst, const CUtensorMap *m, uint32_t bar_cluster_addr, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar_cluster_addr), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

__device__ __forceinline__ void tma_store_3d(const CUtensorMap *m, const void *src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(src)), "r"(x), "r"(y), "r"(z) : "memory");
}
// this row's 32 columns of the addend (rows of the workspace are padded to whole 16-byte pieces)
__device__ __forceinline__ void load_addend(const Product &p, int batch, int row, int c0, uint4 (&r)[4])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) r[q] = uint4{};
    if (p.add == nullptr || row >= p.rows) return;
    const uint4 *add = reinterpret_cast<const uint4 *>((const __half *)p.add + batch * p.add_bs + (long long)row * p.add_ld + c0);
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (c0 + 8 * q < p.cols) r[q] = __ldg(add + q);
}
// The epilogue of 32 rows x 32 columns by one warp: out = alpha acc + beta add, rounded once, staged in shared memory (64-byte
// swizzle: 16-byte piece c of row r at piece c ^ ((r >> 1) & 3)) and stored by TMA, which leaves out what lies outside the matrix; the
// mirrored copy is staged transposed.  of_row: this row's part of beta.
__device__ __forceinline__ void finish_block(const Product &p, const CUtensorMap *tm_out, const CUtensorMap *tm_mirror, uint8_t *stages, int &turn, const Tile &t, int lane,
                                             int row, int c0, float of_row, float d_row, const uint4 (&add)[4], const uint32_t (&acc)[32])
{
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = p.alpha * __uint_as_float(acc[j]);
    if (p.add != nullptr) {
        const float *col_v = p.col_v != nullptr ? p.col_v + t.batch * p.v_bs + c0 : nullptr;   // padded like the rows
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t w[4] = {add[q].x, add[q].y, add[q].z, add[q].w};
            float beta[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) beta[i] = of_row;
            if (col_v != nullptr && c0 + 8 * q < p.cols) {
                const float4 lo = __ldg(reinterpret_cast<const float4 *>(col_v + 8 * q)), hi = __ldg(reinterpret_cast<const float4 *>(col_v + 8 * q + 4));
                const float of_col[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) beta[i] = fmaf(p.gamma, of_col[i], beta[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                v[8 * q + 2 * i] = fmaf(beta[2 * i], f.x, v[8 * q + 2 * i]);
                v[8 * q + 2 * i + 1] = fmaf(beta[2 * i + 1], f.y, v[8 * q + 2 * i + 1]);
            }
        }
    }
    if (p.diag != nullptr && !t.mirror && row >= c0 && row < c0 + 32 && row < p.rows) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (row == c0 + j) {                           // `add` has a zero here: v is alpha times the sum
                p.diag[t.batch * p.v_bs + row] = v[j] + p.q0 + d_row * (p.q1 + p.q2 * d_row);
                v[j] = 0.0f;
            }
    }
    uint32_t h[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) h[j] = p.out_bf16 ? pack2(v[2 * j], v[2 * j + 1]) : pack_half2(v[2 * j], v[2 * j + 1]);
    // two buffers in turn: the store before the last (same elected lane) has read this one
    if (tc::elect_one()) tc::tma_store_wait_read<1>();
    __syncwarp();
    uint8_t *stage = stages + (turn++ & 1) * 2048;
    const int sw = (lane >> 1) & 3;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<uint4 *>(stage + lane * 64 + ((q ^ sw) << 4)) = make_uint4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
    tc::fence_proxy_async();
    __syncwarp();
    if (tc::elect_one()) {                                 // the election is deterministic: always the same lane of the warp
        tma_store_3d(tm_out, stage, c0, row - lane, t.batch);
        tc::tma_store_commit();
    }
    if (!t.mirror) return;
    // lanes hold consecutive rows of the same columns: a pair of lanes exchanges halves, the even one writes rows (r, r + 1) of
    // column c, the odd one rows (r - 1, r) of column c + 1: 128 contiguous bytes per store
    if (tc::elect_one()) tc::tma_store_wait_read<1>();
    __syncwarp();
    stage = stages + (turn++ & 1) * 2048;
    const bool odd = lane & 1;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, h[j], 1);
        const uint32_t w = odd ? __byte_perm(other, h[j], 0x7632) : __byte_perm(h[j], other, 0x5410);
        *reinterpret_cast<uint32_t *>(stage + (2 * j + (odd ? 1 : 0)) * 64 + (lane & ~1) * 2) = w;
    }
    tc::fence_proxy_async();
    __syncwarp();
    if (tc::elect_one()) {
        tma_store_3d(tm_mirror, stage, row - lane, c0, t.batch);
        tc::tma_store_commit();
    }
}

template <bool A_MN, bool B_MN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NUM_THREADS, 1)
orth_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_out,
                 const __grid_constant__ CUtensorMap tm_mirror, const Product p, const __grid_constant__ UnitTable tb)
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
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const long long n_units = tb.n > 0 ? tb.n : (long long)p.units * p.batch;

    if (threadIdx.x == 0) {
        for (int i = 0; i < BAR_TMEM; ++i) tc::mbar_init(&bars[i], 1);
        for (int b = 0; b < 2; ++b) { tc::mbar_init(&tmem_full[b], 1); tc::mbar_init(&tmem_empty[b], 2 * EPI_WARPS); }
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tmap(&tm_a);
        tc::prefetch_tmap(&tm_b);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();
    tc::tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();

    if (warp == 0 || warp == 18) {
        const bool load_a = warp == 0;
        int cur = 0, s = 0, n_st = 0, st_bytes = 0;
        uint32_t phase = 0;
        uint64_t *full = bars, *empty = bars;
        bool ok = true;
        for (long long u = pair; u < n_units && ok; u += n_pairs) {
            const Unit w = unit_of(p, tb, u);
            const int c = w.width >> 7;
            if (c != cur) {
                // the new class's stages lie over the old one's: every old stage must have been released
                for (int i = 0; i < n_st && ok; ++i) {
                    ok = __all_sync(0xffffffffu, tc::mbar_wait(&empty[s], phase ^ 1, abort_flag, p.err, tc::ERR_WAIT_EMPTY));
                    if (++s == n_st) { s = 0; phase ^= 1; }
                }
                if (!ok) break;
                cur = c; n_st = cls_stages(c); st_bytes = cls_stage_bytes(c);
                full = bars + cls_bar_base(c); empty = full + n_st;
                s = 0; phase = 0;
            }
            // the first MMA of a 16-deep step covers 2 h0 columns, the second 2 h1; this block holds h0 + h1 of them
            const int h0 = c == 1 ? 64 : 128, h1 = c == 3 ? 64 : c == 4 ? 128 : 0;
            const int m0 = w.m0 + (int)rank * 128;
            const int na = w.n0 + (int)rank * h0, nb = w.n0 + 2 * h0 + (int)rank * h1;
            const int boxes0 = h0 >> 6, boxes = (h0 + h1) >> 6;
            const uint32_t tx = 2u * (uint32_t)st_bytes;                            // bytes of both blocks
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(&empty[s], phase ^ 1, abort_flag, p.err, tc::ERR_WAIT_EMPTY));
                if (!ok) break;
                uint8_t *sa = smem + (size_t)s * st_bytes, *sb = sa + A_BYTES;
                const uint32_t bar = tc::mapa(tc::smem_u32(&full[s]), 0);           // the leader's barrier
                const int k0 = kb * BK;
                if (tc::elect_one()) {
                    if (load_a) {
                        if (rank == 0) tc::mbar_expect_tx_cluster(bar, tx);
                        if (A_MN) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) tma_load_3d_pair(sa + i * MN_BOX_BYTES, &tm_a, bar, m0 + i * 64, k0, w.batch);
                        } else {
                            tma_load_3d_pair(sa, &tm_a, bar, k0, m0, w.batch);
                        }
                    } else {
                        for (int i = 0; i < boxes; ++i) {
                            const int n = i < boxes0 ? na + i * 64 : nb + (i - boxes0) * 64;
                            if (B_MN) tma_load_3d_pair(sb + i * MN_BOX_BYTES, &tm_b, bar, n, k0, w.batch);
                            else tma_load_3d_pair(sb + i * MN_BOX_BYTES, &tm_b, bar, k0, n, w.batch);
                        }
                    }
                }
                __syncwarp();
                if (++s == n_st) { s = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            constexpr uint32_t idesc_256 = instr_desc_f16(256, 256, A_MN, B_MN), idesc_128 = instr_desc_f16(256, 128, A_MN, B_MN);
            constexpr uint32_t a_lbo = A_MN ? MN_BOX_BYTES : 16, b_lbo = B_MN ? MN_BOX_BYTES : 16;
            constexpr uint32_t a_step = A_MN ? 2048 : 32, b_step = B_MN ? 2048 : 32;
            constexpr uint32_t b1_off = (2 * CHUNK_BYTES) >> 4;   // the second MMA's columns follow the first's 128 in this block
            const uint64_t desc_a0 = tc::smem_desc(tc::smem_u32(smem), a_lbo, 1024);
            const uint64_t desc_b0 = tc::smem_desc(tc::smem_u32(smem) + A_BYTES, b_lbo, 1024);
            uint32_t t_local = 0, phase = 0, stage_off = 0;       // t_local counts accumulators handed to the epilogue
            int cur = 0, s = 0, n_st = 0, st_bytes = 0;
            uint64_t *full = bars, *empty = bars;
            bool ok = true;
            for (long long u = pair; u < n_units && ok; u += n_pairs) {
                const Unit w = unit_of(p, tb, u);
                const int c = w.width >> 7;
                if (c != cur) {
                    cur = c; n_st = cls_stages(c); st_bytes = cls_stage_bytes(c);
                    full = bars + cls_bar_base(c); empty = full + n_st;
                    s = 0; phase = 0; stage_off = 0;
                }
                const bool both = c >= 3;                  // both accumulators (t_local is even: such units come first)
                const int buf = t_local & 1;
                const uint32_t par = ((t_local >> 1) & 1) ^ 1;
                if (!__all_sync(0xffffffffu, tc::mbar_wait(&tmem_empty[buf], par, abort_flag, p.err, tc::ERR_WAIT_TMEM_EMPTY))) break;
                if (both && !__all_sync(0xffffffffu, tc::mbar_wait(&tmem_empty[1], par, abort_flag, p.err, tc::ERR_WAIT_TMEM_EMPTY))) break;
                tc::tc_fence_after_sync();
                const uint32_t d0 = tmem_base + buf * BN, d1 = tmem_base + BN;
                const uint32_t idesc0 = c == 1 ? idesc_128 : idesc_256, idesc1 = c == 3 ? idesc_128 : idesc_256;
                for (int kb = 0; kb < p.k_blocks; ++kb) {
                    ok = __all_sync(0xffffffffu, tc::mbar_wait(&full[s], phase, abort_flag, p.err, tc::ERR_WAIT_FULL));
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
                if (both) tc::mma_commit_pair_elect(&tmem_full[1]);
                t_local += both ? 2 : 1;
            }
        }
    } else {
        const int quarter = warp & 3;                      // TMEM lanes [32 quarter, 32 quarter + 32)
        const int slot = (warp - 2) >> 2;                  // which quarter of an accumulator's 32-column groups this warp drains
        uint8_t *my_stage = staging + (size_t)(warp - 2) * 4096;
        int turn = 0;
        const bool by_tma = !p.out_bf16 || p.out_ld % 8 == 0;
        uint32_t t_local = 0;
        bool ok_all = true;
        for (long long u = pair; u < n_units && ok_all; u += n_pairs) {
            const Unit w = unit_of(p, tb, u);
            const int items = w.width > BN ? 2 : 1;        // accumulators of this unit
            const int row = w.m0 + (int)rank * 128 + quarter * 32 + lane;
            const float d_row = p.row_v != nullptr && row < p.rows ? p.row_v[w.batch * p.v_bs + row] : 0.0f;
            const float of_row = fmaf(p.gamma, d_row, p.beta);
            for (int item = 0; item < items; ++item, ++t_local) {
                const int buf = t_local & 1;
                const int n0 = w.n0 + item * BN, width = item == 0 ? min(w.width, BN) : w.width - BN;
                const int per = width / 128;               // 32-column groups per warp: 2 for a 256-column accumulator, 1 for 128
                uint4 add[4];                              // requested a group ahead: before the wait, and before the group at hand is finished
                load_addend(p, w.batch, row, n0 + slot * per * 32, add);
                int ok = 1;
                if (lane == 0) ok = tc::mbar_wait(&tmem_full[buf], (t_local >> 1) & 1, abort_flag, p.err, tc::ERR_WAIT_TMEM_FULL) ? 1 : 0;
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) { ok_all = false; break; }
                tc::tc_fence_after_sync();
                const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * BN;
#pragma unroll 1
                for (int g = slot * per; g < slot * per + per; ++g) {
                    uint32_t acc[32];
                    tc::tmem_ld_32x32(taddr + g * 32, acc);
                    uint4 next[4];
                    if (g + 1 < slot * per + per) load_addend(p, w.batch, row, n0 + (g + 1) * 32, next);
                    tc::tmem_ld_wait();
                    const int c0 = n0 + g * 32;
                    // right of the diagonal's 256 x 256 block the mirrored place is not computed by anyone
                    const Tile t{w.batch, w.m0, c0, p.symmetric && c0 >= w.m0 + 256};
                    if (by_tma) {
                        if (row - lane < p.rows && c0 < p.cols) finish_block(p, &tm_out, &tm_mirror, my_stage, turn, t, lane, row, c0, of_row, d_row, add, acc);
                    } else {
                        finish_columns(p, t, lane, row, c0, acc);
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) add[q] = next[q];
                }
                tc::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive_cluster(tc::mapa(tc::smem_u32(&tmem_empty[buf]), 0));
            }
        }
        __syncwarp();
        if (tc::elect_one()) tc::tma_store_wait_all<0>();
    }

    tc::tc_fence_before_sync();
    __syncthreads();
    tc::cluster_sync();                                    // neither block leaves while the other may still signal it
    if (warp == 1) {
        tc::tc_fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// ---- plan --------------------------------------------------------------------------------------------------------------
// cycles of a unit of c chunks: its k-steps, and its epilogue where that is not overlapped
double unit_cycles(int c, int k_blocks) { return k_blocks * std::max(256.0 * c, (16.0 + 8.0 * c) * 1024.0 / 48.0) + (c >= 3 ? 3000.0 : 400.0); }

// Cuts the rows of chunks of all matrices into units, taking widths from `rounds` (one width per round over the pairs, the last
// one for whatever follows); false if they are more than the table holds.
bool cut(const Product &p, int pairs, const std::vector<int> &rounds, std::vector<uint32_t> *units)
{
    const int cpr = (p.cols + 127) / 128;
    units->clear();
    size_t r = 0;
    int quota = pairs;
    for (int b = 0; b < p.batch; ++b)
        for (int m = 0; m < p.tiles_m; ++m) {
            int at = p.symmetric ? 2 * m : 0;
            while (at < cpr) {
                const int c = std::min(rounds[std::min(r, rounds.size() - 1)], cpr - at);
                if (units->size() == (size_t)UnitTable::kMax) return false;
                units->push_back((uint32_t)m | ((uint32_t)at << 8) | ((uint32_t)c << 17) | ((uint32_t)b << 20));
                at += c;
                if (--quota == 0) { quota = pairs; ++r; }
            }
        }
    std::stable_sort(units->begin(), units->end(), [](uint32_t a, uint32_t b) { return ((a >> 17) & 7) > ((b >> 17) & 7); });
    return true;
}
double finish_time(const std::vector<uint32_t> &units, int pairs, int k_blocks)
{
    double t = 0;
    for (size_t i = 0; i < units.size(); i += pairs) t += unit_cycles((int)((units[i] >> 17) & 7), k_blocks);   // each round's widest
    return t;
}
Product in_tiles(const Product &q)
{
    Product p = q;
    p.tiles_m = (p.rows + 255) / 256; p.tiles_n = (p.cols + 255) / 256;
    p.units = p.symmetric ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
    return p;
}

}  // namespace

// the cut that finishes first: one width throughout, or as many chunks as a pair's share has, the widest first
void plan_units(const Product &q, int sms, UnitTable *tb)
{
    const Product p = in_tiles(q);
    const int pairs = sms / 2;
    tb->n = 0;
    if (p.batch >= 4096 || p.tiles_m > 256 || p.cols > 65536) return;
    const int cpr = (p.cols + 127) / 128;
    long long total = 0;
    for (int m = 0; m < p.tiles_m; ++m) total += std::max(0, cpr - (p.symmetric ? 2 * m : 0));
    total *= p.batch;
    std::vector<uint32_t> units, best;
    double best_time = 0;
    for (int widest = 1; widest <= 4; ++widest)
        for (int share = 0; share < 2; ++share) {
            std::vector<int> rounds;
            if (share) for (long long left = (total + pairs - 1) / pairs; left > 0; left -= rounds.back()) rounds.push_back((int)std::min<long long>(widest, left));
            else rounds.push_back(widest);
            if (!cut(p, pairs, rounds, &units)) continue;
            const double t = finish_time(units, pairs, p.k_blocks);
            if (best.empty() || t < best_time) { best = units; best_time = t; }
        }
    tb->n = (int)best.size();
    std::copy(best.begin(), best.end(), tb->e);
}

relay_status_t launch_product_pair(const Product &q, bool a_mn, bool b_mn, const CUtensorMap &ta, const CUtensorMap &tb, const UnitTable &table, int sms,
                                   cudaStream_t st)
{
    const Product p = in_tiles(q);
    const long long n = table.n > 0 ? table.n : (long long)p.units * p.batch;
    const dim3 grid((unsigned)(2 * std::min<long long>(n, sms / 2)));
    CUtensorMap out, mirror;
    out = mirror = ta;                                     // not used where rows of the result are not whole 16-byte pieces
    if (p.out_ld % 8 == 0) {
        RELAY_TRY(make_tmap_3d_block(&out, p.out_bf16 != 0, p.out, p.cols, p.rows, p.batch, p.out_ld, p.out_bs, true));
        if (p.symmetric) RELAY_TRY(make_tmap_3d_block(&mirror, p.out_bf16 != 0, p.out, p.cols, p.rows, p.batch, p.out_ld, p.out_bs, false));
    }
#define LAUNCH(AMN, BMN)                                                                                                          \
    do {                                                                                                                          \
        RELAY_CUDA(cudaFuncSetAttribute(orth_pair_kernel<AMN, BMN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_BYTES)); \
        RELAY_CUDA(launch_pdl(orth_pair_kernel<AMN, BMN>, grid, dim3(NUM_THREADS), SMEM_BYTES, st, ta, tb, out, mirror, p, table));             \
    } while (0)
    if (a_mn && b_mn) LAUNCH(true, true);
    else if (b_mn) LAUNCH(false, true);
    else LAUNCH(false, false);
#undef LAUNCH
    return check_launch("orthogonalize_product_pair");
}

}  // namespace orth
}  // namespace relay
