// Device code that the one-block and the two-block product kernels of an orthogonalisation share: the tile's place, and the
// epilogue of one row's 32 columns.
#pragma once
#include <cuda_fp16.h>

#include "ewise_kernels.cuh"
#include "orthogonalize.h"
#include "tc_common.cuh"

namespace relay {
namespace orth {

__host__ __device__ constexpr uint32_t instr_desc_f16(int m, int n, bool a_mn, bool b_mn)
{   // fp32 accumulator, fp16 A and B (format 0), majorness, N / 8, M / 16
    return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

struct Tile { int batch, m0, n0; bool mirror; };
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
}

// 32 accumulator columns of one row: out = alpha acc + beta add, rounded once, and the mirrored copy
__device__ __forceinline__ void finish_columns(const Product &p, const Tile &t, int lane, int row, int c0, const uint32_t (&acc)[32])
{
    float v[32];
    const bool row_ok = row < p.rows;
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = p.alpha * __uint_as_float(acc[j]);
    if (p.add != nullptr && row_ok) {
        const __half *add = (const __half *)p.add + t.batch * p.add_bs + (long long)row * p.add_ld;
        const float of_row = p.row_v != nullptr ? fmaf(p.gamma, p.row_v[t.batch * p.v_bs + row], p.beta) : p.beta;
        const float *col_v = p.col_v != nullptr ? p.col_v + t.batch * p.v_bs : nullptr;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (c0 + 8 * q < p.cols) {                 // rows and vectors of the workspace are padded to whole 16-byte pieces
                const uint4 r = *reinterpret_cast<const uint4 *>(add + c0 + 8 * q);
                const uint32_t w[4] = {r.x, r.y, r.z, r.w};
                float beta[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) beta[i] = of_row;
                if (col_v != nullptr) {
                    const float4 lo = *reinterpret_cast<const float4 *>(col_v + c0 + 8 * q), hi = *reinterpret_cast<const float4 *>(col_v + c0 + 8 * q + 4);
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
    }
    if (p.diag != nullptr && !t.mirror && row_ok && row >= c0 && row < c0 + 32) {
        const float d = p.row_v != nullptr ? p.row_v[t.batch * p.v_bs + row] : 0.0f;
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (row == c0 + j) {                       // `add` has a zero here: v is alpha times the sum
                p.diag[t.batch * p.v_bs + row] = v[j] + p.q0 + d * (p.q1 + p.q2 * d);
                v[j] = 0.0f;
            }
    }
    if (p.out_bf16) {
        if (!row_ok) return;
        __nv_bfloat16 *out = (__nv_bfloat16 *)p.out + t.batch * p.out_bs + (long long)row * p.out_ld;
        if (p.out_ld % 8 == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (c0 + 8 * q < p.cols)
                    *reinterpret_cast<uint4 *>(out + c0 + 8 * q) = make_uint4(pack2(v[8 * q], v[8 * q + 1]), pack2(v[8 * q + 2], v[8 * q + 3]),
                                                                              pack2(v[8 * q + 4], v[8 * q + 5]), pack2(v[8 * q + 6], v[8 * q + 7]));
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (c0 + j < p.cols) out[c0 + j] = __float2bfloat16_rn(v[j]);
        }
        return;
    }
    uint32_t h[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) h[j] = pack_half2(v[2 * j], v[2 * j + 1]);
    __half *base = (__half *)p.out + t.batch * p.out_bs;
    if (row_ok) {
        __half *out = base + (long long)row * p.out_ld;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (c0 + 8 * q < p.cols) *reinterpret_cast<uint4 *>(out + c0 + 8 * q) = make_uint4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
    }
    if (t.mirror) {
        // lanes hold consecutive rows of the same columns: a pair of lanes exchanges halves, the even one stores rows
        // (r, r + 1) of column c, the odd one rows (r - 1, r) of column c + 1: two 64-byte pieces of two output rows per store
        const bool odd = lane & 1;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, h[j], 1);
            const uint32_t w = odd ? __byte_perm(other, h[j], 0x7632) : __byte_perm(h[j], other, 0x5410);
            const int c = c0 + 2 * j + (odd ? 1 : 0), r = row & ~1;
            if (c < p.cols && r < p.rows) *reinterpret_cast<uint32_t *>(base + (long long)c * p.out_ld + r) = w;
        }
    }
}

}  // namespace orth
}  // namespace relay
