// The product that every step of an orthogonalisation is made of, on batches of fp16 matrices in the workspace:
//   out[r,c] = alpha sum_k A(r,k) B(k,c) + (beta + gamma (row_v[r] + col_v[c])) add[r,c]
// and, for the symmetric ones, the diagonal apart from it in fp32 (out then has a zero there):
//   diag[r] = alpha sum_k A(r,k) B(k,r) + q0 + q1 d[r] + q2 d[r]^2,  d = row_v (zero if null)
#pragma once
#include <cuda.h>

#include "common.h"

namespace relay {
namespace orth {

struct Product {
    int rows, cols;                    // of one result
    int tiles_m, tiles_n, k_blocks;
    int units, batch;                  // tiles to compute per matrix, matrices
    int symmetric;                     // tiles on and above the diagonal only, stored to both places
    float alpha, beta, gamma;
    const float *row_v, *col_v;        // [batch][v_bs] or null (zero)
    long long v_bs;
    float *diag;                       // [batch][v_bs] or null
    float q0, q1, q2;
    const void *add;                   // fp16 or null
    long long add_ld, add_bs;          // row and matrix strides in elements
    void *out;                         // fp16, or bf16 where out_bf16 is set
    long long out_ld, out_bs;
    int out_bf16;
    int *err;
};

// How the two-SM kernel cuts a product into units, made once for the products of equal shape.  n = 0: 256 x 256 units in order.
struct UnitTable {
    static constexpr int kMax = 640;
    int n;
    uint32_t e[kMax];                  // row block (256 rows) | first 128-column chunk << 8 | chunks << 17 | matrix << 20
};
void plan_units(const Product &p, int sms, UnitTable *table);

// two-SM kernel (orthogonalize_pair.cu); boxes of its operands: 128 rows of A, 64 of B where the contraction index is contiguous,
// else 64 x 64
relay_status_t launch_product_pair(const Product &p, bool a_mn, bool b_mn, const CUtensorMap &a, const CUtensorMap &b, const UnitTable &units, int sms,
                                   cudaStream_t st);

}  // namespace orth

// 3-D tensor map of `batch` fp16 matrices: `inner` contiguous elements per row, 128-byte swizzle, zero outside
relay_status_t make_tmap_3d_f16(CUtensorMap *m, const void *base, uint64_t inner, uint64_t outer, uint64_t batch, uint64_t row_stride,
                                uint64_t batch_stride, uint32_t box_inner, uint32_t box_outer);
// 3-D tensor map for stores of 32 x 32 blocks of 16-bit elements, 64-byte swizzle or none
relay_status_t make_tmap_3d_block(CUtensorMap *m, bool bf16, const void *base, uint64_t inner, uint64_t outer, uint64_t batch, uint64_t row_stride,
                                  uint64_t batch_stride, bool swizzle64);

}  // namespace relay
