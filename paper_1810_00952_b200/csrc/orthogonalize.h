// The products of an orthogonalisation: what the host describes and the tensor-core kernel (orthogonalize_tc.cu) runs.
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>

#include "common.h"
#include "ewise_kernels.cuh"

namespace relay {
namespace orth {

// The coefficients of each step.  X is kept times 2^-r, r by step, where the iteration leaves the 16-bit operands' range: see steps_of.
constexpr int kMostSteps = 16;
struct Steps {
    int n;
    float a[kMostSteps], b[kMostSteps], c[kMostSteps];
    float scale;                       // of the result
};
Steps steps_of(const relay_orthogonalize_attrs_t &at, double s);

// One product on a batch of fp16 matrices:
//   out[r,c] = alpha sum_k A(r,k) B(k,c) + (beta + gamma (row_v[r] + col_v[c])) add[r,c]
// and, for the symmetric ones, the diagonal apart from it in fp32 (out then has a zero there):
//   diag[r] = alpha sum_k A(r,k) B(k,r) + q0 + q1 d[r] + q2 d[r]^2,  d = row_v (zero if null)
struct Product {
    int rows, cols, k_blocks;          // of one result; contraction steps of 64
    int tiles_m, units;                // row blocks of 256; units per matrix
    int symmetric;                     // units on and above the diagonal only, stored to both places
    int a_mn, b_mn;                    // operand's row / column index contiguous in memory (else the contraction index)
    float alpha, beta, gamma;
    const void *add;                   // fp16 or null
    long long add_ld, add_bs;          // row and matrix strides in elements
    const float *row_v, *col_v;        // [batch][v_bs] or null (zero)
    float *diag;                       // [batch][v_bs] or null
    float q0, q1, q2;
    long long v_bs;
    void *out;                         // fp16, or bf16 where out_bf16 is set
    long long out_ld, out_bs;
    int out_bf16;
};

// How a product of one matrix is cut into units, widest first.  n = 0: 256 x 256 units in order.
struct UnitTable {
    static constexpr int kMax = 640;
    int n;
    uint32_t e[kMax];                  // row block (256 rows) | first piece of 64 columns << 8 | pieces << 19
};

// tensor maps of one launch: X in both buffers, with its columns or its rows as contraction index, G and P (64: boxes for B)
enum Map { X_K0, X_K1, X_K64_0, X_K64_1, X_MN0, X_MN1, G_K, G_K64, P_K, P_K64, MAPS };

struct Launch {
    CUtensorMap map[MAPS];
    Product product[4];                // G, P, X; X of the last step
    void *x[2];                        // X's buffers: step k reads x[k & 1] and writes the other
    UnitTable table[3];
    Steps step;
    unsigned int *done;                // per matrix, zero at the start: epilogue warps that have finished a unit
    int tall, batch;
    int *err;
};

relay_status_t launch_products(Launch &l, int sms, cudaStream_t st);

// Matrices that stay on the chip (orthogonalize_resident.cu): all of a call in one launch.
bool resident_fits(int64_t m, int64_t n);
relay_status_t launch_resident(const relay_tensor_t *x, const Steps &steps, float eps, const relay_tensor_t *y, int64_t L, int M, int N, float s, cudaStream_t st);

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t instr_desc_f16(int m, int n, int a_mn, int b_mn)
{   // fp32 accumulator, fp16 A and B (format 0), majorness, N / 8, M / 16
    return (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <typename T>
__device__ __forceinline__ float element(const T *p)
{
    if (!relay_in_bounds(p, sizeof(T))) return 0.0f;
    if constexpr (sizeof(T) == 2) return __bfloat162float(*p);
    else return *p;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&v);
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
// s / (norm + eps) in two factors, each of them within fp32's range where the whole may not be
__device__ __forceinline__ void normalizer(double squares, float eps, float s, float &f1, float &f2)
{
    const double f = (double)s / (sqrt(squares) + (double)eps);
    int e;
    const float lo = (float)frexp(f, &e);
    f1 = ldexpf(lo, e / 2);
    f2 = ldexpf(1.0f, e - e / 2);
}
#endif

}  // namespace orth

// 3-D tensor map of `batch` fp16 matrices: `inner` contiguous elements per row, 128-byte swizzle, zero outside
relay_status_t make_tmap_3d_f16(CUtensorMap *m, const void *base, uint64_t inner, uint64_t outer, uint64_t batch, uint64_t row_stride,
                                uint64_t batch_stride, uint32_t box_inner, uint32_t box_outer);

}  // namespace relay
