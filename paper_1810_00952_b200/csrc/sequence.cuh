// Pieces shared by the operators over sequences of a state space language model (causal_conv.cu, selective_scan*.cu): vectors of
// consecutive channels in memory, activations, and the checks of tensors (T,B,D).
#pragma once
#include <initializer_list>

#include "common.h"
#include "ewise_kernels.cuh"

namespace relay {
namespace seq {

// ---- V consecutive channels in memory, as fp32 in registers ------------------------------------------------
template <int BYTES> struct RawOf;
template <> struct RawOf<2> { using type = unsigned short; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<16> { using type = uint4; };
template <typename T, int V> using Raw = typename RawOf<(int)sizeof(T) * V>::type;

// each value is touched once: past L1
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> load_raw(const void *base, long long at)
{
    const T *p = (const T *)base + at;
    if (!relay_in_bounds(p, sizeof(T) * V)) return Raw<T, V>{};
    return __ldcs((const Raw<T, V> *)p);
}
__device__ __forceinline__ void widen(unsigned short r, float (&x)[1], __nv_bfloat16) { x[0] = __uint_as_float((uint32_t)r << 16); }
__device__ __forceinline__ void widen(uint32_t r, float (&x)[2], __nv_bfloat16) { x[0] = __uint_as_float(r << 16); x[1] = __uint_as_float(r & 0xffff0000u); }
__device__ __forceinline__ void widen(uint2 r, float (&x)[4], __nv_bfloat16)
{
    x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xffff0000u);
    x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xffff0000u);
}
__device__ __forceinline__ void widen(uint4 r, float (&x)[8], __nv_bfloat16) { unpack(r, x); }
__device__ __forceinline__ void widen(uint32_t r, float (&x)[1], float) { x[0] = __uint_as_float(r); }
__device__ __forceinline__ void widen(uint2 r, float (&x)[2], float) { x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); }
__device__ __forceinline__ void widen(uint4 r, float (&x)[4], float) { unpack(r, x); }
__device__ __forceinline__ void narrow(const float (&x)[1], unsigned short &r) { r = __bfloat16_as_ushort(__float2bfloat16_rn(x[0])); }
__device__ __forceinline__ void narrow(const float (&x)[2], uint32_t &r) { r = pack2(x[0], x[1]); }
__device__ __forceinline__ void narrow(const float (&x)[4], uint2 &r) { r = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3])); }
__device__ __forceinline__ void narrow(const float (&x)[8], uint4 &r) { r = pack(x); }
__device__ __forceinline__ void narrow(const float (&x)[1], uint32_t &r) { r = __float_as_uint(x[0]); }
__device__ __forceinline__ void narrow(const float (&x)[2], uint2 &r) { r = make_uint2(__float_as_uint(x[0]), __float_as_uint(x[1])); }
__device__ __forceinline__ void narrow(const float (&x)[4], uint4 &r) { r = pack(x); }

template <typename T, int V>
__device__ __forceinline__ void load(const void *base, long long at, float (&x)[V])
{
    widen(load_raw<T, V>(base, at), x, T());
}
template <typename T, int V>
__device__ __forceinline__ void store(void *base, long long at, const float (&x)[V])
{
    T *p = (T *)base + at;
    Raw<T, V> r;
    narrow(x, r);
    if (relay_in_bounds(p, sizeof(T) * V)) __stcs((Raw<T, V> *)p, r);
}
// one value of an operand whose base type is known at run time (small operands: filters, biases)
__device__ __forceinline__ float load_one(const void *p, bool bf16, long long at)
{
    if (!relay_in_bounds((const char *)p + at * (bf16 ? 2 : 4), bf16 ? 2 : 4)) return 0.0f;
    return bf16 ? __bfloat162float(((const __nv_bfloat16 *)p)[at]) : ((const float *)p)[at];
}

// V of them
template <int V>
__device__ __forceinline__ void load_operand(const void *p, bool bf16, long long at, float (&x)[V])
{
    if (V == 1) { x[0] = load_one(p, bf16, at); return; }
    if (bf16) load<__nv_bfloat16, V>(p, at, x);
    else {
        constexpr int W = V < 4 ? V : 4;
#pragma unroll
        for (int i = 0; i < V; i += W) {
            float q[W];
            load<float, W>(p, at + i, q);
#pragma unroll
            for (int j = 0; j < W; ++j) x[i + j] = q[j];
        }
    }
}

// ---- two fp32 values at a time (one instruction for both) ------------------------------------------------------
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(f32x2 r, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(r)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 neg2(f32x2 a) { return a ^ 0x8000000080000000ull; }
__device__ __forceinline__ float sum2(f32x2 a) { float x, y; unpair(a, x, y); return x + y; }
// r = a b + c and r = a b of V values, in pairs where V is even
template <int V>
__device__ __forceinline__ void muladd(const float (&a)[V], const float (&b)[V], const float (&c)[V], float (&r)[V])
{
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) unpair(fma2(pair(a[i], a[i + 1]), pair(b[i], b[i + 1]), pair(c[i], c[i + 1])), r[i], r[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = fmaf(a[i], b[i], c[i]);
    }
}
template <int V>
__device__ __forceinline__ void mul(const float (&a)[V], const float (&b)[V], float (&r)[V])
{
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) unpair(mul2(pair(a[i], a[i + 1]), pair(b[i], b[i + 1])), r[i], r[i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = a[i] * b[i];
    }
}
__device__ __forceinline__ float rcp_(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float exp2_(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// ---- activations ---------------------------------------------------------------------------------------------
// 1 / (1 + exp(-x)), a few units off: a bf16 result hides that, and fp32 results take the accurate routines (FINE).  The form
// with tanh costs one instruction less, but what it leaves of the sigmoid of -6 has three bits fewer than bf16.
template <bool FINE>
__device__ __forceinline__ float logistic(float x)
{
    if constexpr (FINE) return 1.0f / (1.0f + expf(-x));
    else return rcp_(1.0f + exp2_(-1.44269504f * x));     // 1 / inf = 0 far below zero, as it should be
}

// Sums of the columns of partial sums (rows,cols) in a fixed order: the first n[0] columns to out[0], the next n[1] to out[1] and so on, cols
// in all (an out may be null: not wanted).
constexpr int kSums = 3;
struct ColumnSums { float *out[kSums]; long long n[kSums]; };
relay_status_t launch_column_sums(const float *in, long long rows, const ColumnSums &to, cudaStream_t st);

// ---- checks ----------------------------------------------------------------------------------------------------
// an optional tensor of one of two base types and the given extents
inline relay_status_t check_tensor(const relay_tensor_t *t, int32_t d0, int32_t d1, std::initializer_list<int64_t> shape, const char *name)
{
    if (!t) return RELAY_OK;
    RELAY_TRY(check_type(t, name));
    RELAY_TRY(check_rank(t, (int)shape.size(), name));
    if (t->dtype != d0 && t->dtype != d1)
        return fail(RELAY_ERR_DTYPE, "%s: base type %s, needs %s%s%s", name, dtype_name(t->dtype), dtype_name(d0), d0 == d1 ? "" : " or ",
                    d0 == d1 ? "" : dtype_name(d1));
    RELAY_TRY(check_layout(t, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
    return check_shape(t, shape, name);
}
// (T,B,D) of a float type, the operand that gives the sizes
struct Sizes { int64_t T, B, D; };
inline relay_status_t check_sequence(const relay_tensor_t *t, Sizes *s, const char *name)
{
    RELAY_TRY(check_type(t, name));
    RELAY_TRY(check_rank(t, 3, name));
    if (!is_float(t->dtype)) return fail(RELAY_ERR_DTYPE, "%s: base type %s, needs f32 or bf16", name, dtype_name(t->dtype));
    RELAY_TRY(check_layout(t, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
    s->T = t->shape[0]; s->B = t->shape[1]; s->D = t->shape[2];
    return RELAY_OK;
}
template <int NI, int NO>
inline relay_status_t check_buffers(const relay_tensor_t *const (&ins)[NI], const relay_tensor_t *const (&outs)[NO])
{
    for (const relay_tensor_t *t : ins) if (t) RELAY_TRY(check_data(t, "input"));
    for (const relay_tensor_t *t : outs) if (t) RELAY_TRY(check_data(t, "output"));
    return check_no_overlap(outs, NO, ins, NI);
}
// (of this file alone: the table of the bounds-check build is one per source file)
template <int NI, int NO>
static relay_status_t register_buffers(const relay_tensor_t *const (&ins)[NI], const relay_tensor_t *const (&outs)[NO], void *ws, size_t ws_bytes,
                                       cudaStream_t st)
{
    BoundsReg reg;
    for (const relay_tensor_t *t : ins) reg.add(t);
    for (const relay_tensor_t *t : outs) reg.add(t);
    reg.add(ws, ws_bytes);
    return reg.commit(st);
}

}  // namespace seq
}  // namespace relay
