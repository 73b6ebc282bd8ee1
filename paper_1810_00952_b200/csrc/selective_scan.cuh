// Pieces shared by the selective scan (selective_scan.cu) and its gradient (selective_scan_grad.cu).
//
// Per step, channel and state: an exponential, and a multiply-add each for its argument, for what is added, for the state and for the
// result.  With N = 16 the special-function pipe (16 lanes an SM) is what bounds the forward call before memory does: 2048 x 8 x 2048 x 16 are 537 M
// exponentials and 134 M of steps and gates, 150 us, beside 41 us of bytes.
#pragma once
#include <cfloat>

#include "sequence.cuh"
#include "tc_common.cuh"

namespace relay {
namespace scan {

using namespace seq;

constexpr int kSpan = RELAY_SCAN_SPAN;
constexpr float kLog2e = 1.44269504f;

struct Args {
    const void *u, *delta, *z;             // [T][B][D]; z or null
    const float *a;                        // [D][N]
    const void *b, *c;                     // row of step t, batch element i: + (t * B + i) * ld_bc, N entries
    const float *d, *delta_bias;           // [D] or null
    const float *h0;                       // [B][D][N] or null
    const int *lengths;                    // [B] or null
    void *y;                               // [T][B][D]
    float *h_final, *states;               // [B][D][N], [spans][B][D][N]; each or null
    // gradient
    const void *dy;                        // [T][B][D]
    const float *dh_final;                 // [B][D][N] or null
    void *du, *ddelta, *dz;                // [T][B][D]; dz or null
    float *dh0;                            // [B][D][N] or null
    float *part_bc;                        // [groups][T * B][2N]: each group of channels' sums of db and dc
    float *part_a;                         // [B][D N | D | D]: each batch element's sums of da, dd and ddelta_bias
    long long T, B, D;
    int N, ld_bc, softplus, groups;
    int pairs;                             // two neighbouring channels are one aligned access
    int four;                              // four are
    int quads;                             // four neighbouring states are one aligned access
    int tma_x, tma_w;                      // rows of channels, and of b and c, are whole 16-byte pieces: TMA fetches them
    int *err;
};
// what TMA fetches, as (B*D columns, T rows) and (B * ld_bc columns, T rows)
struct Maps { CUtensorMap u, delta, z, dy, b, c; };

__device__ __forceinline__ long long end_of(const Args &p, long long i)
{
    if (p.lengths == nullptr) return p.T;
    const long long n = relay_in_bounds(p.lengths + i, 4) ? p.lengths[i] : 0;
    return n < 0 ? 0 : n > p.T ? p.T : n;
}

// softplus(x) = max(x, 0) + log(1 + w), w = exp(-|x|) <= 1, of two values, and its slope, the logistic function.  log(1 + w) = w q(w), q
// the polynomial of degree nine with q(0) = 1 whose largest relative error on [0,1] is the least (5.3e-9): steps are small numbers, and a relative
// error in one moves a whole state.  w = 2^t with what the rounding of t = -|x| log2(e) left put back; from 128 on w is zero, and x may be infinite
// (a step of -inf is one of no length) or so large that t would be.
struct Softplus { f32x2 value, w; };
__device__ __forceinline__ float down_to_128(float x) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(-fabsf(x)), "f"(-128.0f)); return y; }
__device__ __forceinline__ Softplus softplus2(f32x2 x)
{
    constexpr float of[10] = {1.0f, -4.999993145e-01f, 3.333046436e-01f, -2.495802045e-01f, 1.969212145e-01f, -1.534497738e-01f, 1.066137105e-01f,
                              -5.746048316e-02f, 2.008846030e-02f, -3.291074187e-03f};
    float a, b;
    unpair(x, a, b);
    const f32x2 m = pair(down_to_128(a), down_to_128(b));                  // -|x|
    const f32x2 t = mul2(m, pair(kLog2e, kLog2e));
    f32x2 left = fma2(m, pair(kLog2e, kLog2e), neg2(t));
    left = fma2(m, pair(1.925963033e-8f, 1.925963033e-8f), left);          // log2(e) beyond fp32
    unpair(t, a, b);
    const f32x2 p = pair(exp2_(a), exp2_(b)), w = fma2(p, mul2(left, pair(0.693147181f, 0.693147181f)), p);
    f32x2 r = pair(of[9], of[9]);
#pragma unroll
    for (int k = 8; k >= 0; --k) r = fma2(r, w, pair(of[k], of[k]));
    unpair(x, a, b);
    return Softplus{fma2(r, w, pair(fmaxf(a, 0.0f), fmaxf(b, 0.0f))), w};
}
__device__ __forceinline__ float softplus_slope(float x, float w)
{
    const float small = __fdividef(w, 1.0f + w);
    return x >= 0.0f ? 1.0f - small : small;
}

// two or four neighbouring channels
template <typename T, int G>
__device__ __forceinline__ void store_some(const Args &p, void *base, long long row, long long c, const float (&x)[G])
{
    if (G == 2 ? p.pairs : p.four) {
        if (c < p.D) store<T, G>(base, row + c, x);
        return;
    }
#pragma unroll
    for (int j = 0; j < G; ++j) {
        const float q[1] = {x[j]};
        if (c + j < p.D) store<T, 1>(base, row + c + j, q);
    }
}
// one value as it is stored
template <typename T>
__device__ __forceinline__ T load_raw_one(const void *base, long long at)
{
    const T *p = (const T *)base + at;
    return relay_in_bounds(p, sizeof(T)) ? *p : T(0.0f);
}
// two or four neighbouring values in shared memory, as fp32
__device__ __forceinline__ void widen_shared(const __nv_bfloat16 *p, float (&x)[4]) { widen(*reinterpret_cast<const uint2 *>(p), x, __nv_bfloat16()); }
__device__ __forceinline__ void widen_shared(const float *p, float (&x)[4]) { unpack(*reinterpret_cast<const uint4 *>(p), x); }
__device__ __forceinline__ void widen_shared(const __nv_bfloat16 *p, float (&x)[2]) { widen(*reinterpret_cast<const uint32_t *>(p), x, __nv_bfloat16()); }
__device__ __forceinline__ void widen_shared(const float *p, float (&x)[2]) { widen(*reinterpret_cast<const uint2 *>(p), x, float()); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }

// 2^x of two exponents.  The hardware's exponential is 2e-8 low on average, and a state adds that up over the steps in which it forgets: a
// thousand of them where |x| is 1/1000.  So up to 1/32 (a memory of 46 steps) the value comes from 2^x = 1 + z + z^2 / 2 + z^3 / 6, z = x log 2, which
// leaves out 9e-9 at 1/32 and sixteen times less at every halving; its last rounding is to the nearest.  One more term and 1/16 as the border: 5 % slower.
__device__ __forceinline__ f32x2 decay2(f32x2 x)
{
    f32x2 q = fma2(x, pair(5.55041087e-2f, 5.55041087e-2f), pair(0.240226507f, 0.240226507f));
    q = fma2(q, x, pair(0.693147181f, 0.693147181f));
    q = fma2(q, x, pair(1.0f, 1.0f));
    float a, b, c, d;
    unpair(x, a, b);
    unpair(q, c, d);
    return pair(fabsf(a) <= 0.03125f ? c : exp2_(a), fabsf(b) <= 0.03125f ? d : exp2_(b));
}

// a log2(e), what a step multiplies for its exponent: finite, so that a step of no length (those behind a sequence's end are such) has the decay 1
// even where a, or this product, is beyond fp32: 0 inf would be NaN.  Any step that is not as small as 1e-36 leaves nothing then, as it should.
__device__ __forceinline__ float exponent_of(float a)
{
    float x;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(a * kLog2e), "f"(-FLT_MAX));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(x), "f"(FLT_MAX));
    return x;
}

// ---- rows that TMA cannot fetch ------------------------------------------------------------------------------------------
// A copy of four bytes to shared memory that nothing waits for until copies_done.
__device__ __forceinline__ void copy_four(void *to, const void *from)
{
    if (relay_in_bounds(from, 4)) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(tc::smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// all but the last `younger` (0 or 1) groups of this thread's copies have arrived
__device__ __forceinline__ void copies_done(int younger)
{
    if (younger > 0) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
// `rows` rows of `width` values from `from`, `ld` values apart, to rows of `to_ld` values; four bytes at a time where both sides' rows are
// whole four bytes, else one by one (bf16 rows of odd length)
template <typename T>
__device__ __forceinline__ void copy_rows(T *to, int to_ld, const T *from, long long ld, int rows, int width, int tid, int threads)
{
    constexpr int E = 4 / sizeof(T);
    if (sizeof(T) == 4 || (ld % 2 == 0 && width % 2 == 0 && ((uintptr_t)from & 3) == 0)) {
        const int per = width / E, down = threads / per, along = threads - down * per;
        int t = tid / per, c = tid - t * per;
        while (t < rows) {
            copy_four(to + t * to_ld + c * E, from + t * ld + c * E);
            t += down;
            c += along;
            if (c >= per) { c -= per; ++t; }
        }
        return;
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll 4
        for (int e = tid; e < rows * width; e += threads) {
            const int t = e / width, c = e - t * width;
            to[t * to_ld + c] = load_raw_one<T>(from, t * ld + c);
        }
    }
}

// four neighbouring states n .. n + 3 of an f32 tensor [..][N] at entry `at`; those from N on are zero
__device__ __forceinline__ void load_states(const Args &p, const float *base, long long at, int n, float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = 0.0f;
    if (base == nullptr) return;
    if (p.quads) {
        if (n < p.N) load<float, 4>(base, at + n, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < p.N && relay_in_bounds(base + at + n + i, 4)) x[i] = __ldcs(base + at + n + i);
}
__device__ __forceinline__ void store_states(const Args &p, float *base, long long at, int n, const float (&x)[4])
{
    if (base == nullptr) return;
    if (p.quads) {
        if (n < p.N) store<float, 4>(base, at + n, x);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < p.N && relay_in_bounds(base + at + n + i, 4)) __stcs(base + at + n + i, x[i]);
}
// one value of b or c
template <typename T>
__device__ __forceinline__ float load_weight(const void *base, long long at)
{
    float q[1];
    load<T, 1>(base, at, q);
    return q[0];
}

// Sums over the lanes that differ in the bits BIT, 2 BIT, .. of V values each: half of the values change hands at every bit, so that a
// lane ends with the sums of V / LANES of them: those at j LANES + (the lane's position among the LANES).
template <int V, int BIT, int LANES>
__device__ __forceinline__ void reduce_lanes(float (&x)[V], int lane, float (&out)[V / LANES])
{
    if constexpr (LANES == 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = x[i];
    } else {
        float y[V / 2];
        const bool odd = lane & BIT;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float keep = odd ? x[2 * i + 1] : x[2 * i], send = odd ? x[2 * i] : x[2 * i + 1];
            y[i] = keep + __shfl_xor_sync(0xffffffffu, send, BIT);
        }
        reduce_lanes<V / 2, 2 * BIT, LANES / 2>(y, lane, out);
    }
}

// ---- the boundary's part that both calls share ---------------------------------------------------------------------------
struct Inputs { const relay_tensor_t *u, *delta, *a, *b, *c, *d, *z, *delta_bias, *lengths; };
relay_status_t make_maps(Args *p, Maps *m, bool f32, int channels, int steps);
relay_status_t check_sizes(const relay_tensor_t *u, const relay_tensor_t *a, Sizes *s, int64_t *N);
relay_status_t check_inputs(const Inputs &in, Sizes *s, int64_t *N);
relay_status_t check_softplus(int32_t softplus);
Args make_args(const Inputs &in, int32_t softplus, const Sizes &s, int64_t N);

}  // namespace scan
}  // namespace relay
