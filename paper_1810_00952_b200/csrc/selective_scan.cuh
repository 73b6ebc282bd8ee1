// Pieces shared by the selective scan (selective_scan.cu) and its gradient (selective_scan_grad.cu).
//
// Both cut a sequence into chunks and a chunk into runs of a few steps, one run per warp of a row of warps.  A lane holds four
// neighbouring states of a channel, four lanes a block of sixteen.  Every warp sums its run up from a zero state, once, keeping the decays
// exp(delta a) in registers (the exponentials are what the forward call is bounded by); the runs' products and sums meet in shared memory,
// every warp joins those before its own, and the run is summed again from the state that it really starts with.
#pragma once
#include "sequence.cuh"

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
    float *part_a, *part_d, *part_bias;    // [B][D][N], [B][D], [B][D]; the last two or null
    long long T, B, D;
    int N, ld_bc, softplus, groups;
    int pairs;                             // two neighbouring channels are one aligned access
    int quads;                             // four neighbouring states are one aligned access
};

__device__ __forceinline__ long long end_of(const Args &p, long long i)
{
    if (p.lengths == nullptr) return p.T;
    const long long n = relay_in_bounds(p.lengths + i, 4) ? p.lengths[i] : 0;
    return n < 0 ? 0 : n > p.T ? p.T : n;
}

// softplus(x) = max(x, 0) + log(1 + w), w = exp(-|x|) <= 1, and its slope, the logistic function.  log(1 + w) = 2 atanh(s), s = w / (2 + w) <=
// 1/3, by the series of atanh up to s^13 (the rest is below 3^-15 / 15 = 5e-9 of one): steps are small numbers, and a relative error in one
// moves a whole state.  w = 2^t with what the rounding of t = -|x| log2(e) left put back.
__device__ __forceinline__ float softplus_(float x, float &slope)
{
    const float m = -fabsf(x), t = m * kLog2e;
    const float left = fmaf(m, kLog2e, -t) + m * 1.925963033e-8f;            // log2(e) beyond fp32
    const float p = exp2_(t), w = fmaf(p, left * 0.693147181f, p);
    const float s = __fdividef(w, 2.0f + w), q = s * s;
    float r = fmaf(q, 1.0f / 13.0f, 1.0f / 11.0f);
    r = fmaf(r, q, 1.0f / 9.0f);
    r = fmaf(r, q, 1.0f / 7.0f);
    r = fmaf(r, q, 0.2f);
    r = fmaf(r, q, 1.0f / 3.0f);
    r = fmaf(r, q, 1.0f);
    const float small = __fdividef(w, 1.0f + w);
    slope = x >= 0.0f ? 1.0f - small : small;
    return fmaxf(x, 0.0f) + 2.0f * s * r;
}

// two neighbouring channels c, c + 1 of a row that starts at `row`; those from D on are zero
template <typename T>
__device__ __forceinline__ void load_channels(const Args &p, const void *base, long long row, long long c, float (&x)[2])
{
    if (p.pairs) { load<T, 2>(base, row + c, x); return; }
    float q[1];
    load<T, 1>(base, row + c, q);
    x[0] = q[0];
    x[1] = 0.0f;
    if (c + 1 < p.D) { load<T, 1>(base, row + c + 1, q); x[1] = q[0]; }
}
template <typename T>
__device__ __forceinline__ void store_channels(const Args &p, void *base, long long row, long long c, const float (&x)[2])
{
    if (p.pairs) { store<T, 2>(base, row + c, x); return; }
    const float lo[1] = {x[0]}, hi[1] = {x[1]};
    store<T, 1>(base, row + c, lo);
    if (c + 1 < p.D) store<T, 1>(base, row + c + 1, hi);
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
relay_status_t check_sizes(const relay_tensor_t *u, const relay_tensor_t *a, Sizes *s, int64_t *N);
relay_status_t check_inputs(const Inputs &in, Sizes *s, int64_t *N);
relay_status_t check_softplus(int32_t softplus);
Args make_args(const Inputs &in, int32_t softplus, const Sizes &s, int64_t N);

}  // namespace scan
}  // namespace relay
