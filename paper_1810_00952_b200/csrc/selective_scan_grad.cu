// Gradient group of the selective scan (Section 4.2 of the paper: reverse mode through the recursion over time).
#include <algorithm>

#include "selective_scan.cuh"

namespace relay {
namespace {

using namespace scan;

// A block: WC warps side by side, of sixteen channels each (two a lane), WT rows of them, each with a run of RUN steps; the chunk is the span
// whose starting states the forward call saved.
constexpr int RUN = 4, WT = kSpan / RUN, STEPS = kSpan;
__host__ __device__ constexpr int columns_of(int NB) { return NB == 1 ? 2 : 1; }

template <int NB>
struct Tile {
    static constexpr int WC = columns_of(NB), THREADS = 32 * WT * WC, CHANNELS = 16 * WC, NP = 16 * NB, SLOTS = NB == 1 ? 1 : 2;
    float2 step[STEPS][CHANNELS];                          // delta, delta u
    float e[STEPS][CHANNELS];                              // dy silu(z)
    float b[STEPS][NP], c[STEPS][NP];
    float4 decay[SLOTS][WT][WC][2][32], sum[SLOTS][WT][WC][2][32], back[SLOTS][WT][WC][2][32];
    float along[STEPS][CHANNELS], kept[STEPS][CHANNELS], plain[STEPS][CHANNELS];   // sum_n g b, sum_n a G h[t-1], sum_n c h
    float dbc[WC][STEPS][2 * NP];
    float2 u[THREADS], slope[THREADS], gate[THREADS];      // what a thread needs again at the end of a chunk
    float4 slots[NB == 1 ? 1 : NB][4][NB == 1 ? 1 : THREADS];   // more than sixteen states: carries and sums of da wait here
};

template <typename T, int NB>
__global__ void __launch_bounds__(32 * WT * columns_of(NB), 1) selective_scan_grad_kernel(const Args p)
{
    using S = Tile<NB>;
    constexpr bool FINE = sizeof(T) == 4;
    constexpr int WC = S::WC, WEIGHTS = (STEPS * S::NP + S::THREADS - 1) / S::THREADS;
    extern __shared__ uint4 shared_raw[];
    S &s = *reinterpret_cast<S *>(shared_raw);
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wt = warp / WC, wc = warp % WC, nl = lane & 3, cl = lane >> 2;
    const long long i = blockIdx.x / p.groups;
    const int group = (int)(blockIdx.x - i * p.groups);
    const long long c0 = (long long)group * S::CHANNELS, end = end_of(p, i);
    const int ch = wc * 16 + cl * 2;                       // this lane's channels: ch, ch + 1 of the block
    const long long mine = c0 + ch;
    // sixteen states: everything that lives from chunk to chunk is in registers
    f32x2 a1[2][2], G1[2][2], dA1[2][2];                   // a log2(e), what flows back into the chunk, sums of da
    auto load_a = [&](int k, f32x2 (&a)[2][2]) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float x[4];
            load_states(p, mine + j < p.D ? p.a : nullptr, (mine + j) * p.N, k * 16 + nl * 4, x);
            a[j][0] = pair(x[0] * kLog2e, x[1] * kLog2e);
            a[j][1] = pair(x[2] * kLog2e, x[3] * kLog2e);
        }
    };
    auto to_slot = [&](int k, int at, const f32x2 (&v)[2][2]) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float4 x;
            unpair(v[j][0], x.x, x.y); unpair(v[j][1], x.z, x.w);
            s.slots[k][at + j][tid] = x;
        }
    };
    auto from_slot = [&](int k, int at, f32x2 (&v)[2][2]) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float4 x = s.slots[k][at + j][tid];
            v[j][0] = pair(x.x, x.y); v[j][1] = pair(x.z, x.w);
        }
    };
#pragma unroll
    for (int k = 0; k < NB; ++k) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float x[4];
            load_states(p, mine + j < p.D ? p.dh_final : nullptr, (i * p.D + mine + j) * p.N, k * 16 + nl * 4, x);
            G1[j][0] = pair(x[0], x[1]); G1[j][1] = pair(x[2], x[3]);
            dA1[j][0] = dA1[j][1] = pair(0.0f, 0.0f);
        }
        if constexpr (NB > 1) { to_slot(k, 0, G1); to_slot(k, 2, dA1); }
    }
    if constexpr (NB == 1) load_a(0, a1);
    // this thread's pair of channels and step of the chunk in what surrounds the scan
    const int pt = tid / (S::CHANNELS / 2), pc = 2 * (tid % (S::CHANNELS / 2));
    const long long two = c0 + pc;
    float skip[2] = {0.0f, 0.0f}, bias[2] = {0.0f, 0.0f}, dd[2] = {0.0f, 0.0f}, dbias[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 2; ++j)
        if (two + j < p.D) {
            if (p.d && relay_in_bounds(p.d + two + j, 4)) skip[j] = p.d[two + j];
            if (p.delta_bias && relay_in_bounds(p.delta_bias + two + j, 4)) bias[j] = p.delta_bias[two + j];
        }
    float u[2], raw[2], z[2], dy[2], wb[WEIGHTS], wc_[WEIGHTS];
    auto fetch = [&](long long t0) {
        const long long t = t0 + pt;
#pragma unroll
        for (int j = 0; j < 2; ++j) u[j] = raw[j] = z[j] = dy[j] = 0.0f;
        if (t < end && two < p.D) {
            const long long row = (t * p.B + i) * p.D;
            load_channels<T>(p, p.u, row, two, u);
            load_channels<T>(p, p.delta, row, two, raw);
            load_channels<T>(p, p.dy, row, two, dy);
            if (p.z) load_channels<T>(p, p.z, row, two, z);
        }
#pragma unroll
        for (int k = 0; k < WEIGHTS; ++k) {
            const int q = tid + k * S::THREADS, tt = q / S::NP, n = q % S::NP;
            wb[k] = wc_[k] = 0.0f;
            if (t0 + tt < end && n < p.N) {
                const long long at = ((t0 + tt) * p.B + i) * p.ld_bc + n;
                wb[k] = load_weight<T>(p.b, at);
                wc_[k] = load_weight<T>(p.c, at);
            }
        }
    };
    const long long chunks = (p.T + STEPS - 1) / STEPS;
    if (chunks > 0) fetch((chunks - 1) * STEPS);
    for (long long chunk = chunks - 1; chunk >= 0; --chunk) {
        const long long t0 = chunk * STEPS, row = ((t0 + pt) * p.B + i) * p.D;
        const bool stored = t0 + pt < p.T && two < p.D;
        if (t0 >= end) {                                   // behind the sequence (the whole block): nothing flows back
            if (stored) {
                const float zero[2] = {0.0f, 0.0f};
                store_channels<T>(p, p.du, row, two, zero);
                store_channels<T>(p, p.ddelta, row, two, zero);
                if (p.dz) store_channels<T>(p, p.dz, row, two, zero);
            }
            for (int q = tid; q < STEPS * 2 * p.N; q += S::THREADS) {
                const int t = q / (2 * p.N), n = q - t * 2 * p.N;
                float *out = p.part_bc + (((long long)group * p.T + t0 + t) * p.B + i) * 2 * p.N + n;
                if (t0 + t < p.T && relay_in_bounds(out, 4)) *out = 0.0f;
            }
            if (chunk > 0) fetch(t0 - STEPS);
            continue;
        }
        const bool inside = t0 + pt < end;
        {
            float2 uu, sl, gz;
            float step[2], slope[2], e[2], gate[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                step[j] = raw[j] + bias[j];
                slope[j] = 1.0f;
                if (p.softplus) {
                    const Softplus q = softplus2(pair(step[j], step[j]));
                    float v, w;
                    unpair(q.w, w, v);
                    slope[j] = softplus_slope(step[j], w);
                    unpair(q.value, step[j], v);
                }
                if (!inside || two + j >= p.D) step[j] = 0.0f;             // nothing decays and nothing is added
                e[j] = dy[j];
                gate[j] = 0.0f;
                if (p.z) {
                    const float q = logistic<FINE>(z[j]);
                    e[j] *= z[j] * q;
                    gate[j] = dy[j] * q * fmaf(z[j], 1.0f - q, 1.0f);
                }
                s.step[pt][pc + j] = make_float2(step[j], step[j] * u[j]);
                s.e[pt][pc + j] = e[j];
                dd[j] = fmaf(e[j], u[j], dd[j]);
            }
            uu = make_float2(u[0], u[1]); sl = make_float2(slope[0], slope[1]); gz = make_float2(gate[0], gate[1]);
            s.u[tid] = uu; s.slope[tid] = sl; s.gate[tid] = gz;
        }
#pragma unroll
        for (int k = 0; k < WEIGHTS; ++k) {
            const int q = tid + k * S::THREADS;
            if (q < STEPS * S::NP) {
                (&s.b[0][0])[q] = wb[k];
                (&s.c[0][0])[q] = wc_[k];
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int k = 0; k < NB; ++k) {
            const int slot = NB == 1 ? 0 : k & 1;
            if constexpr (NB > 1) { load_a(k, a1); from_slot(k, 0, G1); }
            f32x2 from[2][2];                              // the state at the start of the chunk, then of this run
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x[4];
                load_states(p, mine + j < p.D ? p.states : nullptr, ((chunk * p.B + i) * p.D + mine + j) * p.N, k * 16 + nl * 4, x);
                from[j][0] = pair(x[0], x[1]); from[j][1] = pair(x[2], x[3]);
            }
            if (k == 0 && chunk > 0) fetch(t0 - STEPS);
            f32x2 da[RUN][2][2], h[RUN][2][2];             // decays; what is added, then the states
            {
                f32x2 P[2][2], H[2][2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int q = 0; q < 2; ++q) { P[j][q] = pair(1.0f, 1.0f); H[j][q] = pair(0.0f, 0.0f); }
#pragma unroll
                for (int r = 0; r < RUN; ++r) {
                    const float4 st = *reinterpret_cast<const float4 *>(&s.step[wt * RUN + r][ch]);
                    const float4 b = *reinterpret_cast<const float4 *>(&s.b[wt * RUN + r][k * 16 + nl * 4]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f32x2 dt = j ? pair(st.z, st.z) : pair(st.x, st.x), du = j ? pair(st.w, st.w) : pair(st.y, st.y);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            float lo, hi;
                            unpair(mul2(dt, a1[j][q]), lo, hi);
                            da[r][j][q] = pair(exp2_(lo), exp2_(hi));
                            h[r][j][q] = mul2(du, q ? pair(b.z, b.w) : pair(b.x, b.y));
                            H[j][q] = fma2(da[r][j][q], H[j][q], h[r][j][q]);
                            P[j][q] = mul2(da[r][j][q], P[j][q]);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float4 v;
                    unpair(P[j][0], v.x, v.y); unpair(P[j][1], v.z, v.w);
                    s.decay[slot][wt][wc][j][lane] = v;
                    unpair(H[j][0], v.x, v.y); unpair(H[j][1], v.z, v.w);
                    s.sum[slot][wt][wc][j][lane] = v;
                }
            }
            // what flows back through the run from a zero carry
            {
                f32x2 G[2][2];
#pragma unroll
                for (int j = 0; j < 2; ++j) G[j][0] = G[j][1] = pair(0.0f, 0.0f);
#pragma unroll
                for (int r = RUN - 1; r >= 0; --r) {
                    const float2 e = *reinterpret_cast<const float2 *>(&s.e[wt * RUN + r][ch]);
                    const float4 c = *reinterpret_cast<const float4 *>(&s.c[wt * RUN + r][k * 16 + nl * 4]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f32x2 ee = j ? pair(e.y, e.y) : pair(e.x, e.x);
                        G[j][0] = mul2(da[r][j][0], fma2(ee, pair(c.x, c.y), G[j][0]));
                        G[j][1] = mul2(da[r][j][1], fma2(ee, pair(c.z, c.w), G[j][1]));
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float4 v;
                    unpair(G[j][0], v.x, v.y); unpair(G[j][1], v.z, v.w);
                    s.back[slot][wt][wc][j][lane] = v;
                }
            }
            __syncthreads();
            for (int w = 0; w < wt; ++w)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float4 pw = s.decay[slot][w][wc][j][lane], hw = s.sum[slot][w][wc][j][lane];
                    from[j][0] = fma2(pair(pw.x, pw.y), from[j][0], pair(hw.x, hw.y));
                    from[j][1] = fma2(pair(pw.z, pw.w), from[j][1], pair(hw.z, hw.w));
                }
            f32x2 G[2][2];                                 // what flows back into this run
            for (int w = WT - 1; w >= 0; --w)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float4 pw = s.decay[slot][w][wc][j][lane], gw = s.back[slot][w][wc][j][lane];
                    if (w == wt) { G[j][0] = G1[j][0]; G[j][1] = G1[j][1]; }
                    G1[j][0] = fma2(pair(pw.x, pw.y), G1[j][0], pair(gw.x, gw.y));
                    G1[j][1] = fma2(pair(pw.z, pw.w), G1[j][1], pair(gw.z, gw.w));
                }
            if constexpr (NB > 1) { to_slot(k, 0, G1); from_slot(k, 2, dA1); }
#pragma unroll
            for (int r = 0; r < RUN; ++r)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int q = 0; q < 2; ++q) h[r][j][q] = fma2(da[r][j][q], r ? h[r ? r - 1 : 0][j][q] : from[j][q], h[r][j][q]);
            if (p.z) {                                     // y before the gate
                float y[2 * RUN], out[RUN / 2];
#pragma unroll
                for (int r = 0; r < RUN; ++r) {
                    const float4 c = *reinterpret_cast<const float4 *>(&s.c[wt * RUN + r][k * 16 + nl * 4]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) y[2 * r + j] = sum2(fma2(pair(c.x, c.y), h[r][j][0], mul2(pair(c.z, c.w), h[r][j][1])));
                }
                reduce_lanes<2 * RUN, 1, 4>(y, lane, out);
#pragma unroll
                for (int j = 0; j < RUN / 2; ++j) {        // value 4 j + nl: step 2 j + (nl >> 1), channel nl & 1
                    float *at = &s.plain[wt * RUN + 2 * j + (nl >> 1)][ch + (nl & 1)];
                    *at = k ? *at + out[j] : out[j];
                }
            }
#pragma unroll
            for (int r = RUN - 1; r >= 0; --r) {
                const float4 st = *reinterpret_cast<const float4 *>(&s.step[wt * RUN + r][ch]);
                const float2 e = *reinterpret_cast<const float2 *>(&s.e[wt * RUN + r][ch]);
                const float4 b = *reinterpret_cast<const float4 *>(&s.b[wt * RUN + r][k * 16 + nl * 4]);
                const float4 c = *reinterpret_cast<const float4 *>(&s.c[wt * RUN + r][k * 16 + nl * 4]);
                f32x2 db[2], dc[2];
                float v[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const f32x2 ee = j ? pair(e.y, e.y) : pair(e.x, e.x), dt = j ? pair(st.z, st.z) : pair(st.x, st.x);
                    const f32x2 du = j ? pair(st.w, st.w) : pair(st.y, st.y);
                    f32x2 along = pair(0.0f, 0.0f), kept = pair(0.0f, 0.0f);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const f32x2 cc = q ? pair(c.z, c.w) : pair(c.x, c.y), bb = q ? pair(b.z, b.w) : pair(b.x, b.y);
                        const f32x2 g = fma2(ee, cc, G[j][q]);
                        G[j][q] = mul2(da[r][j][q], g);
                        const f32x2 left = mul2(G[j][q], r ? h[r ? r - 1 : 0][j][q] : from[j][q]);
                        dA1[j][q] = fma2(left, dt, dA1[j][q]);
                        kept = fma2(left, a1[j][q], kept);
                        along = fma2(g, bb, along);
                        db[q] = j ? fma2(g, du, db[q]) : mul2(g, du);
                        dc[q] = j ? fma2(ee, h[r][j][q], dc[q]) : mul2(ee, h[r][j][q]);
                    }
                    v[j] = sum2(along);
                    v[2 + j] = sum2(kept);
                }
                float one[1], w[8];
                reduce_lanes<4, 1, 4>(v, lane, one);
                float *at = nl < 2 ? &s.along[wt * RUN + r][ch + nl] : &s.kept[wt * RUN + r][ch + nl - 2];
                *at = k ? *at + one[0] : one[0];
                unpair(db[0], w[0], w[1]); unpair(db[1], w[2], w[3]);
                unpair(dc[0], w[4], w[5]); unpair(dc[1], w[6], w[7]);
                reduce_lanes<8, 4, 8>(w, lane, one);
                s.dbc[wc][wt * RUN + r][(cl < 4 ? 0 : S::NP) + k * 16 + nl * 4 + (cl & 3)] = one[0];
            }
            if constexpr (NB > 1) to_slot(k, 2, dA1);
        }
        __syncthreads();
        if (stored) {
            const float2 uu = s.u[tid], sl = s.slope[tid], gz = s.gate[tid];
            float du[2], ddelta[2], dz[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float along = s.along[pt][pc + j], uj = j ? uu.y : uu.x;
                du[j] = fmaf(s.e[pt][pc + j], skip[j], along * s.step[pt][pc + j].x);
                ddelta[j] = fmaf(s.kept[pt][pc + j], 0.693147181f, along * uj) * (j ? sl.y : sl.x);
                dz[j] = 0.0f;
                if (p.z) dz[j] = (j ? gz.y : gz.x) * fmaf(skip[j], uj, s.plain[pt][pc + j]);
                if (!inside) du[j] = ddelta[j] = dz[j] = 0.0f;
                dbias[j] += ddelta[j];
            }
            store_channels<T>(p, p.du, row, two, du);
            store_channels<T>(p, p.ddelta, row, two, ddelta);
            if (p.dz) store_channels<T>(p, p.dz, row, two, dz);
        }
        for (int q = tid; q < STEPS * 2 * p.N; q += S::THREADS) {
            const int t = q / (2 * p.N), n = q - t * 2 * p.N, at = n < p.N ? n : S::NP + n - p.N;
            float *out = p.part_bc + (((long long)group * p.T + t0 + t) * p.B + i) * 2 * p.N + n;
            if (t0 + t < p.T && relay_in_bounds(out, 4)) {
                float x = s.dbc[0][t][at];
#pragma unroll
                for (int w = 1; w < WC; ++w) x += s.dbc[w][t][at];
                __stcs(out, x);
            }
        }
        __syncthreads();
    }
    // sums over the runs (da) and over the steps of a chunk (dd, ddelta_bias)
#pragma unroll 1
    for (int k = 0; k < NB; ++k) {
        if constexpr (NB > 1) { from_slot(k, 0, G1); from_slot(k, 2, dA1); }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float4 v;
            unpair(dA1[j][0], v.x, v.y); unpair(dA1[j][1], v.z, v.w);
            s.sum[0][wt][wc][j][lane] = v;
        }
        __syncthreads();
        if (wt != 0) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (mine + j >= p.D) continue;
            float x[4] = {0.0f, 0.0f, 0.0f, 0.0f}, g[4];
            for (int w = 0; w < WT; ++w) {
                const float4 v = s.sum[0][w][wc][j][lane];
                x[0] += v.x; x[1] += v.y; x[2] += v.z; x[3] += v.w;
            }
            store_states(p, p.part_a, (i * p.D + mine + j) * p.N, k * 16 + nl * 4, x);
            unpair(G1[j][0], g[0], g[1]); unpair(G1[j][1], g[2], g[3]);
            store_states(p, p.dh0, (i * p.D + mine + j) * p.N, k * 16 + nl * 4, g);
        }
    }
    __syncthreads();
    s.step[pt][pc] = make_float2(dd[0], dbias[0]);
    s.step[pt][pc + 1] = make_float2(dd[1], dbias[1]);
    __syncthreads();
    if (tid < S::CHANNELS && c0 + tid < p.D) {
        float x = 0.0f, y = 0.0f;
        for (int t = 0; t < STEPS; ++t) { x += s.step[t][tid].x; y += s.step[t][tid].y; }
        const long long at = i * p.D + c0 + tid;
        if (p.part_d && relay_in_bounds(p.part_d + at, 4)) p.part_d[at] = x;
        if (p.part_bias && relay_in_bounds(p.part_bias + at, 4)) p.part_bias[at] = y;
    }
}

// db and dc: sums over the groups of channels, in their order
template <typename T>
__global__ void __launch_bounds__(256) join_weights_kernel(const float *part, long long rows, int N, int groups, void *db, void *dc)
{
    pdl_wait();
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, all = rows * 2 * N;
    if (at >= all) return;
    float x = 0.0f;
#pragma unroll 8
    for (int g = 0; g < groups; ++g)
        if (relay_in_bounds(part + g * all + at, 4)) x += __ldcs(part + g * all + at);
    const float out[1] = {x};
    if (dc == nullptr) { store<T, 1>(db, at, out); return; }
    const long long row = at / (2 * N);
    const int n = (int)(at - row * 2 * N);
    if (n < N) store<T, 1>(db, row * N + n, out);
    else store<T, 1>(dc, row * N + n - N, out);
}

// ---- workspace: partial sums of db and dc, of da, dd and ddelta_bias ----------------------------------------------------
int blocks_of_states(int64_t N) { return N <= 16 ? 1 : N <= 32 ? 2 : 4; }
int64_t groups_of(int64_t D, int64_t N)
{
    const int64_t channels = 16 * columns_of(blocks_of_states(N));
    return (D + channels - 1) / channels;
}
struct Parts { size_t bc, a, d, bias, bytes; };
Parts parts_of(const Sizes &s, int64_t N)
{
    Parts q{};
    q.a = align_up((size_t)groups_of(s.D, N) * s.T * s.B * 2 * N * sizeof(float), 256);
    q.d = q.a + align_up((size_t)s.B * s.D * N * sizeof(float), 256);
    q.bias = q.d + align_up((size_t)s.B * s.D * sizeof(float), 256);
    q.bytes = q.bias + align_up((size_t)s.B * s.D * sizeof(float), 256);
    return q;
}

template <typename T, int NB>
relay_status_t launch_chunks(const Args &p, cudaStream_t st)
{
    using S = Tile<NB>;
    const long long blocks = p.B * p.groups;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "selective_scan_grad: %lld x %lld channels", p.B, p.D);
    RELAY_CUDA(cudaFuncSetAttribute(selective_scan_grad_kernel<T, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(S)));
    RELAY_CUDA(launch_pdl(selective_scan_grad_kernel<T, NB>, dim3((unsigned)blocks), dim3(S::THREADS), sizeof(S), st, p));
    return check_launch("selective_scan_grad");
}
template <typename T>
relay_status_t launch_gradient(const Args &p, void *db, void *dc, cudaStream_t st)
{
    if (p.N <= 16) RELAY_TRY((launch_chunks<T, 1>(p, st)));
    else if (p.N <= 32) RELAY_TRY((launch_chunks<T, 2>(p, st)));
    else RELAY_TRY((launch_chunks<T, 4>(p, st)));
    const long long rows = p.T * p.B, blocks = (rows * 2 * p.N + 255) / 256;
    if (blocks == 0) return RELAY_OK;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "selective_scan_grad: %lld steps", rows);
    RELAY_CUDA(launch_pdl(join_weights_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, p.part_bc, rows, p.N, p.groups, db, dc));
    return check_launch("selective_scan_grad");
}

}  // namespace
}  // namespace relay

using namespace relay;

extern "C" size_t relay_workspace_bytes_selective_scan_grad(const relay_tensor_t *u, const relay_tensor_t *a)
{
    clear_error();
    seq::Sizes s;
    int64_t N;
    if (!u || !a || scan::check_sizes(u, a, &s, &N) != RELAY_OK) return 0;
    if (s.B == 0 || s.D == 0) return 0;
    return parts_of(s, N).bytes;
}

extern "C" relay_status_t relay_selective_scan_grad(const relay_tensor_t *u, const relay_tensor_t *delta, const relay_tensor_t *a,
                                                    const relay_tensor_t *b, const relay_tensor_t *c, const relay_tensor_t *d,
                                                    const relay_tensor_t *z, const relay_tensor_t *delta_bias, const relay_tensor_t *lengths,
                                                    int32_t softplus, const relay_tensor_t *states, const relay_tensor_t *dy,
                                                    const relay_tensor_t *dh_final, const relay_tensor_t *du, const relay_tensor_t *ddelta,
                                                    const relay_tensor_t *da, const relay_tensor_t *db, const relay_tensor_t *dc,
                                                    const relay_tensor_t *dd, const relay_tensor_t *dz, const relay_tensor_t *ddelta_bias,
                                                    const relay_tensor_t *dh0, void *ws, size_t ws_bytes, void *stream)
{
    clear_error();
    const scan::Inputs in{u, delta, a, b, c, d, z, delta_bias, lengths};
    RELAY_TRY(check_not_null(states, "states"));
    RELAY_TRY(check_not_null(dy, "dy"));
    RELAY_TRY(check_not_null(du, "du"));
    RELAY_TRY(check_not_null(ddelta, "ddelta"));
    RELAY_TRY(check_not_null(da, "da"));
    RELAY_TRY(check_not_null(db, "db"));
    if (c) RELAY_TRY(check_not_null(dc, "dc"));
    if (z) RELAY_TRY(check_not_null(dz, "dz"));
    seq::Sizes s;
    int64_t N;
    RELAY_TRY(scan::check_inputs(in, &s, &N));
    const int32_t t = u->dtype;
    RELAY_TRY(seq::check_tensor(states, RELAY_F32, RELAY_F32, {(s.T + RELAY_SCAN_SPAN - 1) / RELAY_SCAN_SPAN, s.B, s.D, N}, "states"));
    RELAY_TRY(seq::check_tensor(dy, t, t, {s.T, s.B, s.D}, "dy"));
    RELAY_TRY(seq::check_tensor(dh_final, RELAY_F32, RELAY_F32, {s.B, s.D, N}, "dh_final"));
    RELAY_TRY(seq::check_tensor(du, t, t, {s.T, s.B, s.D}, "du"));
    RELAY_TRY(seq::check_tensor(ddelta, t, t, {s.T, s.B, s.D}, "ddelta"));
    RELAY_TRY(seq::check_tensor(da, RELAY_F32, RELAY_F32, {s.D, N}, "da"));
    RELAY_TRY(seq::check_tensor(db, t, t, {s.T, s.B, c ? N : 2 * N}, "db"));
    RELAY_TRY(seq::check_tensor(dc, t, t, {s.T, s.B, N}, "dc"));
    RELAY_TRY(seq::check_tensor(dd, RELAY_F32, RELAY_F32, {s.D}, "dd"));
    RELAY_TRY(seq::check_tensor(dz, t, t, {s.T, s.B, s.D}, "dz"));
    RELAY_TRY(seq::check_tensor(ddelta_bias, RELAY_F32, RELAY_F32, {s.D}, "ddelta_bias"));
    RELAY_TRY(seq::check_tensor(dh0, RELAY_F32, RELAY_F32, {s.B, s.D, N}, "dh0"));
    RELAY_TRY(scan::check_softplus(softplus));
    if (!c && dc) return fail(RELAY_ERR_ATTR, "dc is given, but c is part of b: its partial is part of db");
    if (!z && dz) return fail(RELAY_ERR_ATTR, "dz is given, but there is no gate");
    if (!d && dd) return fail(RELAY_ERR_ATTR, "dd is given, but there is no d");
    if (!delta_bias && ddelta_bias) return fail(RELAY_ERR_ATTR, "ddelta_bias is given, but there is no delta_bias");
    const relay_tensor_t *ins[12] = {u, delta, a, b, c, d, z, delta_bias, lengths, states, dy, dh_final};
    const relay_tensor_t *outs[9] = {du, ddelta, da, db, dc, dd, dz, ddelta_bias, dh0};
    RELAY_TRY(seq::check_buffers(ins, outs));
    const bool empty = s.B == 0 || s.D == 0;
    const Parts q = parts_of(s, N);
    RELAY_TRY(check_workspace(ws, ws_bytes, empty ? 0 : q.bytes));
    cudaStream_t st = (cudaStream_t)stream;
    RELAY_TRY(seq::register_buffers(ins, outs, ws, empty ? 0 : q.bytes, st));
    if (empty) {                                           // sums over nothing
        for (const relay_tensor_t *o : {da, db, dc, dd, ddelta_bias})
            if (o && nbytes(o)) RELAY_CUDA(cudaMemsetAsync(o->data, 0, nbytes(o), st));
        return RELAY_OK;
    }
    scan::Args p = scan::make_args(in, softplus, s, N);
    p.states = (float *)states->data;
    p.dy = dy->data;
    p.dh_final = dh_final ? (const float *)dh_final->data : nullptr;
    p.du = du->data; p.ddelta = ddelta->data; p.dz = dz ? dz->data : nullptr;
    p.dh0 = dh0 ? (float *)dh0->data : nullptr;
    p.groups = (int)groups_of(s.D, N);
    char *w = (char *)ws;
    p.part_bc = (float *)w;
    p.part_a = (float *)(w + q.a);
    p.part_d = dd ? (float *)(w + q.d) : nullptr;
    p.part_bias = ddelta_bias ? (float *)(w + q.bias) : nullptr;
    void *dcp = dc ? dc->data : nullptr;
    RELAY_TRY(t == RELAY_F32 ? launch_gradient<float>(p, db->data, dcp, st) : launch_gradient<__nv_bfloat16>(p, db->data, dcp, st));
    RELAY_TRY(seq::launch_column_sums(p.part_a, s.B, s.D * N, s.D * N, (float *)da->data, s.D * N, nullptr, st));
    if (dd) RELAY_TRY(seq::launch_column_sums(p.part_d, s.B, s.D, s.D, (float *)dd->data, s.D, nullptr, st));
    if (ddelta_bias) RELAY_TRY(seq::launch_column_sums(p.part_bias, s.B, s.D, s.D, (float *)ddelta_bias->data, s.D, nullptr, st));
    return RELAY_OK;
}
