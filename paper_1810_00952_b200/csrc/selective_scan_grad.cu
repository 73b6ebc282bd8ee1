// Gradient group of the selective scan (Section 4.2 of the paper: reverse mode through the recursion over time).
//
// The decays exp(delta a) of a run stay in registers and serve three times: the run summed up from a zero state, its states from the one that it
// really starts with, and what flows back.  Sums over states end in four lanes, sums over channels in eight and then over the groups of
// sixteen channels, through the workspace in a fixed order.
// Measured, bf16, 2048 x 8 x 2048 x 16, gated: 1.13 ms, 47 us for the sums over groups, 1.55 ms with the forward call.  Counters (T = 512): 53 % of issue
// slots, 56 % of shared memory's cycles, 16 warps an SM (128 registers).  Taken out one at a time, reductions between lanes cost 85 us, the
// joins 170, and what follows the scan 190, of which 72 are bytes.
#include <algorithm>
#include <type_traits>

#include "selective_scan.cuh"

namespace relay {
namespace {

using namespace scan;

// A block: sixteen channels of a batch element, eight warps; a lane has two neighbouring channels and four neighbouring states of every sixteen,
// and each warp a run of RUN steps of the chunk, which is the span whose starting states the forward call saved.  The runs' products and sums
// meet in shared memory, in both directions at once.  Chunks are taken from the last to the first; rows are fetched a chunk ahead by TMA.
constexpr int RUN = 4, WT = kSpan / RUN, STEPS = kSpan, CHANNELS = 16, THREADS = 32 * WT, STAGES = 2;

template <typename T, int NB>
struct Tile {
    static constexpr int NP = 16 * NB, SLOTS = NB == 1 ? 1 : 2;
    struct Stage { alignas(128) T u[STEPS][CHANNELS]; alignas(128) T delta[STEPS][CHANNELS]; alignas(128) T z[STEPS][CHANNELS]; alignas(128) T dy[STEPS][CHANNELS]; alignas(128) T bc[STEPS * 2 * NP]; };
    Stage stage[STAGES];
    alignas(16) float2 step[STEPS][CHANNELS];              // delta, delta u
    alignas(16) float e[STEPS][CHANNELS];                  // dy silu(z)
    alignas(16) float b[STEPS][NP], c[STEPS][NP];
    // Of every run: its decay, the state it leaves from zero, what flows back through it from zero.  Joined in place, a thread each of the
    // 256 chains of states: the state a run starts from, and what flows back into it.
    ulonglong2 decay[SLOTS][WT][2][32], sum[SLOTS][WT][2][32], back[SLOTS][WT][2][32];
    float carry[NB == 1 ? 1 : NB][NB == 1 ? 1 : THREADS];  // more than sixteen states: what flows back into the chunk
    alignas(16) float along[STEPS][CHANNELS], kept[STEPS][CHANNELS], plain[STEPS][CHANNELS];   // sum_n g b, sum_n a G h[t-1], sum_n c h
    alignas(16) float dbc[STEPS][2 * NP];
    float2 u[THREADS], slope[THREADS], gate[THREADS];      // what a thread needs again at the end of a chunk
    ulonglong2 da[NB == 1 ? 1 : NB][2][NB == 1 ? 1 : THREADS];   // more than sixteen states: sums of da wait here
    uint64_t full[STAGES];
    int gave_up;
};

// ENDS: a sequence may end inside a chunk (without: 1548 us for 2048 x 8 x 2048 x 16 with the forward call, 1568 with)
template <typename T, int NB, bool ENDS>
__global__ void __launch_bounds__(THREADS, NB == 1 ? 2 : 1) selective_scan_grad_kernel(const Args p, const __grid_constant__ Maps maps)
{
    using S = Tile<T, NB>;
    constexpr bool FINE = sizeof(T) == 4;
    extern __shared__ uint8_t shared_raw[];
    S &s = *reinterpret_cast<S *>(((uintptr_t)shared_raw + 127) & ~(uintptr_t)127);
    const int tid = threadIdx.x, lane = tid & 31, wt = tid >> 5, nl = lane & 3, cl = lane >> 2;
    const long long i = blockIdx.x / p.groups;
    const int group = (int)(blockIdx.x - i * p.groups);
    const long long c0 = (long long)group * CHANNELS;
    if (tid == 0) {
        for (int q = 0; q < STAGES; ++q) tc::mbar_init(&s.full[q], 1);
        s.gave_up = 0;
        tc::fence_barrier_init();
    }
    __syncthreads();
    pdl_wait();
    const long long end = end_of(p, i);
    const int chunks = (int)((p.T + STEPS - 1) / STEPS), live_chunks = (int)((end + STEPS - 1) / STEPS);
    // the q-th fetch: rows of chunk live_chunks - 1 - q
    auto fetch = [&](int q) {
        typename S::Stage &g = s.stage[q % STAGES];
        const long long t0 = (long long)(live_chunks - 1 - q) * STEPS;
        if (tid == 0 && (p.tma_x || p.tma_w)) {
            uint64_t *full = &s.full[q % STAGES];
            const uint32_t x = p.tma_x ? (p.z ? 4u : 3u) * (uint32_t)sizeof(g.u) : 0u, w = p.tma_w ? (uint32_t)(STEPS * 2 * p.N * sizeof(T)) : 0u;
            tc::mbar_expect_tx(full, x + w);
            const int col = (int)(i * p.D + c0), row = (int)t0;
            if (p.tma_x) {
                tc::tma_load_2d(g.u, &maps.u, full, col, row);
                tc::tma_load_2d(g.delta, &maps.delta, full, col, row);
                tc::tma_load_2d(g.dy, &maps.dy, full, col, row);
                if (p.z) tc::tma_load_2d(g.z, &maps.z, full, col, row);
            }
            if (p.tma_w) {
                tc::tma_load_2d(g.bc, &maps.b, full, (int)(i * p.ld_bc), row);
                if (p.ld_bc == p.N) tc::tma_load_2d(g.bc + STEPS * p.N, &maps.c, full, (int)(i * p.ld_bc), row);
            }
        }
        const int rows = (int)min((long long)STEPS, end - t0);
        if (!p.tma_x) {
            const int width = (int)min((long long)CHANNELS, p.D - c0);
            const long long at = (t0 * p.B + i) * p.D + c0;
            copy_rows<T>(&g.u[0][0], CHANNELS, (const T *)p.u + at, p.B * p.D, rows, width, tid, THREADS);
            copy_rows<T>(&g.delta[0][0], CHANNELS, (const T *)p.delta + at, p.B * p.D, rows, width, tid, THREADS);
            copy_rows<T>(&g.dy[0][0], CHANNELS, (const T *)p.dy + at, p.B * p.D, rows, width, tid, THREADS);
            if (p.z) copy_rows<T>(&g.z[0][0], CHANNELS, (const T *)p.z + at, p.B * p.D, rows, width, tid, THREADS);
        }
        if (!p.tma_w) {
            const long long at = (t0 * p.B + i) * p.ld_bc;
            copy_rows<T>(g.bc, p.ld_bc, (const T *)p.b + at, p.B * p.ld_bc, rows, p.ld_bc, tid, THREADS);
            if (p.ld_bc == p.N) copy_rows<T>(g.bc + STEPS * p.N, p.N, (const T *)p.c + at, p.B * p.ld_bc, rows, p.N, tid, THREADS);
        }
        copies_end();
    };
    for (int q = 0; q < STAGES && q < live_chunks; ++q) fetch(q);
    const int ch = cl * 2;                                 // this lane's channels: ch, ch + 1 of the block
    const long long mine = c0 + ch;
    f32x2 a[2][2], dA[2][2];                               // a log2(e), sums of da
    auto load_a = [&](int k) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float x[4];
            load_states(p, mine + j < p.D ? p.a : nullptr, (mine + j) * p.N, k * 16 + nl * 4, x);
            a[j][0] = pair(exponent_of(x[0]), exponent_of(x[1]));
            a[j][1] = pair(exponent_of(x[2]), exponent_of(x[3]));
        }
    };
#pragma unroll
    for (int j = 0; j < 2; ++j) dA[j][0] = dA[j][1] = 0;
    // this thread's chain in the joins: channel and first state of every sixteen
    const int chain = (tid >> 2 & 31);                     // the lane that holds it
    const long long chain_d = c0 + (chain >> 2) * 2 + (tid >> 7);
    const int chain_n = (chain & 3) * 4 + (tid & 3);
    auto chain_load = [&](const float *base, long long row, int k) {
        const int n = k * 16 + chain_n;
        const float *at = base + (row + chain_d) * p.N + n;
        return base != nullptr && chain_d < p.D && n < p.N && relay_in_bounds(at, 4) ? __ldcs(at) : 0.0f;
    };
    auto chain_store = [&](float *base, long long row, int k, float x) {
        const int n = k * 16 + chain_n;
        float *at = base + (row + chain_d) * p.N + n;
        if (base != nullptr && chain_d < p.D && n < p.N && relay_in_bounds(at, 4)) __stcs(at, x);
    };
    float carry = 0.0f;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        carry = chain_load(p.dh_final, i * p.D, k);
        if constexpr (NB > 1) {
            s.carry[k][tid] = carry;
#pragma unroll
            for (int j = 0; j < 2; ++j) s.da[k][j][tid] = make_ulonglong2(0, 0);
        }
    }
    if constexpr (NB == 1) load_a(0);
    // this thread's pair of channels and step of the chunk in what surrounds the scan
    const int pt = tid / (CHANNELS / 2), pc = 2 * (tid % (CHANNELS / 2));
    const long long two = c0 + pc;
    f32x2 skip, bias, dd = 0, dbias = 0;
    {
        float x[2], y[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool in = two + j < p.D;
            x[j] = p.d && in && relay_in_bounds(p.d + two + j, 4) ? p.d[two + j] : 0.0f;
            y[j] = p.delta_bias && in && relay_in_bounds(p.delta_bias + two + j, 4) ? p.delta_bias[two + j] : 0.0f;
        }
        skip = pair(x[0], x[1]); bias = pair(y[0], y[1]);
    }
    for (int chunk = chunks - 1; chunk >= live_chunks; --chunk) {            // behind the sequence nothing flows back
        const long long t0 = (long long)chunk * STEPS, row = ((t0 + pt) * p.B + i) * p.D;
        if (t0 + pt < p.T && two < p.D) {
            const float zero[2] = {0.0f, 0.0f};
            store_some<T>(p, p.du, row, two, zero);
            store_some<T>(p, p.ddelta, row, two, zero);
            if (p.dz) store_some<T>(p, p.dz, row, two, zero);
        }
        for (int q = tid; q < STEPS * 2 * p.N; q += THREADS) {
            const int t = q / (2 * p.N), n = q - t * 2 * p.N;
            float *out = p.part_bc + (((long long)group * p.T + t0 + t) * p.B + i) * 2 * p.N + n;
            if (t0 + t < p.T && relay_in_bounds(out, 4)) *out = 0.0f;
        }
    }
    for (int done = 0; done < live_chunks; ++done) {
        const long long chunk = live_chunks - 1 - done, t0 = chunk * STEPS;
        typename S::Stage &g = s.stage[done % STAGES];
        // the state that the first run starts from: on its way while the rows are made fp32
        float start = 0.0f;
        if constexpr (NB == 1) start = chain_load(p.states, (chunk * p.B + i) * p.D, 0);
        if (p.tma_x || p.tma_w) tc::mbar_wait(&s.full[done % STAGES], (done / STAGES) & 1, &s.gave_up, p.err, tc::ERR_WAIT_FULL);
        if (!p.tma_x || !p.tma_w) { copies_done(min(live_chunks - done, STAGES) - 1); __syncthreads(); }   // everyone's own copies
        const int in = (int)min((long long)STEPS, end - t0);                 // steps of the chunk that are inside the sequence
        const bool inside = pt < in;
        {
            float u[2], x[2], z[2], dy[2], lo, hi;
            widen_shared(&g.u[pt][pc], u);
            widen_shared(&g.delta[pt][pc], x);
            widen_shared(&g.dy[pt][pc], dy);
            f32x2 step = add2(pair(x[0], x[1]), bias);
            float slope[2] = {1.0f, 1.0f}, gate[2] = {0.0f, 0.0f};
            if (p.softplus) {
                const Softplus q = softplus2(step);
                float w[2];
                unpair(step, x[0], x[1]);
                unpair(q.w, w[0], w[1]);
                slope[0] = softplus_slope(x[0], w[0]); slope[1] = softplus_slope(x[1], w[1]);
                step = q.value;
            }
            if (p.z) {
                widen_shared(&g.z[pt][pc], z);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float q = logistic<FINE>(z[j]);
                    gate[j] = dy[j] * q * fmaf(z[j], 1.0f - q, 1.0f);
                    dy[j] *= z[j] * q;
                }
            }
            if (!inside) {                                 // behind the end nothing decays and nothing is added
                step = 0;
                u[0] = u[1] = dy[0] = dy[1] = 0.0f;
            }
            unpair(step, lo, hi);
            if (two >= p.D) lo = u[0] = dy[0] = 0.0f;      // channels that do not exist have no part in db and dc
            if (two + 1 >= p.D) hi = u[1] = dy[1] = 0.0f;
            *reinterpret_cast<float4 *>(&s.step[pt][pc]) = make_float4(lo, lo * u[0], hi, hi * u[1]);
            *reinterpret_cast<float2 *>(&s.e[pt][pc]) = make_float2(dy[0], dy[1]);
            dd = fma2(pair(dy[0], dy[1]), pair(u[0], u[1]), dd);
            s.u[tid] = make_float2(u[0], u[1]); s.slope[tid] = make_float2(slope[0], slope[1]); s.gate[tid] = make_float2(gate[0], gate[1]);
        }
        if (p.N == S::NP) {                                // four states at a time
            for (int e = tid; e < STEPS * S::NP / 4; e += THREADS) {
                const int t = e / (S::NP / 4), n = e % (S::NP / 4) * 4;
                float b[4], c[4];
                widen_shared(p.ld_bc != p.N ? &g.bc[t * 2 * S::NP + n] : &g.bc[t * S::NP + n], b);
                widen_shared(p.ld_bc != p.N ? &g.bc[t * 2 * S::NP + S::NP + n] : &g.bc[STEPS * S::NP + t * S::NP + n], c);
                if (t >= in) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) b[j] = c[j] = 0.0f;
                }
                *reinterpret_cast<float4 *>(&s.b[t][n]) = make_float4(b[0], b[1], b[2], b[3]);
                *reinterpret_cast<float4 *>(&s.c[t][n]) = make_float4(c[0], c[1], c[2], c[3]);
            }
        } else {
            for (int e = tid; e < STEPS * S::NP; e += THREADS) {
                const int t = e / S::NP, n = e % S::NP;
                const bool on = t < in && n < p.N, packed = p.ld_bc != p.N;
                s.b[t][n] = on ? to_f32(g.bc[packed ? t * 2 * p.N + n : t * p.N + n]) : 0.0f;
                s.c[t][n] = on ? to_f32(g.bc[packed ? t * 2 * p.N + p.N + n : STEPS * p.N + t * p.N + n]) : 0.0f;
            }
        }
        __syncthreads();
        if (done + STAGES < live_chunks) fetch(done + STAGES);               // everyone has read this chunk's rows
        const int r0 = wt * RUN;
#pragma unroll 1
        for (int k = 0; k < NB; ++k) {
            const int slot = NB == 1 ? 0 : k & 1;
            if constexpr (NB > 1) {
                load_a(k);
                start = chain_load(p.states, (chunk * p.B + i) * p.D, k);
                carry = s.carry[k][tid];
            }
            f32x2 da[RUN][2][2], h[RUN][2][2];             // decays; what is added, then the states
            {
                f32x2 P[2][2], H[2][2];
#pragma unroll
                for (int r = 0; r < RUN; ++r) {
                    const float4 st = *reinterpret_cast<const float4 *>(&s.step[r0 + r][ch]);
                    const ulonglong2 b = *reinterpret_cast<const ulonglong2 *>(&s.b[r0 + r][k * 16 + nl * 4]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f32x2 dt = j ? pair(st.z, st.z) : pair(st.x, st.x), du = j ? pair(st.w, st.w) : pair(st.y, st.y);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            da[r][j][q] = decay2(mul2(dt, a[j][q]));
                            h[r][j][q] = mul2(du, q ? b.y : b.x);
                            H[j][q] = r ? fma2(da[r][j][q], H[j][q], h[r][j][q]) : h[r][j][q];
                            P[j][q] = r ? mul2(da[r][j][q], P[j][q]) : da[r][j][q];
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s.decay[slot][wt][j][lane] = make_ulonglong2(P[j][0], P[j][1]);
                    s.sum[slot][wt][j][lane] = make_ulonglong2(H[j][0], H[j][1]);
                }
                // what flows back through the run from a zero carry
#pragma unroll
                for (int r = RUN - 1; r >= 0; --r) {
                    const float2 e = *reinterpret_cast<const float2 *>(&s.e[r0 + r][ch]);
                    const ulonglong2 c = *reinterpret_cast<const ulonglong2 *>(&s.c[r0 + r][k * 16 + nl * 4]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f32x2 ee = j ? pair(e.y, e.y) : pair(e.x, e.x);
                        H[j][0] = mul2(da[r][j][0], r == RUN - 1 ? mul2(ee, c.x) : fma2(ee, c.x, H[j][0]));
                        H[j][1] = mul2(da[r][j][1], r == RUN - 1 ? mul2(ee, c.y) : fma2(ee, c.y, H[j][1]));
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) s.back[slot][wt][j][lane] = make_ulonglong2(H[j][0], H[j][1]);
            }
            __syncthreads();
            {
                float *P = reinterpret_cast<float *>(&s.decay[slot][0][0][0]) + tid, *H = reinterpret_cast<float *>(&s.sum[slot][0][0][0]) + tid;
                float *R = reinterpret_cast<float *>(&s.back[slot][0][0][0]) + tid, d[WT], x[WT], y[WT];
#pragma unroll
                for (int w = 0; w < WT; ++w) { d[w] = P[w * THREADS]; x[w] = H[w * THREADS]; y[w] = R[w * THREADS]; }
#pragma unroll
                for (int w = 0; w < WT; ++w) {
                    H[w * THREADS] = start;
                    start = fmaf(d[w], start, x[w]);
                }
#pragma unroll
                for (int w = WT - 1; w >= 0; --w) {
                    R[w * THREADS] = carry;
                    carry = fmaf(d[w], carry, y[w]);
                }
                if constexpr (NB > 1) s.carry[k][tid] = carry;
            }
            __syncthreads();
            f32x2 from[2][2], G[2][2];                     // the state at the start of this run, what flows back into it
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const ulonglong2 x = s.sum[slot][wt][j][lane], y = s.back[slot][wt][j][lane];
                from[j][0] = x.x; from[j][1] = x.y;
                G[j][0] = y.x; G[j][1] = y.y;
            }
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
                    const ulonglong2 c = *reinterpret_cast<const ulonglong2 *>(&s.c[r0 + r][k * 16 + nl * 4]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) y[2 * r + j] = sum2(fma2(c.x, h[r][j][0], mul2(c.y, h[r][j][1])));
                }
                reduce_lanes<2 * RUN, 1, 4>(y, lane, out);
#pragma unroll
                for (int j = 0; j < RUN / 2; ++j) {        // value 4 j + nl: step 2 j + (nl >> 1), channel nl & 1
                    float *at = &s.plain[r0 + 2 * j + (nl >> 1)][ch + (nl & 1)];
                    *at = k ? *at + out[j] : out[j];
                }
            }
            if constexpr (NB > 1) {
#pragma unroll
                for (int j = 0; j < 2; ++j) { const ulonglong2 v = s.da[k][j][tid]; dA[j][0] = v.x; dA[j][1] = v.y; }
            }
            auto backwards = [&](auto whole) {             // whole: all steps of the chunk are inside the sequence
#pragma unroll
                for (int r = RUN - 1; r >= 0; --r) {
                    if (!whole && r0 + r >= in) {          // behind the end: a zero partial of an infinite state would be NaN
                        s.dbc[r0 + r][(cl < 4 ? 0 : S::NP) + k * 16 + nl * 4 + (cl & 3)] = 0.0f;
                        continue;
                    }
                    const float4 st = *reinterpret_cast<const float4 *>(&s.step[r0 + r][ch]);
                    const float2 e = *reinterpret_cast<const float2 *>(&s.e[r0 + r][ch]);
                    const ulonglong2 b = *reinterpret_cast<const ulonglong2 *>(&s.b[r0 + r][k * 16 + nl * 4]);
                    const ulonglong2 c = *reinterpret_cast<const ulonglong2 *>(&s.c[r0 + r][k * 16 + nl * 4]);
                    f32x2 db[2], dc[2];
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f32x2 ee = j ? pair(e.y, e.y) : pair(e.x, e.x), dt = j ? pair(st.z, st.z) : pair(st.x, st.x);
                        const f32x2 du = j ? pair(st.w, st.w) : pair(st.y, st.y);
                        f32x2 along, kept;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const f32x2 gq = fma2(ee, q ? c.y : c.x, G[j][q]), bb = q ? b.y : b.x;
                            G[j][q] = mul2(da[r][j][q], gq);
                            const f32x2 left = mul2(G[j][q], r ? h[r ? r - 1 : 0][j][q] : from[j][q]);
                            dA[j][q] = fma2(left, dt, dA[j][q]);
                            kept = q ? fma2(left, a[j][q], kept) : mul2(left, a[j][q]);
                            along = q ? fma2(gq, bb, along) : mul2(gq, bb);
                            db[q] = j ? fma2(gq, du, db[q]) : mul2(gq, du);
                            dc[q] = j ? fma2(ee, h[r][j][q], dc[q]) : mul2(ee, h[r][j][q]);
                        }
                        v[j] = sum2(along);
                        v[2 + j] = sum2(kept);
                    }
                    float one[1], w[8];
                    reduce_lanes<4, 1, 4>(v, lane, one);
                    float *at = nl < 2 ? &s.along[r0 + r][ch + nl] : &s.kept[r0 + r][ch + nl - 2];
                    *at = k ? *at + one[0] : one[0];
                    unpair(db[0], w[0], w[1]); unpair(db[1], w[2], w[3]);
                    unpair(dc[0], w[4], w[5]); unpair(dc[1], w[6], w[7]);
                    reduce_lanes<8, 4, 8>(w, lane, one);
                    s.dbc[r0 + r][(cl < 4 ? 0 : S::NP) + k * 16 + nl * 4 + (cl & 3)] = one[0];
                }
            };
            if (!ENDS || in == STEPS) backwards(std::true_type());
            else if constexpr (ENDS) backwards(std::false_type());
            if constexpr (NB > 1) {
#pragma unroll
                for (int j = 0; j < 2; ++j) s.da[k][j][tid] = make_ulonglong2(dA[j][0], dA[j][1]);
            }
        }
        __syncthreads();
        if (t0 + pt < p.T && two < p.D) {
            const float2 u = s.u[tid], sl = s.slope[tid], gz = s.gate[tid], e = *reinterpret_cast<const float2 *>(&s.e[pt][pc]);
            const float4 st = *reinterpret_cast<const float4 *>(&s.step[pt][pc]);
            const float2 al = *reinterpret_cast<const float2 *>(&s.along[pt][pc]), ke = *reinterpret_cast<const float2 *>(&s.kept[pt][pc]);
            const f32x2 along = pair(al.x, al.y), uu = pair(u.x, u.y);
            f32x2 du = mul2(along, pair(st.x, st.z));
            if (p.d) du = fma2(pair(e.x, e.y), skip, du);
            f32x2 ddelta = mul2(fma2(pair(ke.x, ke.y), pair(0.693147181f, 0.693147181f), mul2(along, uu)), pair(sl.x, sl.y));
            if (!inside) du = ddelta = 0;
            float x[2];
            unpair(ddelta, x[0], x[1]);                    // a step of no length passes nothing, also where a state times a is beyond fp32
            ddelta = pair(sl.x == 0.0f ? 0.0f : x[0], sl.y == 0.0f ? 0.0f : x[1]);
            dbias = add2(dbias, ddelta);
            const long long row = ((t0 + pt) * p.B + i) * p.D;
            unpair(du, x[0], x[1]);
            store_some<T>(p, p.du, row, two, x);
            unpair(ddelta, x[0], x[1]);
            store_some<T>(p, p.ddelta, row, two, x);
            if (p.dz) {
                const float2 pl = *reinterpret_cast<const float2 *>(&s.plain[pt][pc]);
                f32x2 plain = pair(pl.x, pl.y);
                if (p.d) plain = fma2(skip, uu, plain);
                unpair(mul2(pair(gz.x, gz.y), plain), x[0], x[1]);
                if (!inside) x[0] = x[1] = 0.0f;
                store_some<T>(p, p.dz, row, two, x);
            }
        }
        if (p.N == S::NP) {
            for (int q = tid; q < STEPS * 2 * S::NP / 4; q += THREADS) {
                const int t = q / (S::NP / 2), n = q % (S::NP / 2) * 4;
                float *out = p.part_bc + (((long long)group * p.T + t0 + t) * p.B + i) * (2 * S::NP) + n;
                if (t0 + t < p.T && relay_in_bounds(out, 16)) __stcs((float4 *)out, *reinterpret_cast<const float4 *>(&s.dbc[t][n]));
            }
        } else {
            const int N = p.N, down = THREADS / (2 * N), along = THREADS - down * 2 * N, rows = (int)min((long long)STEPS, p.T - t0);
            const long long step = p.B * 2 * N;
            float *first = p.part_bc + (((long long)group * p.T + t0) * p.B + i) * 2 * N;
            for (int t = tid / (2 * N), n = tid - t * 2 * N; t < rows;) {
                float *out = first + t * step + n;
                if (relay_in_bounds(out, 4)) __stcs(out, s.dbc[t][n < N ? n : S::NP + n - N]);
                t += down;
                n += along;
                if (n >= 2 * N) { n -= 2 * N; ++t; }
            }
        }
    }
    // sums over the runs (da) and over the steps of a chunk (dd, ddelta_bias)
#pragma unroll 1
    for (int k = 0; k < NB; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (NB > 1) s.sum[0][wt][j][lane] = s.da[k][j][tid];
            else s.sum[0][wt][j][lane] = make_ulonglong2(dA[j][0], dA[j][1]);
        }
        __syncthreads();
        float x = 0.0f;
#pragma unroll
        for (int w = 0; w < WT; ++w) x += reinterpret_cast<const float *>(&s.sum[0][0][0][0])[w * THREADS + tid];
        chain_store(p.part_a + i * 2 * p.D, i * p.D, k, x);
        if constexpr (NB > 1) carry = s.carry[k][tid];
        chain_store(p.dh0, i * p.D, k, carry);
    }
    __syncthreads();
    {
        float x[2], y[2];
        unpair(dd, x[0], x[1]); unpair(dbias, y[0], y[1]);
        *reinterpret_cast<float4 *>(&s.step[pt][pc]) = make_float4(x[0], y[0], x[1], y[1]);
    }
    __syncthreads();
    if (tid < CHANNELS && c0 + tid < p.D) {
        float x = 0.0f, y = 0.0f;
        for (int t = 0; t < STEPS; ++t) { x += s.step[t][tid].x; y += s.step[t][tid].y; }
        float *at = p.part_a + i * p.D * (p.N + 2) + p.D * p.N + c0 + tid;
        if (relay_in_bounds(at, 4)) *at = x;
        if (relay_in_bounds(at + p.D, 4)) at[p.D] = y;
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
int64_t groups_of(int64_t D) { return (D + CHANNELS - 1) / CHANNELS; }
struct Parts { size_t a, bytes; };                         // the first are at the start
Parts parts_of(const Sizes &s, int64_t N)
{
    Parts q{};
    q.a = align_up((size_t)groups_of(s.D) * s.T * s.B * 2 * N * sizeof(float), 256);
    q.bytes = q.a + align_up((size_t)s.B * s.D * (N + 2) * sizeof(float), 256);
    return q;
}

template <typename T, int NB, bool ENDS>
relay_status_t launch_chunks(Args p, cudaStream_t st)
{
    const long long blocks = p.B * p.groups;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "selective_scan_grad: %lld x %lld channels", p.B, p.D);
    if (!p.err) return fail(RELAY_ERR_CUDA, "no device error word");
    Maps maps;
    RELAY_TRY(make_maps(&p, &maps, sizeof(T) == 4, CHANNELS, STEPS));
    const size_t bytes = sizeof(Tile<T, NB>) + 128;
    RELAY_CUDA(cudaFuncSetAttribute(selective_scan_grad_kernel<T, NB, ENDS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    RELAY_CUDA(launch_pdl(selective_scan_grad_kernel<T, NB, ENDS>, dim3((unsigned)blocks), dim3(THREADS), bytes, st, p, maps));
    return check_launch("selective_scan_grad");
}
template <typename T, int NB>
relay_status_t launch_ends(const Args &p, cudaStream_t st)
{
    return p.lengths == nullptr && p.T % STEPS == 0 ? launch_chunks<T, NB, false>(p, st) : launch_chunks<T, NB, true>(p, st);
}
template <typename T>
relay_status_t launch_gradient(const Args &p, void *db, void *dc, cudaStream_t st)
{
    if (p.N <= 16) RELAY_TRY((launch_ends<T, 1>(p, st)));
    else if (p.N <= 32) RELAY_TRY((launch_ends<T, 2>(p, st)));
    else RELAY_TRY((launch_ends<T, 4>(p, st)));
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
    p.groups = (int)groups_of(s.D);
    char *w = (char *)ws;
    p.part_bc = (float *)w;
    p.part_a = (float *)(w + q.a);
    void *dcp = dc ? dc->data : nullptr;
    RELAY_TRY(t == RELAY_F32 ? launch_gradient<float>(p, db->data, dcp, st) : launch_gradient<__nv_bfloat16>(p, db->data, dcp, st));
    return seq::launch_column_sums(p.part_a, s.B, {{(float *)da->data, dd ? (float *)dd->data : nullptr, ddelta_bias ? (float *)ddelta_bias->data : nullptr},
                                                   {s.D * N, s.D, s.D}}, st);
}
