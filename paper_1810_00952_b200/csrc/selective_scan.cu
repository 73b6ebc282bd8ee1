// Selective scan: h = exp(delta a) h + delta u b per channel and state, y = sum_n c h + d u, with an optional gate silu(z).
//
// Measured, bf16, N = 16, gate and softplus: 2048 x 8 x 2048 344 us, 16384 x 1 x 2048 608 us (two passes), one step of 64 x 2048 12 us (9.5 in a
// captured graph: 65 % of issue slots).  Counters of the first (T = 512): 53 % of issue slots, 40 % of the special-function pipe, two thirds of
// shared memory's cycles, with 14 warps an SM, all there are: waits of fixed length are what is left.
#include <algorithm>
#include <type_traits>

#include "selective_scan.cuh"

namespace relay {

relay_status_t make_tmap_2d(CUtensorMap *m, bool f32, const void *base, uint64_t inner, uint64_t outer, uint64_t row_stride,
                            uint32_t box_inner, uint32_t box_outer, bool swizzle128);

namespace {

using namespace scan;

// ---- few steps: four lanes a channel, the states in registers from step to step ----------------------------------------
constexpr int kStepThreads = 128;

template <typename T, int NB>
__global__ void __launch_bounds__(kStepThreads) selective_scan_steps_kernel(const Args p)
{
    constexpr bool FINE = sizeof(T) == 4;
    pdl_wait();
    const long long at = ((long long)blockIdx.x * kStepThreads + threadIdx.x) >> 2;      // b * D + d
    const int nl = threadIdx.x & 3;
    const bool live = at < p.B * p.D;                                                    // the lanes of a warp stay together
    const long long i = live ? at / p.D : 0, d = live ? at - i * p.D : 0;
    const long long end = live ? end_of(p, i) : 0;
    float h[NB][4], a[NB][4];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        load_states(p, live ? p.h0 : nullptr, at * p.N, k * 16 + nl * 4, h[k]);
        load_states(p, live ? p.a : nullptr, d * p.N, k * 16 + nl * 4, a[k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) a[k][j] = exponent_of(a[k][j]);
    }
    const float skip = p.d && live && relay_in_bounds(p.d + d, 4) ? p.d[d] : 0.0f;
    const float bias = p.delta_bias && live && relay_in_bounds(p.delta_bias + d, 4) ? p.delta_bias[d] : 0.0f;
    for (long long t = 0; t < p.T; ++t) {
        const long long row = (t * p.B + i) * p.D;
        float y = 0.0f, u = 0.0f;
        if (live && p.states && t % kSpan == 0) {
#pragma unroll
            for (int k = 0; k < NB; ++k) store_states(p, p.states, ((t / kSpan) * p.B * p.D + at) * p.N, k * 16 + nl * 4, h[k]);
        }
        if (t < end) {
            u = load_weight<T>(p.u, row + d);
            float step = load_weight<T>(p.delta, row + d) + bias, other;
            if (p.softplus) unpair(softplus2(pair(step, step)).value, step, other);
            const long long bc = (t * p.B + i) * p.ld_bc;
#pragma unroll
            for (int k = 0; k < NB; ++k)
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    float decay[2];
                    unpair(decay2(pair(step * a[k][j], step * a[k][j + 1])), decay[0], decay[1]);
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int n = k * 16 + nl * 4 + j + q;
                        if (n >= p.N) continue;
                        h[k][j + q] = fmaf(decay[q], h[k][j + q], step * u * load_weight<T>(p.b, bc + n));
                        y = fmaf(load_weight<T>(p.c, bc + n), h[k][j + q], y);
                    }
                }
        }
        y += __shfl_xor_sync(0xffffffffu, y, 1);
        y += __shfl_xor_sync(0xffffffffu, y, 2);
        if (live && nl == 0) {
            float out[1] = {0.0f};
            if (t < end) {
                out[0] = p.d ? fmaf(skip, u, y) : y;       // no term, not one of zero: u may be infinite
                if (p.z) {
                    const float z = load_weight<T>(p.z, row + d);
                    out[0] *= z * logistic<FINE>(z);
                }
            }
            store<T, 1>(p.y, row + d, out);
        }
    }
    if (!live) return;
#pragma unroll
    for (int k = 0; k < NB; ++k) store_states(p, p.h_final, at * p.N, k * 16 + nl * 4, h[k]);
}

// ---- chunks -----------------------------------------------------------------------------------------------------------
// A block: two warps of eight channels each; four lanes a channel, with four neighbouring states of every sixteen each.  A chunk's rows are
// fetched a chunk ahead by TMA.  Three phases: steps and weights are made fp32, four channels a thread; the scan itself; and skip, gate and
// rounding of the results, whose four parts a channel the scan leaves side by side.  Several blocks on an SM are in different phases.
//
// Where there are too few channels for that, the blocks of a cluster take a part of the sequence each.  Every block first takes its part from
// a zero state, for the state that it leaves and the sum of its steps alone; then the blocks read each other's (shared memory of the cluster),
// join those before their own, exp(a sum of steps) being the part's decay, and take their part again from the state that it starts with.
constexpr int STAGES = 2, STEPS = 32, WARPS = 2, THREADS = 32 * WARPS, CHANNELS = 8 * WARPS;

template <typename T, int NB>
struct Tile {
    static constexpr int NP = 16 * NB;
    struct Stage { alignas(128) T u[STEPS][CHANNELS]; alignas(128) T delta[STEPS][CHANNELS]; alignas(128) T z[STEPS][CHANNELS]; alignas(128) T bc[STEPS * 2 * NP]; };
    Stage stage[STAGES];
    alignas(16) float2 step[STEPS][CHANNELS];              // delta, delta u
    alignas(16) float b[STEPS][NP], c[STEPS][NP];
    // The four lanes' parts of sum_n c h, channel ch of lane l at ch ^ 8 (l >> 1): no two lanes of a warp in one bank.  Between the passes of a
    // shared sequence: the state from zero and the sum of steps of every lane, for the cluster.
    union {
        alignas(16) float y[STEPS][4][CHANNELS];
        struct { ulonglong2 left[NB][THREADS]; float sum[THREADS]; };
    };
    uint64_t full[STAGES];
    int gave_up;
};

template <typename T, int NB, bool SPLIT>
__global__ void __launch_bounds__(THREADS) selective_scan_kernel(const Args p, const __grid_constant__ Maps maps, const int parts)
{
    using S = Tile<T, NB>;
    constexpr bool FINE = sizeof(T) == 4;
    extern __shared__ uint8_t shared_raw[];
    S &s = *reinterpret_cast<S *>(((uintptr_t)shared_raw + 127) & ~(uintptr_t)127);
    const int tid = threadIdx.x, lane = tid & 31, wc = tid >> 5, nl = lane & 3, cl = lane >> 2;
    const long long block = SPLIT ? blockIdx.x / parts : blockIdx.x;
    const int part = SPLIT ? (int)(blockIdx.x - block * parts) : 0;        // rank in the cluster
    const long long i = block / p.groups;
    const long long c0 = (block - i * p.groups) * CHANNELS;
    if (tid == 0) {
        for (int q = 0; q < STAGES; ++q) tc::mbar_init(&s.full[q], 1);
        s.gave_up = 0;
        tc::fence_barrier_init();
    }
    __syncthreads();
    pdl_wait();
    const long long end = end_of(p, i);
    const int all = (int)((p.T + STEPS - 1) / STEPS), each = SPLIT ? (all + parts - 1) / parts : all;
    const int first = min(all, part * each), last = min(all, first + each);                  // this block's chunks
    const int live = max(0, min(last, (int)((end + STEPS - 1) / STEPS)) - first);             // those of them inside the sequence
    // rows of the k-th live chunk into the stage of the q-th fetch, by TMA (one thread) or by everyone's own copies
    auto fetch = [&](int q, int k, bool with_z) {
        typename S::Stage &g = s.stage[q % STAGES];
        const long long t0 = (long long)(first + k) * STEPS;
        if (tid == 0 && (p.tma_x || p.tma_w)) {
            uint64_t *full = &s.full[q % STAGES];
            const uint32_t x = p.tma_x ? (with_z ? 3u : 2u) * (uint32_t)sizeof(g.u) : 0u, w = p.tma_w ? (uint32_t)(STEPS * 2 * p.N * sizeof(T)) : 0u;
            tc::mbar_expect_tx(full, x + w);
            const int col = (int)(i * p.D + c0), row = (int)t0;
            if (p.tma_x) {
                tc::tma_load_2d(g.u, &maps.u, full, col, row);
                tc::tma_load_2d(g.delta, &maps.delta, full, col, row);
                if (with_z) tc::tma_load_2d(g.z, &maps.z, full, col, row);
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
            if (with_z) copy_rows<T>(&g.z[0][0], CHANNELS, (const T *)p.z + at, p.B * p.D, rows, width, tid, THREADS);
        }
        if (!p.tma_w) {
            const long long at = (t0 * p.B + i) * p.ld_bc;
            copy_rows<T>(g.bc, p.ld_bc, (const T *)p.b + at, p.B * p.ld_bc, rows, p.ld_bc, tid, THREADS);
            if (p.ld_bc == p.N) copy_rows<T>(g.bc + STEPS * p.N, p.N, (const T *)p.c + at, p.B * p.ld_bc, rows, p.N, tid, THREADS);
        }
        copies_end();
    };
    int fetched = 0, used = 0;                             // fetches so far, and chunks taken from them
    // this thread's states: of channel mine
    const int ch = wc * 8 + cl;
    const long long mine = c0 + ch;
    f32x2 a[NB][2], h[NB][2];                              // a log2(e); the state
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        float x[4];
        load_states(p, mine < p.D ? p.a : nullptr, mine * p.N, k * 16 + nl * 4, x);
        a[k][0] = pair(exponent_of(x[0]), exponent_of(x[1]));
        a[k][1] = pair(exponent_of(x[2]), exponent_of(x[3]));
    }
    auto from_start = [&] {
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            float x[4];
            load_states(p, mine < p.D ? p.h0 : nullptr, (i * p.D + mine) * p.N, k * 16 + nl * 4, x);
            h[k][0] = pair(x[0], x[1]);
            h[k][1] = pair(x[2], x[3]);
        }
    };
    auto write = [&](float *to, long long row, int k) {
        float g[4];
        unpair(h[k][0], g[0], g[1]); unpair(h[k][1], g[2], g[3]);
        if (mine < p.D) store_states(p, to, (row + mine) * p.N, k * 16 + nl * 4, g);
    };
    // four channels that this thread turns into steps, and whose results it finishes: always the same ones
    constexpr int G = 4, UNITS = CHANNELS / G, PASSES = STEPS * UNITS / THREADS;
    static_assert(THREADS % UNITS == 0 && PASSES * THREADS == STEPS * UNITS, "a thread's channels are the same in every row");
    const int pc = G * (tid % UNITS);
    f32x2 skip[G / 2], bias[G / 2];
#pragma unroll
    for (int j = 0; j < G; j += 2) {
        float x[2], y[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const long long d = c0 + pc + j + q;
            x[q] = p.d && d < p.D && relay_in_bounds(p.d + d, 4) ? p.d[d] : 0.0f;
            y[q] = p.delta_bias && d < p.D && relay_in_bounds(p.delta_bias + d, 4) ? p.delta_bias[d] : 0.0f;
        }
        skip[j / 2] = pair(x[0], x[1]);
        bias[j / 2] = pair(y[0], y[1]);
    }
    // waits for a chunk's rows; steps and weights in fp32
    auto prepare = [&](const typename S::Stage &g, int in) {
        if (p.tma_x || p.tma_w) tc::mbar_wait(&s.full[used % STAGES], (used / STAGES) & 1, &s.gave_up, p.err, tc::ERR_WAIT_FULL);
        if (!p.tma_x || !p.tma_w) { copies_done(fetched - used - 1); __syncthreads(); }      // everyone's own copies
#pragma unroll
        for (int k = 0; k < PASSES; ++k) {
            const int t = tid / UNITS + k * (THREADS / UNITS);
            float u[G], x[G];
            widen_shared(&g.u[t][pc], u);
            widen_shared(&g.delta[t][pc], x);
            f32x2 step[G / 2];
#pragma unroll
            for (int j = 0; j < G / 2; ++j) step[j] = add2(pair(x[2 * j], x[2 * j + 1]), bias[j]);
            if (p.softplus) {
#pragma unroll
                for (int j = 0; j < G / 2; ++j) step[j] = softplus2(step[j]).value;
            }
            if (t >= in) {                                 // behind the end nothing decays and nothing is added
#pragma unroll
                for (int j = 0; j < G; ++j) { step[j / 2] = 0; u[j] = 0.0f; }
            }
#pragma unroll
            for (int j = 0; j < G / 2; ++j) {
                float lo, hi;
                unpair(step[j], lo, hi);
                *reinterpret_cast<float4 *>(&s.step[t][pc + 2 * j]) = make_float4(lo, lo * u[2 * j], hi, hi * u[2 * j + 1]);
            }
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
        ++used;
        __syncthreads();
    };
    // A few steps at a time: first their decays and what they add, all independent, then the chain.  RESULTS: leaves the parts of sum_n c h.
    float sum = 0.0f;
    auto chain = [&](auto results) {
        constexpr bool RESULTS = decltype(results)::value;
        constexpr int AT_ONCE = NB == 1 ? 8 : 2;
#pragma unroll (NB == 1 ? 4 : 2)
        for (int r0 = 0; r0 < STEPS; r0 += AT_ONCE) {
            f32x2 da[AT_ONCE][NB][2], x[AT_ONCE][NB][2];
#pragma unroll
            for (int r = 0; r < AT_ONCE; ++r) {
                const float2 st = s.step[r0 + r][ch];
                const f32x2 dd = pair(st.x, st.x), du = pair(st.y, st.y);
                if (!RESULTS) sum += st.x;
#pragma unroll
                for (int k = 0; k < NB; ++k) {
                    const ulonglong2 b = *reinterpret_cast<const ulonglong2 *>(&s.b[r0 + r][k * 16 + nl * 4]);
                    da[r][k][0] = decay2(mul2(dd, a[k][0]));
                    da[r][k][1] = decay2(mul2(dd, a[k][1]));
                    x[r][k][0] = mul2(du, b.x);
                    x[r][k][1] = mul2(du, b.y);
                }
            }
#pragma unroll
            for (int r = 0; r < AT_ONCE; ++r) {
                f32x2 y = 0;
#pragma unroll
                for (int k = 0; k < NB; ++k) {
                    h[k][0] = fma2(da[r][k][0], h[k][0], x[r][k][0]);
                    h[k][1] = fma2(da[r][k][1], h[k][1], x[r][k][1]);
                    if (!RESULTS) continue;
                    const ulonglong2 c = *reinterpret_cast<const ulonglong2 *>(&s.c[r0 + r][k * 16 + nl * 4]);
                    y = k ? fma2(c.x, h[k][0], y) : mul2(c.x, h[k][0]);
                    y = fma2(c.y, h[k][1], y);
                }
                if (RESULTS) s.y[r0 + r][nl][ch ^ ((nl >> 1) << 3)] = sum2(y);
            }
        }
    };
    if constexpr (SPLIT) {
#pragma unroll
        for (int k = 0; k < NB; ++k) h[k][0] = h[k][1] = 0;
        if (part < parts - 1) {                            // nobody joins the last part
            for (int k = 0; k < STAGES && k < live; ++k) fetch(fetched++, k, false);
            for (int chunk = 0; chunk < live; ++chunk) {
                prepare(s.stage[used % STAGES], (int)min((long long)STEPS, end - (long long)(first + chunk) * STEPS));
                if (chunk + STAGES < live) fetch(fetched++, chunk + STAGES, false);           // its rows have been read
                chain(std::false_type());
                __syncthreads();                           // steps and weights have been read
            }
        }
#pragma unroll
        for (int k = 0; k < NB; ++k) s.left[k][tid] = make_ulonglong2(h[k][0], h[k][1]);
        s.sum[tid] = sum;
    }
    // the rows that the second pass begins with are on their way while the blocks meet
    for (int k = 0; k < STAGES && k < live; ++k) fetch(fetched++, k, p.z != nullptr);
    from_start();
    if constexpr (SPLIT) {
        tc::cluster_sync();
        for (int r = 0; r < part; ++r) {
            const uint32_t at = tc::mapa(tc::smem_u32(&s.sum[tid]), (uint32_t)r);
            float total;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(total) : "r"(at));
#pragma unroll
            for (int k = 0; k < NB; ++k) {
                const uint32_t from = tc::mapa(tc::smem_u32(&s.left[k][tid]), (uint32_t)r);
                unsigned long long x, y;
                asm volatile("ld.shared::cluster.v2.u64 {%0, %1}, [%2];" : "=l"(x), "=l"(y) : "r"(from));
                h[k][0] = fma2(decay2(mul2(pair(total, total), a[k][0])), h[k][0], x);
                h[k][1] = fma2(decay2(mul2(pair(total, total), a[k][1])), h[k][1], y);
            }
        }
        tc::cluster_sync();                                // every block has read what it needs of the others
    }
    for (int chunk = 0; chunk < live; ++chunk) {
        typename S::Stage &g = s.stage[used % STAGES];
        const long long t0 = (long long)(first + chunk) * STEPS;
        const int in = (int)min((long long)STEPS, end - t0);                 // steps of the chunk that are inside the sequence
        prepare(g, in);
        if (p.states) {
#pragma unroll
            for (int k = 0; k < NB; ++k) write(p.states, ((first + chunk) * p.B + i) * p.D, k);
        }
        chain(std::true_type());
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PASSES; ++k) {
            const int t = tid / UNITS + k * (THREADS / UNITS);
            if (t0 + t >= p.T) break;
            f32x2 out[G / 2];
            float q[G];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(&s.y[t][j][pc ^ ((j >> 1) << 3)]);
                out[0] = j ? add2(out[0], v.x) : v.x;
                out[1] = j ? add2(out[1], v.y) : v.y;
            }
            widen_shared(&g.u[t][pc], q);
            if (p.d) { out[0] = fma2(skip[0], pair(q[0], q[1]), out[0]); out[1] = fma2(skip[1], pair(q[2], q[3]), out[1]); }
            if (p.z) {
                widen_shared(&g.z[t][pc], q);
                out[0] = mul2(out[0], pair(q[0] * logistic<FINE>(q[0]), q[1] * logistic<FINE>(q[1])));
                out[1] = mul2(out[1], pair(q[2] * logistic<FINE>(q[2]), q[3] * logistic<FINE>(q[3])));
            }
            unpair(out[0], q[0], q[1]); unpair(out[1], q[2], q[3]);
            if (t >= in) q[0] = q[1] = q[2] = q[3] = 0.0f;
            store_some<T>(p, p.y, ((t0 + t) * p.B + i) * p.D, c0 + pc, q);
        }
        __syncthreads();                                   // the stage is free
        if (chunk + STAGES < live) fetch(fetched++, chunk + STAGES, p.z != nullptr);
    }
    // behind the sequence
    const float zero[G] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (long long t = (long long)(first + live) * STEPS + tid / UNITS; t < min(p.T, (long long)last * STEPS); t += THREADS / UNITS)
        store_some<T>(p, p.y, (t * p.B + i) * p.D, c0 + pc, zero);
#pragma unroll
    for (int k = 0; k < NB; ++k) {
        if (p.states)
            for (int q = first + live; q < last; ++q) write(p.states, (q * p.B + i) * p.D, k);
        if (p.h_final && part == parts - 1) write(p.h_final, i * p.D, k);
    }
}
static_assert(STEPS == kSpan, "a chunk starts where a state is saved");

// ---- launches ------------------------------------------------------------------------------------------------------
// Up to few_steps() step by step, longer ones by chunks, whose time grows with the number of chunks alone.  bf16, 64 x 2048 channels, us step by step and
// by chunks: N = 16, 8 steps 40 and 43, 10 steps 49 and 44; N = 32, 10 steps 73 and 80, 12 steps 86 and 80; N = 64, 16 steps 150 and 158, 20 steps 182 and 161.
// Few channels wait for each step's rows in turn: 4 x 2048, N = 16, 4 steps 8.4 and 8.7, 8 steps 13.6 and 8.7; 10 x 2048, 5 steps 10.5 and 11.8, 8 steps
// 15.1 and 11.8; 16 x 2048, 8 steps 15.4 and 14.8.
constexpr long long kSms = 148;

template <int NB>
long long few_steps(const Args &p)
{
    return p.B * p.D < 32768 ? 4 : NB == 1 ? 8 : NB == 2 ? 12 : 16;
}

template <typename T, int NB>
relay_status_t launch_steps(const Args &p, cudaStream_t st)
{
    const long long blocks = (p.B * p.D * 4 + kStepThreads - 1) / kStepThreads;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "selective_scan: %lld x %lld channels", p.B, p.D);
    RELAY_CUDA(launch_pdl(selective_scan_steps_kernel<T, NB>, dim3((unsigned)blocks), dim3(kStepThreads), 0, st, p));
    return check_launch("selective_scan");
}
template <typename T, int NB, bool SPLIT>
relay_status_t launch_chunks(Args p, int parts, cudaStream_t st)
{
    using S = Tile<T, NB>;
    p.groups = (int)((p.D + CHANNELS - 1) / CHANNELS);
    const long long blocks = p.B * p.groups * parts;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "selective_scan: %lld x %lld channels", p.B, p.D);
    if (!p.err) return fail(RELAY_ERR_CUDA, "no device error word");
    Maps maps;
    RELAY_TRY(make_maps(&p, &maps, sizeof(T) == 4, CHANNELS, STEPS));
    const size_t bytes = sizeof(S) + 128;
    RELAY_CUDA(cudaFuncSetAttribute(selective_scan_kernel<T, NB, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if constexpr (SPLIT)
        RELAY_CUDA(launch_pdl_cluster(selective_scan_kernel<T, NB, SPLIT>, dim3((unsigned)blocks), dim3(THREADS), dim3(parts), bytes, st, p, maps, parts));
    else
        RELAY_CUDA(launch_pdl(selective_scan_kernel<T, NB, SPLIT>, dim3((unsigned)blocks), dim3(THREADS), bytes, st, p, maps, parts));
    return check_launch("selective_scan");
}
// Blocks that share a sequence.  A second pass costs them three quarters as much again, so it pays where one pass leaves most of the chip empty, and
// later with more states, whose blocks hold more of it.  us alone, by four and by eight; bf16, N = 16: 2048 steps of 2048 warps 345, 575, 610; 4096
// of 1024 505, 598, 587; 4096 of 640 447, 496, 397; 8192 of 512 768, 603, 602; 16384 of 256 1490, 851, 603; 256 of 512 28, 25, 30; 256 of 256 27, 21, 17;
// 256 of 128 27, 16, 14; 128 of 256 16, 13.  f32: 2048 of 640 258, 242, 244; 256 of 512 31, 39, 38; 256 of 256 29, 21, 26.  N = 64: 2048 of 512 538,
// 554, 572; 2048 of 256 472, 280, 289; 256 of 256 63, 43, 55.
int parts_of(const Args &p)
{
    const long long warps = p.B * ((p.D + 7) / 8), chunks = (p.T + STEPS - 1) / STEPS;
    if (warps > (p.N <= 16 ? 5 : 3) * kSms) return 1;
    if (chunks >= (warps <= kSms ? 8 : 16)) return 8;
    return warps <= 2 * kSms && chunks >= 4 ? 4 : 1;
}
template <typename T, int NB>
relay_status_t launch_form(const Args &p, cudaStream_t st)
{
    if (p.T <= few_steps<NB>(p)) return launch_steps<T, NB>(p, st);
    const int parts = parts_of(p);
    return parts > 1 ? launch_chunks<T, NB, true>(p, parts, st) : launch_chunks<T, NB, false>(p, 1, st);
}
template <typename T>
relay_status_t launch_states(const Args &p, cudaStream_t st)
{
    if (p.N <= 16) return launch_form<T, 1>(p, st);
    return p.N <= 32 ? launch_form<T, 2>(p, st) : launch_form<T, 4>(p, st);
}

}  // namespace

namespace scan {

// TMA takes rows of whole 16-byte pieces that start at such pieces for every batch element, and coordinates of 31 bits.
relay_status_t make_maps(Args *p, Maps *m, bool f32, int channels, int steps)
{
    const int64_t e = f32 ? 4 : 2, row = p->B * p->D, weights = p->B * p->ld_bc;
    p->tma_x = p->T > 0 && p->D * e % 16 == 0 && row < 0x7fffff00LL && p->T < 0x7fffff00LL;
    p->tma_w = p->T > 0 && p->ld_bc * e % 16 == 0 && weights < 0x7fffff00LL && p->T < 0x7fffff00LL;
    *m = Maps{};
    if (p->tma_x) {
        RELAY_TRY(make_tmap_2d(&m->u, f32, p->u, row, p->T, row, channels, steps, false));
        RELAY_TRY(make_tmap_2d(&m->delta, f32, p->delta, row, p->T, row, channels, steps, false));
        if (p->z) RELAY_TRY(make_tmap_2d(&m->z, f32, p->z, row, p->T, row, channels, steps, false));
        if (p->dy) RELAY_TRY(make_tmap_2d(&m->dy, f32, p->dy, row, p->T, row, channels, steps, false));
    }
    if (p->tma_w) {
        RELAY_TRY(make_tmap_2d(&m->b, f32, p->b, weights, p->T, weights, p->ld_bc, steps, false));
        if (p->ld_bc == p->N) RELAY_TRY(make_tmap_2d(&m->c, f32, p->c, weights, p->T, weights, p->ld_bc, steps, false));
    }
    return RELAY_OK;
}

relay_status_t check_inputs(const Inputs &in, Sizes *s, int64_t *N)
{
    RELAY_TRY(check_not_null(in.u, "u"));
    RELAY_TRY(check_not_null(in.delta, "delta"));
    RELAY_TRY(check_not_null(in.a, "a"));
    RELAY_TRY(check_not_null(in.b, "b"));
    RELAY_TRY(check_sizes(in.u, in.a, s, N));
    const int32_t t = in.u->dtype;
    RELAY_TRY(check_tensor(in.delta, t, t, {s->T, s->B, s->D}, "delta"));
    RELAY_TRY(check_tensor(in.b, t, t, {s->T, s->B, in.c ? *N : 2 * *N}, "b"));
    RELAY_TRY(check_tensor(in.c, t, t, {s->T, s->B, *N}, "c"));
    RELAY_TRY(check_tensor(in.d, RELAY_F32, RELAY_F32, {s->D}, "d"));
    RELAY_TRY(check_tensor(in.z, t, t, {s->T, s->B, s->D}, "z"));
    RELAY_TRY(check_tensor(in.delta_bias, RELAY_F32, RELAY_F32, {s->D}, "delta_bias"));
    return check_tensor(in.lengths, RELAY_I32, RELAY_I32, {s->B}, "lengths");
}
relay_status_t check_sizes(const relay_tensor_t *u, const relay_tensor_t *a, Sizes *s, int64_t *N)
{
    RELAY_TRY(check_sequence(u, s, "u"));
    RELAY_TRY(check_type(a, "a"));
    RELAY_TRY(check_rank(a, 2, "a"));
    *N = a->shape[1];
    RELAY_TRY(check_tensor(a, RELAY_F32, RELAY_F32, {s->D, *N}, "a"));
    if (*N < 1 || *N > RELAY_MAX_SCAN_STATES)
        return fail(RELAY_ERR_SHAPE, "a: %lld states, needs 1..%d", (long long)*N, RELAY_MAX_SCAN_STATES);
    return RELAY_OK;
}
relay_status_t check_softplus(int32_t softplus)
{
    if (softplus != 0 && softplus != 1) return fail(RELAY_ERR_ATTR, "softplus = %d, needs 0 or 1", softplus);
    return RELAY_OK;
}
Args make_args(const Inputs &in, int32_t softplus, const Sizes &s, int64_t N)
{
    Args p{};
    p.u = in.u->data; p.delta = in.delta->data; p.a = (const float *)in.a->data;
    p.b = in.b->data;
    p.c = in.c ? in.c->data : (const char *)in.b->data + N * dtype_size(in.b->dtype);
    p.d = in.d ? (const float *)in.d->data : nullptr;
    p.z = in.z ? in.z->data : nullptr;
    p.delta_bias = in.delta_bias ? (const float *)in.delta_bias->data : nullptr;
    p.lengths = in.lengths ? (const int *)in.lengths->data : nullptr;
    p.T = s.T; p.B = s.B; p.D = s.D; p.N = (int)N;
    p.ld_bc = (int)(in.c ? N : 2 * N);
    p.softplus = softplus;
    p.pairs = s.D % 2 == 0;
    p.four = s.D % 4 == 0;
    p.err = device_error_word();
    p.quads = N % 4 == 0;
    return p;
}

}  // namespace scan
}  // namespace relay

using namespace relay;

extern "C" relay_status_t relay_infer_selective_scan(const relay_tensor_t *u, const relay_tensor_t *a, relay_tensor_t *y,
                                                     relay_tensor_t *h_final, relay_tensor_t *states)
{
    clear_error();
    RELAY_TRY(check_not_null(u, "u"));
    RELAY_TRY(check_not_null(a, "a"));
    RELAY_TRY(check_not_null(y, "y"));
    RELAY_TRY(check_not_null(h_final, "h_final"));
    RELAY_TRY(check_not_null(states, "states"));
    seq::Sizes s;
    int64_t N;
    RELAY_TRY(scan::check_sizes(u, a, &s, &N));
    *y = *u;
    y->data = nullptr;
    *h_final = relay_tensor_t{};
    h_final->dtype = RELAY_F32; h_final->rank = 3; h_final->layout = RELAY_ROWMAJOR;
    h_final->shape[0] = s.B; h_final->shape[1] = s.D; h_final->shape[2] = N;
    *states = relay_tensor_t{};
    states->dtype = RELAY_F32; states->rank = 4; states->layout = RELAY_ROWMAJOR;
    states->shape[0] = (s.T + RELAY_SCAN_SPAN - 1) / RELAY_SCAN_SPAN;
    states->shape[1] = s.B; states->shape[2] = s.D; states->shape[3] = N;
    return RELAY_OK;
}

extern "C" relay_status_t relay_selective_scan(const relay_tensor_t *u, const relay_tensor_t *delta, const relay_tensor_t *a,
                                               const relay_tensor_t *b, const relay_tensor_t *c, const relay_tensor_t *d,
                                               const relay_tensor_t *z, const relay_tensor_t *delta_bias, const relay_tensor_t *h0,
                                               const relay_tensor_t *lengths, int32_t softplus, const relay_tensor_t *y,
                                               const relay_tensor_t *h_final, const relay_tensor_t *states, void *stream)
{
    clear_error();
    const scan::Inputs in{u, delta, a, b, c, d, z, delta_bias, lengths};
    seq::Sizes s;
    int64_t N;
    RELAY_TRY(check_not_null(y, "y"));
    RELAY_TRY(scan::check_inputs(in, &s, &N));
    RELAY_TRY(seq::check_tensor(h0, RELAY_F32, RELAY_F32, {s.B, s.D, N}, "h0"));
    RELAY_TRY(seq::check_tensor(y, u->dtype, u->dtype, {s.T, s.B, s.D}, "y"));
    RELAY_TRY(seq::check_tensor(h_final, RELAY_F32, RELAY_F32, {s.B, s.D, N}, "h_final"));
    RELAY_TRY(seq::check_tensor(states, RELAY_F32, RELAY_F32, {(s.T + RELAY_SCAN_SPAN - 1) / RELAY_SCAN_SPAN, s.B, s.D, N}, "states"));
    RELAY_TRY(scan::check_softplus(softplus));
    const relay_tensor_t *ins[10] = {u, delta, a, b, c, d, z, delta_bias, h0, lengths}, *outs[3] = {y, h_final, states};
    RELAY_TRY(seq::check_buffers(ins, outs));
    if (s.B == 0 || s.D == 0) return RELAY_OK;
    scan::Args p = scan::make_args(in, softplus, s, N);
    p.h0 = h0 ? (const float *)h0->data : nullptr;
    p.y = y->data;
    p.h_final = h_final ? (float *)h_final->data : nullptr;
    p.states = states ? (float *)states->data : nullptr;
    cudaStream_t st = (cudaStream_t)stream;
    RELAY_TRY(seq::register_buffers(ins, outs, nullptr, 0, st));
    return u->dtype == RELAY_F32 ? launch_states<float>(p, st) : launch_states<__nv_bfloat16>(p, st);
}
