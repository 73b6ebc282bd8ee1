// The contraction on pairs of SMs (gemm_tc2.cuh) with the dense groups' epilogue: bias, activation, rounding, TMA tile stores.
#include "gemm_tc2.cuh"

namespace relay {

using namespace gemm_tc;
using namespace gemm_tc2;

relay_status_t make_tmap_2d_sw64(CUtensorMap *m, bool f32, const void *base, uint64_t inner, uint64_t outer, uint64_t row_stride,
                                 uint32_t box_outer);
relay_status_t make_tmap_2d_bf16(CUtensorMap *m, const void *base, uint64_t inner, uint64_t outer, uint64_t row_stride,
                                 uint32_t box_inner, uint32_t box_outer);

namespace {

// One epilogue warp drains its 32 accumulator rows, the 32-column groups [g_begin, g_end) of an accumulator that
// starts at column n0: both groups' TMEM loads are issued before the first is awaited (a load takes several hundred
// cycles), then per group bias + activation + rounding, a 32-row x 64-byte staging buffer in the 64-byte swizzle
// pattern (16-byte piece c of row r at piece c ^ ((r >> 1) & 3)) and one TMA tile store (two for f32 output).
// The drain is spread over sixteen warps because one warp alone issues these instructions only every few cycles.
template <bool OUT_F32, bool TRANSC>
__device__ __forceinline__ void finish_group(const Params &p, const CUtensorMap *tm_c, uint8_t *stage, int lane, int row0, int nc,
                                             float bias_lane, uint32_t (&r)[32])
{
    float v[32];
    if (p.bias != nullptr) {                             // warp-uniform; lane j holds the bias of column nc + j
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]) + __shfl_sync(0xffffffffu, bias_lane, j);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
    }
    if (TRANSC) {                                        // tanh / sigmoid: their own instantiation (they need many registers)
        if (p.gate_block > 0) {                          // LSTM gates: a 32-column group lies inside one gate block (warp-uniform)
            if (nc / p.gate_block == 2) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = 1.0f - __fdividef(2.0f, 1.0f + __expf(2.0f * v[j]));
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __fdividef(1.0f, 1.0f + __expf(-v[j]));
            }
        } else if (p.act == RELAY_ACT_TANH) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = OUT_F32 ? tanh_<false>(v[j]) : tanh_<true>(v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = OUT_F32 ? sigmoid_<false>(v[j]) : sigmoid_<true>(v[j]);
        }
    } else if (p.act == RELAY_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = fmaxf(v[j], 0.0f);
    }
    const int sw = (lane >> 1) & 3;
#pragma unroll
    for (int h = 0; h < (OUT_F32 ? 2 : 1); ++h) {        // 64 bytes of every row at a time
        if (tc::elect_one()) tc::tma_store_wait_read<0>();   // the previous store (same elected lane) has read the buffer
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            uint4 piece;
            if (OUT_F32) piece = make_uint4(__float_as_uint(v[16 * h + 4 * c]), __float_as_uint(v[16 * h + 4 * c + 1]),
                                            __float_as_uint(v[16 * h + 4 * c + 2]), __float_as_uint(v[16 * h + 4 * c + 3]));
            else piece = make_uint4(pack2(v[8 * c], v[8 * c + 1]), pack2(v[8 * c + 2], v[8 * c + 3]), pack2(v[8 * c + 4], v[8 * c + 5]),
                                    pack2(v[8 * c + 6], v[8 * c + 7]));
            *reinterpret_cast<uint4 *>(stage + lane * 64 + ((c ^ sw) << 4)) = piece;
        }
        tc::fence_proxy_async();
        __syncwarp();
        if (tc::elect_one()) {                           // the election is deterministic: always the same lane of the warp
            tc::tma_store_2d(tm_c, stage, nc + h * (OUT_F32 ? 16 : 0), row0);
            tc::tma_store_commit();
        }
    }
}

// One epilogue warp drains its 32 accumulator rows, `per` (1 or 2) 32-column groups starting at group g0 of an
// accumulator that starts at column n0: the TMEM loads of both groups are issued before the first is awaited (a load
// takes several hundred cycles), then per group bias + activation + rounding, a 32-row x 64-byte staging buffer in
// the 64-byte swizzle pattern (16-byte piece c of row r at piece c ^ ((r >> 1) & 3)) and one TMA tile store (two for
// f32 output).  The drain is spread over sixteen warps because one warp alone issues these instructions only every
// few cycles.
template <bool OUT_F32, bool TRANSC>
__device__ __forceinline__ void drain_groups(const Params &p, const CUtensorMap *tm_c, uint32_t taddr, uint8_t *stage, int lane, int row0,
                                             int n0, const float (&bias_r)[8], int g0, int per)
{
    uint32_t ra[32], rb[32];
    const int g1 = g0 + per - 1;                         // per == 1: the same group again (its copy is not used)
    tc::tmem_ld_32x32(taddr + g0 * 32, ra);
    tc::tmem_ld_32x32(taddr + g1 * 32, rb);
    tc::tmem_ld_wait();
    float bl0 = 0.0f, bl1 = 0.0f;
#pragma unroll
    for (int q = 0; q < 8; ++q) { if (q == g0) bl0 = bias_r[q]; if (q == g1) bl1 = bias_r[q]; }
    if (n0 + g0 * 32 < p.N) finish_group<OUT_F32, TRANSC>(p, tm_c, stage, lane, row0, n0 + g0 * 32, bl0, ra);
    if (per == 2 && n0 + g1 * 32 < p.N) finish_group<OUT_F32, TRANSC>(p, tm_c, stage, lane, row0, n0 + g1 * 32, bl1, rb);
}

template <bool TRANSC>
struct StoreEpilogue {
    using Params = gemm_tc::Params;
    static constexpr int kDepth = 0;
    float bias_r[8];
    __device__ __forceinline__ void prepare(const Params &p, int lane, int, int n0, int width) { load_bias(p, lane, n0, width, bias_r); }
    __device__ __forceinline__ void drain(const Params &p, const CUtensorMap *tm_c, uint32_t taddr, uint8_t *stage, int lane, int row0, int n0,
                                          int width, int slot)
    {
        const int per = width / 128;                     // 32-column groups per warp: 2 for a 256-column accumulator, 1 for 128
        if (p.out_f32) drain_groups<true, TRANSC>(p, tm_c, taddr, stage, lane, row0, n0, bias_r, slot * per, per);
        else drain_groups<false, TRANSC>(p, tm_c, taddr, stage, lane, row0, n0, bias_r, slot * per, per);
    }
    __device__ __forceinline__ void finish() { if (tc::elect_one()) tc::tma_store_wait_all<0>(); }
};

}  // namespace

bool gemm_tc2_eligible(const GemmDesc &g, int sms)
{
    if (g.M < 256 || sms < 2) return false;
    const int64_t t2 = ((g.M + 255) / 256) * ((g.N + BN - 1) / BN);
    return t2 >= sms;                                 // at least two 256 x 256 tiles per pair of SMs
}

relay_status_t launch_gemm_tc2(const GemmDesc &g, int sms, cudaStream_t st)
{
    const bool a_mn = g.a_sk != 1, b_mn = g.b_sk != 1;
    CUtensorMap tm_a, tm_b, tm_c;
    if (a_mn) RELAY_TRY(make_tmap_2d_bf16(&tm_a, g.a, g.M, g.K, g.a_sk, 64, BK));
    else RELAY_TRY(make_tmap_2d_bf16(&tm_a, g.a, g.K, g.M, g.a_sm, BK, 128));
    if (b_mn) RELAY_TRY(make_tmap_2d_bf16(&tm_b, g.b, g.N, g.K, g.b_sk, 64, BK));
    else RELAY_TRY(make_tmap_2d_bf16(&tm_b, g.b, g.K, g.N, g.b_sn, BK, 64));
    const bool f32 = g.out_dtype == RELAY_F32;
    RELAY_TRY(make_tmap_2d_sw64(&tm_c, f32, g.c, g.N, g.M, g.ldc, 32));
    Params p{};
    p.M = (int)g.M; p.N = (int)g.N; p.K = (int)g.K;
    p.c = g.c; p.ldc = g.ldc;
    p.bias = g.bias; p.bias_bf16 = g.bias_dtype == RELAY_BF16; p.act = g.act; p.out_f32 = f32;
    p.gate_block = (int)g.gate_block;
    p.tiles_m = (int)((g.M + 255) / 256); p.tiles_n = (int)((g.N + BN - 1) / BN); p.k_blocks = (int)((g.K + BK - 1) / BK);
    p.err = device_error_word();
    if (!p.err) return fail(RELAY_ERR_CUDA, "no device error word");
    const int n_tiles = p.tiles_m * p.tiles_n;
    const int pairs = std::min(n_tiles, sms / 2);
    static thread_local UnitTable tb;
    tb.n = 0;
    p.tail_split = 1;
    if (!plan_units(p.tiles_m, (int)((g.N + 127) / 128), pairs, p.k_blocks, &tb)) {
        // fixed scheme: class-4 units for whole rounds over the pairs (only for a contraction long enough to pay for
        // their exposed epilogue), then 256 x 256 tiles; the tiles of a last, partly filled round become two
        // half-width units each when they then still fit one round
        tb.n = 0;
        const int wide_rounds = p.k_blocks >= kWideMinKBlocks ? std::min(n_tiles / (2 * pairs), (p.tiles_m * (p.tiles_n / 2)) / pairs) : 0;
        p.wide_units = wide_rounds * pairs;
        const int narrow = n_tiles - 2 * p.wide_units;
        const int rem = narrow % pairs;
        p.tail_split = (rem > 0 && 2 * rem <= pairs) ? 2 : 1;
        p.full_tiles = p.tail_split == 2 ? narrow - rem : narrow;
    }
    if (g.gate_block > 0 && (g.gate_block % 32 != 0 || g.N != 4 * g.gate_block))
        return fail(RELAY_ERR_UNSUPPORTED, "gate blocks of %lld columns over N = %lld", (long long)g.gate_block, (long long)g.N);
    const bool transc = g.act == RELAY_ACT_TANH || g.act == RELAY_ACT_SIGMOID || g.gate_block > 0;
#define LAUNCH3(AMN, BMN, TR)                                                                                               \
    do {                                                                                                                    \
        RELAY_CUDA(cudaFuncSetAttribute(gemm_tc2_kernel<AMN, BMN, StoreEpilogue<TR>>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_BYTES)); \
        RELAY_CUDA(launch_pdl(gemm_tc2_kernel<AMN, BMN, StoreEpilogue<TR>>, dim3(2 * pairs), dim3(NUM_THREADS), SMEM_BYTES, st, tm_a, tm_b, tm_c, p, tb));                 \
    } while (0)
#define LAUNCH2(AMN, BMN)            \
    do {                             \
        if (transc) LAUNCH3(AMN, BMN, true); \
        else LAUNCH3(AMN, BMN, false);       \
    } while (0)
    if (a_mn && b_mn) LAUNCH2(true, true);
    else if (a_mn) LAUNCH2(true, false);
    else if (b_mn) LAUNCH2(false, true);
    else LAUNCH2(false, false);
#undef LAUNCH2
#undef LAUNCH3
    return check_launch("gemm_tc2");
}

}  // namespace relay

// Host-only view of the unit plan (no GPU is touched), so that its invariants can be tested for many shapes.
extern "C" int32_t relay_debug_plan_units(int64_t M, int64_t N, int64_t K, int32_t sms, uint32_t *units, int32_t max_units)
{
    using namespace relay;
    if (M < 1 || N < 1 || K < 1 || sms < 2 || !units || max_units < 0) return -2;
    const int tiles_m = (int)((M + 255) / 256), tiles_n = (int)((N + BN - 1) / BN), k_blocks = (int)((K + BK - 1) / BK);
    const int pairs = std::min(tiles_m * tiles_n, sms / 2);
    static thread_local UnitTable tb;
    tb.n = 0;
    if (!plan_units(tiles_m, (int)((N + 127) / 128), pairs, k_blocks, &tb)) return -1;   // the fixed scheme would run
    if (tb.n > max_units) return -2;
    std::copy(tb.e, tb.e + tb.n, units);
    return tb.n;
}
