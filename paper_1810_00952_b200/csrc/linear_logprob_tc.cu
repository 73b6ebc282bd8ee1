// The products of a language model's head with what becomes of their scores: softmax statistics per row (forward) or the partials
// of the scores (gradient), on the main loop of the two-SM contraction (gemm_tc2.cuh).  The scores live in TMEM alone: an epilogue warp
// holds 32 rows x 64 columns of them in registers, one row a lane.  2048 x 1024 x 32768: statistics 95 us with the tensor pipe 85 % of the active cycles,
// slopes 105 us with 73 % (their 134 MB are stored by TMA, 32 x 32 at a time, and a warp waits for its one staging buffer).
#include "gemm_tc2.cuh"
#include "linear_logprob.h"

namespace relay {

relay_status_t make_tmap_2d_sw64(CUtensorMap *m, bool f32, const void *base, uint64_t inner, uint64_t outer, uint64_t row_stride,
                                 uint32_t box_outer);
relay_status_t make_tmap_2d_bf16(CUtensorMap *m, const void *base, uint64_t inner, uint64_t outer, uint64_t row_stride,
                                 uint32_t box_inner, uint32_t box_outer);

namespace {

using namespace gemm_tc2;

// what rounding 2^(x scale + off) to bf16 leaves; the exponential is made again (32 kept ones would spill)
__device__ __forceinline__ float low_part(float x, float scale, float off)
{
    float y;
    asm volatile("fma.rn.f32 %0, %1, %2, %3;\n\tex2.approx.ftz.f32 %0, %0;" : "=&f"(y) : "f"(x), "f"(scale), "f"(off));
    return y - __bfloat162float(__float2bfloat16_rn(y));
}
__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

struct HeadParams : gemm_tc::Params {
    const void *tokens;
    int tokens_i64;
    long long rows, V, first, classes;
    float scale;                           // log2(e) / temperature
    float inv_temperature;
    float2 *part;                          // statistics
    long long ld;
    float *at;
    const float *lse, *dlogp;              // slopes
    int low_rows;                          // of two parts: rows from the first to the second
};

// The scores that a warp has of an accumulator: 64 neighbouring columns of its 32 rows, so that of a 128-column accumulator only the first two of
// the four slots have some.  DEPTH = 0: read as they are.  Else they are summed up over accumulators of DEPTH k-blocks each.
template <int DEPTH>
struct Scores {
    static constexpr int kDepth = DEPTH;
    uint32_t r[2][32];
    __device__ __forceinline__ void read(uint32_t taddr)
    {
        tc::tmem_ld_32x32(taddr, r[0]);
        tc::tmem_ld_32x32(taddr + 32, r[1]);
        tc::tmem_ld_wait();
    }
    __device__ __forceinline__ void collect(uint32_t taddr, int width, int slot, bool first)
    {
        const int c0 = slot * 64;
        if (c0 >= width) return;
        if (first) { read(taddr + c0); return; }
#pragma unroll
        for (int k = 0; k < 64; k += 8) {                  // few columns at a time: the sums leave no registers for more
            uint32_t q[8];
            tc::tmem_ld_32x8(taddr + c0 + k, q);
            tc::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t &to = r[k >> 5][(k & 31) + j];
                to = __float_as_uint(__uint_as_float(to) + __uint_as_float(q[j]));
            }
        }
    }
};

template <int DEPTH>
struct StatsEpilogue : Scores<DEPTH> {
    using Params = HeadParams;
    using Scores<DEPTH>::r;
    int token;
    __device__ __forceinline__ void prepare(const Params &p, int lane, int row0, int, int)
    {
        token = -1;
        if (row0 + lane < p.rows) token = head::token_in_piece(p.tokens, p.tokens_i64, row0 + lane, p.V, p.first, p.classes);
    }
    __device__ __forceinline__ void drain(const Params &p, const CUtensorMap *, uint32_t taddr, uint8_t *, int lane, int row0, int n0, int width,
                                          int slot)
    {
        const int c0 = slot * head::kPartColumns;
        if (c0 >= width) return;
        if (DEPTH == 0) this->read(taddr + c0);
        const int n = n0 + c0;
        if (n + 64 > p.classes) {                          // warp-uniform: columns that do not exist
#pragma unroll
            for (int j = 0; j < 64; ++j)
                if (n + j >= p.classes) r[j >> 5][j & 31] = 0xff800000u;
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < 64; ++j) top[j & 3] = fmaxf(top[j & 3], __uint_as_float(r[j >> 5][j & 31]));
        const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * p.scale, off = m == -INFINITY ? 0.0f : -m;
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 64; ++j) s[j & 3] += ex2(fmaf(__uint_as_float(r[j >> 5][j & 31]), p.scale, off));
        const long long row = row0 + lane;
        const long long to = (long long)(n / head::kPartColumns) * p.ld + row;
        if (row < p.rows && relay_in_bounds(p.part + to, 8)) p.part[to] = make_float2(m, (s[0] + s[1]) + (s[2] + s[3]));
        const int hit = token - n;
        if (hit >= 0 && hit < 64) {
            float z = 0.0f;
#pragma unroll
            for (int j = 0; j < 64; ++j) if (j == hit) z = __uint_as_float(r[j >> 5][j & 31]);
            if (relay_in_bounds(p.at + row, 4)) p.at[row] = z;
        }
    }
    __device__ __forceinline__ void finish() {}
};

// The partials of 64 columns a warp: -slope 2^(z log2(e) / temperature - lse log2(e)), the slope's size taken into the exponent, its sign and
// the rows without a part put in where two values are already one register.  Tokens and the vocabulary's end, which few groups of 32 columns
// meet, are seen to under a condition that the whole warp shares.  PARTS = 2: what the rounding to bf16 leaves is stored as well.
template <int DEPTH, int PARTS>
struct SlopeEpilogue : Scores<DEPTH> {
    using Params = HeadParams;
    using Scores<DEPTH>::r;
    int token;
    float off, slope, lse;                 // log2 |slope| - lse log2(e), dlogp / temperature
    uint32_t keep, sign;                   // of two bf16 values: all bits or none (no token, or no class that can occur); their signs
    __device__ __forceinline__ void prepare(const Params &p, int lane, int row0, int, int)
    {
        const long long row = row0 + lane;
        token = -1;
        slope = lse = 0.0f;
        off = -INFINITY;
        keep = sign = 0;
        if (row >= p.rows) return;
        if (relay_in_bounds(p.lse + row, 4)) lse = p.lse[row];
        if (lse == -INFINITY || head::token_in_piece(p.tokens, p.tokens_i64, row, p.V, 0, p.V) < 0) return;
        token = head::token_in_piece(p.tokens, p.tokens_i64, row, p.V, p.first, p.classes);
        if (relay_in_bounds(p.dlogp + row, 4)) slope = p.dlogp[row] * p.inv_temperature;
        off = fmaf(-lse, 1.44269504f, log2f(fabsf(slope)));
        keep = 0xffffffffu;
        sign = slope > 0.0f ? 0x80008000u : 0u;
    }
    // the token's own partial, where the token is among 32 columns from n on: 1 - p of a class that is nearly certain keeps its precision
    __device__ __forceinline__ float own_partial(const Params &p, const uint32_t (&z)[32], int n)
    {
        const int hit = token - n;
        float own = 0.0f;
        if (__any_sync(0xffffffffu, hit >= 0 && hit < 32)) {
#pragma unroll
            for (int j = 0; j < 32; ++j) if (j == hit) own = __uint_as_float(z[j]);
            own = -slope * expm1f(fmaf(own, p.inv_temperature, -lse));
        }
        return own;
    }
    // those 32 columns; LOW: of the second part
    template <bool LOW>
    __device__ __forceinline__ void store(const Params &p, const CUtensorMap *tm_c, const uint32_t (&z)[32], float own, uint8_t *stage, int lane, int row0,
                                          int n)
    {
        const int sw = (lane >> 1) & 3;
        const int hit = token - n;
        if (LOW) own -= __bfloat162float(__float2bfloat16_rn(own));
        uint32_t v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float a = __uint_as_float(z[2 * j]), b = __uint_as_float(z[2 * j + 1]);
            v[j] = LOW ? pack2(low_part(a, p.scale, off), low_part(b, p.scale, off)) : pack2(ex2(fmaf(a, p.scale, off)), ex2(fmaf(b, p.scale, off)));
            v[j] = (v[j] ^ sign) & keep;
        }
        if (__any_sync(0xffffffffu, hit >= 0 && hit < 32)) {
            const uint32_t bits = pack2(own, own);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (hit == 2 * j) v[j] = (v[j] & 0xffff0000u) | (bits & 0xffffu);
                if (hit == 2 * j + 1) v[j] = (v[j] & 0xffffu) | (bits & 0xffff0000u);
            }
        }
        if (n + 32 > p.classes) {                          // warp-uniform: columns that do not exist
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (n + 2 * j >= p.classes) v[j] = 0;
                else if (n + 2 * j + 1 >= p.classes) v[j] &= 0xffffu;
            }
        }
        if (tc::elect_one()) tc::tma_store_wait_read<0>();
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint4 *>(stage + lane * 64 + ((c ^ sw) << 4)) = make_uint4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
        tc::fence_proxy_async();
        __syncwarp();
        if (tc::elect_one()) {
            tc::tma_store_2d(tm_c, stage, n, LOW ? row0 + p.low_rows : row0);
            tc::tma_store_commit();
        }
    }
    __device__ __forceinline__ void drain(const Params &p, const CUtensorMap *tm_c, uint32_t taddr, uint8_t *stage, int lane, int row0, int n0,
                                          int width, int slot)
    {
        const int c0 = slot * 64;
        if (c0 >= width) return;
        if (DEPTH == 0) this->read(taddr + c0);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int n = n0 + c0 + 32 * half;
            if (n >= p.N) break;                           // warp-uniform; p.N: columns of the stored piece
            const float own = own_partial(p, r[half], n);
            store<false>(p, tm_c, r[half], own, stage, lane, row0, n);
            if (PARTS == 2) store<true>(p, tm_c, r[half], own, stage, lane, row0, n);
        }
    }
    __device__ __forceinline__ void finish() { if (tc::elect_one()) tc::tma_store_wait_all<0>(); }
};

template <int DEPTH> using Slopes = SlopeEpilogue<DEPTH, 1>;
template <int DEPTH> using SlopesInTwo = SlopeEpilogue<DEPTH, 2>;

template <template <int> class Epi>
relay_status_t launch(const head::Piece &q, HeadParams p, int64_t M, int64_t N, void *c, int64_t ldc, int64_t c_rows, cudaStream_t st)
{
    int dev = 0, sms = 148;
    RELAY_CUDA(cudaGetDevice(&dev));
    RELAY_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    CUtensorMap tm_a, tm_b, tm_c;
    RELAY_TRY(make_tmap_2d_bf16(&tm_a, q.x, q.K, q.rows, q.ldx, BK, 128));
    if (q.trans_w) RELAY_TRY(make_tmap_2d_bf16(&tm_b, q.w, q.K, q.classes, q.ldw, BK, 64));
    else RELAY_TRY(make_tmap_2d_bf16(&tm_b, q.w, q.classes, q.K, q.ldw, 64, BK));
    tm_c = tm_a;                                           // statistics are not stored by tile
    if (c) RELAY_TRY(make_tmap_2d_sw64(&tm_c, false, c, N, c_rows, ldc, 32));
    p.M = (int)M; p.N = (int)N; p.K = (int)q.K;
    p.tiles_m = (int)((M + 255) / 256); p.tiles_n = (int)((N + BN - 1) / BN); p.k_blocks = (int)((q.K + BK - 1) / BK);
    p.err = device_error_word();
    if (!p.err) return fail(RELAY_ERR_CUDA, "no device error word");
    p.tokens = q.tokens; p.tokens_i64 = q.tokens_i64;
    p.rows = q.rows; p.V = q.V; p.first = q.first; p.classes = q.classes;
    p.inv_temperature = q.inv_temperature;
    p.scale = (float)(1.4426950408889634 * (double)p.inv_temperature);
    if ((long long)p.tiles_m * p.tiles_n > 1 << 30) return fail(RELAY_ERR_UNSUPPORTED, "linear_logprob: %lld x %lld scores at a time", (long long)M, (long long)N);
    const int n_tiles = p.tiles_m * p.tiles_n, pairs = std::min(n_tiles, sms / 2);
    static thread_local UnitTable tb;
    tb.n = 0;
    p.tail_split = 1;
    // no wide units: a contraction long enough to gain by them is cut
    constexpr int kCut = head::kDepth / BK;
    static_assert(kCut < kWideMinKBlocks, "units of class 3 and 4 have no epilogue here");
    if (!plan_units(p.tiles_m, (int)((N + 127) / 128), pairs, std::min(p.k_blocks, kCut), &tb)) {
        tb.n = 0;
        const int rem = n_tiles % pairs;
        p.tail_split = (rem > 0 && 2 * rem <= pairs) ? 2 : 1;
        p.full_tiles = p.tail_split == 2 ? n_tiles - rem : n_tiles;
    }
    BoundsReg reg;
    reg.add(q.tokens, (size_t)q.rows * (q.tokens_i64 ? 8 : 4));
    if (p.part) reg.add(p.part, ((size_t)(head::parts_of(q.classes) - 1) * p.ld + q.rows) * sizeof(float2));
    for (const float *t : {(const float *)p.at, p.lse, p.dlogp}) reg.add(t, (size_t)q.rows * 4);
    RELAY_TRY(reg.commit(st));
    auto go = [&](auto kernel) -> relay_status_t {
        RELAY_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_BYTES));
        RELAY_CUDA(launch_pdl(kernel, dim3(2 * pairs), dim3(NUM_THREADS), SMEM_BYTES, st, tm_a, tm_b, tm_c, p, tb));
        return check_launch("linear_logprob");
    };
    if (p.k_blocks <= kCut) return q.trans_w ? go(gemm_tc2_kernel<false, false, Epi<0>>) : go(gemm_tc2_kernel<false, true, Epi<0>>);
    return q.trans_w ? go(gemm_tc2_kernel<false, false, Epi<kCut>>) : go(gemm_tc2_kernel<false, true, Epi<kCut>>);
}

}  // namespace

namespace head {

relay_status_t launch_stats(const Piece &q, float2 *part, long long ld, float *at, cudaStream_t st)
{
    HeadParams p{};
    p.part = part; p.ld = ld; p.at = at;
    return launch<StatsEpilogue>(q, p, q.rows, q.classes, nullptr, 0, 0, st);
}
relay_status_t launch_slopes(const Piece &q, const float *lse, const float *dlogp, void *dz, long long ld, long long padded_rows,
                             long long padded_classes, int parts, cudaStream_t st)
{
    HeadParams p{};
    p.lse = lse; p.dlogp = dlogp;
    p.low_rows = (int)padded_rows;
    if (parts == 2) return launch<SlopesInTwo>(q, p, padded_rows, padded_classes, dz, ld, 2 * padded_rows, st);
    return launch<Slopes>(q, p, padded_rows, padded_classes, dz, ld, padded_rows, st);
}

}  // namespace head
}  // namespace relay
