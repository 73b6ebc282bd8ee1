// Log-probabilities of given tokens straight from the operands of a language model's head, and the gradient group: the N x V scores are
// made a piece of the vocabulary at a time and never kept.
//
// bf16: the forward call is one product whose epilogue leaves (maximum, sum of exponentials) per row and 64 columns, which a second
// kernel joins.  The gradient makes the partials dz of a piece of the scores (the same product with another epilogue), and multiplies
// them with w and x; the sum of dx over the pieces is kept in fp32.  TMA wants rows of whole 16 bytes: pieces of w that have others
// (odd vocabularies, odd widths) are copied to padded rows first, and dw of such a piece back.
// f32: the same pieces through the fp32 contraction, with the scores of a piece in the workspace.
//
// Measured, bf16: 8192 x 1024 x 32768 360 us (1.53 PFLOP/s) and 1.53 ms with the gradient in a short series, 424 us and 1.82 ms in a long one (power);
// 4096 x 2048 x 131072 tied with the gradient 6.2 to 6.4 and 6.8 ms; 509 x 1024 x 50021, rows of odd length, 102 to 107 us, 47 of them the copy of w.
// f32: 2048 x 1024 x 32768 5.0 ms, with the gradient 20.1.
#include <algorithm>
#include <cfloat>

#include "gemm.h"
#include "linear_logprob.h"
#include "sequence.cuh"

namespace relay {
namespace {

using head::Piece;

constexpr long long kPieceElements = 1ll << 27;            // scores (or copied weights) of a piece, at most: 256 MB in bf16

// ---- small kernels -----------------------------------------------------------------------------------------------
// Joins the partial statistics of a row: kJoin groups of them, each in its order.
constexpr int kJoin = 32;
__global__ void __launch_bounds__(32 * kJoin) join_stats_kernel(const float2 *part, long long ld, long long parts, const float *at, const void *tokens,
                                                                int tokens_i64, long long rows, long long V, float inv_temperature, float *logp,
                                                                float *lse)
{
    __shared__ float2 joint[kJoin][32];
    pdl_wait();
    const long long row = (long long)blockIdx.x * 32 + threadIdx.x;
    float m = -INFINITY, s = 0.0f;
    auto add = [&](const float2 &q) {
        const float top = fmaxf(m, q.x), off = top == -INFINITY ? 0.0f : top;
        s = s * exp2f(m - off) + q.y * exp2f(q.x - off);
        m = top;
    };
    constexpr int U = 8;                                   // on their way at once
    for (long long j = threadIdx.y; j < parts; j += kJoin * U) {
        float2 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float2 *from = part + (j + u * kJoin) * ld + row;
            q[u] = make_float2(-INFINITY, 0.0f);
            if (row < rows && j + u * kJoin < parts && relay_in_bounds(from, 8)) q[u] = __ldcs(from);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) add(q[u]);
    }
    joint[threadIdx.y][threadIdx.x] = make_float2(m, s);
    for (int n = kJoin / 2; n > 0; n /= 2) {
        __syncthreads();
        if (threadIdx.y >= n) continue;
        add(joint[threadIdx.y + n][threadIdx.x]);
        joint[threadIdx.y][threadIdx.x] = make_float2(m, s);
    }
    if (threadIdx.y != 0 || row >= rows) return;
    const float l = m == -INFINITY && s == 0.0f ? -INFINITY : fmaf(m, 0.693147181f, logf(s));
    float lp = 0.0f;
    if (head::token_in_piece(tokens, tokens_i64, row, V, 0, V) >= 0 && relay_in_bounds(at + row, 4))
        lp = l == -INFINITY ? l : fmaf(at[row], inv_temperature, -l);
    if (relay_in_bounds(logp + row, 4)) logp[row] = lp;
    if (relay_in_bounds(lse + row, 4)) lse[row] = l;
}

// 16 bytes from an address of any 2-byte alignment: the two aligned pieces that hold them, shifted
__device__ __forceinline__ uint4 load_shifted(const char *p)
{
    const unsigned skew = (unsigned)((uintptr_t)p & 15);
    const uint4 *q = (const uint4 *)(p - skew);
    if (skew == 0) return relay_in_bounds(q, 16) ? __ldg(q) : make_uint4(0, 0, 0, 0);
    if (!relay_in_bounds(p, 16)) return make_uint4(0, 0, 0, 0);
    const uint4 a = __ldg(q), b = __ldg(q + 1);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t v[5];
    const unsigned words = skew >> 2, bits = (skew & 3) * 8;
#pragma unroll
    for (int j = 0; j < 5; ++j) v[j] = words == 0 ? w[j] : words == 1 ? w[j + 1 < 8 ? j + 1 : 7] : words == 2 ? w[j + 2 < 8 ? j + 2 : 7] : w[j + 3 < 8 ? j + 3 : 7];
    return make_uint4(__funnelshift_r(v[0], v[1], bits), __funnelshift_r(v[1], v[2], bits), __funnelshift_r(v[2], v[3], bits),
                      __funnelshift_r(v[3], v[4], bits));
}
// Which rows have a part in a gradient: those whose token names a class and which have a class that can occur.
struct Rows {
    const void *tokens;                    // null: all of them
    int i64;
    long long V;
    const float *lse;
    __device__ __forceinline__ bool part(long long row) const
    {
        if (tokens == nullptr) return true;
        if (head::token_in_piece(tokens, i64, row, V, 0, V) < 0 || !relay_in_bounds(lse + row, 4)) return false;
        return lse[row] != -INFINITY;
    }
};
// to (to_rows, to_cols) <- from (rows, cols), zero beyond; rows without a part are zero too: whatever x holds there (infinities and NaN too) takes
// no part in dw.  A thread has the elements that share 16 aligned bytes of the result: one access each way
// unless the row's end or what must not be read lies in between.
template <typename T>
__global__ void __launch_bounds__(256) copy_padded_kernel(const T *from, long long ld_from, long long rows, long long cols, T *to, long long ld_to,
                                                          long long to_rows, long long to_cols, const Rows some)
{
    constexpr int E = 16 / sizeof(T);
    pdl_wait();
    for (long long r = blockIdx.y; r < to_rows; r += gridDim.y) {
        const bool live = r < rows && some.part(r);
        const T *src = from + r * ld_from;
        T *dst = to + r * ld_to;
        const int skew = (int)(((uintptr_t)dst & 15) / sizeof(T));
        // the last piece that may be read whole: an aligned 16-byte piece behind the tensor's end may not be there
        const long long safe = r + 1 < rows ? cols : cols - E;
        for (long long g = (long long)blockIdx.x * 256 + threadIdx.x; g * E < skew + to_cols; g += (long long)gridDim.x * 256) {
            const long long c = g * E - skew;
            if (c >= 0 && c + E <= to_cols && (!live || c + E <= safe || c >= cols)) {
                const uint4 v = live && c < cols ? load_shifted((const char *)(src + c)) : make_uint4(0, 0, 0, 0);
                if (relay_in_bounds(dst + c, 16)) *(uint4 *)(dst + c) = v;
                continue;
            }
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (c + j >= 0 && c + j < to_cols) {
                    const T x = live && c + j < cols && relay_in_bounds(src + c + j, sizeof(T)) ? src[c + j] : T(0.0f);
                    if (relay_in_bounds(dst + c + j, sizeof(T))) dst[c + j] = x;
                }
        }
    }
}
// out (rows, cols) <- a + b, both fp32 with rows of `ld` values, whole 16-byte pieces (b may be null), rounded once; rows without a part are zero
// (their sums are, unless a weight is infinite)
template <typename T>
__global__ void __launch_bounds__(256) add_kernel(const float *a, const float *b, long long ld, T *out, long long ld_out, long long rows,
                                                  long long cols, const Rows some)
{
    pdl_wait();
    const bool whole = ld % 4 == 0 && ld_out % 4 == 0;
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        const bool part = some.part(r);
        for (long long c = ((long long)blockIdx.x * 256 + threadIdx.x) * 4; c < cols; c += (long long)gridDim.x * 1024) {
            const long long at = r * ld + c;
            T *q = out + r * ld_out + c;
            float x[4] = {0.0f, 0.0f, 0.0f, 0.0f}, y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (whole && c + 4 <= cols) {
                if (part) seq::load<float, 4>(a, at, x);
                if (part && b != nullptr) seq::load<float, 4>(b, at, y);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] += y[j];
                seq::store<T, 4>(q, 0, x);
                continue;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c + j >= cols || !relay_in_bounds(a + at + j, 4)) continue;
                const float one[1] = {part ? a[at + j] + (b != nullptr && relay_in_bounds(b + at + j, 4) ? b[at + j] : 0.0f) : 0.0f};
                seq::store<T, 1>(q, j, one);
            }
        }
    }
}
// f32, whose products write dx themselves: zeros in the rows without a part
__global__ void __launch_bounds__(256) clear_rows_kernel(float *dx, long long rows, long long cols, const Rows some)
{
    pdl_wait();
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        if (some.part(r)) continue;
        for (long long c = (long long)blockIdx.x * 256 + threadIdx.x; c < cols; c += (long long)gridDim.x * 256)
            if (relay_in_bounds(dx + r * cols + c, 4)) dx[r * cols + c] = 0.0f;
    }
}

// f32: statistics of a piece of scores in memory, one block a row (base 2, as the other path's)
__global__ void __launch_bounds__(256) stats_kernel(const float *z, long long ld, const Piece p, float scale, float2 *part, float *at)
{
    __shared__ float2 joint[256];
    pdl_wait();
    const long long row = blockIdx.x;
    const float *zr = z + row * ld;
    float m = -INFINITY, s = 0.0f;
    auto add = [&](float qm, float qs) {
        const float top = fmaxf(m, qm), off = top == -INFINITY ? 0.0f : top;
        s = s * exp2f(m - off) + qs * exp2f(qm - off);
        m = top;
    };
    for (long long j = threadIdx.x; j < p.classes; j += 256) {
        const float v = relay_in_bounds(zr + j, 4) ? zr[j] * scale : 0.0f;
        if (v == -INFINITY) continue;
        add(v, v != v ? v : 1.0f);
    }
    joint[threadIdx.x] = make_float2(m, s);
    __syncthreads();
    for (int n = 128; n > 0; n >>= 1) {
        if (threadIdx.x < n) {
            m = joint[threadIdx.x].x; s = joint[threadIdx.x].y;
            add(joint[threadIdx.x + n].x, joint[threadIdx.x + n].y);
            joint[threadIdx.x] = make_float2(m, s);
        }
        __syncthreads();
    }
    if (threadIdx.x != 0) return;
    if (relay_in_bounds(part + row, 8)) part[row] = make_float2(m, s);
    const int t = head::token_in_piece(p.tokens, p.tokens_i64, row, p.V, p.first, p.classes);
    if (t >= 0 && relay_in_bounds(zr + t, 4) && relay_in_bounds(at + row, 4)) at[row] = zr[t];
}
// f32: dz of a piece, over its scores
__global__ void __launch_bounds__(256) slopes_kernel(float *z, long long ld, const Piece p, const float *lse, const float *dlogp)
{
    pdl_wait();
    for (long long row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const int t = head::token_in_piece(p.tokens, p.tokens_i64, row, p.V, p.first, p.classes);
        const float l = relay_in_bounds(lse + row, 4) ? lse[row] : 0.0f;
        const bool nothing = l == -INFINITY || head::token_in_piece(p.tokens, p.tokens_i64, row, p.V, 0, p.V) < 0;
        const float slope = nothing || !relay_in_bounds(dlogp + row, 4) ? 0.0f : dlogp[row] * p.inv_temperature;
        for (long long j = (long long)blockIdx.x * 256 + threadIdx.x; j < p.classes; j += (long long)gridDim.x * 256) {
            float *q = z + row * ld + j;
            if (!relay_in_bounds(q, 4)) continue;
            const float lp = fmaf(*q, p.inv_temperature, -l);
            *q = nothing ? 0.0f : -slope * (j == t ? expm1f(lp) : expf(lp));
        }
    }
}

dim3 grid_of(long long rows, long long cols)               // cols: threads along a row
{
    return dim3((unsigned)std::min<long long>(std::max<long long>(1, (cols + 255) / 256), 64), (unsigned)std::min<long long>(std::max<long long>(1, rows), 16384));
}
template <typename T>
relay_status_t copy_padded(const void *from, long long ld_from, long long rows, long long cols, void *to, long long ld_to, long long to_rows,
                           long long to_cols, const Rows &some, cudaStream_t st)
{
    RELAY_CUDA(launch_pdl(copy_padded_kernel<T>, grid_of(to_rows, (to_cols * sizeof(T) + 31) / 16), dim3(256), 0, st, (const T *)from, ld_from, rows, cols, (T *)to, ld_to,
                          to_rows, to_cols, some));
    return check_launch("linear_logprob");
}
template <typename T>
relay_status_t add(const float *a, const float *b, long long ld, void *out, long long ld_out, long long rows, long long cols, const Rows &some,
                   cudaStream_t st)
{
    RELAY_CUDA(launch_pdl(add_kernel<T>, grid_of(rows, (cols + 3) / 4), dim3(256), 0, st, a, b, ld, (T *)out, ld_out, rows, cols, some));
    return check_launch("linear_logprob");
}

// ---- sizes and the workspace --------------------------------------------------------------------------------------
struct Sizes { int64_t rows, K, V; int rank; };            // rank of the row vectors

int64_t padded(int64_t n) { return std::max<int64_t>(64, (n + 7) / 8 * 8); }
// classes of a piece, whole tiles of 256: pieces of nearly the same size
int64_t piece_of(int64_t V, int64_t other)
{
    const int64_t most = std::max<int64_t>(256, kPieceElements / std::max<int64_t>(1, other) / 256 * 256), n = (V + most - 1) / most;
    return std::min<int64_t>((V + 255) / 256 * 256, ((V + n - 1) / n + 255) / 256 * 256);
}
bool rows_fit(const Sizes &s, bool trans_w) { return (trans_w ? s.K : s.V) % 8 == 0; }                // rows of w are whole 16 bytes

// The forward call takes as many rows at a time as have a quarter of a gigabyte of partial statistics, whole tiles of 256; in fp32 as many as
// have a whole piece of scores.
int64_t slab_of(const Sizes &s, bool bf16)
{
    if (!bf16) return std::min<int64_t>(s.rows, kPieceElements / 256);
    const int64_t per_row = head::parts_of(s.V) * (int64_t)sizeof(float2);
    return std::min<int64_t>(s.rows, std::max<int64_t>(256, (1ll << 28) / per_row / 256 * 256));
}

struct Layout {
    int64_t piece, pieces;                 // classes of a piece
    int64_t N, K, C;                       // padded rows, width and classes of a piece (bf16)
    int parts;                             // of the partials of the scores (bf16)
    bool copy_x, copy_w;
    size_t part, at, x, w, z, dx, dx_more, dw, bytes;
};
Layout forward_layout(const Sizes &s, bool trans_w, bool bf16)
{
    Layout q{};
    q.copy_x = bf16 && s.K % 8 != 0;
    q.copy_w = bf16 && !rows_fit(s, trans_w);
    q.K = padded(s.K); q.N = s.rows;
    q.piece = !bf16 ? piece_of(s.V, s.rows) : q.copy_w ? piece_of(s.V, q.K) : s.V;
    q.pieces = (s.V + q.piece - 1) / q.piece;
    q.C = padded(q.piece);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, 256); return here; };
    q.part = take((size_t)(bf16 ? head::parts_of(q.piece) : 1) * q.pieces * s.rows * sizeof(float2));
    q.at = take((size_t)s.rows * 4);
    q.x = take(q.copy_x ? (size_t)s.rows * q.K * 2 : 0);
    q.w = take(q.copy_w ? (size_t)q.K * q.C * 2 : 0);
    q.z = take(bf16 ? 0 : (size_t)s.rows * q.piece * 4);
    q.bytes = at;
    return q;
}
// The partials of the scores are operands of the products and so rounded to bf16.  A row's error is mostly that of its token's own partial, a factor
// that all of its part in dx and dw has in common, and over few rows such errors do not average out: dx and dw are 1.9 times as far from 64 bits as
// the rounding of the results alone leaves them with one row, 1.66 with nine, 1.5 with 128 or 300, 1.44 from 500 rows on, at the worst of six seeds.  So up
// to 512 rows, whose products wait for their other operand anyway, the partials come in two bf16 numbers, one below the other in a contraction
// twice as long (1.00).  (The slopes on dx's fp32 sums and on x instead: 1.15 in dx, but 1.53 in dw, and the products of x with a slope near a power
// of two round alike.)  1024 x 32768: 1 row 220 -> 232 us, 128 rows 222 -> 242, 512 rows 255 -> 291; 2048 x 131072 tied: 64 rows 0.98 -> 1.04 ms, 512
// rows 1.18 -> 1.49; at 8192 rows they would cost half as much again.
constexpr int64_t kTwoPartRows = 512;
Layout gradient_layout(const Sizes &s, bool trans_w, bool bf16)
{
    Layout q{};
    q.parts = bf16 && s.rows <= kTwoPartRows ? 2 : 1;
    q.N = !bf16 ? s.rows : q.parts == 2 ? std::max<int64_t>(64, (s.rows + 31) / 32 * 32) : padded(s.rows); q.K = bf16 ? padded(s.K) : s.K;
    q.piece = piece_of(s.V, std::max(q.N * q.parts, q.K));
    q.pieces = (s.V + q.piece - 1) / q.piece;
    q.C = bf16 ? padded(q.piece) : q.piece;
    q.copy_x = true;                                       // masked
    const int64_t last = s.V - (q.pieces - 1) * q.piece;   // the pieces before it are whole tiles
    q.copy_w = bf16 && (!rows_fit(s, trans_w) || padded(last) != last || q.K != s.K);                     // some piece is copied
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, 256); return here; };
    const size_t rows = (size_t)q.N * q.parts;
    q.x = take(rows * q.K * (bf16 ? 2 : 4));
    q.z = take(rows * q.C * (bf16 ? 2 : 4));
    q.dx = take(bf16 ? rows * q.K * 4 : 0);
    q.dx_more = take(q.pieces > 1 ? rows * q.K * 4 : 0);
    q.w = take(q.copy_w ? (size_t)q.K * q.C * 2 : 0);
    q.dw = take(q.copy_w ? (size_t)q.K * q.C * 2 : 0);
    q.bytes = at;
    return q;
}

// ---- the calls --------------------------------------------------------------------------------------------------------
GemmDesc product(int64_t M, int64_t N, int64_t K, const void *a, int64_t a_sm, int64_t a_sk, const void *b, int64_t b_sk, int64_t b_sn, void *c,
                 int64_t ldc, int32_t in, int32_t out)
{
    GemmDesc g;
    g.M = M; g.N = N; g.K = K;
    g.a = a; g.a_sm = a_sm; g.a_sk = a_sk;
    g.b = b; g.b_sk = b_sk; g.b_sn = b_sn;
    g.c = c; g.ldc = ldc;
    g.in_dtype = in; g.out_dtype = out;
    return g;
}

// the piece of w that starts at class `first`: as it is, or copied to padded rows
relay_status_t weights_of(Piece *p, const Sizes &s, const char *w, const Layout &q, char *ws, bool copy, cudaStream_t st)
{
    p->w = w + (p->trans_w ? p->first * s.K : p->first) * 2;
    p->ldw = p->trans_w ? s.K : s.V;
    if (!copy) return RELAY_OK;
    const int64_t rows = p->trans_w ? p->classes : s.K, cols = p->trans_w ? s.K : p->classes;
    const int64_t to_rows = p->trans_w ? padded(p->classes) : q.K, to_cols = p->trans_w ? q.K : padded(p->classes);
    RELAY_TRY(copy_padded<__nv_bfloat16>(p->w, p->ldw, rows, cols, ws + q.w, to_cols, to_rows, to_cols, Rows{}, st));
    p->w = ws + q.w;
    p->ldw = to_cols;
    return RELAY_OK;
}

relay_status_t run_forward(Piece p, const Sizes &s, const void *w, bool bf16, float *logp, float *lse, char *ws, cudaStream_t st)
{
    const Layout q = forward_layout(s, p.trans_w, bf16);
    float2 *part = (float2 *)(ws + q.part);
    float *at = (float *)(ws + q.at);
    const float scale = (float)(1.4426950408889634 * (double)p.inv_temperature);
    const long long per_piece = bf16 ? head::parts_of(q.piece) : 1;
    long long parts = 0;
    if (q.copy_x) {
        RELAY_TRY(copy_padded<__nv_bfloat16>(p.x, s.K, s.rows, s.K, ws + q.x, q.K, s.rows, q.K, Rows{}, st));
        p.x = ws + q.x;
        p.ldx = q.K;
    }
    for (p.first = 0; p.first < s.V; p.first += q.piece) {
        p.classes = std::min<int64_t>(q.piece, s.V - p.first);
        if (bf16) {
            RELAY_TRY(weights_of(&p, s, (const char *)w, q, ws, q.copy_w, st));
            RELAY_TRY(head::launch_stats(p, part + p.first / q.piece * per_piece * s.rows, s.rows, at, st));
            parts += (p.classes + 127) / 128 * 2;
        } else {
            const float *b = (const float *)w + (p.trans_w ? p.first * s.K : p.first);
            RELAY_TRY(launch_gemm(product(s.rows, p.classes, s.K, p.x, s.K, 1, b, p.trans_w ? 1 : s.V, p.trans_w ? s.K : 1, ws + q.z, q.piece,
                                          RELAY_F32, RELAY_F32), st));
            RELAY_CUDA(launch_pdl(stats_kernel, dim3((unsigned)s.rows), dim3(256), 0, st, (const float *)(ws + q.z), (long long)q.piece, p, scale,
                                  part + p.first / q.piece * s.rows, at));
            RELAY_TRY(check_launch("linear_logprob"));
            parts += 1;
        }
    }
    RELAY_CUDA(launch_pdl(join_stats_kernel, dim3((unsigned)((s.rows + 31) / 32)), dim3(32, kJoin), 0, st, (const float2 *)part, (long long)s.rows, parts,
                          (const float *)at, p.tokens, p.tokens_i64, (long long)s.rows, (long long)s.V,
                          p.inv_temperature, logp, lse));
    return check_launch("linear_logprob");
}

relay_status_t run_gradient_f32(Piece p, const Sizes &s, const float *w, const float *lse, const float *dlogp, float *dx, float *dw, char *ws,
                                cudaStream_t st)
{
    const Layout q = gradient_layout(s, p.trans_w, false);
    float *x = (float *)(ws + q.x), *z = (float *)(ws + q.z), *more = (float *)(ws + q.dx_more);
    const Rows some{p.tokens, p.tokens_i64, p.V, lse};
    RELAY_TRY(copy_padded<float>(p.x, s.K, s.rows, s.K, x, s.K, s.rows, s.K, some, st));
    for (p.first = 0; p.first < s.V; p.first += q.piece) {
        p.classes = std::min<int64_t>(q.piece, s.V - p.first);
        const int64_t at = p.trans_w ? p.first * s.K : p.first, w_k = p.trans_w ? 1 : s.V, w_v = p.trans_w ? s.K : 1;
        RELAY_TRY(launch_gemm(product(s.rows, p.classes, s.K, x, s.K, 1, w + at, w_k, w_v, z, q.piece, RELAY_F32, RELAY_F32), st));
        RELAY_CUDA(launch_pdl(slopes_kernel, grid_of(s.rows, p.classes), dim3(256), 0, st, z, (long long)q.piece, p, lse, dlogp));
        RELAY_TRY(check_launch("linear_logprob_grad"));
        if (dx) {
            float *to = p.first == 0 ? dx : more;
            RELAY_TRY(launch_gemm(product(s.rows, s.K, p.classes, z, q.piece, 1, w + at, w_v, w_k, to, s.K, RELAY_F32, RELAY_F32), st));
            if (to == more) RELAY_TRY(add<float>(dx, more, s.K, dx, s.K, s.rows, s.K, Rows{}, st));
        }
        if (!dw) continue;
        if (p.trans_w) RELAY_TRY(launch_gemm(product(p.classes, s.K, s.rows, z, 1, q.piece, x, s.K, 1, dw + at, s.K, RELAY_F32, RELAY_F32), st));
        else RELAY_TRY(launch_gemm(product(s.K, p.classes, s.rows, x, 1, s.K, z, q.piece, 1, dw + at, s.V, RELAY_F32, RELAY_F32), st));
    }
    if (!dx) return RELAY_OK;
    RELAY_CUDA(launch_pdl(clear_rows_kernel, grid_of(s.rows, s.K), dim3(256), 0, st, dx, (long long)s.rows, (long long)s.K, some));
    return check_launch("linear_logprob_grad");
}

relay_status_t run_gradient_bf16(Piece p, const Sizes &s, const void *w, const float *lse, const float *dlogp, __nv_bfloat16 *dx, __nv_bfloat16 *dw,
                                 char *ws, cudaStream_t st)
{
    const Layout q = gradient_layout(s, p.trans_w, true);
    void *x = ws + q.x, *z = ws + q.z;
    float *sum = (float *)(ws + q.dx), *more = (float *)(ws + q.dx_more);
    const Rows some{p.tokens, p.tokens_i64, p.V, lse};
    for (int part = q.parts - 1; part >= 0; --part)
        RELAY_TRY(copy_padded<__nv_bfloat16>(p.x, s.K, s.rows, s.K, (char *)x + part * q.N * q.K * 2, q.K, q.N, q.K, some, st));
    const int64_t N = q.N * q.parts;                       // rows of the products
    float *low = q.parts == 2 ? sum + q.N * q.K : nullptr;
    p.x = x;
    p.ldx = q.K;
    for (p.first = 0; p.first < s.V; p.first += q.piece) {
        p.classes = std::min<int64_t>(q.piece, s.V - p.first);
        const int64_t C = padded(p.classes), at = p.trans_w ? p.first * s.K : p.first;
        const bool copy = !rows_fit(s, p.trans_w) || C != p.classes || q.K != s.K;
        RELAY_TRY(weights_of(&p, s, (const char *)w, q, ws, copy, st));
        RELAY_TRY(head::launch_slopes(p, lse, dlogp, z, C, q.N, C, q.parts, st));
        const int64_t w_k = p.trans_w ? 1 : p.ldw, w_v = p.trans_w ? p.ldw : 1;
        if (dx) {
            float *to = p.first == 0 ? sum : more;
            RELAY_TRY(launch_gemm(product(N, q.K, C, z, C, 1, p.w, w_v, w_k, to, q.K, RELAY_BF16, RELAY_F32), st));
            const bool last = p.first + q.piece >= s.V;
            const float *b = to == more ? more : nullptr;
            if (b && (low || !last)) {
                RELAY_TRY(add<float>(sum, b, q.K, sum, q.K, N, q.K, Rows{}, st));
                b = nullptr;
            }
            if (last) RELAY_TRY(add<__nv_bfloat16>(sum, low ? low : b, q.K, dx, s.K, s.rows, s.K, some, st));
        }
        if (!dw) continue;
        void *to = copy ? (void *)(ws + q.dw) : (void *)(dw + at);
        const int64_t ld = copy ? (p.trans_w ? q.K : C) : p.ldw;
        if (p.trans_w) RELAY_TRY(launch_gemm(product(C, q.K, N, z, 1, C, x, q.K, 1, to, ld, RELAY_BF16, RELAY_BF16), st));
        else RELAY_TRY(launch_gemm(product(q.K, C, N, x, 1, q.K, z, C, 1, to, ld, RELAY_BF16, RELAY_BF16), st));
        if (copy) {
            const int64_t rows = p.trans_w ? p.classes : s.K, cols = p.trans_w ? s.K : p.classes;
            RELAY_TRY(copy_padded<__nv_bfloat16>(to, ld, rows, cols, dw + at, p.trans_w ? s.K : s.V, rows, cols, Rows{}, st));
        }
    }
    return RELAY_OK;
}

// ---- boundary -----------------------------------------------------------------------------------------------------------
relay_status_t check_operands(const relay_tensor_t *x, const relay_tensor_t *w, int32_t trans_w, Sizes *s)
{
    RELAY_TRY(check_type(x, "x"));
    RELAY_TRY(check_type(w, "w"));
    if (x->rank < 1) return fail(RELAY_ERR_RANK, "x: rank 0, a row is needed");
    RELAY_TRY(check_rank(w, 2, "w"));
    if (!is_float(x->dtype)) return fail(RELAY_ERR_DTYPE, "x: base type %s, needs f32 or bf16", dtype_name(x->dtype));
    RELAY_TRY(check_dtype(w, x->dtype, "w"));
    RELAY_TRY(check_layout(x, RELAY_ROWMAJOR, RELAY_ROWMAJOR, "x"));
    RELAY_TRY(check_layout(w, RELAY_ROWMAJOR, RELAY_ROWMAJOR, "w"));
    s->rank = x->rank - 1;
    s->K = x->shape[s->rank];
    s->rows = 1;
    for (int d = 0; d < s->rank; ++d) s->rows *= x->shape[d];
    s->V = w->shape[trans_w ? 0 : 1];
    if (w->shape[trans_w ? 1 : 0] != s->K)
        return fail(RELAY_ERR_SHAPE, "w: contraction extent %lld, x has %lld", (long long)w->shape[trans_w ? 1 : 0], (long long)s->K);
    if (s->V == 0) return fail(RELAY_ERR_SHAPE, "w: a row without classes has no softmax");
    if (s->K == 0) return fail(RELAY_ERR_SHAPE, "x: a contraction over nothing");
    if (s->V > INT32_MAX - 512) return fail(RELAY_ERR_SHAPE, "w: %lld classes do not fit an i32", (long long)s->V);
    if (s->K > (1 << 20) || s->rows > (1 << 28)) return fail(RELAY_ERR_UNSUPPORTED, "x: %lld rows of %lld", (long long)s->rows, (long long)s->K);
    return RELAY_OK;
}
relay_status_t check_rows(const relay_tensor_t *t, const relay_tensor_t *x, const Sizes &s, int32_t d0, int32_t d1, const char *name)
{
    RELAY_TRY(check_type(t, name));
    RELAY_TRY(check_rank(t, s.rank, name));
    if (t->dtype != d0 && t->dtype != d1) return fail(RELAY_ERR_DTYPE, "%s: base type %s", name, dtype_name(t->dtype));
    RELAY_TRY(check_layout(t, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
    return check_shape_n(t, x->shape, s.rank, name);
}
relay_status_t check_temperature(float t)
{
    if (!(t > 0.0f) || t > 3.0e38f) return fail(RELAY_ERR_ATTR, "temperature = %g, needs a positive finite number", (double)t);
    return RELAY_OK;
}
Piece make_piece(const relay_tensor_t *x, const relay_tensor_t *tokens, int32_t trans_w, float temperature, const Sizes &s)
{
    Piece p{};
    p.x = x->data; p.ldx = s.K;
    p.trans_w = trans_w != 0;
    p.rows = s.rows; p.K = s.K; p.V = s.V;
    p.tokens = tokens->data; p.tokens_i64 = tokens->dtype == RELAY_I64;
    p.inv_temperature = 1.0f / std::max(temperature, FLT_MIN);
    return p;
}

}  // namespace
}  // namespace relay

using namespace relay;

extern "C" size_t relay_workspace_bytes_linear_logprob(const relay_tensor_t *x, const relay_tensor_t *w, int32_t trans_w)
{
    clear_error();
    Sizes s;
    if (!x || !w || check_operands(x, w, trans_w, &s) != RELAY_OK || s.rows == 0) return 0;
    s.rows = slab_of(s, x->dtype == RELAY_BF16);
    return forward_layout(s, trans_w != 0, x->dtype == RELAY_BF16).bytes;
}
extern "C" size_t relay_workspace_bytes_linear_logprob_grad(const relay_tensor_t *x, const relay_tensor_t *w, int32_t trans_w)
{
    clear_error();
    Sizes s;
    if (!x || !w || check_operands(x, w, trans_w, &s) != RELAY_OK || s.rows == 0) return 0;
    return gradient_layout(s, trans_w != 0, x->dtype == RELAY_BF16).bytes;
}

extern "C" relay_status_t relay_linear_logprob(const relay_tensor_t *x, const relay_tensor_t *w, int32_t trans_w, const relay_tensor_t *tokens,
                                               float temperature, const relay_tensor_t *logp, const relay_tensor_t *lse, void *ws, size_t ws_bytes,
                                               void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(x, "x"));
    RELAY_TRY(check_not_null(w, "w"));
    RELAY_TRY(check_not_null(tokens, "tokens"));
    RELAY_TRY(check_not_null(logp, "logp"));
    RELAY_TRY(check_not_null(lse, "lse"));
    Sizes s;
    RELAY_TRY(check_operands(x, w, trans_w, &s));
    RELAY_TRY(check_rows(tokens, x, s, RELAY_I32, RELAY_I64, "tokens"));
    RELAY_TRY(check_rows(logp, x, s, RELAY_F32, RELAY_F32, "logp"));
    RELAY_TRY(check_rows(lse, x, s, RELAY_F32, RELAY_F32, "lse"));
    RELAY_TRY(check_temperature(temperature));
    const relay_tensor_t *ins[3] = {x, w, tokens}, *outs[2] = {logp, lse};
    RELAY_TRY(seq::check_buffers(ins, outs));
    if (s.rows == 0) return RELAY_OK;
    const bool bf16 = x->dtype == RELAY_BF16;
    Sizes slab = s;
    slab.rows = slab_of(s, bf16);
    const size_t need = forward_layout(slab, trans_w != 0, bf16).bytes;
    RELAY_TRY(check_workspace(ws, ws_bytes, need));
    cudaStream_t st = (cudaStream_t)stream;
    RELAY_TRY(seq::register_buffers(ins, outs, ws, need, st));
    Piece p = make_piece(x, tokens, trans_w, temperature, s);
    const size_t x_row = (size_t)s.K * dtype_size(x->dtype), token = dtype_size(tokens->dtype), step = slab.rows;
    for (int64_t r = 0; r < s.rows; r += step) {
        p.rows = slab.rows = std::min<int64_t>(step, s.rows - r);
        p.x = (const char *)x->data + r * x_row; p.ldx = s.K;
        p.tokens = (const char *)tokens->data + r * token;
        RELAY_TRY(run_forward(p, slab, w->data, bf16, (float *)logp->data + r, (float *)lse->data + r, (char *)ws, st));
    }
    return RELAY_OK;
}

extern "C" relay_status_t relay_linear_logprob_grad(const relay_tensor_t *x, const relay_tensor_t *w, int32_t trans_w, const relay_tensor_t *tokens,
                                                    float temperature, const relay_tensor_t *lse, const relay_tensor_t *dlogp,
                                                    const relay_tensor_t *dx, const relay_tensor_t *dw, void *ws, size_t ws_bytes, void *stream)
{
    clear_error();
    RELAY_TRY(check_not_null(x, "x"));
    RELAY_TRY(check_not_null(w, "w"));
    RELAY_TRY(check_not_null(tokens, "tokens"));
    RELAY_TRY(check_not_null(lse, "lse"));
    RELAY_TRY(check_not_null(dlogp, "dlogp"));
    if (!dx && !dw) return fail(RELAY_ERR_NULL, "no output is wanted");
    Sizes s;
    RELAY_TRY(check_operands(x, w, trans_w, &s));
    RELAY_TRY(check_rows(tokens, x, s, RELAY_I32, RELAY_I64, "tokens"));
    RELAY_TRY(check_rows(lse, x, s, RELAY_F32, RELAY_F32, "lse"));
    RELAY_TRY(check_rows(dlogp, x, s, RELAY_F32, RELAY_F32, "dlogp"));
    for (const auto &o : {std::make_pair(dx, x), std::make_pair(dw, w)}) {
        if (!o.first) continue;
        const char *name = o.second == x ? "dx" : "dw";
        RELAY_TRY(check_type(o.first, name));
        RELAY_TRY(check_rank(o.first, o.second->rank, name));
        RELAY_TRY(check_dtype(o.first, o.second->dtype, name));
        RELAY_TRY(check_layout(o.first, RELAY_ROWMAJOR, RELAY_ROWMAJOR, name));
        RELAY_TRY(check_shape_n(o.first, o.second->shape, o.second->rank, name));
    }
    RELAY_TRY(check_temperature(temperature));
    const relay_tensor_t *ins[5] = {x, w, tokens, lse, dlogp}, *outs[2] = {dx, dw};
    RELAY_TRY(seq::check_buffers(ins, outs));
    cudaStream_t st = (cudaStream_t)stream;
    if (s.rows == 0) {                                     // a sum over no rows
        if (dw) RELAY_CUDA(cudaMemsetAsync(dw->data, 0, nbytes(dw), st));
        return RELAY_OK;
    }
    const bool bf16 = x->dtype == RELAY_BF16;
    const size_t need = gradient_layout(s, trans_w != 0, bf16).bytes;
    RELAY_TRY(check_workspace(ws, ws_bytes, need));
    RELAY_TRY(seq::register_buffers(ins, outs, ws, need, st));
    const Piece p = make_piece(x, tokens, trans_w, temperature, s);
    if (bf16)
        return run_gradient_bf16(p, s, w->data, (const float *)lse->data, (const float *)dlogp->data, dx ? (__nv_bfloat16 *)dx->data : nullptr,
                                 dw ? (__nv_bfloat16 *)dw->data : nullptr, (char *)ws, st);
    return run_gradient_f32(p, s, (const float *)w->data, (const float *)lse->data, (const float *)dlogp->data, dx ? (float *)dx->data : nullptr,
                            dw ? (float *)dw->data : nullptr, (char *)ws, st);
}
