// Log-probabilities from a head's operands: the products with their epilogues (linear_logprob_tc.cu) as the boundary
// (linear_logprob.cu) calls them.
#pragma once
#include "common.h"

namespace relay {
namespace head {

// One piece of the vocabulary: scores z = x w of classes first .. first + classes - 1, never stored.
struct Piece {
    const void *x; long long ldx;          // [rows][K] bf16
    const void *w; long long ldw;          // (K, classes) or, trans_w, (classes, K) bf16
    int trans_w;
    long long rows, K, classes, first;
    const void *tokens;
    int tokens_i64;
    long long V;                           // classes of the whole vocabulary
    float inv_temperature;
};
constexpr int kPartColumns = 64;           // columns that one partial sum covers
inline long long parts_of(long long classes) { return (classes + 255) / 256 * (256 / kPartColumns); }      // that a piece writes, or may write

// The tensor cores add the products of sixteen k at a time to an fp32 accumulator and drop what lies below its last bit, towards zero: a score whose
// terms are of all sizes comes out small by 2^-26 of itself for every such addition, on average (measured on normal operands: 4.9e-8, 8.6e-7 and
// 3.8e-6 of a score at K = 64, 1024 and 4096), one whose sums are exact not at all.  So an accumulator takes 1024 k at most; the epilogue adds
// those of a longer contraction up with one rounding each, on units of 256 columns (4096 x 2048 x 131072 with its gradient 6.8 ms; in one accumulator
// on units of up to 512 columns 7.0).
constexpr int kDepth = 1024;

// part[j][row] = (m, s): over the 64 columns from 64 j on, m = max z log2(e) / temperature and s = sum 2^(z log2(e) / temperature - m);
// at[row] = the token's score where the token is in this piece.  `ld` entries from one j to the next.
relay_status_t launch_stats(const Piece &p, float2 *part, long long ld, float *at, cudaStream_t st);
// dz[row][class] (bf16, ld entries a row; `padded_rows` x `padded_classes`, zero outside the piece).  In two parts (padded_rows a multiple of 32):
// the values rounded to bf16, and `padded_rows` rows further what that leaves, rounded to bf16 too.
relay_status_t launch_slopes(const Piece &p, const float *lse, const float *dlogp, void *dz, long long ld, long long padded_rows,
                             long long padded_classes, int parts, cudaStream_t st);

__device__ __forceinline__ int token_in_piece(const void *tokens, int i64, long long row, long long V, long long first, long long classes)
{
    const char *at = (const char *)tokens + row * (i64 ? 8 : 4);
    if (!relay_in_bounds(at, i64 ? 8 : 4)) return -1;
    const long long t = i64 ? *(const long long *)at : *(const int *)at;
    return t >= 0 && t < V && t >= first && t < first + classes ? (int)(t - first) : -1;
}

}  // namespace head
}  // namespace relay
