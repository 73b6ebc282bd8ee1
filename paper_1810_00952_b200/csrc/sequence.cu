// The column sums that end the gradient groups of sequences: partial sums of blocks, added in a fixed order (no float atomics).
#include "sequence.cuh"

namespace relay {
namespace seq {
namespace {

constexpr int kGroups = 8;          // rows are dealt to this many threads per column

__global__ void __launch_bounds__(32 * kGroups) column_sums_kernel(const float *in, long long rows, long long cols, const ColumnSums to)
{
    __shared__ float part[kGroups][32];
    pdl_wait();
    const long long c = (long long)blockIdx.x * 32 + threadIdx.x;
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 4
        for (long long r = threadIdx.y; r < rows; r += kGroups) {
            const float *p = in + r * cols + c;
            if (relay_in_bounds(p, 4)) sum += __ldcs(p);
        }
    }
    part[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y != 0 || c >= cols) return;
#pragma unroll
    for (int g = 1; g < kGroups; ++g) sum += part[g][threadIdx.x];
    long long first = 0;
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        float *out = to.out[k] + (c - first);
        if (c >= first && c < first + to.n[k] && to.out[k] != nullptr && relay_in_bounds(out, 4)) *out = sum;
        first += to.n[k];
    }
}

}  // namespace

relay_status_t launch_column_sums(const float *in, long long rows, const ColumnSums &to, cudaStream_t st)
{
    long long cols = 0;
    bool wanted = false;
    for (int k = 0; k < kSums; ++k) { cols += to.n[k]; wanted |= to.n[k] > 0 && to.out[k] != nullptr; }
    if (!wanted) return RELAY_OK;
    const long long blocks = (cols + 31) / 32;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "%lld columns", cols);
    BoundsReg reg;
    reg.add(in, (size_t)rows * cols * 4);
    for (int k = 0; k < kSums; ++k) reg.add(to.out[k], (size_t)to.n[k] * 4);
    RELAY_TRY(reg.commit(st));
    RELAY_CUDA(launch_pdl(column_sums_kernel, dim3((unsigned)blocks), dim3(32, kGroups), 0, st, in, rows, cols, to));
    return check_launch("column_sums");
}

}  // namespace seq
}  // namespace relay
