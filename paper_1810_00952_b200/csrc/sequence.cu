// The column sums that end the gradient groups of sequences: partial sums of blocks, added in a fixed order (no float atomics).
#include "sequence.cuh"

namespace relay {
namespace seq {
namespace {

constexpr int kGroups = 8;          // rows are dealt to this many threads per column

__global__ void __launch_bounds__(32 * kGroups) column_sums_kernel(const float *in, long long rows, long long cols, long long ld, float *out0,
                                                                   long long n0, float *out1)
{
    __shared__ float part[kGroups][32];
    pdl_wait();
    const long long c = (long long)blockIdx.x * 32 + threadIdx.x;
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 4
        for (long long r = threadIdx.y; r < rows; r += kGroups) {
            const float *p = in + r * ld + c;
            if (relay_in_bounds(p, 4)) sum += __ldcs(p);
        }
    }
    part[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.y != 0 || c >= cols) return;
#pragma unroll
    for (int g = 1; g < kGroups; ++g) sum += part[g][threadIdx.x];
    float *out = c < n0 ? out0 : out1;
    if (out == nullptr) return;
    out += c < n0 ? c : c - n0;
    if (relay_in_bounds(out, 4)) *out = sum;
}

}  // namespace

relay_status_t launch_column_sums(const float *in, long long rows, long long cols, long long ld, float *out0, long long n0, float *out1,
                                  cudaStream_t st)
{
    if (cols == 0 || (out0 == nullptr && out1 == nullptr)) return RELAY_OK;
    const long long blocks = (cols + 31) / 32;
    if (blocks > 0x7fffffffLL) return fail(RELAY_ERR_UNSUPPORTED, "%lld columns", cols);
    RELAY_CUDA(launch_pdl(column_sums_kernel, dim3((unsigned)blocks), dim3(32, kGroups), 0, st, in, rows, cols, ld, out0, n0, out1));
    return check_launch("column_sums");
}

}  // namespace seq
}  // namespace relay
