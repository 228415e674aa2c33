// Sums of the parts that workgroups leave of a gradient that runs over all tokens.  Parts are added in an order of their own, so the same call
// gives the same bits.
#include "msla_device.h"
#include "msla_layer_kernels.h"

namespace msla {
namespace {

// 32 columns a workgroup, 32 runs of parts, then those.
__global__ void __launch_bounds__(1024) sum_parts_kernel(const float* parts, int64_t count, int64_t stride, PartSums to, int64_t columns) {
    __shared__ float room[32][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
    const int run = threadIdx.x / 32;
    float s = 0.0f;
    if (c < columns) {
#pragma unroll 8
        for (int64_t b = run; b < count; b += 32) s += parts[b * stride + c];
    }
    room[run][threadIdx.x % 32] = s;
    __syncthreads();
    if (run != 0 || c >= columns) return;
#pragma unroll
    for (int k = 1; k < 32; ++k) s += room[k][threadIdx.x];
    if (c < to.n[0]) {
        if (to.out[0]) to.out[0][c] = s;
    } else if (c < to.n[0] + to.n[1]) {
        if (to.out[1]) to.out[1][c - to.n[0]] = s;
    } else if (to.out[2]) {
        to.out[2][c - to.n[0] - to.n[1]] = s;
    }
}

}  // namespace

hipError_t launch_sum_parts(const float* parts, int64_t count, int64_t stride, const PartSums& to, hipStream_t stream) {
    const int64_t columns = to.n[0] + to.n[1] + to.n[2];
    if (columns == 0) return hipSuccess;
    hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)((columns + 31) / 32)), dim3(1024), 0, stream, parts, count, stride, to, columns);
    return hipGetLastError();
}

}  // namespace msla
