// The sum of workgroups' parts of a weight gradient.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

// out[i][c] = sum over parts of partial[i][p][c].  A workgroup has 32 columns
// of one worker and 8 sums of every eighth part each, added in a fixed order,
// so equal inputs give equal bits.
__global__ __launch_bounds__(256) void sum_parts_kernel(const float *partial, float *out,
                                                        int64_t out_stride, int32_t parts,
                                                        int32_t width) {
    __shared__ float sums[8][32];
    const unsigned per = (width + 31) / 32;
    const int64_t worker = blockIdx.x / per;
    const int lane = threadIdx.x % 32, group = threadIdx.x / 32;
    const int c = (int)(blockIdx.x % per) * 32 + lane;
    float v = 0.0f;
    if (c < width) {
        const float *p = partial + worker * parts * (int64_t)width + c;
#pragma unroll 4
        for (int k = group; k < parts; k += 8) v += p[(int64_t)k * width];
    }
    sums[group][lane] = v;
    __syncthreads();
    if (group == 0 && c < width) {
#pragma unroll
        for (int k = 1; k < 8; ++k) v += sums[k][lane];
        out[worker * out_stride + c] = v;
    }
}

}  // namespace
