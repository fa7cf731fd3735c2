// Sums over the rows of partial results: what a backward's workgroups leave for the gradients of parameters.
#include <algorithm>

#include "kla_layer.hpp"

namespace kla {

// 64 columns per workgroup, its 16 waves take every sixteenth row, joined in a fixed order.  512 rows of 2048 columns (4 MB): 5 us, of which
// a launch and two trips to memory are most.
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* __restrict__ partial, long P, ColumnSums s, long first)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long col = first + (long)blockIdx.x * 64 + lane, C = s.n[0] + s.n[1] + s.n[2];
    float x = 0.f;
    if (col < C) {
#pragma unroll 8
        for (long r = wave; r < P; r += 16) x += partial[r * C + col];
    }
    red[wave][lane] = x;
    __syncthreads();
    if (wave == 0 && col < C) {
        x = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) x += red[w][lane];
        long at = col;
        int o = 0;
        while (o < 2 && at >= s.n[o]) at -= s.n[o++];
        if (s.out[o]) s.out[o][at] = x;
    }
}
hipError_t launch_column_sums(const float* partial, long P, const ColumnSums& s, hipStream_t st)
{
    const long C = s.n[0] + s.n[1] + s.n[2];
    for (long first = 0; first < C; first += most_blocks(1024) * 64) {
        const long blocks = std::min((C - first + 63) / 64, most_blocks(1024));
        hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)blocks), dim3(1024), 0, st, partial, P, s, first);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace kla
