// Sums over the rows of what workgroups left of a gradient that all tokens share: out[c] = sum_r part[r][c], always in the same order.
#pragma once
#include "common.h"

namespace tfno {

struct ColumnSums {
    const float *part;      // [jobs][rows][C]
    float *out;             // [jobs][C]
    unsigned rows;
};

// A workgroup takes 16 columns of one job (64 bytes of a row) in 64 groups of rows.
template <int JOBS>
struct ColumnSumsArgs {
    ColumnSums kind[JOBS];
    unsigned first[JOBS + 1];       // jobs of each kind begin here
    int C;
};
template <int JOBS>
__global__ __launch_bounds__(1024) void k_column_sums(ColumnSumsArgs<JOBS> a)
{
    __shared__ float sums[64][16];
    const unsigned c = blockIdx.x * 16 + (threadIdx.x & 15), group = threadIdx.x >> 4;
    int k = 0;
#pragma unroll
    for (int i = 1; i < JOBS; ++i) k = blockIdx.y >= a.first[i] ? i : k;
    const ColumnSums job = a.kind[k];
    const size_t at = blockIdx.y - a.first[k];
    float sum = 0.0f;
    if (c < (unsigned)a.C)
#pragma unroll 8
        for (unsigned r = group; r < job.rows; r += 64) sum += job.part[(at * job.rows + r) * a.C + c];
    sums[group][threadIdx.x & 15] = sum;
    __syncthreads();
    if (group == 0 && c < (unsigned)a.C) {
        float all = 0.0f;
        for (int i = 0; i < 64; ++i) all += sums[i][threadIdx.x];
        job.out[at * a.C + c] = all;
    }
}

}  // namespace tfno
