// Sums over the rows of what workgroups left of a gradient that all tokens share: out[c] = sum_r part[r][c], always in the same order.
#pragma once
#include "common.h"

namespace tfno {

struct ColumnSums {
    const float *part;      // [jobs][rows][C]
    float *out;             // [jobs][C]
    unsigned rows, all;     // of a job, and of all of them: the last one may have less
};
template <int KINDS>
struct ColumnSumsArgs {
    ColumnSums kind[KINDS];
    unsigned first[KINDS + 1];      // jobs of each kind begin here
    int C;
};

// A workgroup takes 16 times V columns of one job in up to 64 groups of rows.  Four columns a thread where rows are aligned to that: fewer workgroups, each of which is mostly the
// wait for its rows (512 rows of 2048 columns, 18 sums: 10 -> 7 us).
template <int KINDS, int V>
__global__ __launch_bounds__(1024) void k_column_sums(ColumnSumsArgs<KINDS> a)
{
    __shared__ float sums[64][16 * V];
    const unsigned column = (threadIdx.x & 15) * V, c = blockIdx.x * 16 * V + column, group = threadIdx.x >> 4, groups = blockDim.x >> 4;
    int k = 0;
#pragma unroll
    for (int i = 1; i < KINDS; ++i) k = blockIdx.y >= a.first[i] ? i : k;
    const ColumnSums job = a.kind[k];
    const size_t at = blockIdx.y - a.first[k];
    float sum[V] = {};
    if (c < (unsigned)a.C) {
        const float *p = job.part + at * job.rows * a.C + c;
        const unsigned rows = min(job.rows, job.all - (unsigned)at * job.rows);
#pragma unroll 8
        for (unsigned r = group; r < rows; r += groups) {
            if constexpr (V == 4) {
                const float4 v = *reinterpret_cast<const float4 *>(p + (size_t)r * a.C);
                sum[0] += v.x, sum[1] += v.y, sum[2] += v.z, sum[3] += v.w;
            } else {
                sum[0] += p[(size_t)r * a.C];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) sums[group][column + e] = sum[e];
    __syncthreads();
    const unsigned mine = blockIdx.x * 16 * V + threadIdx.x;
    if (threadIdx.x < 16 * V && mine < (unsigned)a.C) {
        float all = 0.0f;
        for (unsigned i = 0; i < groups; ++i) all += sums[i][threadIdx.x];
        job.out[at * a.C + mine] = all;
    }
}

template <int KINDS>
void column_sums(const ColumnSumsArgs<KINDS> &a, hipStream_t s)
{
    unsigned rows = 0, threads = 64;
    for (const ColumnSums &k : a.kind) rows = k.rows > rows ? k.rows : rows;
    while (threads < 1024 && threads / 16 * 4 < rows) threads *= 2;        // four rows a group, where there are so few
    if (!a.first[KINDS]) return;
    bool four = a.C % 4 == 0;
    for (const ColumnSums &k : a.kind) four = four && ((uintptr_t)k.part & 15) == 0;
    if (four) k_column_sums<KINDS, 4><<<dim3((a.C + 63) / 64, a.first[KINDS]), threads, 0, s>>>(a);
    else k_column_sums<KINDS, 1><<<dim3((a.C + 15) / 16, a.first[KINDS]), threads, 0, s>>>(a);
}

}  // namespace tfno
