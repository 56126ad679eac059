// y = Rot(position)(x r w), r = (mean x^2 + eps)^-1/2, for every head of queries and keys in one pass, and its gradient
//
//   a = Rot(-position) dy,   dw = sum a x r,   dx = r (a w - x r^2 mean(a w x)).
//
// Bound by bytes: x is read once and y written once (backward: x and dy, and dx).  A group of `lpr` lanes holds one head; a lane
// holds pairs of values, the two that one rotation turns into each other, so the rotation needs no exchange between lanes and the
// norm one sum over the group.  The values past the first R go through as pairs that are not turned.  A group takes NH heads
// of one token, whose angles it loads once.  A workgroup takes heads of queries or heads of keys, never both: one set of weights.
//
// What is loaded waits in registers as it stands in memory, so that four waves of a SIMD fit beside all loads of four heads: with its values as
// float32 three did, and the gradient of 16 x 1024 tokens of 16 + 8 heads of 128 in BF16 took 98 us; it takes 60 (302 MB, 5.0 TB/s, what a copy
// reaches), the forward pass 43 (201 MB, 4.6 TB/s).
#pragma once
#include "headnorm.h"

namespace tfno {

constexpr int HEAD_NORM_THREADS = 256;
// Workgroups of the backward kernel, at most: as many as the chip holds at four waves a SIMD, each with one partial sum of the weights' gradient (both
// directions of the batch above: 104 us; with 768 111, with 512 128, with 2048 107).
constexpr int HEAD_NORM_BLOCKS = 1024;
constexpr unsigned HEAD_NORM_LAUNCH = 1u << 22;      // of the forward kernel: 2^30 threads, a launch takes less than 2^32

struct HeadNormShape {
    int lpr;                        // lanes of a head
    unsigned blocks_q;              // workgroups of queries; the others take keys
    unsigned chunks[2], items[2];   // groups of NH heads of a token, and of all tokens: queries, keys
};

// VEC pairs of the head at `p` as they stand in memory (in BF16 half the registers of their values), until they are used.
template <class E, int VEC, bool INTER>
struct Pairs {
    Quad<E> u, v;
    __device__ __forceinline__ void clear() { u = v = {}; }
    __device__ __forceinline__ void load(const E *p, int first, int second, bool) { u.load(p + first), v.load(p + (INTER ? first + 4 : second)); }
    __device__ __forceinline__ void values(float (&x)[VEC], float (&y)[VEC]) const
    {
        if constexpr (INTER) {
            float a[4], b[4];
            u.values(a), v.values(b);
            x[0] = a[0], y[0] = a[1], x[1] = a[2], y[1] = a[3], x[2] = b[0], y[2] = b[1], x[3] = b[2], y[3] = b[3];
        } else {
            u.values(x), v.values(y);
        }
    }
};
template <class E, bool INTER>
struct Pairs<E, 1, INTER> {
    E u, v;
    __device__ __forceinline__ void clear() { u = v = {}; }
    __device__ __forceinline__ void load(const E *p, int first, int second, bool has_second)
    {
        u = p[first];
        if (has_second) v = p[second];
    }
    __device__ __forceinline__ void values(float (&x)[1], float (&y)[1]) const { x[0] = to_float(u), y[0] = to_float(v); }
};
template <class E, int VEC, bool INTER>
__device__ __forceinline__ void store_pairs(E *p, int first, int second, bool has_second, const float (&x)[VEC], const float (&y)[VEC])
{
    if constexpr (VEC == 4 && INTER) {
        const float u[4] = {x[0], y[0], x[1], y[1]}, v[4] = {x[2], y[2], x[3], y[3]};
        store4(p + first, u);
        store4(p + first + 4, v);
    } else if constexpr (VEC == 4) {
        store4(p + first, x);
        store4(p + second, y);
    } else {
        store_element(p + first, x[0]);
        if (has_second) store_element(p + second, y[0]);
    }
}

template <class E, int VEC, int ITER, int NH, bool INTER, bool BACKWARD>
__global__ __launch_bounds__(HEAD_NORM_THREADS) __attribute__((amdgpu_waves_per_eu(4))) void k_head_norm(HeadNormArgs a, HeadNormShape s)
{
    const int lane = threadIdx.x & (s.lpr - 1), group = threadIdx.x / s.lpr, groups = HEAD_NORM_THREADS / s.lpr;
    const int turned = a.R >> 1, rest = (a.D - a.R + 1) >> 1;
    const bool keys = blockIdx.x >= s.blocks_q;
    const unsigned block = keys ? blockIdx.x - s.blocks_q : blockIdx.x, blocks = keys ? gridDim.x - s.blocks_q : s.blocks_q;
    const unsigned chunks = s.chunks[keys], items = s.items[keys];
    const int H = keys ? a.Hk : a.Hq;
    const E *in = (const E *)(keys ? a.k : a.q), *grad = (const E *)(keys ? a.dk_out : a.dq_out);
    E *out = (E *)(BACKWARD ? keys ? a.dk : a.dq : keys ? a.k_out : a.q_out);
    const Strides si = keys ? a.sk : a.sq, sg = keys ? a.sk_out : a.sq_out, so = BACKWARD ? keys ? a.sdk : a.sdq : sg;
    const float *weights = keys ? a.wk : a.wq;
    int first[ITER], second[ITER];
    bool has[ITER], has_second[ITER];
    float w[2][ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int slot = (i * s.lpr + lane) * VEC;
        has[i] = slot < turned + rest;
        first[i] = INTER ? 2 * slot : slot < turned ? slot : a.R + slot - turned;
        second[i] = INTER ? first[i] + 1 : slot < turned ? slot + turned : a.R + rest + slot - turned;
        has_second[i] = has[i] && second[i] < a.D;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c0 = INTER ? first[i] + 2 * e : first[i] + e, c1 = INTER ? c0 + 1 : second[i] + e;
            w[0][i][e] = has[i] ? weights ? weights[c0] : 1.0f : 0.0f;
            w[1][i][e] = has_second[i] ? weights ? weights[c1] : 1.0f : 0.0f;
        }
    }
    float dw[2][ITER][VEC] = {};
    const float over_D = 1.0f / (float)a.D;

    for (unsigned item = block * groups + group; item < items; item += blocks * groups) {
        const unsigned token = item / chunks, chunk = item - token * chunks;
        const unsigned b = token / (unsigned)a.T, t = token - b * (unsigned)a.T;
        Pairs<E, VEC, INTER> in_x[NH][ITER], in_d[BACKWARD ? NH : 1][ITER];
        const E *p = in + (b * si.batch + t * si.token), *o = grad + (b * sg.batch + t * sg.token);
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const int h = chunk * NH + n;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                in_x[n][i].clear();
                if constexpr (BACKWARD) in_d[n][i].clear();
                if (!has[i] || h >= H) continue;
                in_x[n][i].load(p + h * si.head, first[i], second[i], has_second[i]);
                if constexpr (BACKWARD) in_d[n][i].load(o + h * sg.head, first[i], second[i], has_second[i]);
            }
        }
        // the token's angles; a position that the tables do not hold gives NaN, and nothing is read for it
        float c[ITER][VEC], r[ITER][VEC];
        const int position = a.positions ? a.positions[b * a.positions_batch + t] : (int)t;
        const bool known = (unsigned)position < (unsigned)a.P;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int slot = (i * s.lpr + lane) * VEC;
            const bool turns = slot < turned;
            const long long at = (long long)position * turned + slot;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                c[i][e] = !turns ? 1.0f : __uint_as_float(0x7fc00000u);
                r[i][e] = !turns ? 0.0f : __uint_as_float(0x7fc00000u);
            }
            if (turns && known) {
                if constexpr (VEC == 4) {
                    load4(a.cos + at, c[i]);
                    load4(a.sin + at, r[i]);
                } else {
                    c[i][0] = a.cos[at], r[i][0] = a.sin[at];
                }
            }
        }
        E *to = out + (b * so.batch + t * so.token);
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const int h = chunk * NH + n;
            float squares = 0.0f, dot = 0.0f, x[2][ITER][VEC], d[2][ITER][VEC];
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                in_x[n][i].values(x[0][i], x[1][i]);
                if constexpr (BACKWARD) in_d[n][i].values(d[0][i], d[1][i]);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    squares = fmaf(x[0][i][e], x[0][i][e], fmaf(x[1][i][e], x[1][i][e], squares));
                    if constexpr (BACKWARD) {
                        const float u = d[0][i][e], v = d[1][i][e];
                        d[0][i][e] = fmaf(u, c[i][e], v * r[i][e]);
                        d[1][i][e] = fmaf(v, c[i][e], -(u * r[i][e]));
                        dot = fmaf(d[0][i][e] * w[0][i][e], x[0][i][e], dot);
                        dot = fmaf(d[1][i][e] * w[1][i][e], x[1][i][e], dot);
                    }
                }
            }
            squares = group_sum(squares, s.lpr);
            const float norm = 1.0f / sqrtf(fmaf(squares, over_D, a.eps));
            float mean = 0.0f;
            if constexpr (BACKWARD) mean = group_sum(dot, s.lpr) * norm * norm * over_D;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                float y[2][VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    if constexpr (BACKWARD) {
                        // a head past the last one has zeros in d
                        dw[0][i][e] = fmaf(d[0][i][e], x[0][i][e] * norm, dw[0][i][e]);
                        dw[1][i][e] = fmaf(d[1][i][e], x[1][i][e] * norm, dw[1][i][e]);
                        y[0][e] = norm * fmaf(d[0][i][e], w[0][i][e], -(x[0][i][e] * mean));
                        y[1][e] = norm * fmaf(d[1][i][e], w[1][i][e], -(x[1][i][e] * mean));
                    } else {
                        const float n0 = x[0][i][e] * norm * w[0][i][e], n1 = x[1][i][e] * norm * w[1][i][e];
                        y[0][e] = fmaf(n0, c[i][e], -(n1 * r[i][e]));
                        y[1][e] = fmaf(n0, r[i][e], n1 * c[i][e]);
                    }
                }
                if (has[i] && h < H) store_pairs<E, VEC, INTER>(to + h * so.head, first[i], second[i], has_second[i], y[0], y[1]);
            }
        }
    }

    if constexpr (BACKWARD) {
        if (!a.partial) return;          // nobody asks for the weights' gradient
        // the block's part of the weights' gradient: groups of a wave, then the waves, always in the same order
        __shared__ float sums[HEAD_NORM_THREADS / 64][512];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float v[2] = {dw[0][i][e], dw[1][i][e]};
#pragma unroll
                for (int m = 0; m < 2; ++m)
                    for (int step = s.lpr; step < 64; step <<= 1) v[m] += __shfl_xor(v[m], step, 64);
                if ((threadIdx.x & 63) < s.lpr && has[i]) {
                    const int c0 = INTER ? first[i] + 2 * e : first[i] + e, c1 = INTER ? c0 + 1 : second[i] + e;
                    sums[wave][c0] = v[0];
                    if (has_second[i]) sums[wave][c1] = v[1];
                }
            }
        __syncthreads();
        for (int c = threadIdx.x; c < a.D; c += HEAD_NORM_THREADS)
            a.partial[(long long)blockIdx.x * a.D + c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    }
}

// dw[c] = sum of partial[row][c] over the rows of queries resp. of keys: 16 columns and 64 row groups a block.
__global__ __launch_bounds__(1024) static void k_head_norm_weights(const float *partial, unsigned rows_q, unsigned rows, int D, float *dwq, float *dwk)
{
    __shared__ float sums[64][17];
    const int col = threadIdx.x & 15, part = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    float *out = blockIdx.y ? dwk : dwq;
    const unsigned begin = blockIdx.y ? rows_q : 0, end = blockIdx.y ? rows : rows_q;
    if (!out) return;
    float v = 0.0f;
    if (c < D)
#pragma unroll 4
        for (unsigned r = begin + part; r < end; r += 64) v += partial[(long long)r * D + c];
    sums[part][col] = v;
    __syncthreads();
    for (int half = 32; half >= 1; half >>= 1) {
        if (part < half) sums[part][col] += sums[part + half][col];
        __syncthreads();
    }
    if (part == 0 && c < D) out[c] = sums[0][col];
}

}  // namespace tfno
