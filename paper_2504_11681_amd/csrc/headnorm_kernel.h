// y = Rot(position)(x r w), r = (mean x^2 + eps)^-1/2, for every head of queries and keys in one pass, and its gradient
//
//   a = Rot(-position) dy,   dw = sum a x r,   dx = r (a w - x r^2 mean(a w x)).
//
// Bound by bytes: x is read once and y written once (backward: x and dy, and dx).  A group of `lpr` lanes holds one head; a lane
// holds pairs of values, the two that one rotation turns into each other, so the rotation needs no exchange between lanes and the
// norm one sum over the group.  The values past the first R go through as pairs that are not turned.  A group takes NH heads
// of one token, whose angles it loads once.  A workgroup takes heads of queries or heads of keys, never both: one set of weights.
#pragma once
#include "headnorm.h"

namespace tfno {

constexpr int HEAD_NORM_THREADS = 256;
constexpr int HEAD_NORM_BLOCKS = 2048;     // of the backward kernel, at most: each leaves one partial sum of the weights' gradient

struct HeadNormShape {
    int lpr;                        // lanes of a head
    unsigned blocks_q;              // workgroups of queries; the others take keys
    unsigned chunks[2], items[2];   // groups of NH heads of a token, and of all tokens: queries, keys
};

// The two halves of VEC pairs: values first[] and second[] of the head at `p`.
template <class E, int VEC, bool INTER>
__device__ __forceinline__ void load_pairs(const E *p, int first, int second, bool has_second, float (&x)[VEC], float (&y)[VEC])
{
    if constexpr (VEC == 4 && INTER) {
        float u[4], v[4];
        load4(p + first, u);
        load4(p + first + 4, v);
        x[0] = u[0], y[0] = u[1], x[1] = u[2], y[1] = u[3], x[2] = v[0], y[2] = v[1], x[3] = v[2], y[3] = v[3];
    } else if constexpr (VEC == 4) {
        load4(p + first, x);
        load4(p + second, y);
    } else {
        x[0] = to_float(p[first]);
        y[0] = has_second ? to_float(p[second]) : 0.0f;
    }
}
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
__global__ __launch_bounds__(HEAD_NORM_THREADS) void k_head_norm(HeadNormArgs a, HeadNormShape s)
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
        float x[2][NH][ITER][VEC], d[2][NH][ITER][VEC];
        const E *p = in + (b * si.batch + t * si.token), *o = grad + (b * sg.batch + t * sg.token);
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const int h = chunk * NH + n;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[0][n][i][e] = x[1][n][i][e] = d[0][n][i][e] = d[1][n][i][e] = 0.0f;
                if (!has[i] || h >= H) continue;
                load_pairs<E, VEC, INTER>(p + h * si.head, first[i], second[i], has_second[i], x[0][n][i], x[1][n][i]);
                if constexpr (BACKWARD) load_pairs<E, VEC, INTER>(o + h * sg.head, first[i], second[i], has_second[i], d[0][n][i], d[1][n][i]);
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
            float squares = 0.0f, dot = 0.0f;
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    squares = fmaf(x[0][n][i][e], x[0][n][i][e], fmaf(x[1][n][i][e], x[1][n][i][e], squares));
                    if constexpr (BACKWARD) {
                        const float u = d[0][n][i][e], v = d[1][n][i][e];
                        d[0][n][i][e] = fmaf(u, c[i][e], v * r[i][e]);
                        d[1][n][i][e] = fmaf(v, c[i][e], -(u * r[i][e]));
                        dot = fmaf(d[0][n][i][e] * w[0][i][e], x[0][n][i][e], dot);
                        dot = fmaf(d[1][n][i][e] * w[1][i][e], x[1][n][i][e], dot);
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
                        dw[0][i][e] = fmaf(d[0][n][i][e], x[0][n][i][e] * norm, dw[0][i][e]);
                        dw[1][i][e] = fmaf(d[1][n][i][e], x[1][n][i][e] * norm, dw[1][i][e]);
                        y[0][e] = norm * fmaf(d[0][n][i][e], w[0][i][e], -(x[0][n][i][e] * mean));
                        y[1][e] = norm * fmaf(d[1][n][i][e], w[1][i][e], -(x[1][n][i][e] * mean));
                    } else {
                        const float n0 = x[0][n][i][e] * norm * w[0][i][e], n1 = x[1][n][i][e] * norm * w[1][i][e];
                        y[0][e] = fmaf(n0, c[i][e], -(n1 * r[i][e]));
                        y[1][e] = fmaf(n0, r[i][e], n1 * c[i][e]);
                    }
                }
                if (has[i] && h < H) store_pairs<E, VEC, INTER>(to + h * so.head, first[i], second[i], has_second[i], y[0], y[1]);
            }
        }
    }

    if constexpr (BACKWARD) {
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
