// y = Rot(position)(x r w), r = (mean x^2 + eps)^-1/2, for every head of queries and keys in one pass, and its gradient
//
//   a = Rot(-position) dy,   dw = sum a x r,   dx = r (a w - x r^2 mean(a w x)).
//
// Bound by bytes: x is read once and y written once (backward: x and dy, and dx).  A group of `lpr` lanes holds one head; a lane
// holds pairs of values, the two that one rotation turns into each other, so the rotation needs no exchange between lanes and the
// norm one sum over the group.  The values past the first R go through as pairs that are not turned.  A group takes NH heads
// of one token, whose angles it loads once.
#pragma once
#include "headnorm.h"

namespace tfno {

constexpr int HEAD_NORM_THREADS = 256;
constexpr int HEAD_NORM_BLOCKS = 1024;     // of the backward kernel, at most: each leaves one partial sum of the weights' gradients

struct HeadNormShape {
    int lpr;                // lanes of a head
    unsigned chunks;        // groups of NH heads of a token
    unsigned items;         // tokens * chunks
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
__global__ __launch_bounds__(HEAD_NORM_THREADS) void k_head_norm(HeadNormArgs a, HeadNormShape g)
{
    const int lane = threadIdx.x & (g.lpr - 1), group = threadIdx.x / g.lpr, groups = HEAD_NORM_THREADS / g.lpr;
    const int turned = a.R >> 1, rest = (a.D - a.R + 1) >> 1, H = a.Hq + a.Hk;
    int first[ITER], second[ITER];
    bool has[ITER], has_second[ITER];
    float wq[2][ITER][VEC], wk[2][ITER][VEC];
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int slot = (i * g.lpr + lane) * VEC;
        has[i] = slot < turned + rest;
        first[i] = INTER ? 2 * slot : slot < turned ? slot : a.R + slot - turned;
        second[i] = INTER ? first[i] + 1 : slot < turned ? slot + turned : a.R + rest + slot - turned;
        has_second[i] = has[i] && second[i] < a.D;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c0 = INTER ? first[i] + 2 * e : first[i] + e, c1 = INTER ? c0 + 1 : second[i] + e;
            wq[0][i][e] = has[i] ? a.wq ? a.wq[c0] : 1.0f : 0.0f;
            wq[1][i][e] = has_second[i] ? a.wq ? a.wq[c1] : 1.0f : 0.0f;
            wk[0][i][e] = has[i] ? a.wk ? a.wk[c0] : 1.0f : 0.0f;
            wk[1][i][e] = has_second[i] ? a.wk ? a.wk[c1] : 1.0f : 0.0f;
        }
    }
    float dwq[2][ITER][VEC] = {}, dwk[2][ITER][VEC] = {};

    for (unsigned item = blockIdx.x * groups + group; item < g.items; item += gridDim.x * groups) {
        const unsigned token = item / g.chunks, chunk = item - token * g.chunks;
        const unsigned b = token / (unsigned)a.T, t = token - b * (unsigned)a.T;
        float x[2][NH][ITER][VEC], d[2][NH][ITER][VEC];
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const int h = chunk * NH + n;
            const bool key = h >= a.Hq;
            const E *p = key ? (const E *)a.k + (b * a.sk.batch + t * a.sk.token + (h - a.Hq) * a.sk.head)
                             : (const E *)a.q + (b * a.sq.batch + t * a.sq.token + h * a.sq.head);
            const E *o = key ? (const E *)a.dk_out + (b * a.sk_out.batch + t * a.sk_out.token + (h - a.Hq) * a.sk_out.head)
                             : (const E *)a.dq_out + (b * a.sq_out.batch + t * a.sq_out.token + h * a.sq_out.head);
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[0][n][i][e] = x[1][n][i][e] = d[0][n][i][e] = d[1][n][i][e] = 0.0f;
                if (!has[i] || h >= H) continue;
                load_pairs<E, VEC, INTER>(p, first[i], second[i], has_second[i], x[0][n][i], x[1][n][i]);
                if constexpr (BACKWARD) load_pairs<E, VEC, INTER>(o, first[i], second[i], has_second[i], d[0][n][i], d[1][n][i]);
            }
        }
        // the token's angles; a position that the tables do not hold gives NaN, and nothing is read for it
        float c[ITER][VEC], s[ITER][VEC];
        const int position = a.positions ? a.positions[b * a.positions_batch + t] : (int)t;
        const bool known = (unsigned)position < (unsigned)a.P;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int slot = (i * g.lpr + lane) * VEC;
            const bool turns = slot < turned;
            const long long at = (long long)position * turned + slot;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                c[i][e] = !turns ? 1.0f : __uint_as_float(0x7fc00000u);
                s[i][e] = !turns ? 0.0f : __uint_as_float(0x7fc00000u);
            }
            if (turns && known) {
                if constexpr (VEC == 4) {
                    load4(a.cos + at, c[i]);
                    load4(a.sin + at, s[i]);
                } else {
                    c[i][0] = a.cos[at], s[i][0] = a.sin[at];
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NH; ++n) {
            const int h = chunk * NH + n;
            const bool key = h >= a.Hq;
            float squares = 0.0f, dot = 0.0f;
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    squares = fmaf(x[0][n][i][e], x[0][n][i][e], fmaf(x[1][n][i][e], x[1][n][i][e], squares));
                    if constexpr (BACKWARD) {
                        const float u = d[0][n][i][e], v = d[1][n][i][e];
                        d[0][n][i][e] = fmaf(u, c[i][e], v * s[i][e]);
                        d[1][n][i][e] = fmaf(v, c[i][e], -(u * s[i][e]));
                        dot = fmaf(d[0][n][i][e] * (key ? wk[0][i][e] : wq[0][i][e]), x[0][n][i][e], dot);
                        dot = fmaf(d[1][n][i][e] * (key ? wk[1][i][e] : wq[1][i][e]), x[1][n][i][e], dot);
                    }
                }
            squares = group_sum(squares, g.lpr);
            const float r = 1.0f / sqrtf(squares / (float)a.D + a.eps);
            float mean = 0.0f;
            if constexpr (BACKWARD) mean = group_sum(dot, g.lpr) * r * r / (float)a.D;
            E *out = key ? (E *)(BACKWARD ? a.dk : a.k_out) : (E *)(BACKWARD ? a.dq : a.q_out);
            const Strides &so = BACKWARD ? (key ? a.sdk : a.sdq) : (key ? a.sk_out : a.sq_out);
            out += b * so.batch + t * so.token + (key ? h - a.Hq : h) * so.head;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                float y[2][VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float w0 = key ? wk[0][i][e] : wq[0][i][e], w1 = key ? wk[1][i][e] : wq[1][i][e];
                    if constexpr (BACKWARD) {
                        const float n0 = x[0][n][i][e] * r, n1 = x[1][n][i][e] * r;
                        if (h < H) {
                            if (key) {
                                dwk[0][i][e] = fmaf(d[0][n][i][e], n0, dwk[0][i][e]);
                                dwk[1][i][e] = fmaf(d[1][n][i][e], n1, dwk[1][i][e]);
                            } else {
                                dwq[0][i][e] = fmaf(d[0][n][i][e], n0, dwq[0][i][e]);
                                dwq[1][i][e] = fmaf(d[1][n][i][e], n1, dwq[1][i][e]);
                            }
                        }
                        y[0][e] = r * fmaf(d[0][n][i][e], w0, -(x[0][n][i][e] * mean));
                        y[1][e] = r * fmaf(d[1][n][i][e], w1, -(x[1][n][i][e] * mean));
                    } else {
                        const float n0 = x[0][n][i][e] * r * w0, n1 = x[1][n][i][e] * r * w1;
                        y[0][e] = fmaf(n0, c[i][e], -(n1 * s[i][e]));
                        y[1][e] = fmaf(n0, s[i][e], n1 * c[i][e]);
                    }
                }
                if (has[i] && h < H) store_pairs<E, VEC, INTER>(out, first[i], second[i], has_second[i], y[0], y[1]);
            }
        }
    }

    if constexpr (BACKWARD) {
        // the block's part of the weights' gradients: groups of a wave, then the waves, always in the same order
        __shared__ float sums[HEAD_NORM_THREADS / 64][2][512];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float v[4] = {dwq[0][i][e], dwq[1][i][e], dwk[0][i][e], dwk[1][i][e]};
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    for (int step = g.lpr; step < 64; step <<= 1) v[m] += __shfl_xor(v[m], step, 64);
                if ((threadIdx.x & 63) < g.lpr && has[i]) {
                    const int c0 = INTER ? first[i] + 2 * e : first[i] + e, c1 = INTER ? c0 + 1 : second[i] + e;
                    sums[wave][0][c0] = v[0], sums[wave][1][c0] = v[2];
                    if (has_second[i]) sums[wave][0][c1] = v[1], sums[wave][1][c1] = v[3];
                }
            }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * a.D; c += HEAD_NORM_THREADS) {
            const int which = c >= a.D, col = which ? c - a.D : c;
            a.partial[(long long)blockIdx.x * 2 * a.D + c] = (sums[0][which][col] + sums[1][which][col]) + (sums[2][which][col] + sums[3][which][col]);
        }
    }
}

// dw[c] = sum of partial[row][c] over the rows: 16 columns and 64 row groups a block.
__global__ __launch_bounds__(1024) static void k_head_norm_weights(const float *partial, int rows, int D, float *dwq, float *dwk)
{
    __shared__ float sums[64][17];
    const int col = threadIdx.x & 15, part = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    float v = 0.0f;
    if (c < 2 * D)
        for (int r = part; r < rows; r += 64) v += partial[(long long)r * 2 * D + c];
    sums[part][col] = v;
    __syncthreads();
    for (int half = 32; half >= 1; half >>= 1) {
        if (part < half) sums[part][col] += sums[part + half][col];
        __syncthreads();
    }
    if (part == 0 && c < 2 * D) {
        float *out = c < D ? dwq : dwk;
        if (out) out[c < D ? c : c - D] = sums[0][col];
    }
}

}  // namespace tfno
