// m = Norm(y) w_after,   s = scale r + act(gate) m,   n = Norm(s) w_before,   Norm(x) = x (mean x^2 + eps)^-1/2, for every row in one pass, and its gradient
//
//   d = d_s + q (b - s q (q mean(b s))),   b = d_n w_before,   q = (mean s^2 + eps)^-1/2,
//   dr = scale d,   dgate = d m act'(gate),   f = d act(gate),   dy = p (f w_after - y p (p mean(f w_after y))),   p = (mean y^2 + eps)^-1/2,
//   dw_after = sum f y p,   dw_before = sum d_n s q.
//
// Bound by bytes: every row is read once and written once.  A group of lanes (up to a whole workgroup) holds a row in registers, eight or sixteen values a lane;
// the backward pass makes s again from y, r and the gate instead of reading it back: as many bytes, and s as it was before its rounding.  Sums over
// tokens (of the weights' gradients, of a gate that tokens share) stay in registers over a group's rows, then a workgroup leaves one row of each in the
// workspace, which k_column_sums adds up in their order.  A group's rows lie one behind the other, and the next one's values wait in registers as they stand in memory (16 x 1024
// tokens of 2048 in BF16 with a float32 residual: forward 82 us, 403 MB, 4.9 TB/s, gradient 143, 604 MB, 4.2 TB/s; with a row a workgroup and its weights read for each 173 and 187).
// Rows of more than 4096 take sixteen values a lane, for which the gradient has too few registers: 255 or 256, and all but one kernel spill, up to 304 bytes a lane.
#pragma once
#include "blocknorm.h"
#include "gates.h"

namespace tfno {

constexpr int BLOCK_NORM_THREADS = 256, BLOCK_NORM_MOST = 512;      // of a workgroup whose rows are narrow, and of one that holds a wide row
enum { GATE_NONE = 0, GATE_TOKEN = 1, GATE_SEQUENCE = 2, GATE_CHANNEL = 3 };
enum { ACT_NONE = 0, ACT_SILU = 1, ACT_SIGMOID = 2 };

struct BlockNormShape {
    int group_log2;                 // threads of a row
    int by_group;                   // a part's rows are one group's; else a workgroup's, whose groups share them
    unsigned outer, outer_stride;   // parts of the batch, and how many are worked on at once
    unsigned parts, rows;           // parts of a sequence, and their rows; without parts (0) a group takes `rows` rows of the batch in all
    int whole;                      // a part is a whole sequence: its gate's gradient needs no further sum
    float *part_after, *part_before, *part_gate;
};

// Eight values of a thread as they stand in memory: neighbours where VEC, else `step` apart.  `count` of them are inside the row.
template <class E, bool VEC>
struct Eight {
    E at[8];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = E{};
    }
    __device__ __forceinline__ void load(const E *p, int step, int count)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) at[i] = i < count ? p[i * step] : E{};
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_float(at[i]);
    }
    __device__ __forceinline__ static void store(E *p, int step, int count, const float (&v)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) store_element(p + i * step, v[i]);
    }
};
template <>
struct Eight<float, true> {
    float4 lo, hi;
    __device__ __forceinline__ void clear() { lo = hi = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
    __device__ __forceinline__ void load(const float *p, int, int) { lo = reinterpret_cast<const float4 *>(p)[0], hi = reinterpret_cast<const float4 *>(p)[1]; }
    __device__ __forceinline__ void values(float (&v)[8]) const { v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w; }
    __device__ __forceinline__ static void store(float *p, int, int, const float (&v)[8])
    {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
};
template <>
struct Eight<bf16, true> {
    uint4 at;
    __device__ __forceinline__ void clear() { at = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const bf16 *p, int, int) { at = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
        const unsigned w[4] = {at.x, at.y, at.z, at.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    __device__ __forceinline__ static void store(bf16 *p, int, int, const float (&v)[8])
    {
        // whole lines, past the caches: 16 x 1024 of 1024 forward 40 us, else 41, gradient 79 and 79, 131072 heads of 128 29 and 30, 52 and 53.  What reads them next is as fast or
        // faster, but a product behind little: n_out of 16 x 64 of 1024 and a product 25.6 us, else 23.6, of 2 x 256 of 2048 26.9 and 25.6, of 16 x 1024 of 1024 58 and 59, of
        // 16 x 1024 of 2048 131 and 130.  The two halves of a lane's float32 values would be parts of lines
        typedef unsigned vector __attribute__((ext_vector_type(4)));
        __builtin_nontemporal_store(vector{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])}, (vector *)p);
    }
};

// Sums of N values over the threads of a row.  Rows wider than a wave have the workgroup to themselves and meet in LDS, in two buffers by turns.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int group_log2, float (*meet)[2][16], int &turn)
{
    const int width = min(1 << group_log2, 64);
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = group_sum(v[n], width);
    if (group_log2 <= 6) return;
    const int waves = 1 << (group_log2 - 6);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) meet[turn][n][threadIdx.x >> 6] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        float all = 0.0f;
        for (int w = 0; w < waves; ++w) all += meet[turn][n][w];
        v[n] = all;
    }
    turn ^= 1;
}

// A row of one sum over tokens: the groups of a workgroup add up in their order.
template <bool VEC, int ITER>
__device__ __forceinline__ void leave(float (&v)[ITER][8], int group_log2, const int (&count)[ITER], const int (&column)[ITER], int step, float *out, float (*meet)[8])
{
    const int width = 1 << group_log2;
    if (width >= (int)blockDim.x) {
#pragma unroll
        for (int i = 0; i < ITER; ++i)
            if (count[i] > 0) Eight<float, false>::store(out + column[i], VEC ? 1 : step, count[i], v[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) meet[threadIdx.x][e] = v[i][e];
        __syncthreads();
        if ((int)threadIdx.x < width && count[i] > 0) {
            float sum[8] = {};
            for (int g = threadIdx.x; g < (int)blockDim.x; g += width)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += meet[g][e];
            Eight<float, false>::store(out + column[i], VEC ? 1 : step, count[i], sum);
        }
    }
    __syncthreads();
}

// E: type of y, n and of a token's gate.  R: type of the residual.  TOKEN: each token has a gate of its own; else they share one, or there is none.  A thread has ITER times eight values of a row; the next row's are on their way while it works on one.
template <class E, class R, bool VEC, int ITER, bool TOKEN, bool BACKWARD>
__global__ __launch_bounds__(BLOCK_NORM_MOST) __attribute__((amdgpu_waves_per_eu(BACKWARD && TOKEN && ITER == 1 ? 3 : 2))) void k_block_norm(BlockNormArgs a, BlockNormShape s)
{
    __shared__ float meet[2][2][16];
    __shared__ float sums[BACKWARD ? BLOCK_NORM_THREADS : 1][8];
    const int width = 1 << s.group_log2, lane = threadIdx.x & (width - 1), group = threadIdx.x >> s.group_log2, groups = blockDim.x >> s.group_log2;
    const int step = width;
    int column[ITER], count[ITER], turn = 0;
    float wa[ITER][8], wb[ITER][8], gate[TOKEN ? 1 : ITER][8];       // gate: of the channels, or of the sequence that the rows are in
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        column[i] = VEC ? (i * width + lane) * 8 : i * width * 8 + lane;
        count[i] = VEC ? (column[i] < a.C ? 8 : 0) : max(0, min(8, (a.C - column[i] + step - 1) / step));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = column[i] + (VEC ? e : e * step);
            const bool in = e < count[i];
            wa[i][e] = in ? a.w_after && a.norm_after ? a.w_after[c] : 1.0f : 0.0f;
            wb[i][e] = in ? a.w_before ? a.w_before[c] : 1.0f : 0.0f;
            if constexpr (!TOKEN) gate[i][e] = in && a.gate_kind == GATE_CHANNEL ? ((const float *)a.gate)[c] : 0.0f;
        }
    }
    float d_after[ITER][8] = {}, d_before[ITER][8] = {}, d_gate[TOKEN ? 1 : ITER][8] = {};
    const float over_C = 1.0f / (float)a.C;
    const bool before = BACKWARD ? a.d_n_out != nullptr : a.n_out != nullptr;
    const unsigned here = blockIdx.x * groups + group;
    for (unsigned part = s.parts && !s.by_group ? blockIdx.x : s.parts ? here : 0; part < s.outer; part += s.outer_stride) {
        // the group's rows
        unsigned row, end;
        if (s.parts == 0) {
            const unsigned long long from = (unsigned long long)here * s.rows, all = (unsigned long long)a.B * a.T;
            row = (unsigned)min(from, all), end = (unsigned)min(from + s.rows, all);
        } else {
            const unsigned b = part / s.parts, from = (part - b * s.parts) * s.rows, to = min(from + s.rows, (unsigned)a.T);
            const unsigned each = s.by_group ? to - from : (to - from + groups - 1) / groups, first = s.by_group ? from : from + group * each;
            row = b * a.T + min(first, to), end = b * a.T + min(first + each, to);
        }
        unsigned b = a.T ? row / a.T : 0, t = row - b * a.T;
        int seen = -1;                              // the sequence whose gate is in the registers
        int length = a.lengths && row < end ? a.lengths[b] : a.T;
        Eight<E, VEC> in_y[ITER], in_z[TOKEN ? ITER : 1], in_n[BACKWARD ? ITER : 1];
        Eight<R, VEC> in_r[ITER], in_s[BACKWARD ? ITER : 1];
        const auto load = [&] {
            const bool there = (int)t < length;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                in_y[i].clear(), in_r[i].clear();
                if constexpr (TOKEN) in_z[i].clear();
                if constexpr (BACKWARD) in_n[i].clear(), in_s[i].clear();
                if (!there || count[i] == 0) continue;
                in_y[i].load((const E *)a.y + b * a.sy.batch + t * a.sy.token + column[i], step, count[i]);
                if (a.r) in_r[i].load((const R *)a.r + b * a.sr.batch + t * a.sr.token + column[i], step, count[i]);
                if constexpr (TOKEN) in_z[i].load((const E *)a.gate + b * a.sgate.batch + t * a.sgate.token + column[i], step, count[i]);
                if constexpr (BACKWARD) {
                    if (a.d_r_out) in_s[i].load((const R *)a.d_r_out + b * a.sr_out.batch + t * a.sr_out.token + column[i], step, count[i]);
                    if (a.d_n_out) in_n[i].load((const E *)a.d_n_out + b * a.sn_out.batch + t * a.sn_out.token + column[i], step, count[i]);
                }
            }
        };
        if (row < end) load();
        while (row < end) {
            const unsigned cb = b, ct = t;
            const bool there = (int)t < length;
            float y[ITER][8], r[ITER][8], z[ITER][8], dn[ITER][8], ds[ITER][8];
            if (!TOKEN && a.gate_kind == GATE_SEQUENCE && seen != (int)b) {
                seen = (int)b;
#pragma unroll
                for (int i = 0; i < ITER; ++i) {
                    Eight<float, VEC> shared;
                    shared.clear();
                    if (count[i] > 0) shared.load((const float *)a.gate + b * a.sgate.batch + column[i], step, count[i]);
                    shared.values(gate[TOKEN ? 0 : i]);
                }
            }
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                in_y[i].values(y[i]), in_r[i].values(r[i]);
                if constexpr (BACKWARD) in_n[i].values(dn[i]), in_s[i].values(ds[i]);
                if constexpr (TOKEN) {
                    in_z[i].values(z[i]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[i][e] = gate[i][e];
                }
            }
            ++row;
            if (++t == (unsigned)a.T) {
                t = 0, ++b;
                if (a.lengths && row < end) length = a.lengths[b];
            }
            if (row < end) load();
            float p = 1.0f;
            if (a.norm_after) {
                float ss[1] = {};
#pragma unroll
                for (int i = 0; i < ITER; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss[0] = fmaf(y[i][e], y[i][e], ss[0]);
                row_sums(ss, s.group_log2, meet, turn);
                p = rsqrtf(fmaf(ss[0], over_C, a.eps));
            }
            // z: act(gate), slope: its slope
            float st[ITER][8], slope[ITER][8], two[2] = {};
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                if (!TOKEN && a.gate_kind == GATE_NONE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[i][e] = 1.0f, slope[i][e] = 0.0f;
                } else if (a.activation == ACT_NONE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) slope[i][e] = 1.0f;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float open, rest;
                        sigmoid(z[i][e], open, rest);
                        const float through = a.activation == ACT_SILU ? z[i][e] * open : open;
                        slope[i][e] = a.activation == ACT_SILU ? fmaf(through, rest, open) : open * rest;
                        z[i][e] = through;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    st[i][e] = y[i][e] * p * wa[i][e] * z[i][e];
                    if (a.r) st[i][e] = fmaf(a.residual_scale, r[i][e], st[i][e]);
                    two[0] = fmaf(st[i][e], st[i][e], two[0]);
                    if constexpr (BACKWARD) two[1] = fmaf(dn[i][e] * wb[i][e], st[i][e], two[1]);
                }
            }
            float q = 0.0f;
            if (before) {
                if constexpr (BACKWARD) {
                    row_sums(two, s.group_log2, meet, turn);
                } else {
                    float one[1] = {two[0]};
                    row_sums(one, s.group_log2, meet, turn);
                    two[0] = one[0];
                }
                q = rsqrtf(fmaf(two[0], over_C, a.eps));
            }
            if constexpr (!BACKWARD) {
#pragma unroll
                for (int i = 0; i < ITER; ++i) {
                    if (count[i] == 0) continue;
                    float n[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        n[e] = there ? st[i][e] * q * wb[i][e] : 0.0f;
                        st[i][e] = there ? st[i][e] : 0.0f;
                    }
                    if (a.r_out) Eight<R, VEC>::store((R *)a.r_out + cb * a.sr_out.batch + ct * a.sr_out.token + column[i], step, count[i], st[i]);
                    if (a.n_out) Eight<E, VEC>::store((E *)a.n_out + cb * a.sn_out.batch + ct * a.sn_out.token + column[i], step, count[i], n);
                }
            } else {
                // products in an order that stays in range: the third power of an inverse root would not, for rows of 1e13 or 1e-13
                const float back = q * two[1] * over_C * q;
                float dot[1] = {};
                // a row that is not there counts in no sum, whatever gate and weights it would have: selected, not skipped, which took registers (rows of 8192 285 -> 301 us)
#pragma unroll
                for (int i = 0; i < ITER; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float scaled = y[i][e] * p;
                        float d = ds[i][e];
                        if (before) {
                            d = fmaf(q, fmaf(wb[i][e], dn[i][e], -back * st[i][e]), d);
                            d_before[i][e] = there ? fmaf(dn[i][e] * q, st[i][e], d_before[i][e]) : d_before[i][e];
                        }
                        const float f = d * z[i][e], dz = d * (scaled * wa[i][e]) * slope[i][e];
                        d_after[i][e] = there ? fmaf(f, scaled, d_after[i][e]) : d_after[i][e];
                        if constexpr (TOKEN) slope[i][e] = dz;
                        else d_gate[i][e] += there ? dz : 0.0f;
                        r[i][e] = a.residual_scale * d;
                        z[i][e] = f * wa[i][e];
                        dot[0] = fmaf(z[i][e], y[i][e], dot[0]);
                    }
                float along = 0.0f;
                if (a.norm_after) {
                    row_sums(dot, s.group_log2, meet, turn);
                    along = p * dot[0] * over_C * p;
                }
#pragma unroll
                for (int i = 0; i < ITER; ++i) {
                    if (count[i] == 0) continue;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        y[i][e] = there ? p * fmaf(-along, y[i][e], z[i][e]) : 0.0f;
                        r[i][e] = there ? r[i][e] : 0.0f;
                        slope[i][e] = there ? slope[i][e] : 0.0f;
                    }
                    Eight<E, VEC>::store((E *)a.dy + cb * a.sdy.batch + ct * a.sdy.token + column[i], step, count[i], y[i]);
                    if (a.dr) Eight<R, VEC>::store((R *)a.dr + cb * a.sdr.batch + ct * a.sdr.token + column[i], step, count[i], r[i]);
                    if (TOKEN && a.dgate)
                        Eight<E, VEC>::store((E *)a.dgate + cb * a.sdgate.batch + ct * a.sdgate.token + column[i], step, count[i], slope[i]);
                }
            }
        }
        if constexpr (BACKWARD && !TOKEN) {
            if (s.parts && a.gate_kind == GATE_SEQUENCE && a.dgate) {
                // one row of the gate's gradient for the part: where it is a whole sequence, that is the gradient
                float *out = s.whole ? (float *)a.dgate + (long long)part * a.sdgate.batch : s.part_gate + (size_t)part * a.C;
                if (s.by_group) {
#pragma unroll
                    for (int i = 0; i < ITER; ++i)
                        if (count[i] > 0) Eight<float, false>::store(out + column[i], VEC ? 1 : step, count[i], d_gate[i]);
                } else {
                    leave<VEC>(d_gate, s.group_log2, count, column, step, out, sums);
                }
#pragma unroll
                for (int i = 0; i < ITER; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) d_gate[i][e] = 0.0f;
            }
        }
    }
    if constexpr (BACKWARD) {
        if (a.dw_after) leave<VEC>(d_after, s.group_log2, count, column, step, s.part_after + (size_t)blockIdx.x * a.C, sums);
        if (a.dw_before) leave<VEC>(d_before, s.group_log2, count, column, step, s.part_before + (size_t)blockIdx.x * a.C, sums);
        if constexpr (!TOKEN)
            if (a.dgate && a.gate_kind == GATE_CHANNEL) leave<VEC>(d_gate, s.group_log2, count, column, step, s.part_gate + (size_t)blockIdx.x * a.C, sums);
    }
}

}  // namespace tfno
