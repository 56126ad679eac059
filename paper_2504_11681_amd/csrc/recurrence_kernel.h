// h = a h + u for every channel, a = exp(l), u = x sigmoid(input_gate) sqrt(1 - exp(2 l)), and its gradient
//
//   D_t = dy_t + a_{t+1} D_{t+1},   du = D,   dl = D a h_{t-1} - D x sigmoid(input_gate) a^2 / sqrt(1 - a^2).
//
// Bound by bytes: every input is read once and every output written once.  A workgroup takes `lanes` neighbouring pairs of channels and walks
// through a sequence in tiles; a tile is shared out over time among groups of lanes, each with S tokens in a row, whose loads are all under way while the tile
// before is worked on.  A group makes of its tokens one map h -> a h + B (backward also e -> a e + R for what comes from later tokens), the
// maps meet in LDS, and each group then walks its tokens from the state that the maps before it give.
// Sequences too few to fill the chip are cut into segments, whose maps a kernel of its own finds first.
//
#pragma once
#include "recurrence.h"

namespace tfno {

constexpr int RECURRENCE_THREADS = 256;

struct RecurrenceShape {
    int lanes_log2;                 // lanes of a group
    unsigned channel_blocks, segments, first;
    int segment;                    // tokens of a segment
};

// V neighbouring elements as they stand in memory.
template <class E, int V>
struct Some;
template <class E>
struct Some<E, 1> {
    E at;
    __device__ __forceinline__ void load(const E *p) { at = *p; }
    __device__ __forceinline__ float value(int) const { return to_float(at); }
};
template <>
struct Some<float, 2> {
    float2 at;
    __device__ __forceinline__ void load(const float *p) { at = *reinterpret_cast<const float2 *>(p); }
    __device__ __forceinline__ float value(int i) const { return i ? at.y : at.x; }
};
template <>
struct Some<bf16, 2> {
    unsigned at;
    __device__ __forceinline__ void load(const bf16 *p) { at = *reinterpret_cast<const unsigned *>(p); }
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(i ? at & 0xffff0000u : at << 16); }
};
__device__ __forceinline__ void store_some(float *p, const float (&v)[1]) { *p = v[0]; }
__device__ __forceinline__ void store_some(bf16 *p, const float (&v)[1]) { store_element(p, v[0]); }
__device__ __forceinline__ void store_some(float *p, const float (&v)[2]) { *reinterpret_cast<float2 *>(p) = make_float2(v[0], v[1]); }
__device__ __forceinline__ void store_some(bf16 *p, const float (&v)[2]) { *reinterpret_cast<unsigned *>(p) = bf16_pair(v[0], v[1]); }

constexpr float LOG2E = 1.44269504088896340736f;

// 1 / (1 + exp(-z)), and what is left of 1.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * z)); }
__device__ __forceinline__ void sigmoid(float z, float &s, float &rest)
{
    const float e = __builtin_amdgcn_exp2f(-LOG2E * fabsf(z)), big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
    s = z < 0.0f ? small : big;
    rest = z < 0.0f ? big : small;
}
// A decay a = exp(l).  Near 1, where states last long, its distance from 1 is what matters: it is kept as -(1 - a), sign bit set, and from the series
// -l (1 + l/2 + l^2/6 + ...), whose first term left out is l^7 / 40320 of the whole, 2e-8 at the border; rounded to a float32 itself, a decay of 0.9999 would be
// 3e-4 of its distance off, always to the same side.  Elsewhere (and above 1) it is a itself, at least 2^-126.  +0 is a decay of exactly 0, which forgets the state whatever it
// holds: that of one token where exp(l) rounds to 0 in float32; of a sum of logarithms only where one of them was that of 0, whatever the others make of it.
constexpr float NOTHING_LEFT = -104.0f;
struct Decay {
    float at;
    __device__ __forceinline__ Decay() {}
    // a and 1 - a too
    __device__ __forceinline__ Decay(float l, float &a, float &less, float nothing = NOTHING_LEFT)
    {
        float p = fmaf(l, 1.0f / 5040.0f, 1.0f / 720.0f);
        p = fmaf(l, p, 1.0f / 120.0f);
        p = fmaf(l, p, 1.0f / 24.0f);
        p = fmaf(l, p, 1.0f / 6.0f);
        p = fmaf(l, p, 0.5f);
        p = fmaf(l, p, 1.0f);
        a = __builtin_amdgcn_exp2f(l * LOG2E);
        a = a == 0.0f ? 1.17549435e-38f : a;
        const bool near = l > -0.35f && l <= 0.0f;
        less = near ? fabsf(l * p) : 1.0f - a;
        at = near ? -less : l < nothing ? 0.0f : a;
    }
    __device__ __forceinline__ static Decay of_sum(float l)
    {
        float a, less;
        return Decay(l, a, less, -3.4e38f);
    }
    __device__ __forceinline__ bool forgets() const { return __float_as_uint(at) == 0; }
    __device__ __forceinline__ float of(float h) const { return forgets() ? 0.0f : fmaf(at, h, (int)__float_as_uint(at) < 0 ? h : 0.0f); }
    // a h + u
    __device__ __forceinline__ float of(float h, float u) const { return forgets() ? u : fmaf(at, h, ((int)__float_as_uint(at) < 0 ? h : 0.0f) + u); }
};
// The part of a sum of logarithms that a token has.
__device__ __forceinline__ float part_of_sum(float l) { return l < NOTHING_LEFT ? -INFINITY : l; }

// What tokens in their order do to the state before them: h -> a h + B.
struct Map { Decay a; float B; };

// What the workgroup's place in the launch means.
template <int V>
struct Place {
    int b, segment, group, groups, c, len, begin, end;      // tokens begin .. end - 1 of the segment
    bool live;                                             // the lane has channels
    __device__ __forceinline__ Place(const RecurrenceArgs &a, const RecurrenceShape &s)
    {
        const unsigned item = s.first + blockIdx.x, block = item % s.channel_blocks, rest = item / s.channel_blocks;
        segment = rest % s.segments;
        b = rest / s.segments;
        const int lane = threadIdx.x & ((1 << s.lanes_log2) - 1);
        group = threadIdx.x >> s.lanes_log2, groups = RECURRENCE_THREADS >> s.lanes_log2;
        c = ((int)(block << s.lanes_log2) + lane) * V;
        live = c < a.C;
        if (!live) c = 0;           // loads stay inside
        len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
        begin = segment * s.segment, end = min(a.T, begin + s.segment);
    }
};

// The decays and inputs of S tokens of the thread from token t on, past `end` as if they were not there.
template <class E, int V, int S>
struct Tile {
    Some<E, V> x[S], gate[S], input[S];
    __device__ __forceinline__ void load(const RecurrenceArgs &a, int b, int c, int t, int last)
    {
#pragma unroll
        for (int j = 0; j < S; ++j) {
            const long long at = min(t + j, last);
            x[j].load((const E *)a.x + b * a.sx.batch + at * a.sx.token + c);
            gate[j].load((const E *)a.gate + b * a.sgate.batch + at * a.sgate.token + c);
            if (a.input_gate) input[j].load((const E *)a.input_gate + b * a.sinput.batch + at * a.sinput.token + c);
        }
    }
};

template <class E, int V>
__device__ __forceinline__ void decay_and_input(const RecurrenceArgs &a, const float (&rate)[V], const Some<E, V> &x, const Some<E, V> &gate,
                                                const Some<E, V> &input, bool there, Decay (&decay)[V], float (&u)[V], float (&log)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float l = gate.value(e), full, less;
        if (a.rate) l = -rate[e] * sigmoid(l);
        l = there ? l : 0.0f;
        decay[e] = Decay(l, full, less);
        float w = x.value(e);
        if (a.input_gate) w *= sigmoid(input.value(e));
        if (a.normalise) w *= __builtin_amdgcn_sqrtf(less * (2.0f - less));       // 1 - a^2
        u[e] = there ? w : 0.0f;
        log[e] += part_of_sum(l);
    }
}

template <int V>
__device__ __forceinline__ void load_rates(const RecurrenceArgs &a, int c, float (&rate)[V])
{
#pragma unroll
    for (int e = 0; e < V; ++e) rate[e] = a.rate ? a.rate[c + e] : 0.0f;
}

template <class E, int V, int S>
__global__ __launch_bounds__(RECURRENCE_THREADS) void k_recurrence(RecurrenceArgs a, RecurrenceShape s)
{
    __shared__ Map maps[2][V][RECURRENCE_THREADS];
    const Place<V> at(a, s);
    const int lanes = 1 << s.lanes_log2, lane = threadIdx.x & (lanes - 1), tile = at.groups * S;
    float rate[V], carry[V];
    load_rates(a, at.c, rate);
    // the state before the segment
#pragma unroll
    for (int e = 0; e < V; ++e) carry[e] = a.initial ? a.initial[(long long)at.b * a.C + at.c + e] : 0.0f;
    for (int i = 0; i < at.segment; ++i) {
        const float2 *m = a.effects + ((long long)at.b * s.segments + i) * a.C + at.c;
#pragma unroll
        for (int e = 0; e < V; ++e) carry[e] = Decay::of_sum(m[e].x).of(carry[e], m[e].y);
    }
    const int last = max(min(at.len, at.end) - 1, 0);
    E *y = (E *)a.y + at.b * a.sy.batch + at.c;
    Tile<E, V, S> in;
    int t = at.begin + at.group * S, buffer = 0;
    if (at.begin < at.len) in.load(a, at.b, at.c, t, last);
    for (int start = at.begin; start < at.end; start += tile, t += tile, buffer ^= 1) {
        if (start >= at.len) {              // past the sequence: zeros, and nothing on the tape, which is not read there
            const float zeros[V] = {};
#pragma unroll
            for (int j = 0; j < S; ++j)
                if (t + j < at.end && at.live) store_some(y + (long long)(t + j) * a.sy.token, zeros);
            continue;
        }
        Decay d[S][V];
        float u[S][V], log[V] = {};
#pragma unroll
        for (int j = 0; j < S; ++j) decay_and_input<E, V>(a, rate, in.x[j], in.gate[j], in.input[j], t + j <= last, d[j], u[j], log);
        in.load(a, at.b, at.c, t + tile, last);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float B = u[0][e];
#pragma unroll
            for (int j = 1; j < S; ++j) B = d[j][e].of(B, u[j][e]);
            maps[buffer][e][threadIdx.x] = Map{Decay::of_sum(log[e]), B};
        }
        __syncthreads();                    // the other buffer is written next: a wave that is here has read it
        float h[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float all = carry[e];
            h[e] = all;
            for (int g = 0; g < at.groups; ++g) {
                h[e] = g == at.group ? all : h[e];
                const Map m = maps[buffer][e][g * lanes + lane];
                all = m.a.of(all, m.B);
            }
            carry[e] = all;
        }
        if (a.tape && (t & (RECURRENCE_TAPE - 1)) == 0 && t < at.end && at.live)
#pragma unroll
            for (int e = 0; e < V; ++e)
                a.tape[((long long)at.b * ((a.T + RECURRENCE_TAPE - 1) / RECURRENCE_TAPE) + t / RECURRENCE_TAPE) * a.C + at.c + e] = h[e];
#pragma unroll
        for (int j = 0; j < S; ++j) {
            float out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                h[e] = d[j][e].of(h[e], u[j][e]);
                out[e] = t + j < at.len ? h[e] : 0.0f;
            }
            if (t + j < at.end && at.live) store_some(y + (long long)(t + j) * a.sy.token, out);
        }
    }
    if (a.final_state && at.segment == (int)s.segments - 1 && at.group == 0 && at.live)
#pragma unroll
        for (int e = 0; e < V; ++e) a.final_state[(long long)at.b * a.C + at.c + e] = carry[e];
}

// What each segment does to the state (to the gradient that comes from later tokens, where BACKWARD): every group finds the map of its part, the first group joins them.
template <class E, int V, int S, bool BACKWARD>
__global__ __launch_bounds__(RECURRENCE_THREADS) void k_recurrence_effects(RecurrenceArgs a, RecurrenceShape s)
{
    __shared__ float2 maps[V][RECURRENCE_THREADS];       // logarithm of the decay, B
    const Place<V> at(a, s);
    if (at.segment == (BACKWARD ? 0 : (int)s.segments - 1)) return;          // nobody asks
    const int lanes = 1 << s.lanes_log2, lane = threadIdx.x & (lanes - 1);
    float rate[V], log[V] = {}, B[V] = {};
    load_rates(a, at.c, rate);
    const int stop = min(at.end, at.len), part = (s.segment / at.groups + S - 1) / S * S;
    const int from = at.begin + at.group * part, to = min(from + part, stop);
    const int last = max(stop - 1, 0);
    if (BACKWARD) {
        const E *dy = (const E *)a.dy + at.b * a.sy.batch + at.c;
        for (int t = from + part - S; t >= from && at.begin < at.len; t -= S) {
            Some<E, V> gate[S], in[S];
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const long long k = min(t + j, last);
                gate[j].load((const E *)a.gate + at.b * a.sgate.batch + k * a.sgate.token + at.c);
                in[j].load(dy + k * a.sy.token);
            }
#pragma unroll
            for (int j = S - 1; j >= 0; --j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float l = gate[j].value(e);
                    if (a.rate) l = -rate[e] * sigmoid(l);
                    const bool there = t + j < to;
                    l = there ? l : 0.0f;
                    float full, less;
                    B[e] = Decay(l, full, less).of(B[e] + (there ? in[j].value(e) : 0.0f));
                    log[e] += part_of_sum(l);
                }
        }
    } else {
        for (int t = from; t < to; t += S) {
            Tile<E, V, S> in;
            in.load(a, at.b, at.c, t, last);
#pragma unroll
            for (int j = 0; j < S; ++j) {
                Decay d[V];
                float u[V];
                decay_and_input<E, V>(a, rate, in.x[j], in.gate[j], in.input[j], t + j < to, d, u, log);
#pragma unroll
                for (int e = 0; e < V; ++e) B[e] = d[e].of(B[e], u[e]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) maps[e][threadIdx.x] = make_float2(log[e], B[e]);
    __syncthreads();
    if (at.group != 0 || !at.live) return;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float2 all = make_float2(0.0f, 0.0f);
        for (int i = 0; i < at.groups; ++i) {
            const float2 m = maps[e][(BACKWARD ? at.groups - 1 - i : i) * lanes + lane];
            all = make_float2(all.x + m.x, Decay::of_sum(m.x).of(all.y, m.y));
        }
        a.effects[((long long)at.b * s.segments + at.segment) * a.C + at.c + e] = all;
    }
}

template <class E, int V, int S>
__global__ __launch_bounds__(RECURRENCE_THREADS) void k_recurrence_back(RecurrenceArgs a, RecurrenceShape s)
{
    __shared__ Map maps[2][V][RECURRENCE_THREADS];
    __shared__ float later[2][V][RECURRENCE_THREADS];
    const Place<V> at(a, s);
    const int lanes = 1 << s.lanes_log2, lane = threadIdx.x & (lanes - 1), tile = at.groups * S;
    float rate[V], carry[V], drate[V];          // carry: the gradient that reaches the state before the tile from its later tokens
    load_rates(a, at.c, rate);
#pragma unroll
    for (int e = 0; e < V; ++e) carry[e] = a.d_final ? a.d_final[(long long)at.b * a.C + at.c + e] : 0.0f, drate[e] = 0.0f;
    for (int i = (int)s.segments - 1; i > at.segment; --i) {
        const float2 *m = a.effects + ((long long)at.b * s.segments + i) * a.C + at.c;
#pragma unroll
        for (int e = 0; e < V; ++e) carry[e] = Decay::of_sum(m[e].x).of(carry[e], m[e].y);
    }
    const int last = max(min(at.len, at.end) - 1, 0), tiles = (at.end - at.begin + tile - 1) / tile;
    const float *tape = a.tape + (long long)at.b * ((a.T + RECURRENCE_TAPE - 1) / RECURRENCE_TAPE) * a.C + at.c;
    const E *dy = (const E *)a.dy + at.b * a.sy.batch + at.c;
    E *dx = (E *)a.dx + at.b * a.sdx.batch + at.c, *dgate = (E *)a.dgate + at.b * a.sdgate.batch + at.c;
    E *dinput = (E *)a.dinput_gate + at.b * a.sdinput.batch + at.c;
    Tile<E, V, S> in;
    Some<E, V> in_dy[S];
    float in_h[V] = {};
    int start = at.begin + (tiles - 1) * tile, t = start + at.group * S, buffer = 0;
    const auto load = [&](int t, int start) {
        in.load(a, at.b, at.c, t, last);
#pragma unroll
        for (int j = 0; j < S; ++j) in_dy[j].load(dy + (long long)min(t + j, last) * a.sy.token);
#pragma unroll
        for (int e = 0; e < V; ++e) in_h[e] = tape[(long long)(start / RECURRENCE_TAPE) * a.C + e];
    };
    for (; start >= at.begin && start >= at.len; start -= tile, t -= tile) {      // past the sequence: zeros
        const float zeros[V] = {};
#pragma unroll
        for (int j = 0; j < S; ++j)
            if (t + j < at.end && at.live) {
                store_some(dx + (long long)(t + j) * a.sdx.token, zeros);
                store_some(dgate + (long long)(t + j) * a.sdgate.token, zeros);
                if (a.input_gate) store_some(dinput + (long long)(t + j) * a.sdinput.token, zeros);
            }
    }
    if (start >= at.begin) load(t, start);
    for (; start >= at.begin; start -= tile, t -= tile, buffer ^= 1) {
        // of each token: decay, input, and with the state before it known: dx = D by_x, dinput = D by_input, dl = D by_log, dgate = dl by_gate, drate = dl by_rate
        Decay d[S][V];
        float log[V] = {}, u[S][V], by_x[S][V], by_input[S][V], by_log[S][V], by_gate[S][V], by_rate[S][V], g[S][V];
#pragma unroll
        for (int j = 0; j < S; ++j) {
            const bool there = t + j <= last;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float l = in.gate[j].value(e), sigma, rest;
                by_gate[j][e] = 1.0f, by_rate[j][e] = 0.0f;
                if (a.rate) {
                    sigmoid(l, sigma, rest);
                    l = -rate[e] * sigma;
                    by_gate[j][e] = l * rest, by_rate[j][e] = -sigma;
                }
                l = there ? l : 0.0f;
                float full, less;
                d[j][e] = Decay(l, full, less);
                log[e] += part_of_sum(l);
                const float x = in.x[j].value(e);
                float open = 1.0f, left = 1.0f, by_open = 0.0f;
                if (a.input_gate) {
                    sigmoid(in.input[j].value(e), open, rest);
                    by_open = open * rest;
                }
                by_log[j][e] = 0.0f;
                if (a.normalise) {
                    left = __builtin_amdgcn_sqrtf(less * (2.0f - less));
                    by_log[j][e] = left == 0.0f ? 0.0f : -x * open * full * full * __builtin_amdgcn_rcpf(left);
                }
                by_x[j][e] = open * left, by_input[j][e] = x * left * by_open;
                u[j][e] = there ? x * by_x[j][e] : 0.0f;
                g[j][e] = there ? in_dy[j].value(e) : 0.0f;
            }
        }
        float first[V];
#pragma unroll
        for (int e = 0; e < V; ++e) first[e] = in_h[e];
        if (start > at.begin) load(t - tile, start - tile);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float B = u[0][e], R = 0.0f;
#pragma unroll
            for (int j = 1; j < S; ++j) B = d[j][e].of(B, u[j][e]);
#pragma unroll
            for (int j = S - 1; j >= 0; --j) R = d[j][e].of(g[j][e] + R);
            maps[buffer][e][threadIdx.x] = Map{Decay::of_sum(log[e]), B};
            later[buffer][e][threadIdx.x] = R;
        }
        __syncthreads();
        float h[V], D[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float all = first[e], back = carry[e];
            for (int i = 0; i < at.group; ++i) {
                const Map m = maps[buffer][e][i * lanes + lane];
                all = m.a.of(all, m.B);
            }
            for (int i = at.groups - 1; i >= 0; --i) {
                D[e] = i == at.group ? back : D[e];
                back = maps[buffer][e][i * lanes + lane].a.of(back, later[buffer][e][i * lanes + lane]);
            }
            h[e] = all, carry[e] = back;
        }
#pragma unroll
        for (int j = 0; j < S; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float kept = d[j][e].of(h[e]);
                by_log[j][e] += kept;
                h[e] = kept + u[j][e];
            }
#pragma unroll
        for (int j = S - 1; j >= 0; --j) {
            const bool there = t + j < at.len;
            float ox[V], og[V], oi[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                D[e] += g[j][e];
                const float dl = D[e] * by_log[j][e];
                ox[e] = there ? D[e] * by_x[j][e] : 0.0f;
                oi[e] = there ? D[e] * by_input[j][e] : 0.0f;
                og[e] = there ? dl * by_gate[j][e] : 0.0f;
                drate[e] += there ? dl * by_rate[j][e] : 0.0f;
                D[e] = d[j][e].of(D[e]);
            }
            if (t + j < at.end && at.live) {
                store_some(dx + (long long)(t + j) * a.sdx.token, ox);
                store_some(dgate + (long long)(t + j) * a.sdgate.token, og);
                if (a.input_gate) store_some(dinput + (long long)(t + j) * a.sdinput.token, oi);
            }
        }
    }
    if (a.d_initial && at.segment == 0 && at.group == 0 && at.live)
#pragma unroll
        for (int e = 0; e < V; ++e) a.d_initial[(long long)at.b * a.C + at.c + e] = carry[e];
    if (!a.drate) return;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) later[0][e][threadIdx.x] = drate[e];
    __syncthreads();
    if (at.group == 0 && at.live)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float sum = 0.0f;
            for (int i = 0; i < at.groups; ++i) sum += later[0][e][i * lanes + lane];
            a.partial[((long long)at.b * s.segments + at.segment) * a.C + at.c + e] = sum;
        }
}

}  // namespace tfno
