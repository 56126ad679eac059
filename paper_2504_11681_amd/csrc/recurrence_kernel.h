// h = a h + u for every channel, a = exp(l), u = x sigmoid(input_gate) sqrt(1 - exp(2 l)), and its gradient
//
//   D_t = dy_t + a_{t+1} D_{t+1},   du = D,   dl = D a h_{t-1} - D x sigmoid(input_gate) a^2 / sqrt(1 - a^2).
//
// Every input is read once and every output written once; a value takes 46 vector instructions (56 where groups of 32 lanes are joined, backward 100), five of them of the slow kind
// (exp2, 1/x, square root), so with BF16 both sides are near: 256 x 1024 tokens of 128 channels 62 us (269 MB, 4.3 TB/s; vector pipes busy for 44).  A workgroup takes 64 or 32 neighbouring channels and walks through a sequence
// in tiles; a tile is shared out over time among groups of as many lanes, each with S tokens in a row, whose loads are all under way while the tile before is worked on.  A
// group makes of its tokens one map h -> a h + B (backward also e -> a e + R for what comes from later tokens); the maps are joined along the wave by shuffles and along the
// workgroup in LDS, and each group then walks its tokens from the state that the maps before it give.  Sequences too few to fill the chip are cut into segments, whose maps a
// kernel of its own finds first.  One channel a lane: with two the maps of a lane are joined twice and the gradient has 256 registers.  Workgroups that are neighbours in memory share an XCD: half lines of
// channels were read twice otherwise (4 x 2048 tokens of 2048 channels, both directions, 143 -> 129 us).
#pragma once
#include "gates.h"
#include "recurrence.h"

namespace tfno {

// Tokens of a group in a tile.  Forward four waves a SIMD have registers for that (with 16, which two have, 70 -> 82 us for the batch above, each time on other inputs); backward two
// (with 4 129 -> 146 us for the two directions above: twice the joining).
constexpr int RECURRENCE_TOKENS = 8, RECURRENCE_TOKENS_BACK = 8;

// What a kernel knows of its gates: ALL has rates, an input gate and `normalise`, NONE neither, RATES all but an input gate; ANY asks.
enum { ANY = 0, ALL = 1, NONE = 2, RATES = 3 };
struct RecurrenceShape {
    int lanes_log2;                 // lanes of a group
    unsigned channel_blocks, segments, first;
    int segment;                    // tokens of a segment
};

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// A decay a = exp(l).  Near 1, where states last long, its distance from 1 is what matters: it is kept as -(1 - a), sign bit set, and from the series
// -l (1 + l/2 + l^2/6 + ...), whose first term left out is l^5 / 720 of the whole, 4e-8 at the border; rounded to a float32 itself, a decay of 0.9999 would be
// 3e-4 of its distance off, always to the same side.  Elsewhere (and above 1) it is a itself, at least 2^-126.  +0 is a decay of exactly 0, which forgets the state whatever it
// holds: where exp(l) rounds to 0 in float32.
constexpr float NOTHING_LEFT = -104.0f, HARDLY = -87.0f, LEAST = 1.17549435e-38f;
struct Decay {
    float at;
    __device__ __forceinline__ Decay() {}
    // For l no less than HARDLY (or NaN); a and 1 - a too.
    __device__ __forceinline__ Decay(float l, float &a, float &less)
    {
        float p = fmaf(l, 1.0f / 120.0f, 1.0f / 24.0f);
        p = fmaf(l, p, 1.0f / 6.0f);
        p = fmaf(l, p, 0.5f);
        p = fmaf(l, p, 1.0f) * l;
        a = __builtin_amdgcn_exp2f(l * LOG2E);
        const bool near = __float_as_uint(l) - 0x80000000u < 0x3e000000u;      // -0.125 < l <= -0
        less = near ? -p : 1.0f - a;
        at = near ? p : a;
    }
    // For any l, which is no more than HARDLY.
    __device__ __forceinline__ void hardly(float l) { at = l < NOTHING_LEFT ? 0.0f : LEAST; }
    __device__ __forceinline__ bool forgets() const { return __float_as_uint(at) == 0; }
    // a h, and a h + u
    __device__ __forceinline__ float of(float h) const { return forgets() ? 0.0f : fmaf(at, h, (int)__float_as_uint(at) < 0 ? h : 0.0f); }
    __device__ __forceinline__ float of(float h, float u) const { return forgets() ? u : fmaf(at, h, ((int)__float_as_uint(at) < 0 ? h : 0.0f) + u); }
};
// The same with what the sign bit says as a factor, for the walks through tokens: two instructions where none of a wave's tokens forgets, which nearly always holds.
struct TokenDecay {
    float at, whole;
    __device__ __forceinline__ TokenDecay() {}
    __device__ __forceinline__ TokenDecay(float l, float &a, float &less)
    {
        const Decay d(l, a, less);
        at = d.at, whole = (int)__float_as_uint(d.at) < 0 ? 1.0f : 0.0f;
    }
    __device__ __forceinline__ void hardly(float l) { at = l < NOTHING_LEFT ? 0.0f : LEAST; }
    template <bool RESETS>
    __device__ __forceinline__ float of(float h) const { return RESETS && __float_as_uint(at) == 0 ? 0.0f : fmaf(at, h, whole * h); }
    template <bool RESETS>
    __device__ __forceinline__ float of(float h, float u) const { return RESETS && __float_as_uint(at) == 0 ? u : fmaf(at, h, fmaf(whole, h, u)); }
};
// The logarithm of a token's decay.
__device__ __forceinline__ float log_of(bool rated, float rate, float gate) { return rated ? -rate * sigmoid(gate) : gate; }

__device__ __forceinline__ void set(float &v, float to) { v = to; }
__device__ __forceinline__ void set(bf16 &v, float to) { v.bits = (unsigned short)(__float_as_uint(to) >> 16); }       // 0 and infinity
// Tokens as if they were not there: they add nothing, and their decay is 1.
template <int S, class E>
__device__ __forceinline__ void leave_out(bool rated, int t, int last, E (&x)[S], E (&gate)[S])
{
#pragma unroll
    for (int j = 0; j < S; ++j)
        if (t + j > last) set(x[j], 0.0f), set(gate[j], rated ? -INFINITY : 0.0f);
}
// What tokens in their order do to the state before them, h -> a h + B: their decays' product, its distance from 1 without taking the difference, and B.
struct Span {
    float a, less, B;
    __device__ __forceinline__ void longer(float more, float more_less) { less = fmaf(a, more_less, less), a *= more; }
    __device__ __forceinline__ Decay decay() const
    {
        Decay d;
        d.at = less > 0.0f && a > 0.5f ? -less : a;
        return d;
    }
};
// A product that underflows does not forget; one with a 0 in it does, whatever else is in it: 0 times a NaN or an infinity is no decay, and what such tokens leave behind the 0 is in B.
__device__ __forceinline__ Span after(Span first, Span second)
{
    const float a = first.a * second.a;
    return Span{first.a == 0.0f || second.a == 0.0f ? 0.0f : a == 0.0f ? LEAST : a, fmaf(first.a, second.less, first.less), second.decay().of(first.B, second.B)};
}
struct Joined {
    Decay a;
    float B;
    __device__ __forceinline__ float of(float h) const { return a.of(h, B); }
};
// Decays that are hardly more than 0, or not: seldom, and then looked for in a wave's whole tile, whose gates are read again.  A product that is 0 or NaN (0 times a NaN or an
// infinity) may have one in it.
__device__ __forceinline__ bool may_reset(Span own) { return !(own.a > 0.0f); }
template <int S, class E>
__device__ __forceinline__ bool find_resets(bool rated, float rate, const E (&gate)[S], int t, int last, TokenDecay (&d)[S], Span &own)
{
    bool found = false;
#pragma unroll
    for (int j = 0; j < S; ++j) {
        const float l = t + j <= last ? log_of(rated, rate, to_float(gate[j])) : 0.0f;
        if (l < HARDLY) d[j].hardly(l);
        found = found || l < NOTHING_LEFT;
    }
    own.a = found ? 0.0f : own.a == 0.0f ? LEAST : own.a;
    return __any(found);
}

__device__ __forceinline__ Joined joined(Span s) { return Joined{s.decay(), s.B}; }

__device__ __forceinline__ Span moved(Span m, int d, bool back)
{
    return Span{back ? __shfl_down(m.a, d, 64) : __shfl_up(m.a, d, 64), back ? __shfl_down(m.less, d, 64) : __shfl_up(m.less, d, 64),
                back ? __shfl_down(m.B, d, 64) : __shfl_up(m.B, d, 64)};
}
// What the groups of a wave do, each joined with those before it (behind it, where BACK), without its own, where `others` is true on return; and all of them, in the last group.
template <bool BACK>
__device__ __forceinline__ bool join(int lanes, Span own, Span &others, Span &all)
{
    const int lane = threadIdx.x & 63, order = BACK ? 63 - lane : lane;
    for (int d = lanes; d < 64; d <<= 1) {
        const Span p = moved(own, d, BACK);
        if (order >= d) own = after(p, own);
    }
    if (lanes < 64) others = moved(own, lanes, BACK);
    all = own;
    return order >= lanes;
}

// What the workgroup's place in the launch means.
struct Place {
    int b, segment, lane, wave, group, c, len, begin, end;      // tokens begin .. end - 1 of the segment; group: in its wave
    bool live;                                                 // the lane has a channel
    __device__ __forceinline__ Place(const RecurrenceArgs &a, const RecurrenceShape &s)
    {
        const unsigned place = xcd_contiguous(blockIdx.x, gridDim.x);
        const unsigned item = s.first + place, block = item % s.channel_blocks, rest = item / s.channel_blocks;
        segment = rest % s.segments;
        b = rest / s.segments;
        lane = threadIdx.x & ((1 << s.lanes_log2) - 1);
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        group = (threadIdx.x & 63) >> s.lanes_log2;
        c = (int)(block << s.lanes_log2) + lane;
        live = c < a.C;
        if (!live) c = 0;           // loads stay inside
        len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
        begin = segment * s.segment, end = min(a.T, begin + s.segment);
    }
};

// The state before the segment (the gradient behind it, where BACK): the maps of the other segments, shared out among the workgroup's groups.
template <bool BACK, int WAVES>
__device__ __forceinline__ float through_segments(const RecurrenceArgs &a, const RecurrenceShape &s, const Place &at, float start, Joined (&maps)[WAVES][64])
{
    const int n = BACK ? (int)s.segments - 1 - at.segment : at.segment, groups = 64 >> s.lanes_log2, lanes = 1 << s.lanes_log2;
    if (n == 0) return start;
    const int each = (n + groups * WAVES - 1) / (groups * WAVES), from = (at.wave * groups + at.group) * each;
    Span own = {1.0f, 0.0f, 0.0f};
    const Span *effects = (const Span *)a.effects;
    for (int i = from; i < min(from + each, n); i += 8) {          // eight on their way at once
        Span some[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int which = min(i + k, n - 1);
            some[k] = effects[((long long)at.b * s.segments + (BACK ? (int)s.segments - 1 - which : which)) * a.C + at.c];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k < min(from + each, n)) own = after(own, some[k]);
    }
    Span others, all;
    join<false>(lanes, own, others, all);
    if ((int)(threadIdx.x & 63) >= 64 - lanes) maps[at.wave][at.lane] = joined(all);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) start = maps[w][at.lane].of(start);
    __syncthreads();
    return start;
}

// A tensor's elements of the thread: S tokens from `first` (of the wave) + `ahead` (of its group) on, in one channel.  A token's address is scalar, a lane's offset from it has 32
// bits of bytes, the same for all: tokens of a wave, 16 at most, are less than 2^24 elements apart.
template <class E>
struct Row {
    char *at;                   // of the sequence
    long long wide;             // bytes from token to token
    unsigned offset;            // of the lane
    __device__ __forceinline__ Row(const void *p, const Strides &s, int b, int c, int ahead)
        : at((char *)p + b * s.batch * (long long)sizeof(E)), wide(s.token * (long long)sizeof(E)), offset((unsigned)ahead * (unsigned)wide + (unsigned)c * (unsigned)sizeof(E)) {}
    // The lane's offset, made to look new each time: kept as an address it would be two registers a token instead of none.
    __device__ __forceinline__ unsigned here() const
    {
        unsigned o = offset;
        asm volatile("" : "+v"(o));
        return o;
    }
    // From a token's scalar offset to its element, and on to the next token.
    __device__ __forceinline__ long long from(int token) const { return token * wide; }
    __device__ __forceinline__ E *next(long long &k, unsigned here) const
    {
        E *p = (E *)(at + k + here);
        k += wide;
        asm volatile("" : "+s"(k));         // a sum, not a product for every token
        return p;
    }
    __device__ __forceinline__ E *before(long long &k, unsigned here) const
    {
        E *p = (E *)(at + k + here);
        k -= wide;
        asm volatile("" : "+s"(k));
        return p;
    }
    // S tokens; those past the last one that counts, which is not negative, are that one again: their values are not used.
    template <bool FULL, int S>
    __device__ __forceinline__ void load(int first, int ahead, int c, int last, E (&v)[S]) const
    {
        if (FULL) {
            const unsigned o = here();
            long long k = from(first);
#pragma unroll
            for (int j = 0; j < S; ++j) v[j] = *next(k, o);
            // the loads of both kinds stay apart: as common code behind them the compiler would take addresses of 64 bits from either
            asm volatile("; whole");
        } else {
            const char *p = at + min(first, last) * wide;
            unsigned o = c * (unsigned)sizeof(E) + (unsigned)(min(first + ahead, last) - min(first, last)) * (unsigned)wide;
#pragma unroll
            for (int j = 0; j < S; ++j) {
                v[j] = *(const E *)(p + o);
                o += first + ahead + j < last ? (unsigned)wide : 0u;
            }
            asm volatile("; cut");
        }
    }
};

template <class E, int GATES, int S, int THREADS>
__global__ __launch_bounds__(THREADS) void k_recurrence(RecurrenceArgs a, RecurrenceShape s)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ Joined maps[2][WAVES][64];
    __shared__ float state[2][64];          // before a tile
    const Place at(a, s);
    const int lanes = 1 << s.lanes_log2, ahead = at.group * S, per_wave = (64 >> s.lanes_log2) * S, tile = per_wave * WAVES;
    const bool rated = GATES ? GATES != NONE : a.rate != nullptr, gated = GATES ? GATES == ALL : a.input_gate != nullptr, normalise = GATES ? GATES != NONE : a.normalise;
    const float rate = rated ? a.rate[at.c] : 0.0f;
    // the state before the segment
    float carry = a.initial ? a.initial[(long long)at.b * a.C + at.c] : 0.0f;
    carry = through_segments<false, WAVES>(a, s, at, carry, maps[0]);
    if (at.wave == 0 && at.group == 0) state[1][at.lane] = carry;
    if (a.final_state && at.len == 0 && at.segment == 0 && at.wave == 0 && at.group == 0 && at.live) a.final_state[(long long)at.b * a.C + at.c] = carry;
    const int last = max(min(at.len, at.end) - 1, 0), tape_every = 1 << a.tape_log2, tape_rows = (a.T + tape_every - 1) >> a.tape_log2;
    const Row<E> x(a.x, a.sx, at.b, at.c, ahead), gate(a.gate, a.sgate, at.b, at.c, ahead), input(gated ? a.input_gate : a.x, gated ? a.sinput : a.sx, at.b, at.c, ahead);
    const Row<E> y(a.y, a.sy, at.b, at.c, ahead);
    E in_x[S], in_gate[S], in_input[S];
    const auto load = [&](int first) {          // of the wave
        const auto all = [&](auto full) {
            x.template load<full.value>(first, ahead, at.c, last, in_x);
            gate.template load<full.value>(first, ahead, at.c, last, in_gate);
            if (gated) input.template load<full.value>(first, ahead, at.c, last, in_input);
        };
        if (first + per_wave - 1 <= last) all(Yes());
        else all(No());
    };
    int first = at.begin + at.wave * per_wave, buffer = 0;
    if (at.begin < at.len) load(first);
    for (int start = at.begin; start < at.end; start += tile, first += tile, buffer ^= 1) {
        const int t = first + ahead;
        if (start >= at.len) {
            buffer ^= 1;                    // the state stays where it is
            long long k = y.from(first);    // past the sequence: zeros, and nothing on the tape, which is not read there
#pragma unroll
            for (int j = 0; j < S; ++j) {
                E *p = y.next(k, y.offset);
                if (t + j < at.end && at.live) store_element(p, 0.0f);
            }
            continue;
        }
        TokenDecay d[S];
        float u[S];
        Span own = {1.0f, 0.0f, 0.0f};
        if (first + per_wave - 1 > last) leave_out(rated, t, last, in_x, in_gate);
        const unsigned next_x = x.here(), next_gate = gate.here(), next_input = input.here();
        long long kx = x.from(first + tile), kg = gate.from(first + tile), ki = input.from(first + tile);
        // a token's place in the registers is free once its gates are made: the next tile's is asked for there and then, so that its latency lies under all the rest
        const auto gates = [&](auto next) {
#pragma unroll
            for (int j = 0; j < S; ++j) {
                float part, less;
                const float l = log_of(rated, rate, to_float(in_gate[j]));
                d[j] = TokenDecay(l, part, less);
                u[j] = to_float(in_x[j]);
                if (gated) u[j] *= sigmoid(to_float(in_input[j]));
                if (normalise) u[j] *= __builtin_amdgcn_sqrtf(less * (2.0f - less));       // 1 - a^2
                own.longer(part, less);
                if (next.value) {
                    in_x[j] = *x.next(kx, next_x);
                    in_gate[j] = *gate.next(kg, next_gate);
                    if (gated) in_input[j] = *input.next(ki, next_input);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (first + tile + per_wave - 1 <= last) {
            gates(Yes());
        } else {
            gates(No());
            load(first + tile);
        }
        bool resets = false;
        if (__any(may_reset(own))) {
            E again[S];
            gate.template load<false>(first, ahead, at.c, last, again);
            resets = find_resets(rated, rate, again, t, last, d, own);
        }
        const auto run = [&](float h, auto can, auto each) {
#pragma unroll
            for (int j = 0; j < S; ++j) each(j, h = d[j].template of<can.value>(h, u[j]));
            return h;
        };
        const auto nothing = [](int, float) {};
        own.B = resets ? run(0.0f, Yes(), nothing) : run(0.0f, No(), nothing);
        Span before, all;
        const bool some = join<false>(lanes, own, before, all);
        if ((int)(threadIdx.x & 63) >= 64 - lanes) maps[buffer][at.wave][at.lane] = joined(all);
        __syncthreads();                    // the other buffer is written next: a wave that is here has read it
        float h = state[buffer ^ 1][at.lane];
        for (int w = 0; w < at.wave; ++w) h = maps[buffer][w][at.lane].of(h);
        if (lanes < 64) h = some ? before.decay().of(h, before.B) : h;
        if (a.tape && (t & (tape_every - 1)) == 0 && t < at.end && at.live) a.tape[((long long)at.b * tape_rows + (t >> a.tape_log2)) * a.C + at.c] = h;
        const unsigned o = y.here();
        long long k = y.from(first);
        if (!resets && first + per_wave <= at.end && first + per_wave <= at.len) {
            h = run(h, No(), [&](int, float v) {
                E *p = y.next(k, o);
                if (at.live) store_element(p, v);
            });
        } else {
            h = run(h, Yes(), [&](int j, float v) {
                E *p = y.next(k, o);
                if (t + j < at.end && at.live) store_element(p, t + j < at.len ? v : 0.0f);
            });
        }
        if (a.final_state && at.live && t < at.len && t + S >= at.len) a.final_state[(long long)at.b * a.C + at.c] = h;
        // the last group has the state behind the tile; who reads it is past the next barrier
        if (at.wave == WAVES - 1 && (int)(threadIdx.x & 63) >= 64 - lanes) state[buffer][at.lane] = h;
    }
}

// What each segment does to the state (to the gradient that comes from later tokens, where BACKWARD): every wave goes through a part of it by itself.
template <class E, int GATES, int S, int THREADS, bool BACKWARD>
__global__ __launch_bounds__(THREADS) void k_recurrence_effects(RecurrenceArgs a, RecurrenceShape s)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ Span maps[WAVES][64];
    const Place at(a, s);
    if (at.segment == (BACKWARD ? 0 : (int)s.segments - 1)) return;          // nobody asks
    const int lanes = 1 << s.lanes_log2, ahead = at.group * S, per_wave = (64 >> s.lanes_log2) * S, part = s.segment / WAVES;      // whole tiles, so whole rounds of a wave
    const bool rated = GATES ? GATES != NONE : a.rate != nullptr, gated = !BACKWARD && (GATES ? GATES == ALL : a.input_gate != nullptr), normalise = !BACKWARD && (GATES ? GATES != NONE : a.normalise);
    const float rate = rated ? a.rate[at.c] : 0.0f;
    const int last = max(min(at.end, at.len) - 1, 0), from = at.begin + at.wave * part, end = min(from + part, min(at.end, at.len));
    // in: x, or dy
    const Row<E> in(BACKWARD ? a.dy : a.x, BACKWARD ? a.sy : a.sx, at.b, at.c, ahead), gate(a.gate, a.sgate, at.b, at.c, ahead);
    const Row<E> input(gated ? a.input_gate : a.gate, gated ? a.sinput : a.sgate, at.b, at.c, ahead);
    E in_x[S], in_gate[S], in_input[S];
    const auto load = [&](int first) {
        const auto all = [&](auto full) {
            in.template load<full.value>(first, ahead, at.c, last, in_x);
            gate.template load<full.value>(first, ahead, at.c, last, in_gate);
            if (gated) input.template load<full.value>(first, ahead, at.c, last, in_input);
        };
        if (first + per_wave - 1 <= last) all(Yes());
        else all(No());
    };
    Span sum = {1.0f, 0.0f, 0.0f};
    const int rounds = end > from ? (end - from + per_wave - 1) / per_wave : 0;
    if (rounds > 0) load(BACKWARD ? from + (rounds - 1) * per_wave : from);
    for (int i = 0; i < rounds; ++i) {
        const int first = from + (BACKWARD ? rounds - 1 - i : i) * per_wave, t = first + ahead;
        if (first + per_wave - 1 > last) leave_out(rated, t, last, in_x, in_gate);
        TokenDecay d[S];
        float u[S];
        Span own = {1.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < S; ++j) {
            float decay, less;
            const float l = log_of(rated, rate, to_float(in_gate[j]));
            d[j] = TokenDecay(l, decay, less);
            u[j] = to_float(in_x[j]);
            if (gated) u[j] *= sigmoid(to_float(in_input[j]));
            if (normalise) u[j] *= __builtin_amdgcn_sqrtf(less * (2.0f - less));
            own.longer(decay, less);
        }
        if (i + 1 < rounds) load(BACKWARD ? first - per_wave : first + per_wave);
        if (__any(may_reset(own))) {
            E again[S];
            gate.template load<false>(first, ahead, at.c, last, again);
            find_resets(rated, rate, again, t, last, d, own);
        }
#pragma unroll
        for (int j = 0; j < S; ++j) own.B = BACKWARD ? d[S - 1 - j].template of<true>(own.B + u[S - 1 - j]) : d[j].template of<true>(own.B, u[j]);
        Span others, all;
        join<BACKWARD>(lanes, own, others, all);
        sum = after(sum, all);
    }
    if (BACKWARD ? (int)(threadIdx.x & 63) < lanes : (int)(threadIdx.x & 63) >= 64 - lanes) maps[at.wave][at.lane] = sum;
    __syncthreads();
    if (at.wave != 0 || at.group != 0 || !at.live) return;
    Span all = {1.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all = after(all, maps[BACKWARD ? WAVES - 1 - w : w][at.lane]);
    ((Span *)a.effects)[((long long)at.b * s.segments + at.segment) * a.C + at.c] = all;
}

template <class E, int GATES, int S, int THREADS>
__global__ __launch_bounds__(THREADS) void k_recurrence_back(RecurrenceArgs a, RecurrenceShape s)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ Joined maps[2][WAVES][64];
    __shared__ float later[2][WAVES][64];
    __shared__ float gradient[2][64];       // that reaches a tile from its later tokens
    const Place at(a, s);
    const int lanes = 1 << s.lanes_log2, ahead = at.group * S, per_wave = (64 >> s.lanes_log2) * S, tile = per_wave * WAVES;
    const bool rated = GATES ? GATES != NONE : a.rate != nullptr, gated = GATES ? GATES == ALL : a.input_gate != nullptr, normalise = GATES ? GATES != NONE : a.normalise;
    const float rate = rated ? a.rate[at.c] : 0.0f;
    float drate = 0.0f, carry = a.d_final ? a.d_final[(long long)at.b * a.C + at.c] : 0.0f;      // carry: the gradient that reaches the state before the tile from its later tokens
    carry = through_segments<true, WAVES>(a, s, at, carry, maps[0]);
    if (at.wave == 0 && at.group == 0) gradient[1][at.lane] = carry;
    const int last = max(min(at.len, at.end) - 1, 0), tiles = (at.end - at.begin + tile - 1) / tile;
    const float *tape = a.tape + (long long)at.b * ((a.T + (1 << a.tape_log2) - 1) >> a.tape_log2) * a.C + at.c;      // a tile begins where one is
    const Row<E> x(a.x, a.sx, at.b, at.c, ahead), gate(a.gate, a.sgate, at.b, at.c, ahead), input(gated ? a.input_gate : a.x, gated ? a.sinput : a.sx, at.b, at.c, ahead);
    const Row<E> dy(a.dy, a.sy, at.b, at.c, ahead);
    const Row<E> dx(a.dx, a.sdx, at.b, at.c, ahead), dgate(a.dgate, a.sdgate, at.b, at.c, ahead), dinput(a.dinput_gate, a.sdinput, at.b, at.c, ahead);
    E in_x[S], in_gate[S], in_input[S], in_dy[S];
    float in_h = 0.0f;
    const auto load = [&](int first, int start) {
        const auto all = [&](auto full) {
            x.template load<full.value>(first, ahead, at.c, last, in_x);
            gate.template load<full.value>(first, ahead, at.c, last, in_gate);
            dy.template load<full.value>(first, ahead, at.c, last, in_dy);
            if (gated) input.template load<full.value>(first, ahead, at.c, last, in_input);
        };
        if (first + per_wave - 1 <= last) all(Yes());
        else all(No());
        in_h = tape[(long long)(start >> a.tape_log2) * a.C];
    };
    int start = at.begin + (tiles - 1) * tile, first = start + at.wave * per_wave, buffer = 0;
    for (; start >= at.begin && start >= at.len; start -= tile, first -= tile) {    // past the sequence: zeros
        long long kx = dx.from(first), kg = dgate.from(first), ki = dinput.from(first);
#pragma unroll
        for (int j = 0; j < S; ++j) {
            E *px = dx.next(kx, dx.offset), *pg = dgate.next(kg, dgate.offset), *pi = dinput.next(ki, dinput.offset);
            if (first + ahead + j < at.end && at.live) {
                store_element(px, 0.0f);
                store_element(pg, 0.0f);
                if (gated) store_element(pi, 0.0f);
            }
        }
    }
    if (start >= at.begin) load(first, start);
    for (; start >= at.begin; start -= tile, first -= tile, buffer ^= 1) {
        const int t = first + ahead;
        // of each token: decay, input, and with the state before it known: dx = D by_x, dinput = D by_input, dl = D by_log, dgate = dl by_gate, drate = dl by_rate
        TokenDecay d[S];
        float u[S], by_x[S], by_input[S], by_log[S], by_gate[S], by_rate[S], g[S];
        Span own = {1.0f, 0.0f, 0.0f};
        if (first + per_wave - 1 > last) {
            leave_out(rated, t, last, in_x, in_gate);
#pragma unroll
            for (int j = 0; j < S; ++j)
                if (t + j > last) set(in_dy[j], 0.0f), set(in_input[j], 0.0f);
        }
        const unsigned next_x = x.here(), next_gate = gate.here(), next_input = input.here(), next_dy = dy.here();
        long long kx = x.from(first - tile), kg = gate.from(first - tile), ki = input.from(first - tile), kd = dy.from(first - tile);
        const auto gates = [&](auto next) {
#pragma unroll
            for (int j = 0; j < S; ++j) {
                float l = to_float(in_gate[j]), part, less, sigma, rest;
                by_gate[j] = 1.0f, by_rate[j] = 0.0f;
                if (rated) {
                    sigmoid(l, sigma, rest);
                    l = -rate * sigma;
                    by_gate[j] = l * rest, by_rate[j] = -sigma;
                }
                d[j] = TokenDecay(l, part, less);
                own.longer(part, less);
                const float in = to_float(in_x[j]);
                float open = 1.0f, left = 1.0f, by_open = 0.0f;
                if (gated) {
                    sigmoid(to_float(in_input[j]), open, rest);
                    by_open = open * rest;
                }
                by_log[j] = 0.0f;
                if (normalise) {
                    left = __builtin_amdgcn_sqrtf(less * (2.0f - less));
                    by_log[j] = left == 0.0f ? 0.0f : -in * open * part * part * __builtin_amdgcn_rcpf(left);
                }
                by_x[j] = open * left, by_input[j] = in * left * by_open;
                u[j] = in * by_x[j];
                g[j] = to_float(in_dy[j]);
                if (next.value) {
                    in_x[j] = *x.next(kx, next_x);
                    in_gate[j] = *gate.next(kg, next_gate);
                    in_dy[j] = *dy.next(kd, next_dy);
                    if (gated) in_input[j] = *input.next(ki, next_input);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // the tile before is whole wherever there is one, since tokens are missing at a sequence's end alone
        const float state = in_h;
        if (start > at.begin) {
            gates(Yes());
            in_h = tape[(long long)((start - tile) >> a.tape_log2) * a.C];
        } else {
            gates(No());
        }
        bool resets = false;
        if (__any(may_reset(own))) {
            E again[S];
            gate.template load<false>(first, ahead, at.c, last, again);
            resets = find_resets(rated, rate, again, t, last, d, own);
        }
        const auto local = [&](auto can) {
            float R = 0.0f;
#pragma unroll
            for (int j = 0; j < S; ++j) own.B = d[j].template of<can.value>(own.B, u[j]);
#pragma unroll
            for (int j = S - 1; j >= 0; --j) R = d[j].template of<can.value>(g[j] + R);
            return R;
        };
        const float R = resets ? local(Yes()) : local(No());
        Span before, behind, all, all_back;
        const bool some_before = join<false>(lanes, own, before, all);
        const bool some_behind = join<true>(lanes, Span{own.a, own.less, R}, behind, all_back);
        if ((int)(threadIdx.x & 63) >= 64 - lanes) maps[buffer][at.wave][at.lane] = joined(all);
        if ((int)(threadIdx.x & 63) < lanes) later[buffer][at.wave][at.lane] = all_back.B;
        __syncthreads();
        float h = state, D = gradient[buffer ^ 1][at.lane];
        for (int w = 0; w < at.wave; ++w) h = maps[buffer][w][at.lane].of(h);
        for (int w = WAVES - 1; w > at.wave; --w) D = maps[buffer][w][at.lane].a.of(D, later[buffer][w][at.lane]);
        if (lanes < 64) {
            h = some_before ? before.decay().of(h, before.B) : h;
            D = some_behind ? behind.decay().of(D, behind.B) : D;
        }
        const unsigned ox = dx.here(), og = dgate.here(), oi = dinput.here();
        long long qx = dx.from(first + S - 1), qg = dgate.from(first + S - 1), qi = dinput.from(first + S - 1);
        const auto walk = [&](auto can, auto full) {
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const float kept = d[j].template of<can.value>(h);
                by_log[j] += kept;
                h = kept + u[j];
            }
#pragma unroll
            for (int j = S - 1; j >= 0; --j) {
                const bool there = full.value || t + j < at.len;
                D += g[j];
                const float dl = D * by_log[j];
                drate += there ? dl * by_rate[j] : 0.0f;
                E *px = dx.before(qx, ox), *pg = dgate.before(qg, og), *pi = dinput.before(qi, oi);
                if ((full.value || t + j < at.end) && at.live) {
                    store_element(px, there ? D * by_x[j] : 0.0f);
                    store_element(pg, there ? dl * by_gate[j] : 0.0f);
                    if (gated) store_element(pi, there ? D * by_input[j] : 0.0f);
                }
                D = d[j].template of<can.value>(D);
            }
        };
        if (!resets && first + per_wave <= at.end && first + per_wave <= at.len) walk(No(), Yes());
        else walk(Yes(), No());
        // the first group has the gradient that reaches the state before the tile; who reads it is past the next barrier
        if (at.wave == 0 && at.group == 0) gradient[buffer][at.lane] = D;
    }
    // that of the first token is the first group's own
    if (a.d_initial && at.segment == 0 && at.wave == 0 && at.group == 0 && at.live) a.d_initial[(long long)at.b * a.C + at.c] = gradient[buffer ^ 1][at.lane];
    if (!a.drate) return;
    // the groups' parts in their order
    for (int k = lanes; k < 64; k <<= 1) drate += __shfl_xor(drate, k, 64);
    __syncthreads();
    later[0][at.wave][threadIdx.x & 63] = drate;
    __syncthreads();
    if (at.wave == 0 && at.group == 0 && at.live) {
        float sum = 0.0f;
        for (int w = 0; w < WAVES; ++w) sum += later[0][w][at.lane];
        a.partial[((long long)at.b * s.segments + at.segment) * a.C + at.c] = sum;
    }
}

}  // namespace tfno
