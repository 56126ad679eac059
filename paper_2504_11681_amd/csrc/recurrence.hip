// Launches of the gated linear recurrence, and its step for one token.
#include "columnsums.h"
#include "recurrence_kernel.h"

#include <algorithm>

namespace tfno {

namespace {

constexpr unsigned RECURRENCE_LAUNCH = 1u << 21;            // workgroups: a launch takes less than 2^32 threads

struct Geometry {
    RecurrenceShape s;
    int threads;
};

// Lanes of a group, threads of a workgroup and segments: whole lines of channels and small workgroups where these fill the chip, else more of a sequence in a workgroup, then half
// lines, then segments, in workgroups that are small again (one sequence of 16384 tokens of 512 channels: 64 segments 29 us, 32 31, 128 35; 5 x 777 of 205 in float32 39 -> 32
// with 256 threads instead of 512).
Geometry shape_of(int B, int T, int C, bool bf16, bool back, int tokens)
{
    Geometry g{};
    RecurrenceShape &s = g.s;
    s.lanes_log2 = 6, g.threads = 256;
    const auto blocks = [&] { return (long long)B * ((C + (1 << s.lanes_log2) - 1) >> s.lanes_log2); };
    const auto tile = [&] { return (g.threads >> s.lanes_log2) * tokens; };
    while (s.lanes_log2 > 5 && C <= 1 << (s.lanes_log2 - 1)) --s.lanes_log2;
    constexpr long long full = 256 * 1024;       // threads: four waves a SIMD
    // sequences enough for waves that share little or nothing (BF16, 4096 sequences of 16 tokens of 512 channels 145 -> 72 us, of 64 of 256 in 1024 36 -> 34; float32 62 -> 66 there, so
    // that asks for more), or so short that more waves would have no tokens (4096 of 8 of 512 137 -> 42)
    for (const int few : {128, 64})
        if (blocks() * few >= (bf16 ? full : 4 * full) || (few >> s.lanes_log2) * tokens >= T) g.threads = few;
    if (g.threads == 256 && blocks() * g.threads < full && tile() < T) g.threads = 512;
    while (s.lanes_log2 > 5 && blocks() * g.threads < full && tile() < T) --s.lanes_log2;
    // A workgroup a CU, as large as they come, where most CUs get one and none two.  2048 tokens in BF16, 160 to 252 blocks of channels: 48 to 63 -> 34 to 37 us with 1024 threads instead
    // of segments, 256 blocks 45 -> 37 instead of 512 threads, 260 62 -> 68; 16384 tokens with decays given 144 blocks 200 -> 195, 129 160 -> 180; float32 gains more.  Forward
    // alone: the backward kernel has registers for two waves a SIMD.
    if (g.threads == 512 && !back && blocks() >= 144 && blocks() <= 256 && 2 * tile() <= T) g.threads = 1024;
    else if (g.threads == 512 && blocks() * g.threads < full / 2) g.threads = 256;
    const long long tiles = (T + tile() - 1) / tile();
    long long wanted = 1;
    if (g.threads == 256 && blocks() * g.threads < full / 4) wanted = std::max(1LL, std::min({full / std::max(blocks() * g.threads, 1LL), tiles, 256LL}));
    s.channel_blocks = (unsigned)((C + (1 << s.lanes_log2) - 1) >> s.lanes_log2);
    s.segment = (int)std::max((tiles + wanted - 1) / wanted, 1LL) * tile();
    s.segments = std::max(1, (T + s.segment - 1) / s.segment);
    return g;
}

// Rows of parts of drate that are added up by themselves where there are many, and how many such pieces there are; a grid has 65535 of them at most.
constexpr unsigned SUMS_PIECE = 256;
unsigned pieces_of(unsigned rows) { return rows > 4 * SUMS_PIECE && rows / SUMS_PIECE < 65535 ? (rows + SUMS_PIECE - 1) / SUMS_PIECE : 1; }

// The tape has the state before every tile of the backward kernel, whose tokens are a power of two, but at least before every 32 tokens: a small tile in workgroups of one or two waves.
int tape_log2_of(int B, int T, int C, bool bf16)
{
    const Geometry g = shape_of(B, T, C, bf16, true, RECURRENCE_TOKENS_BACK);
    const int tile = (g.threads >> g.s.lanes_log2) * RECURRENCE_TOKENS_BACK;
    return tile >= 32 ? 5 : tile >= 16 ? 4 : 3;
}

template <class F>
void in_launches(RecurrenceShape s, long long items, F launch)
{
    for (long long first = 0; first < items; first += RECURRENCE_LAUNCH) {
        s.first = (unsigned)first;
        launch(s, (unsigned)std::min<long long>(items - first, RECURRENCE_LAUNCH));
    }
}

template <class E, int GATES, int THREADS>
hipError_t forward(const RecurrenceArgs &a, const RecurrenceShape &s, hipStream_t st)
{
    constexpr int S = RECURRENCE_TOKENS;
    const long long items = (long long)a.B * s.channel_blocks * s.segments;
    if constexpr (THREADS == 256)
        if (s.segments > 1) in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence_effects<E, GATES, S, THREADS, false><<<grid, THREADS, 0, st>>>(a, p); });
    in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence<E, GATES, S, THREADS><<<grid, THREADS, 0, st>>>(a, p); });
    return hipGetLastError();
}

template <class E, int GATES, int THREADS>
hipError_t backward(RecurrenceArgs a, const RecurrenceShape &s, hipStream_t st)
{
    constexpr int S = RECURRENCE_TOKENS_BACK;
    const long long items = (long long)a.B * s.channel_blocks * s.segments;
    a.partial = a.effects + (s.segments > 1 ? 3 * (size_t)a.B * s.segments * a.C : 0);
    if constexpr (THREADS == 256)
        if (s.segments > 1) in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence_effects<E, GATES, S, THREADS, true><<<grid, THREADS, 0, st>>>(a, p); });
    in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence_back<E, GATES, S, THREADS><<<grid, THREADS, 0, st>>>(a, p); });
    if (a.drate) {
        // many sequences' parts first by themselves in pieces: few columns are few workgroups
        const unsigned rows = (unsigned)a.B * s.segments, pieces = pieces_of(rows);
        float *joined = a.partial + (size_t)rows * a.C;
        if (pieces > 1) column_sums(ColumnSumsArgs<1>{{{a.partial, joined, SUMS_PIECE, rows}}, {0, pieces}, a.C}, st);
        column_sums(ColumnSumsArgs<1>{{{pieces > 1 ? joined : a.partial, a.drate, pieces > 1 ? pieces : rows, pieces > 1 ? pieces : rows}}, {0, 1}, a.C}, st);
    }
    return hipGetLastError();
}

template <class E, int GATES>
hipError_t run(RecurrenceArgs a, bool back, hipStream_t st)
{
    a.tape_log2 = tape_log2_of(a.B, a.T, a.C, a.bf16);
    const Geometry g = shape_of(a.B, a.T, a.C, a.bf16, back, back ? RECURRENCE_TOKENS_BACK : RECURRENCE_TOKENS);
    if (g.threads == 64) return back ? backward<E, GATES, 64>(a, g.s, st) : forward<E, GATES, 64>(a, g.s, st);
    if (g.threads == 128) return back ? backward<E, GATES, 128>(a, g.s, st) : forward<E, GATES, 128>(a, g.s, st);
    if (g.threads == 256) return back ? backward<E, GATES, 256>(a, g.s, st) : forward<E, GATES, 256>(a, g.s, st);
    if (g.threads == 1024) return forward<E, GATES, 1024>(a, g.s, st);
    return back ? backward<E, GATES, 512>(a, g.s, st) : forward<E, GATES, 512>(a, g.s, st);
}

constexpr int STEP_THREADS = 256;

// One token: bound by the bytes of states, inputs and outputs, for a single sequence by the launch.  A thread takes four neighbouring channels where every address allows it.
template <class E, int V>
struct Few;
template <class E>
struct Few<E, 4> {
    Quad<E> at;
    __device__ __forceinline__ void load(const E *p) { at.load(p); }
    __device__ __forceinline__ void values(float (&v)[4]) const { at.values(v); }
    __device__ __forceinline__ static void store(E *p, const float (&v)[4]) { store4(p, v); }
};
template <class E>
struct Few<E, 1> {
    E at;
    __device__ __forceinline__ void load(const E *p) { at = *p; }
    __device__ __forceinline__ void values(float (&v)[1]) const { v[0] = to_float(at); }
    __device__ __forceinline__ static void store(E *p, const float (&v)[1]) { store_element(p, v[0]); }
};

template <class E, int V>
__global__ __launch_bounds__(STEP_THREADS) void k_recurrence_step(RecurrenceArgs a, unsigned first)
{
    const unsigned blocks = ((unsigned)a.C / V + STEP_THREADS - 1) / STEP_THREADS, item = first + blockIdx.x;
    const int b = item / blocks, c = (int)((item % blocks) * STEP_THREADS + threadIdx.x) * V;
    if (c >= a.C) return;
    const int slot = a.slots ? a.slots[b] : b;
    E *y = (E *)a.y + b * a.sy.batch + c;
    if ((unsigned)slot >= (unsigned)a.pool) {            // no sequence here (zeros), or one that the pool does not hold (NaN)
        float none[V];
#pragma unroll
        for (int e = 0; e < V; ++e) none[e] = slot < 0 ? 0.0f : __uint_as_float(0x7fc00000u);
        Few<E, V>::store(y, none);
        return;
    }
    float *state = a.states + (long long)slot * a.C + c;
    Few<float, V> in_h, in_rate{};
    Few<E, V> in_x, in_gate, in_input{};
    in_h.load(state);
    in_x.load((const E *)a.x + b * a.sx.batch + c);
    in_gate.load((const E *)a.gate + b * a.sgate.batch + c);
    if (a.input_gate) in_input.load((const E *)a.input_gate + b * a.sinput.batch + c);
    if (a.rate) in_rate.load(a.rate + c);
    float h[V], x[V], gate[V], input[V], rate[V];
    in_h.values(h), in_x.values(x), in_gate.values(gate), in_input.values(input), in_rate.values(rate);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float u = x[e], full, less;
        const float l = log_of(a.rate, rate[e], gate[e]);
        if (a.input_gate) u *= sigmoid(input[e]);
        Decay d(l, full, less);
        if (l < HARDLY) d.hardly(l);
        if (a.normalise) u *= __builtin_amdgcn_sqrtf(less * (2.0f - less));
        h[e] = d.of(h[e], u);
    }
    Few<float, V>::store(state, h);
    Few<E, V>::store(y, h);
}

template <class E, int V>
hipError_t step(const RecurrenceArgs &a, hipStream_t st)
{
    const long long items = (long long)a.B * ((a.C / V + STEP_THREADS - 1) / STEP_THREADS);
    for (long long first = 0; first < items; first += RECURRENCE_LAUNCH)
        k_recurrence_step<E, V><<<(unsigned)std::min<long long>(items - first, RECURRENCE_LAUNCH), STEP_THREADS, 0, st>>>(a, (unsigned)first);
    return hipGetLastError();
}

bool fours(const RecurrenceArgs &a)
{
    const uintptr_t of_elements = (uintptr_t)a.x | (uintptr_t)a.gate | (uintptr_t)a.input_gate | (uintptr_t)a.y, of_floats = (uintptr_t)a.states | (uintptr_t)a.rate;
    const long long s = a.sx.batch | a.sgate.batch | (a.input_gate ? a.sinput.batch : 0) | a.sy.batch | a.C;
    return (of_elements & (a.bf16 ? 7 : 15)) == 0 && (of_floats & 15) == 0 && (s & 3) == 0;
}

}  // namespace

template <class E>
static hipError_t gates(const RecurrenceArgs &a, bool back, hipStream_t s)
{
    if (a.rate && a.normalise) return a.input_gate ? run<E, ALL>(a, back, s) : run<E, RATES>(a, back, s);
    return !a.rate && !a.input_gate && !a.normalise ? run<E, NONE>(a, back, s) : run<E, ANY>(a, back, s);
}
static hipError_t typed(const RecurrenceArgs &a, bool back, hipStream_t s)
{
    return a.bf16 ? gates<bf16>(a, back, s) : gates<float>(a, back, s);
}

hipError_t recurrence_launch(const RecurrenceArgs &a, hipStream_t s) { return typed(a, false, s); }
hipError_t recurrence_backward_launch(const RecurrenceArgs &a, hipStream_t s) { return typed(a, true, s); }
hipError_t recurrence_step_launch(const RecurrenceArgs &a, hipStream_t s) 
{
    if (a.bf16) return fours(a) ? step<bf16, 4>(a, s) : step<bf16, 1>(a, s);
    return fours(a) ? step<float, 4>(a, s) : step<float, 1>(a, s);
}

size_t recurrence_tape_bytes(int B, int T, int C, bool bf16)
{
    const int every = tape_log2_of(B, T, C, bf16);
    return 4 * (size_t)B * (((size_t)T + (1 << every) - 1) >> every) * C;
}

size_t recurrence_workspace_bytes(int B, int T, int C, bool bf16, bool backward)
{
    const size_t maps = (size_t)B * shape_of(B, T, C, bf16, backward, backward ? RECURRENCE_TOKENS_BACK : RECURRENCE_TOKENS).s.segments;
    return (maps > (size_t)B ? 12 * maps * C : 0) + (backward ? 4 * (maps + pieces_of((unsigned)maps)) * C : 0);
}

}  // namespace tfno
