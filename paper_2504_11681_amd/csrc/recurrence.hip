// Launches of the gated linear recurrence, and its step for one token.
#include "columnsums.h"
#include "recurrence_kernel.h"

#include <algorithm>

namespace tfno {

namespace {

constexpr int TOKENS = 8;                                   // of a group in a tile
constexpr unsigned RECURRENCE_LAUNCH = 1u << 23;            // workgroups: a launch takes less than 2^32 threads

// Lanes of a group, and segments.
RecurrenceShape shape_of(int B, int T, int C, int V)
{
    RecurrenceShape s{};
    s.lanes_log2 = 6;
    const auto blocks = [&] { return (unsigned)((C + (V << s.lanes_log2) - 1) / (V << s.lanes_log2)); };
    while (s.lanes_log2 > 4 && (long long)B * blocks() < 1024) --s.lanes_log2;
    s.channel_blocks = blocks();
    const int tile = (RECURRENCE_THREADS >> s.lanes_log2) * TOKENS;
    const long long groups = (long long)B * s.channel_blocks, tiles = (T + tile - 1) / tile;
    const long long wanted = groups < 512 ? std::max(1LL, std::min({1024 / std::max(groups, 1LL), tiles / 2, 64LL})) : 1;
    s.segment = (int)std::max((tiles + wanted - 1) / wanted, 1LL) * tile;
    s.segments = std::max(1, (T + s.segment - 1) / s.segment);
    return s;
}

bool pairs(const RecurrenceArgs &a, bool backward)
{
    const uintptr_t mask = a.bf16 ? 3 : 7;
    uintptr_t p = (uintptr_t)a.x | (uintptr_t)a.gate | (uintptr_t)a.input_gate | (uintptr_t)(backward ? a.dy : a.y);
    long long s = a.sx.batch | a.sx.token | a.sgate.batch | a.sgate.token | a.sy.batch | a.sy.token;
    if (a.input_gate) s |= a.sinput.batch | a.sinput.token;
    if (backward) {
        p |= (uintptr_t)a.dx | (uintptr_t)a.dgate | (uintptr_t)a.dinput_gate;
        s |= a.sdx.batch | a.sdx.token | a.sdgate.batch | a.sdgate.token;
        if (a.input_gate) s |= a.sdinput.batch | a.sdinput.token;
    }
    return a.C % 2 == 0 && (p & mask) == 0 && (s & 1) == 0;
}

template <class F>
void in_launches(RecurrenceShape s, long long items, F launch)
{
    for (long long first = 0; first < items; first += RECURRENCE_LAUNCH) {
        s.first = (unsigned)first;
        launch(s, (unsigned)std::min<long long>(items - first, RECURRENCE_LAUNCH));
    }
}

template <class E, int V>
hipError_t forward(const RecurrenceArgs &a, hipStream_t st)
{
    const RecurrenceShape s = shape_of(a.B, a.T, a.C, V);
    const long long items = (long long)a.B * s.channel_blocks * s.segments;
    if (s.segments > 1)
        in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence_effects<E, V, TOKENS, false><<<grid, RECURRENCE_THREADS, 0, st>>>(a, p); });
    in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence<E, V, TOKENS><<<grid, RECURRENCE_THREADS, 0, st>>>(a, p); });
    return hipGetLastError();
}

template <class E, int V>
hipError_t backward(RecurrenceArgs a, hipStream_t st)
{
    const RecurrenceShape s = shape_of(a.B, a.T, a.C, V);
    const long long items = (long long)a.B * s.channel_blocks * s.segments;
    a.partial = (float *)(a.effects + (s.segments > 1 ? (size_t)a.B * s.segments * a.C : 0));
    if (s.segments > 1)
        in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence_effects<E, V, TOKENS, true><<<grid, RECURRENCE_THREADS, 0, st>>>(a, p); });
    in_launches(s, items, [&](const RecurrenceShape &p, unsigned grid) { k_recurrence_back<E, V, TOKENS><<<grid, RECURRENCE_THREADS, 0, st>>>(a, p); });
    if (a.drate) {
        const ColumnSumsArgs<1> sums{{{a.partial, a.drate, (unsigned)a.B * s.segments}}, {0, 1}, a.C};
        k_column_sums<1><<<dim3((a.C + 15) / 16, 1), 1024, 0, st>>>(sums);
    }
    return hipGetLastError();
}

constexpr int STEP_THREADS = 256;

// One token: bound by the bytes of states, inputs and outputs, for a single sequence by the launch.
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
        for (int e = 0; e < V; ++e) none[e] = slot < 0 ? 0.0f : __uint_as_float(0x7fc00000u);
        store_some(y, none);
        return;
    }
    float *state = a.states + (long long)slot * a.C + c;
    Some<E, V> x, gate, input{};
    Some<float, V> h;
    x.load((const E *)a.x + b * a.sx.batch + c);
    gate.load((const E *)a.gate + b * a.sgate.batch + c);
    if (a.input_gate) input.load((const E *)a.input_gate + b * a.sinput.batch + c);
    h.load(state);
    Decay d[V];
    float rate[V], u[V], out[V], log[V] = {};
    load_rates(a, c, rate);
    decay_and_input<E, V>(a, rate, x, gate, input, true, d, u, log);
#pragma unroll
    for (int e = 0; e < V; ++e) out[e] = d[e].of(h.value(e), u[e]);
    store_some(state, out);
    store_some(y, out);
}

template <class E, int V>
hipError_t step(const RecurrenceArgs &a, hipStream_t st)
{
    const long long items = (long long)a.B * ((a.C / V + STEP_THREADS - 1) / STEP_THREADS);
    for (long long first = 0; first < items; first += RECURRENCE_LAUNCH)
        k_recurrence_step<E, V><<<(unsigned)std::min<long long>(items - first, RECURRENCE_LAUNCH), STEP_THREADS, 0, st>>>(a, (unsigned)first);
    return hipGetLastError();
}

}  // namespace

hipError_t recurrence_launch(const RecurrenceArgs &a, hipStream_t s)
{
    const bool two = pairs(a, false);
    if (a.bf16) return two ? forward<bf16, 2>(a, s) : forward<bf16, 1>(a, s);
    return two ? forward<float, 2>(a, s) : forward<float, 1>(a, s);
}

hipError_t recurrence_backward_launch(const RecurrenceArgs &a, hipStream_t s)
{
    const bool two = pairs(a, true);
    if (a.bf16) return two ? backward<bf16, 2>(a, s) : backward<bf16, 1>(a, s);
    return two ? backward<float, 2>(a, s) : backward<float, 1>(a, s);
}

hipError_t recurrence_step_launch(const RecurrenceArgs &a, hipStream_t s)
{
    const bool two = pairs(a, false) && ((uintptr_t)a.states & 7) == 0;
    if (a.bf16) return two ? step<bf16, 2>(a, s) : step<bf16, 1>(a, s);
    return two ? step<float, 2>(a, s) : step<float, 1>(a, s);
}

size_t recurrence_tape_bytes(int B, int T, int C) { return 4 * (size_t)B * ((T + RECURRENCE_TAPE - 1) / RECURRENCE_TAPE) * C; }

size_t recurrence_workspace_bytes(int B, int T, int C, bool, bool backward)
{
    size_t most = 0;
    for (int V = 1; V <= 2; ++V) {
        const size_t maps = (size_t)B * shape_of(B, T, C, V).segments;
        most = std::max(most, (maps > (size_t)B ? 8 * maps * C : 0) + (backward ? 4 * maps * C : 0));
    }
    return most;
}

}  // namespace tfno
