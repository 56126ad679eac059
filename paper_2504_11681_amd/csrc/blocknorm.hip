// Launches of the norms around a block.
#include "blocknorm_kernel.h"
#include "columnsums.h"

#include <algorithm>

namespace tfno {

namespace {

constexpr unsigned FORWARD_WAVES = 256 * 20;         // five waves a SIMD, which its registers allow

int group_log2_of(int C)
{
    int g = 0;
    while (g < 9 && (8 << g) < C) ++g;
    return g;
}
int threads_of(int group_log2) { return group_log2 > 6 ? 1 << group_log2 : BLOCK_NORM_THREADS; }
// Workgroups of the backward kernel, at most: each leaves a row of every sum over tokens.  As many as are there at once: three waves a SIMD where tokens have gates of their own (131072 heads
// of 128, both directions: 70 us, with two 76), else two (16 x 1024 tokens of 2048: 231, with three 240).
unsigned most_blocks(int C, int gate_kind) { return 1024u * (gate_kind == GATE_TOKEN ? 3 : 2) * 64 / threads_of(group_log2_of(C)); }

// Parts of a sequence for workgroups that sum up a gate's gradient: as many as fill the launch, none without rows.
unsigned parts_of(int B, int T, int C)
{
    const int groups = threads_of(group_log2_of(C)) >> group_log2_of(C);
    if (T <= 2 * groups || (unsigned)B >= most_blocks(C, GATE_SEQUENCE)) return 1;
    const unsigned wanted = (most_blocks(C, GATE_SEQUENCE) + B - 1) / B, most = (T + groups - 1) / groups;
    const unsigned rows = (T + std::min(wanted, most) - 1) / std::min(wanted, most);
    return (T + rows - 1) / rows;
}

template <class E, class R, bool VEC, int ITER, bool TOKEN, bool BACKWARD>
hipError_t launch(const BlockNormArgs &a, hipStream_t st)
{
    BlockNormShape s{};
    s.group_log2 = group_log2_of(a.C);
    const int threads = threads_of(s.group_log2), groups = threads >> s.group_log2;
    const unsigned rows = (unsigned)a.B * (unsigned)a.T;
    unsigned work, most = BACKWARD ? most_blocks(a.C, a.gate_kind) : FORWARD_WAVES * 64 / threads;        // work: workgroups that each have work once
    if (BACKWARD && a.gate_kind == GATE_SEQUENCE && a.dgate) {
        s.parts = parts_of(a.B, a.T, a.C), s.whole = s.parts == 1;
        // Whole sequences are a group's each where there are many or they are short, else a workgroup's, whose groups share them.  Gradient in BF16 with a float32 residual, a group's
        // each and shared: 20000 x 8 tokens of 64 54 and 223 us, 5000 x 2 of 64 17 and 68, 16384 x 64 of 64 298 and 301.  Of a few thousand sequences and fewer, a group's each
        // are too few workgroups for the chip: 8192 x 128 of 64 326 and 258, 2048 x 512 of 64 1062 and 286, 256 x 64 of 64 134 and 20, 1024 x 256 of 128 577 and 142.
        s.by_group = s.whole && (groups == 1 || a.B >= groups * 64 || a.T <= 2 * groups);
        s.outer = a.B * s.parts, s.rows = (a.T + s.parts - 1) / s.parts;
        work = s.by_group ? (s.outer + groups - 1) / groups : s.outer;
    } else {
        s.outer = rows > 0;
        s.rows = (unsigned)std::max(1ull, ((unsigned long long)rows + (unsigned long long)most * groups - 1) / ((unsigned long long)most * groups));
        work = (unsigned)(((unsigned long long)rows + (unsigned long long)s.rows * groups - 1) / ((unsigned long long)s.rows * groups));
    }
    const unsigned grid = std::min(work, most);
    s.outer_stride = s.parts == 0 ? 1 : s.by_group ? grid * groups : grid;
    if (BACKWARD) {
        s.part_after = a.workspace, s.part_before = s.part_after + (size_t)grid * a.C, s.part_gate = s.part_before + (size_t)grid * a.C;
    }
    if (grid) k_block_norm<E, R, VEC, ITER, TOKEN, BACKWARD><<<grid, threads, 0, st>>>(a, s);
    if (BACKWARD) {
        ColumnSumsArgs<3> sums{};
        const bool of_sequences = a.gate_kind == GATE_SEQUENCE && a.dgate && !s.whole && grid;
        sums.kind[0] = {s.part_after, a.dw_after, grid, grid};
        sums.kind[1] = {s.part_before, a.dw_before, grid, grid};
        sums.kind[2] = {s.part_gate, (float *)a.dgate, of_sequences ? s.parts : grid, of_sequences ? s.parts * a.B : grid};
        sums.first[1] = a.dw_after ? 1 : 0;
        sums.first[2] = sums.first[1] + (a.dw_before ? 1 : 0);
        sums.first[3] = sums.first[2] + (a.dgate && a.gate_kind == GATE_CHANNEL ? 1 : of_sequences ? a.B : 0);
        sums.C = a.C;
        column_sums(sums, st);
    }
    return hipGetLastError();
}

bool vectors(const BlockNormArgs &a, bool backward)
{
    if (a.C % 8) return false;
    uintptr_t p = (uintptr_t)a.y;
    long long s = 0;
    const auto of = [&](const void *at, const Strides &v) {
        if (at) p |= (uintptr_t)at, s |= v.batch | v.token;
    };
    of(a.y, a.sy), of(a.r, a.sr);
    if (a.gate_kind == GATE_TOKEN || a.gate_kind == GATE_SEQUENCE) of(a.gate, Strides{a.sgate.batch, a.gate_kind == GATE_TOKEN ? a.sgate.token : 0, 0});
    if (backward) {
        of(a.d_r_out, a.sr_out), of(a.d_n_out, a.sn_out), of(a.dy, a.sdy), of(a.dr, a.sdr);
        if (a.gate_kind == GATE_TOKEN) of(a.dgate, a.sdgate);
    } else {
        of(a.r_out, a.sr_out), of(a.n_out, a.sn_out);
    }
    return (p & 15) == 0 && (s & 7) == 0;
}

template <class E, class R, bool TOKEN, bool BACKWARD>
hipError_t choose(const BlockNormArgs &a, hipStream_t s)
{
    const bool vec = vectors(a, BACKWARD);
    if ((8 << group_log2_of(a.C)) < a.C) return vec ? launch<E, R, true, 2, TOKEN, BACKWARD>(a, s) : launch<E, R, false, 2, TOKEN, BACKWARD>(a, s);
    return vec ? launch<E, R, true, 1, TOKEN, BACKWARD>(a, s) : launch<E, R, false, 1, TOKEN, BACKWARD>(a, s);
}
template <class E, class R, bool BACKWARD>
hipError_t choose(const BlockNormArgs &a, hipStream_t s)
{
    return a.gate_kind == GATE_TOKEN ? choose<E, R, true, BACKWARD>(a, s) : choose<E, R, false, BACKWARD>(a, s);
}

template <bool BACKWARD>
hipError_t typed(const BlockNormArgs &a, hipStream_t s)
{
    if (!a.bf16) return choose<float, float, BACKWARD>(a, s);
    return a.residual_bf16 ? choose<bf16, bf16, BACKWARD>(a, s) : choose<bf16, float, BACKWARD>(a, s);
}

}  // namespace

hipError_t block_norm_launch(const BlockNormArgs &a, hipStream_t s) { return typed<false>(a, s); }
hipError_t block_norm_backward_launch(const BlockNormArgs &a, hipStream_t s) { return typed<true>(a, s); }

size_t block_norm_workspace_bytes(int B, int T, int C, int gate_kind)
{
    size_t rows = 3 * (size_t)most_blocks(C, gate_kind);
    if (gate_kind == GATE_SEQUENCE) rows = 2 * (size_t)most_blocks(C, gate_kind) + (size_t)B * parts_of(B, T, C);
    return sizeof(float) * rows * C;
}

}  // namespace tfno
