// Gradient of the gated delta rule, from the tape of the forward pass (the names are those of the forward kernels).  With dO already
// times scale and dS' the gradient of a chunk's outgoing state:
//
//   dU = P' dO + e^(GL-G) (K dS'),   Y = T' (beta dU) = dV,
//   dS = e^GL dS' + Q' (e^G dO) - K' (e^G Y)                                        (k_delta_scan_back, from the last chunk to the first)
//
// and for every chunk by itself (k_delta_gradients), with C = Y E', D = dO E', X = P . D - A . C and strict() resp. tril() of M:
//
//   dbeta_j = sum_i X_ij + e^(GL-G_j) k_j (dS' E_j),
//   dq = e^G (dO S') + (M . D beta) K,
//   dk = -e^G (Y S') + e^(GL-G) beta (E dS'') + (M . D beta)' Q - (W + W') K,   W = strict(M . C beta),
//   dG_i = sum_j X_ij beta_j - beta_i sum_j X_ji + q_i e^G (dO S')_i - k_i e^G (Y S')_i - c_i,   c_i = e^(GL-G_i) beta_i k_i (dS' E_i),
//   dG_L += sum c + e^GL <S, dS'>,   dg = sum of dG from the token on, up to the next decay of 0 (whose own dg is 0).
//
// Value heads that share a key head are summed by the workgroup of that key head, in their order.
#pragma once
#include "deltarule_kernel.h"

namespace tfno {

// LDS of a chunk: K, gates, P', T' | K', Q'
template <class E, int KB>
struct BackwardLds : ScanLds<DeltaUnits<E, KB>::Q + 1 + 2 * DeltaUnits<E, KB>::TRI * DELTA_PM, DeltaUnits<E, KB>::KEY_TAPE - DeltaUnits<E, KB>::KT> {};

// EFFECTS: what each segment but the first adds to the gradient of the state before it, without anything else.  Bound as the forward walk by the issue of a wave (B 4,
// T 2048, 16 heads of 128 in BF16: 185 us, 5.8 a chunk); two chunks' K' and Q' do not fit LDS for heads of 128, they come during the chunk.
template <class E, int KB, bool EFFECTS>
__global__ __launch_bounds__(SCAN_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_delta_scan_back(DeltaArgs a, DeltaMemory mem, int blocks_per_head)
{
    typedef DeltaUnits<E, KB> U;
    constexpr int L = U::L, NT = U::NT, LB = U::LB, DT = U::DT, PI = U::PI, PM = DELTA_PM;
    typedef BackwardLds<E, KB> Lds;
    constexpr int K_UNITS = U::Q, TRI_UNITS = U::TRI * PM;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = (blockDim.x >> 6) - 1;      // and one that loads
    const int m = lane & 15, g = lane >> 4;
    const int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int some = EFFECTS ? mem.segments - 1 : mem.segments;
    const int block = id % blocks_per_head, part = id / blocks_per_head, segment = part % some + (EFFECTS ? 1 : 0), head = part / some;
    const long long at = (long long)head * mem.segments + segment;
    const int b = head / a.Hv, h = head - b * a.Hv, hk = h / (a.Hv / a.Hk);
    const int len = sequence_length(a, b), all = (len + L - 1) / L;
    const int begin = segment * mem.segment_chunks, n = all < begin + mem.segment_chunks ? all : begin + mem.segment_chunks;   // chunks begin .. n - 1
    const unsigned char *key = mem.key + (long long)(b * a.Hk + hk) * mem.chunks * mem.key_units * 1024;
    const unsigned char *value = mem.value + (long long)head * mem.chunks * mem.value_units * 1024;
    const int col0 = (block * waves + wave) * 16, col = col0 + m;
    const bool all_columns = a.Dv % 32 == 0;

    floatx4 S[DT];          // dS', laid out as the state is
    if (EFFECTS) load_state<DT>(nullptr, 0, 0, col, g, S);
    else if (mem.segments > 1) load_state<DT>(mem.segment_d_states + at * U::DKP * mem.dvp, U::DKP, mem.dvp, col, g, S);
    else load_state<DT>(a.d_final ? a.d_final + (long long)head * a.Dk * a.Dv : nullptr, a.Dk, a.Dv, col, g, S);
    const E *d_o = (const E *)a.d_o + (b * a.sdo.batch + h * a.sdo.head);
    E *dv = (E *)a.dv + (b * a.sdv.batch + h * a.sdv.head);
    const unsigned at_do = (8 * g * (unsigned)a.sdo.token + (col < a.Dv ? col : 0)) * sizeof(E);
    const unsigned at_tape = tiles_at(mem.dvp, col0, lane);
    const int lane_token = 8 * g + (lane & 3), lane_col = col0 + (lane & 12);       // of the transposed tiles: four columns of a token
    const unsigned at_dv = (lane_token * (unsigned)a.sdv.token + lane_col) * sizeof(E);

    auto load_first = [&](int chunk, int parity) {
        unsigned char *to = Lds::first(lds, parity);
        const unsigned char *v = value + (long long)chunk * mem.value_units * 1024;
        units_to_lds(key + ((long long)chunk * mem.key_units + U::K) * 1024, to, K_UNITS, lane);
        units_to_lds(v + U::GATES * 1024, to + K_UNITS * 1024, 1, lane);
        units_to_lds(v + U::PT * 1024, to + (K_UNITS + 1) * 1024, TRI_UNITS, lane);
        units_to_lds(v + U::TT * 1024, to + (K_UNITS + 1 + TRI_UNITS) * 1024, TRI_UNITS, lane);
    };
    auto load_last = [&](int chunk, int parity) {
        units_to_lds(key + ((long long)chunk * mem.key_units + U::KT) * 1024, Lds::last(lds, parity), Lds::LAST, lane);
    };
    E next[LB][8];
    auto load_do = [&](int chunk) { load_columns<E, LB>(d_o + (long long)chunk * L * a.sdo.token, a.sdo.token, at_do, g, len - chunk * L, next); };
    auto load_next = [&](int chunk) {
        if (!Lds::DOUBLE) load_last(chunk, chunk & 1);
        if (chunk > begin) {
            load_first(chunk - 1, (chunk - 1) & 1);
            if (Lds::DOUBLE) load_last(chunk - 1, (chunk - 1) & 1);
        }
    };
    if (wave == waves) {
        if (n > begin) {
            load_first(n - 1, (n - 1) & 1);
            if (Lds::DOUBLE) load_last(n - 1, (n - 1) & 1);
        }
        for (int chunk = n - 1; chunk >= begin; --chunk) {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            load_next(chunk);
            if (!Lds::DOUBLE) {
                __builtin_amdgcn_s_waitcnt(0);
                __syncthreads();
            }
        }
        return;
    }
    if (n > begin) load_do(n - 1);
    __builtin_amdgcn_s_waitcnt(0);
    for (int chunk = n - 1; chunk >= begin; --chunk) {
        const int t0 = chunk * L, parity = chunk & 1;
        const unsigned char *ldsK = Lds::first(lds, parity), *ldsG = ldsK + K_UNITS * 1024, *ldsPT = ldsG + 1024, *ldsTT = ldsPT + TRI_UNITS * 1024,
                            *ldsKT = Lds::last(lds, parity);
        const DeltaGates<L> *gates = (const DeltaGates<L> *)ldsG;
        __syncthreads();
        mask_columns<E, LB>(next, all_columns, col < a.Dv, g, len - t0);
        float x[LB][8];
#pragma unroll
        for (int s = 0; s < LB; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[s][e] = to_float(next[s][e]);
        const int before = chunk > begin ? chunk - 1 : begin;
        load_do(before);
        if (!EFFECTS && col0 < mem.dvp) store_tiles<DT>(mem.d_states + ((long long)head * mem.chunks + chunk) * U::DKP * mem.dvp, mem.dvp, at_tape, lane, S);
        // K dS' and P' dO, a pair of tiles of tokens at a time
        floatx4 KS[NT], PO_[NT];
        {
            Frag<PI> Of[LB];
#pragma unroll
            for (int s = 0; s < LB; ++s) Of[s] = make_frag<PI>(x[s]);
#pragma unroll
            for (int s = 0; s < LB; ++s) {
                Frag<PM> pf[LB][2];
#pragma unroll
                for (int kb = s; kb < LB; ++kb)
#pragma unroll
                    for (int p = 0; p < 2; ++p) pf[kb][p] = load_frag<PM>(ldsPT + U::upper(2 * s + p, kb) * PM * 1024, lane);
                PO_[2 * s] = PO_[2 * s + 1] = floatx4{0, 0, 0, 0};
                floatx4 *to[2] = {&PO_[2 * s], &PO_[2 * s + 1]};
#pragma unroll
                for (int kb = s; kb < LB; ++kb) mm_many<3, false>(pf[kb], Of[kb], to, NoWeave());
            }
            Frag<PM> Sf[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                float u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = S[2 * kb + (e >> 2)][e & 3];
                Sf[kb] = make_frag<PM>(u);
            }
            Frag<PI> kf[2][2];
            auto read = [&](int step, int to) {
                const int i = step / KB * 2, kb = step % KB;
#pragma unroll
                for (int p = 0; p < 2; ++p) kf[to][p] = load_frag<PI>(ldsK + ((i + p) * KB + kb) * PI * 1024, lane);
            };
            read(0, 0);
#pragma unroll
            for (int step = 0; step < LB * KB; ++step) {
                const int i = step / KB * 2, kb = step % KB, at = step & 1;
                if (step + 1 < LB * KB) read(step + 1, at ^ 1);
                __builtin_amdgcn_sched_barrier(0);
                if (kb == 0) KS[i] = KS[i + 1] = floatx4{0, 0, 0, 0};
                floatx4 *to[2] = {&KS[i], &KS[i + 1]};
                mm_many<3, false>(kf[at], Sf[kb], to, NoWeave());
                __builtin_amdgcn_sched_barrier(0);
            }
        }

        // Y = T' (beta dU)
        floatx4 Y[NT];
        {
            Frag<PM> R[LB];
#pragma unroll
            for (int s = 0; s < LB; ++s) {
                float be[8], left[8], u[8];
                load_gates(gates->beta + 32 * s + 8 * g, be);
                load_gates(gates->left + 32 * s + 8 * g, left);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = be[e] * fmaf(left[e], KS[2 * s + (e >> 2)][e & 3], a.scale * PO_[2 * s + (e >> 2)][e & 3]);
                R[s] = make_frag<PM>(u);
            }
#pragma unroll
            for (int s = 0; s < LB; ++s) {
                Frag<PM> tf[LB][2];
#pragma unroll
                for (int kb = s; kb < LB; ++kb)
#pragma unroll
                    for (int p = 0; p < 2; ++p) tf[kb][p] = load_frag<PM>(ldsTT + U::upper(2 * s + p, kb) * PM * 1024, lane);
                Y[2 * s] = Y[2 * s + 1] = floatx4{0, 0, 0, 0};
                floatx4 *to[2] = {&Y[2 * s], &Y[2 * s + 1]};
#pragma unroll
                for (int kb = s; kb < LB; ++kb) mm_many<3, false>(tf[kb], R[kb], to, NoWeave());
            }
        }
        Frag<PM> Wo[LB], Wy[LB];
#pragma unroll
        for (int s = 0; s < LB; ++s) {
            float decay[8], u[8], w[8];
            load_gates(gates->decay + 32 * s + 8 * g, decay);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[e] = a.scale * decay[e] * x[s][e];
                w[e] = -decay[e] * Y[2 * s + (e >> 2)][e & 3];
            }
            Wo[s] = make_frag<PM>(u);
            Wy[s] = make_frag<PM>(w);
        }
        const float whole = gates->whole;
        if (!Lds::DOUBLE) {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
        }
        {
            Frag<PI> kf[2][2], qf[2][2];
            auto read = [&](int step, int to) {
                const int t = step / LB * 2, kb = step % LB;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    kf[to][p] = load_frag<PI>(ldsKT + ((t + p) * LB + kb) * PI * 1024, lane);
                    qf[to][p] = load_frag<PI>(ldsKT + ((DT + t + p) * LB + kb) * PI * 1024, lane);
                }
            };
            read(0, 0);
#pragma unroll
            for (int step = 0; step < KB * LB; ++step) {
                const int t = step / LB * 2, kb = step % LB, at = step & 1;
                if (step + 1 < KB * LB) read(step + 1, at ^ 1);
                __builtin_amdgcn_sched_barrier(0);
                if (kb == 0) S[t] *= whole, S[t + 1] *= whole;
                floatx4 *to[2] = {&S[t], &S[t + 1]};
                mm_many<3, false>(kf[at], Wy[kb], to, NoWeave());
                mm_many<3, false>(qf[at], Wo[kb], to, NoWeave());
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (Lds::DOUBLE) __builtin_amdgcn_s_waitcnt(0);      // what the next chunk needs is there; the stores have its time
        if (!EFFECTS && col0 < mem.dvp) {
            store_tiles<NT>(mem.d_values + ((long long)head * mem.chunks + chunk) * L * mem.dvp, mem.dvp, at_tape, lane, Y);
            const bool plain = mem.vec_dv && t0 + L <= a.T && (all_columns || col0 + 16 <= a.Dv);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const floatx4 y = quad_transpose(Y[i], lane);
                const int row = t0 + 32 * (i >> 1) + 4 * (i & 1);
                float u[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) u[r] = row + lane_token < len ? y[r] : 0.0f;       // past the end zeros beside a NaN too
                E *to = dv + row * a.sdv.token;
                if (plain) {
                    if (col0 < a.Dv) store4(behind(to, at_dv), u);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (row + lane_token < a.T && lane_col + r < a.Dv) store_element(behind(to, at_dv) + r, u[r]);
                }
            }
        }
    }
    if (EFFECTS) {
        if (col0 < mem.dvp) store_tiles<DT>(mem.back_effects + at * U::DKP * mem.dvp, mem.dvp, at_tape, lane, S);
        return;
    }
    const int last = min((begin + mem.segment_chunks) * L, a.T);
    for (int t = (n > begin ? n : begin) * L + g; t < last; t += 4)
        if (col < a.Dv) store_element(dv + t * a.sdv.token + col, 0.0f);
    if (a.d_initial && segment == 0) store_state<DT>(a.d_initial + (long long)head * a.Dk * a.Dv, a.Dk, a.Dv, col, g, S);
}

// LDS of the gradients, 32 columns of the states at a time: operand blocks of S and dS' (rows: Dk), of E and Y (rows: tokens), for two rounds.
template <class E, int KB>
struct GradientLds {
    typedef DeltaUnits<E, KB> U;
    static constexpr int S = 0, D = U::DT * DELTA_PM, ERR = 2 * U::DT * DELTA_PM, Y = ERR + U::NT * DELTA_PM, UNITS = Y + U::NT * DELTA_PM;
    static constexpr int COL = U::L + 4, MATRICES = 2 * U::L * COL * 4;
    static constexpr int BYTES = 2 * UNITS * 1024 > MATRICES ? 2 * UNITS * 1024 : MATRICES;
};

// One workgroup for a chunk of a key head.  L / 16 waves take the products of pairs of tokens and bring the states in, as many the products with the states,
// each for 16 tokens, whose errors and values' gradients they bring in.  What comes is split once for all and left in LDS, a round of 32 columns ahead of its
// products.  B 4, T 2048, 8 key heads and 16 value heads of 128 in BF16: 228 us for 580 MB, a round 8000 cycles, the products of a SIMD's two waves 3000 of them; the rest is the
// splits and the loads' issue, which stands still while their queues are full, some 20000 cycles a workgroup before the first round and after the last, alone on its CU, and
// some 8000 between two value heads, whose sums of dq and dk pass through memory (14 us of the call).
// (All of it in every wave took 512 registers, so one wave a SIMD, and waited for memory in every round: 338 us; all loads and splits in the waves of the
// states 266; loads one after the other behind all splits 256.)
template <class E, int KB>
__global__ __launch_bounds__((8 * DeltaKind<E>::L)) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_delta_gradients(DeltaArgs a, DeltaMemory mem, DeltaVec vec)
{
    typedef DeltaUnits<E, KB> U;
    typedef GradientLds<E, KB> Lds;
    constexpr int L = U::L, NT = U::NT, LB = U::LB, DT = U::DT, DKP = U::DKP, PI = U::PI, PM = DELTA_PM, COL = Lds::COL;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    float *Mq = (float *)lds, *Mk = Mq + L * COL;                    // once the states are done with
    __shared__ float hi[L], lo[L], beta[L], column_sums[NT][L], row_sums[L], token_g[L], token_beta[L], inner[NT];
    __shared__ float whole;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int chunk = id % mem.chunks, kh = id / mem.chunks;
    const int b = kh / a.Hk, hk = kh - b * a.Hk, group = a.Hv / a.Hk;
    const int len = sequence_length(a, b), t0 = chunk * L;
    const bool pairs = wave < NT;
    const int i = pairs ? wave : wave - NT, token = t0 + tile_index(i, m);          // the lane's token where tokens are columns
    E *dq = (E *)a.dq + (b * a.sdq.batch + (long long)token * a.sdq.token + hk * a.sdq.head);
    E *dk = (E *)a.dk + (b * a.sdk.batch + (long long)token * a.sdk.token + hk * a.sdk.head);

    if (t0 >= len) {                     // past the sequence's end
        const float zero[8] = {};
        if (token < a.T && !pairs)
#pragma unroll
            for (int s = 0; s < KB; ++s) {
                store8(dq + 32 * s + 8 * g, a.Dk - 32 * s - 8 * g, vec.dq, zero);
                store8(dk + 32 * s + 8 * g, a.Dk - 32 * s - 8 * g, vec.dk, zero);
            }
        for (int x = tid; x < L * group; x += 128 * NT) {
            const int t = t0 + x % L, h = hk * group + x / L;
            if (t < a.T) {
                if (a.dg) a.dg[b * a.sdg.batch + (long long)t * a.sdg.token + h * a.sdg.head] = 0.0f;
                a.dbeta[b * a.sdbeta.batch + (long long)t * a.sdbeta.token + h * a.sdbeta.head] = 0.0f;
            }
        }
        return;
    }

    const unsigned char *key = mem.key + ((long long)kh * mem.chunks + chunk) * mem.key_units * 1024;
    const int rounds = mem.dvp / 32;
    auto part = [&](int member) { return ((long long)(b * a.Hv + hk * group + member)) * mem.chunks + chunk; };
    // dO of the lane's token in a round: 8 columns
    const unsigned at_do = ((8 * (m >> 2) + (m & 3)) * (unsigned)a.sdo.token + 8 * g) * sizeof(E);
    auto load_do = [&](int member, int kb, float (&u)[8]) {
        const E *p = uniform((const E *)a.d_o + (b * a.sdo.batch + (t0 + tile_index(i, 0)) * a.sdo.token + (hk * group + member) * a.sdo.head + 32 * kb));
        unsigned off = at_do;
        asm("" : "+v"(off));
        load8(behind(p, off), token < len ? a.Dv - 32 * kb - 8 * g : 0, vec.d_o, u);
    };

    // rows of 32 columns between the kernels: a uniform address, and the lane's row of a tile and its eight columns
    const unsigned at_row = ((8 * (m >> 2) + (m & 3)) * mem.dvp + 8 * g) * 4;
    auto load_row = [&](const float *p, int tile, float (&x)[8]) {
        unsigned off = at_row;
        asm("" : "+v"(off));
        load8(behind(uniform(p + tile_index(tile, 0) * mem.dvp), off), 8, true, x);
    };

    if (pairs) {
        constexpr int TILES = DT > NT ? DT / NT : 1;
        struct Round { float s[TILES][8], d[TILES][8]; } next;
        float next_o[8], dot = 0.0f;
        // Splits what waits in `next` as round `split` (-1: nothing does) and loads round `load` (from `count` on: none), a row of tiles after the other: all loads
        // at once fill the queues, and the wave stands still until they have room.
        const int count = group * rounds;
        auto turn = [&](int split, int load) {
            unsigned char *panel = lds + (split & 1) * Lds::UNITS * 1024;
            const int member = load / rounds, kb = load - member * rounds;
            const long long at = part(member);
#pragma unroll
            for (int p = 0; p < TILES; ++p) {
                const int t = i + p * NT;
                if (t < DT) {
                    if (split >= 0) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) dot = fmaf(next.s[p][e], next.d[p][e], dot);
                        store_frag<PM>(panel + (Lds::S + t * PM) * 1024, lane, make_frag<PM>(next.s[p]));
                        store_frag<PM>(panel + (Lds::D + t * PM) * 1024, lane, make_frag<PM>(next.d[p]));
                    }
                    if (load < count) {
                        load_row(mem.states + at * DKP * mem.dvp + 32 * kb, t, next.s[p]);
                        load_row(mem.d_states + at * DKP * mem.dvp + 32 * kb, t, next.d[p]);
                    }
                }
            }
        };
        turn(-1, 0);
        load_do(0, 0, next_o);
        float gate[4];             // of the next member: the lane's token, and the chunk's decay
        auto load_gates_of = [&](int member) {
            const long long at = part(member);
            const DeltaGates<L> *gates = (const DeltaGates<L> *)(mem.value + at * mem.value_units * 1024);
            const int tok = lane & (L - 1);
            gate[0] = mem.logs[at * 2 * L + tok], gate[1] = mem.logs[at * 2 * L + L + tok], gate[2] = gates->beta[tok], gate[3] = gates->whole;
        };
        load_gates_of(0);
        floatx4 kk[NT], qk[NT], mq[NT], mk[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) kk[j] = qk[j] = mq[j] = mk[j] = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const Frag<PI> kf = load_frag<PI>(key + (U::K + (i * KB + kb) * PI) * 1024, lane), qf = load_frag<PI>(key + (U::Q + (i * KB + kb) * PI) * 1024, lane);
#pragma unroll
            for (int j = 0; j < NT; ++j) {            // all tiles, the unused ones too: no branches between the products
                const Frag<PI> other = load_frag<PI>(key + (U::K + (j * KB + kb) * PI) * 1024, lane);
                kk[j] = mm<3>(kf, other, kk[j]);
                qk[j] = mm<3>(qf, other, qk[j]);
            }
        }
        turn(0, 1);
        for (int member = 0; member < group; ++member) {
            if (tid < L) {
                hi[tid] = gate[0], lo[tid] = gate[1], beta[tid] = gate[2];
                if (tid == 0) whole = gate[3];
            }
            load_gates_of(min(member + 1, group - 1));
            floatx4 D[NT], C[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) D[j] = C[j] = floatx4{0, 0, 0, 0};
            for (int kb = 0; kb < rounds; ++kb) {
                const int round = member * rounds + kb;
                const unsigned char *panel = lds + (round & 1) * Lds::UNITS * 1024;
                const Frag<PI> of = make_frag<PI>(next_o);
                __syncthreads();
                if (kb + 1 < rounds) load_do(member, kb + 1, next_o);
                else {
                    if (member + 1 < group) load_do(member + 1, 0, next_o);
                    dot = group_sum(dot, 64);                  // the member's states have all been through
                    if (lane == 0) inner[i] = dot;
                    dot = 0.0f;
                }
                if (round + 1 < count) turn(round + 1, round + 2);
                const Frag<PM> yf = load_frag<PM>(panel + (Lds::Y + i * PM) * 1024, lane);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const Frag<PM> f = load_frag<PM>(panel + (Lds::ERR + j * PM) * 1024, lane);
                    D[j] = mm<3>(of, f, D[j]);
                    C[j] = mm<3>(yf, f, C[j]);
                }
            }
            // matrices of token pairs: rows tile_index(i, 4 g + r), column tile_index(j, m)
            float rows[4] = {};
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                float column = 0.0f;
                const int col = tile_index(j, m);
                const float be = beta[col];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = tile_index(i, 4 * g + r);
                    const float M = col <= row ? decay_between(hi[row], lo[row], hi[col], lo[col]) : 0.0f, strict = col < row ? M : 0.0f;
                    const float Dm = a.scale * M * D[j][r], Cm = strict * C[j][r];
                    const float x = qk[j][r] * Dm - kk[j][r] * Cm;
                    rows[r] = fmaf(x, be, rows[r]);
                    column += x;
                    mq[j][r] = fmaf(Dm, be, mq[j][r]);
                    mk[j][r] = fmaf(-Cm, be, mk[j][r]);
                }
                column += __shfl_xor(column, 16, 64);
                column += __shfl_xor(column, 32, 64);
                if (g == 0) column_sums[i][col] = column;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                rows[r] = group_sum(rows[r], 16);
                if (m == 0) row_sums[tile_index(i, 4 * g + r)] = rows[r];
            }
            __syncthreads();
            if (wave == 0) {
                const int tok = lane < L ? lane : 0, h = hk * group + member;
                float column = 0.0f, all = 0.0f;
#pragma unroll
                for (int w = 0; w < NT; ++w) column += column_sums[w][tok], all += inner[w];
                const float c = lane < L ? beta[tok] * token_beta[tok] : 0.0f;
                float dG = lane < L ? row_sums[tok] - beta[tok] * column + token_g[tok] - c : 0.0f;
                const float sum = group_sum(c, 64);
                if (lane == L - 1) dG += sum + whole * all;
                // Sums from each token on.  A decay of 0 ends them: what comes from there on adds up to nothing, and would leave its rounding with the tokens before it.
                const float factor = lane > 0 ? decay_between(hi[tok], lo[tok], hi[lane < L ? lane - 1 : 0], lo[lane < L ? lane - 1 : 0]) : __builtin_amdgcn_exp2f(hi[0] + lo[0]);
                const unsigned long long resets = __ballot(lane < L && factor == 0.0f), behind_it = lane < 63 ? resets >> (lane + 1) : 0;
                const int end = behind_it ? lane + 1 + __builtin_ctzll(behind_it) : 64;
                for (int step = 1; step < 64; step <<= 1) {
                    const float u = __shfl_down(dG, step, 64);
                    if (lane + step < end) dG += u;
                }
                if (resets >> lane & 1) dG = 0.0f;
                const int t = t0 + lane;
                if (lane < L && t < a.T) {
                    const bool live = t < len;
                    if (a.dg) a.dg[b * a.sdg.batch + (long long)t * a.sdg.token + h * a.sdg.head] = live ? dG : 0.0f;
                    a.dbeta[b * a.sdbeta.batch + (long long)t * a.sdbeta.token + h * a.sdbeta.head] = live ? column + token_beta[tok] : 0.0f;
                }
            }
            __syncthreads();
        }
        // products of token pairs with K and Q, once for the group: the other waves take them
#pragma unroll
        for (int j = 0; j < NT; ++j)
            if (j <= (i | 1))
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = tile_index(i, 4 * g + r) * COL + tile_index(j, m);
                    Mq[at] = mq[j][r], Mk[at] = mk[j][r];
                }
        __syncthreads();
        return;
    }

    // the waves of the states.  Factors of a token go into its operand, so that dq and dk add up in one set of accumulators.  They are one value head's: what it adds to q.dq and
    // k.dk goes into the gradients of its gates (as the difference of running sums it would be lost beside a head whose gradients are some orders larger, and NaN behind one with
    // a NaN).  The sum over the heads of a key head waits in memory between them, 64 KiB for heads of 128.
    floatx4 accq[DT], acck[DT];
    const int tok = tile_index(i, m);
    // sums over the state's rows of q times accq and k times x
    auto dots = [&](const floatx4 (&x)[DT], float &q_sum, float &k_sum) {
        q_sum = k_sum = 0.0f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const Frag<PI> kf = load_frag<PI>(key + (U::K + (i * KB + kb) * PI) * 1024, lane), qf = load_frag<PI>(key + (U::Q + (i * KB + kb) * PI) * 1024, lane);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int t = 2 * kb + (e >> 2), r = e & 3;
                q_sum = fmaf(frag_value<PI>(qf, e), accq[t][r], q_sum);
                k_sum = fmaf(frag_value<PI>(kf, e), x[t][r], k_sum);
            }
        }
        q_sum += __shfl_xor(q_sum, 16, 64), q_sum += __shfl_xor(q_sum, 32, 64);
        k_sum += __shfl_xor(k_sum, 16, 64), k_sum += __shfl_xor(k_sum, 32, 64);
    };
    // sums over the heads before: tile t of dq (of dk from DT on), 16 bytes a lane
    auto sum_of = [&](int t) {
        unsigned off = lane * 16;
        asm volatile("" : "+v"(off));
        return behind(uniform((floatx4 *)mem.sums + ((((long long)kh * mem.chunks + chunk) * NT + i) * 2 * DT + t) * 64), off);
    };
    const int count = group * rounds;
    struct { float e[8], y[8], o[8]; } next;
    Frag<PM> ef, of, yf;
    auto load_round = [&](int round) {
        const int member = round / rounds, kb = round - member * rounds;
        load_row(mem.errors + part(member) * L * mem.dvp + 32 * kb, i, next.e);
        load_row(mem.d_values + part(member) * L * mem.dvp + 32 * kb, i, next.y);
        load_do(member, kb, next.o);
    };
    // Splits the errors and gradients of a round: for the waves of token pairs, and with the token's factor for this one.
    auto split_round = [&](int round, float decay) {
        unsigned char *panel = lds + (round & 1) * Lds::UNITS * 1024;
        ef = make_frag<PM>(next.e);
        store_frag<PM>(panel + (Lds::ERR + i * PM) * 1024, lane, ef);
        store_frag<PM>(panel + (Lds::Y + i * PM) * 1024, lane, make_frag<PM>(next.y));
        float u[8], w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = a.scale * decay * next.o[e], w[e] = -decay * next.y[e];
        of = make_frag<PM>(u), yf = make_frag<PM>(w);
    };
    auto gates_of = [&](int member) { return (const DeltaGates<L> *)(mem.value + part(member) * mem.value_units * 1024); };
    load_round(0);
    split_round(0, gates_of(0)->decay[tok]);
    if (count > 1) load_round(1);
    float next_fe = gates_of(0)->left[tok], next_be = gates_of(0)->beta[tok], next_decay = gates_of(0)->decay[tok];
    for (int member = 0; member < group; ++member) {
        const float fe = next_fe, be = next_be, decay = next_decay;
        const DeltaGates<L> *gates = gates_of(min(member + 1, group - 1));          // those of the next one come during this one's rounds
        next_fe = gates->left[tok], next_be = gates->beta[tok], next_decay = gates->decay[tok];
        floatx4 he[DT];
#pragma unroll
        for (int t = 0; t < DT; ++t) accq[t] = acck[t] = he[t] = floatx4{0, 0, 0, 0};
        float q_sum, k_sum, e_sum, unused;
        for (int kb = 0; kb < rounds; ++kb) {
            const unsigned char *panel = lds + ((member * rounds + kb) & 1) * Lds::UNITS * 1024;
            __syncthreads();
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const Frag<PM> sf = load_frag<PM>(panel + (Lds::S + t * PM) * 1024, lane), df = load_frag<PM>(panel + (Lds::D + t * PM) * 1024, lane);
#pragma unroll
                for (int sum = 2; sum >= 0; --sum)
#pragma unroll
                    for (int p = 0; p <= sum; ++p) {
                        accq[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sf.part(p), of.part(sum - p), accq[t], 0, 0, 0);
                        acck[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sf.part(p), yf.part(sum - p), acck[t], 0, 0, 0);
                        he[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(df.part(p), ef.part(sum - p), he[t], 0, 0, 0);
                    }
            }
            const int round = member * rounds + kb + 1;
            if (round < count) split_round(round, kb + 1 < rounds ? decay : next_decay);
            if (round + 1 < count) load_round(round + 1);
        }
        dots(acck, q_sum, k_sum);
        dots(he, unused, e_sum);
        const float tb = fe * e_sum;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) acck[t][r] = fmaf(be * fe, he[t][r], acck[t][r]);
        if (g == 0) token_g[tok] = q_sum + k_sum, token_beta[tok] = tb;
        if (member > 0) {              // all loads of a half on their way before the first is waited for
            floatx4 before[DT];
#pragma unroll
            for (int t = 0; t < DT; ++t) before[t] = *sum_of(t);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < DT; ++t) accq[t] += before[t], before[t] = *sum_of(DT + t);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < DT; ++t) acck[t] += before[t];
        }
        if (member + 1 < group)
#pragma unroll
            for (int t = 0; t < DT; ++t) *sum_of(t) = accq[t], *sum_of(DT + t) = acck[t];
        __syncthreads();
        __syncthreads();
    }
    __syncthreads();             // the matrices of token pairs are there
    const int row = tile_index(i, m);
#pragma unroll
    for (int kb = 0; kb < LB; ++kb) {
        float u[8];
        Frag<PM> lowq{}, highq{}, sym{};
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = 0.0f;
        if (kb <= i / 2) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = Mq[row * COL + 32 * kb + 8 * g + e], u[e] += Mk[row * COL + 32 * kb + 8 * g + e];
            lowq = make_frag<PM>(w);
        }
        if (kb >= i / 2) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = Mq[(32 * kb + 8 * g + e) * COL + row], u[e] += Mk[(32 * kb + 8 * g + e) * COL + row];
            highq = make_frag<PM>(w);
        }
        sym = make_frag<PM>(u);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            const Frag<PI> kt = load_frag<PI>(key + (U::KT + (t * LB + kb) * PI) * 1024, lane);
            acck[t] = mm<3>(kt, sym, acck[t]);
            accq[t] = mm<3>(kt, lowq, accq[t]);           // zeros where the block lies above the diagonal
            acck[t] = mm<3>(load_frag<PI>(key + (U::QT + (t * LB + kb) * PI) * 1024, lane), highq, acck[t]);
        }
    }
    if (token < a.T)
#pragma unroll
        for (int s = 0; s < KB; ++s) {
            float u[8], w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = token < len ? accq[2 * s + (e >> 2)][e & 3] : 0.0f, w[e] = token < len ? acck[2 * s + (e >> 2)][e & 3] : 0.0f;
            store8(dq + 32 * s + 8 * g, a.Dk - 32 * s - 8 * g, vec.dq, u);
            store8(dk + 32 * s + 8 * g, a.Dk - 32 * s - 8 * g, vec.dk, w);
        }
}

}  // namespace tfno
