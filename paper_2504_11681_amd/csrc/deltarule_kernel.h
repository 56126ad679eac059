// The gated delta rule over whole sequences, by chunks of L tokens.  Token by token a head's state S [Dk, Dv] follows
//
//   Sb = exp(g_t) S,   e_t = v_t - Sb' k_t,   S <- Sb + k_t (beta_t e_t)',   o_t = scale S' q_t.
//
// With a chunk's incoming state S, G the running sum of g in it, M_ij = exp(G_i - G_j) for j <= i (no exponent of a sum is ever
// taken apart, so nothing overflows where decays are strong):
//
//   A = strict(M . K K'),   T = (I + A diag(beta))^-1,   P = M . Q K',
//   E = T (V - e^G (K S)),   U = beta E,
//   O = scale (e^G (Q S) + P U),   S <- e^GL S + K' (e^(GL-G) U).
//
// k_delta_prepare forms what does not depend on S for all chunks at once, k_delta_scan walks through the chunks.  Everything of it
// that the scan reads is laid out as operands of the matrix instructions.
//
// An operand block is 16 rows by 32 columns: lane (m, g) = (lane % 16, lane / 16) holds row m, columns 8 g .. 8 g + 7.  A result tile
// has its column in m and rows 4 g .. 4 g + 3.  Rows of tiles 2 s and 2 s + 1 are taken in the order
//
//   row r of tile 2 s + p  <->  index 32 s + 8 (r / 4) + 4 p + r % 4,
//
// so that the two results of a pair hold in each lane just the eight consecutive indexes that an operand block needs: a result becomes
// an operand without leaving its registers.
//
// Float32 values (the state, E, U, T, P, and float32 inputs) are operands as three BF16 parts that add up to them: the second is below 2^-7 of the value, the third
// at most 2^-16 and of either sign.  Products of the second and the third are left out, 2^-22 of a product at most and 2^-24 in the mean square, so sums have float32's accuracy.
// BF16 inputs are one part.  What goes into a BF16 output alone (P, U, and S as the
// outputs read it) has three parts too: where a key is written over, Q S and P U are large and cancel, and with two parts, 2^-15 off, outputs a
// thousandth of the old value were 2e-2 off.  That is a tenth of the time (256 x 1024 tokens, 2 heads of 64: 205 -> 224 us).
#pragma once
#include "bf16x3.h"
#include "deltarule.h"

namespace tfno {

typedef float floatx4 __attribute__((ext_vector_type(4)));

// An operand block: a lane's eight values in P parts of BF16 each.
template <int P>
struct Frag {
    uintx4 w[P];
    __device__ __forceinline__ bf16x8 part(int i) const { return __builtin_bit_cast(bf16x8, w[i]); }
};

// x minus the low (high) one of the two BF16 values in w: a dot product of pairs with (-1, 0) resp. (0, -1), exact, one instruction instead of a mask
// and a subtraction.  The constants are held in registers behind the compiler's back: as an inline constant -1.0 means the high half alone.
__device__ __forceinline__ float minus_low(unsigned w, float x)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    unsigned c = 0x0000bf80u;
    asm("" : "+s"(c));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, w), __builtin_bit_cast(pair, c), x, false);
}
__device__ __forceinline__ float minus_high(unsigned w, float x)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    unsigned c = 0xbf800000u;
    asm("" : "+s"(c));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair, w), __builtin_bit_cast(pair, c), x, false);
}

// Values 4 e .. 4 e + 3: two pairs in step, since a dot product's result is not there for the next instruction.  The first part is cut off, which no value overflows,
// the others are rounded to nearest: cut off too, the last one would have its value's sign, and what products leave out would add up.
template <int P>
__device__ __forceinline__ void set_four(Frag<P> &f, int e, const float (&x)[4])
{
    float r[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const unsigned u = p ? bf16_pair(r[0], r[1]) : pack_bf16(r[0], r[1]), v = p ? bf16_pair(r[2], r[3]) : pack_bf16(r[2], r[3]);
        if (p + 1 < P) r[0] = minus_low(u, r[0]), r[1] = minus_high(u, r[1]), r[2] = minus_low(v, r[2]), r[3] = minus_high(v, r[3]);
        f.w[p][2 * e] = u, f.w[p][2 * e + 1] = v;
    }
}
template <int P>
__device__ __forceinline__ Frag<P> make_frag(const float (&x)[8])
{
    Frag<P> f;
    set_four<P>(f, 0, {x[0], x[1], x[2], x[3]});
    set_four<P>(f, 1, {x[4], x[5], x[6], x[7]});
    return f;
}

// c + A B with the products of parts i, j that have i + j < CUT
template <int CUT, int PA, int PB>
__device__ __forceinline__ floatx4 mm(const Frag<PA> &a, const Frag<PB> &b, floatx4 c)
{
#pragma unroll
    for (int sum = CUT - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (sum - i >= 0 && sum - i < PB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part(i), b.part(sum - i), c, 0, 0, 0);
    return c;
}

// Work that is spread over the matrix instructions of a region: piece(k) after every EVERY of them, in exactly that order.  A wave issues in order
// and a matrix instruction runs for 16 cycles, so what stands between two of them costs nothing until it fills those.
template <int EVERY, int PIECES, class F>
struct Weave {
    F piece;
    int count = 0;
    __device__ __forceinline__ explicit Weave(F f) : piece(f) {}
    __device__ __forceinline__ void step()
    {
        if (++count % EVERY == 0 && count / EVERY <= PIECES) {
            __builtin_amdgcn_sched_barrier(0);
            piece(count / EVERY - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __device__ __forceinline__ void rest()
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
            if (k >= count / EVERY) piece(k);
        __builtin_amdgcn_sched_barrier(0);
    }
};
template <int EVERY, int PIECES, class F>
__device__ __forceinline__ Weave<EVERY, PIECES, F> weave(F f) { return Weave<EVERY, PIECES, F>(f); }
struct NoWeave { __device__ __forceinline__ void step() {} };

// c[n] + A[n] B (with SWAP c[n] + B A[n]) for N accumulators that do not depend on each other.
template <int CUT, bool SWAP, int N, int PA, int PB, class W>
__device__ __forceinline__ void mm_many(const Frag<PA> (&a)[N], const Frag<PB> &b, floatx4 *const (&c)[N], W &&between)
{
#pragma unroll
    for (int sum = CUT - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (sum - i >= 0 && sum - i < PB)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    *c[n] = SWAP ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.part(sum - i), a[n].part(i), *c[n], 0, 0, 0)
                                 : __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[n].part(i), b.part(sum - i), *c[n], 0, 0, 0);
                    between.step();
                }
}
// Matrix instructions of a product of PA and PB parts.
constexpr int products(int PA, int PB, int CUT)
{
    int n = 0;
    for (int i = 0; i < PA; ++i)
        for (int j = 0; j < PB; ++j) n += i + j < CUT;
    return n;
}
constexpr int at_least_1(int n) { return n > 0 ? n : 1; }
__device__ __forceinline__ void region_end() { __builtin_amdgcn_sched_barrier(0); }
// Values that are wanted here and not where the compiler would rather compute them, behind the branches that follow.
template <int P>
__device__ __forceinline__ void hold(Frag<P> &f)
{
#pragma unroll
    for (int p = 0; p < P; ++p) asm volatile("" : "+v"(f.w[p]));
}

template <int P>
__device__ __forceinline__ Frag<P> load_frag(const unsigned char *unit, int lane)
{
    Frag<P> f;
#pragma unroll
    for (int p = 0; p < P; ++p) f.w[p] = *reinterpret_cast<const uintx4 *>(unit + p * 1024 + lane * 16);
    return f;
}
template <int P>
__device__ __forceinline__ void store_frag(unsigned char *unit, int lane, const Frag<P> &f)
{
#pragma unroll
    for (int p = 0; p < P; ++p) *reinterpret_cast<uintx4 *>(unit + p * 1024 + lane * 16) = f.w[p];
}
// The value that the parts of element e add up to.
template <int P>
__device__ __forceinline__ float frag_value(const Frag<P> &f, int e)
{
    float v = 0.0f;
#pragma unroll
    for (int p = P - 1; p >= 0; --p) v += __uint_as_float(e & 1 ? f.w[p][e >> 1] & 0xffff0000u : f.w[p][e >> 1] << 16);
    return v;
}

// index of row r of tile i
__device__ __forceinline__ int tile_index(int i, int r) { return 32 * (i >> 1) + 8 * (r >> 2) + 4 * (i & 1) + (r & 3); }

// What the kernels are built for.  BF16: chunks of 64, one part an input; float32: chunks of 32 (its operands are three times as large),
// three parts.
template <class E> struct DeltaKind;
template <> struct DeltaKind<bf16> { static constexpr int L = 64, PI = 1; };
template <> struct DeltaKind<float> { static constexpr int L = 32, PI = 3; };

constexpr int DELTA_PM = 3;      // parts of float32 operands

// Memory of a chunk, in units of 1024 bytes (one part of an operand block).  KB = ceil(Dk / 32).
template <class E, int KB>
struct DeltaUnits {
    static constexpr int L = DeltaKind<E>::L, PI = DeltaKind<E>::PI;
    static constexpr int NT = L / 16, LB = L / 32, DT = 2 * KB, DKP = 32 * KB;
    static constexpr int TRI = NT == 2 ? 2 : 6;                    // blocks on and below the diagonal
    // of a key head: K, Q [NT][KB], K', Q' [DT][LB]
    static constexpr int K = 0, Q = NT * KB * PI, KT = 2 * NT * KB * PI, QT = KT + DT * LB * PI;
    static constexpr int KEY_FORWARD = QT, KEY_TAPE = QT + DT * LB * PI;
    // of a value head: gates, T, P; with a tape T', P'
    static constexpr int GATES = 0, T = 1, P = T + TRI * DELTA_PM, VALUE_FORWARD = P + TRI * DELTA_PM;
    static constexpr int TT = VALUE_FORWARD, PT = TT + TRI * DELTA_PM, VALUE_TAPE = PT + TRI * DELTA_PM;
    static constexpr int lower(int i, int kb) { return NT == 2 ? i : i < 2 ? i : 2 + 2 * (i - 2) + kb; }   // kb <= i / 2
    static constexpr int upper(int i, int kb) { return NT == 2 ? i : i < 2 ? 2 * i + kb : 4 + (i - 2); }   // kb >= i / 2
};

// Gates of a chunk of a value head, as they lie in its first unit.
template <int L>
struct DeltaGates {
    float decay[L];        // exp(G)
    float beta[L];
    float left[L];         // exp(GL - G)
    float whole;           // exp(GL)
};
constexpr int DELTA_ZEROS = 1024 - 16;      // behind them in that unit: 16 bytes of zeros, where `rows` is set


// Where the parts of a call's memory lie.
struct DeltaMemory {
    unsigned char *key, *value;      // units of the key heads' and of the value heads' chunks, [b][head][chunk]
    float *logs;                     // tape: [b][hv][chunk][2][L] running sums of g in powers of two, as sums of two floats
    float *states, *errors;          // tape: S before each chunk [DKP][DVP], E [L][DVP]
    float *d_states, *d_values;      // backward: gradient of the state after each chunk, Y [L][DVP]
    float *sums;                     // backward, where value heads share key heads: gradients of q and k from the value heads so far, [b][hk][chunk][2][L][DKP]
    int chunks, dvp, key_units, value_units;
    // Where there are few heads, the chunks of a head are walked through in segments at once: a segment's effect on the state is S -> A S + B.
    int segments, segment_chunks;
    float *effects;                  // [b][hv][segment][DKP][DVP + DKP]: B and A (tape)
    float *segment_states;           // [b][hv][segment][DKP][DVP]: the state before each
    float *back_effects;             // backward: [b][hv][segment][DKP][DVP]: the gradient that a segment itself adds to that of the state before it
    float *segment_d_states;         // backward: the gradient of the state after each segment
    bool rows;                       // the scans take K and Q from the caller's tensors: no blocks of them
    bool vec_o, vec_dv;              // rows of o and of the gradient of v take four elements at a time
};

__device__ __forceinline__ int sequence_length(const DeltaArgs &a, int b)
{
    if (!a.lengths) return a.T;
    const int n = __builtin_amdgcn_readfirstlane(a.lengths[b]);
    return n < 0 ? 0 : n < a.T ? n : a.T;
}

// Eight neighbouring elements of which the first n count (the others are 0); one access where `vec` says that addresses allow it.
__device__ __forceinline__ void load8(const float *p, int n, bool vec, float (&x)[8])
{
    if (vec && n >= 8) {
        const float4 u = reinterpret_cast<const float4 *>(p)[0], v = reinterpret_cast<const float4 *>(p)[1];
        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
    } else if (n > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p[e < n ? e : 0];       // loads without branches between them
#pragma unroll
        for (int e = 1; e < 8; ++e) x[e] = e < n ? x[e] : 0.0f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    }
}
__device__ __forceinline__ void load8(const bf16 *p, int n, bool vec, float (&x)[8])
{
    if (vec && n >= 8) {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(w[e] << 16), x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    } else if (n > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = to_float(p[e < n ? e : 0]);       // loads without branches between them
#pragma unroll
        for (int e = 1; e < 8; ++e) x[e] = e < n ? x[e] : 0.0f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    }
}
__device__ __forceinline__ void store8(float *p, int n, bool vec, const float (&x)[8])
{
    if (vec && n >= 8) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = x[e];
    }
}
__device__ __forceinline__ void store8(bf16 *p, int n, bool vec, const float (&x)[8])
{
    if (vec && n >= 8) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) store_element(p + e, x[e]);
    }
}

// Eight float32 values of LDS whose address is a multiple of 16.
__device__ __forceinline__ void load_gates(const float *p, float (&x)[8])
{
    const float4 u = reinterpret_cast<const float4 *>(p)[0], v = reinterpret_cast<const float4 *>(p)[1];
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
}

struct DeltaVec { bool q, k, d_o, dq, dk; };       // which tensors' rows may be read eight elements at a time

// ---------------------------------------------------------------------------------------------------------------------------------
// An operand block from LDS: eight elements of one row.
template <int P>
__device__ __forceinline__ Frag<P> row_frag(const float *p)
{
    float u[8];
    load8(p, 8, true, u);
    return make_frag<P>(u);
}
template <int P>
__device__ __forceinline__ Frag<P> row_frag(const bf16 *p)
{
    static_assert(P == 1, "BF16 is one part");
    Frag<P> f;
    f.w[0] = *reinterpret_cast<const uintx4 *>(p);
    return f;
}
// The same of one column, rows `stride` apart.
template <int P>
__device__ __forceinline__ Frag<P> column_frag(const float *p, int stride)
{
    float u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = p[e * stride];
    return make_frag<P>(u);
}
template <int P>
__device__ __forceinline__ Frag<P> column_frag(const bf16 *p, int stride)
{
    static_assert(P == 1, "BF16 is one part");
    Frag<P> f;
#pragma unroll
    for (int e = 0; e < 4; ++e) f.w[0][e] = p[2 * e * stride].bits | (unsigned)p[(2 * e + 1) * stride].bits << 16;
    return f;
}
// Eight elements of a row of memory to LDS, zeros past the n-th.
template <class E>
__device__ __forceinline__ void row_to_lds(const E *p, int n, bool vec, E *to)
{
    if (vec && n >= 8) {
        constexpr int W = 8 * sizeof(E) / 16;
#pragma unroll
        for (int w = 0; w < W; ++w) reinterpret_cast<uint4 *>(to)[w] = reinterpret_cast<const uint4 *>(p)[w];
    } else {
        float u[8];
        load8(p, n, false, u);
        store8(to, 8, true, u);
    }
}

// exp(G_i - G_j) from running sums in powers of two that are sums of two floats: exact differences also after a reset.
__device__ __forceinline__ float decay_between(float hi_i, float lo_i, float hi_j, float lo_j) { return __builtin_amdgcn_exp2f((hi_i - hi_j) + (lo_i - lo_j)); }

// One workgroup for a chunk of a value head: L / 16 waves.  256 x 1024 tokens of 2 heads of 64 in BF16 without a tape: 105 us in one piece for 61 KiB a chunk, 4.9 TB/s
// of the 5.1 that a copy reaches, 60 in each of two; its chain of barriers was the bound while its loads came one after the other (by a quarter).  Nothing passes through LDS
// that need not: a wave takes the pairs of tokens whose column is in its own tile, and P comes out as an operand block as it is.  The inverse T of the unit lower triangular matrix I + N is found by blocks of 16: each diagonal
// block by substitution, a column after the other, the blocks below it from T_IJ = -T_II sum_{J<=M<I} N_IM T_MJ, one wave for a block column.
// Substitution and not the product (I - N)(I + N^2)(I + N^4)..: its powers grow like binomials where keys are alike, and cancel.
template <class E, int KB, bool TAPE>
__global__ __launch_bounds__((4 * DeltaKind<E>::L)) void k_delta_prepare(DeltaArgs a, DeltaMemory mem, DeltaVec vec)
{
    typedef DeltaUnits<E, KB> U;
    constexpr int L = U::L, NT = U::NT, LB = U::LB, DT = U::DT, DKP = U::DKP, PI = U::PI, PM = DELTA_PM;
    constexpr int ROW = DKP + 16 / sizeof(E), COL = L + 4;
    constexpr int ROWS_BYTES = 2 * L * ROW * sizeof(E), MATRIX_BYTES = L * COL * 4;
    __shared__ __attribute__((aligned(16))) unsigned char shared[ROWS_BYTES > MATRIX_BYTES ? ROWS_BYTES : MATRIX_BYTES];
    __shared__ __attribute__((aligned(16))) float N[L * COL];      // its columns: N[j * COL + i] is row i, column j
    __shared__ float hi[L], lo[L], beta[L];
    E *Ks = (E *)shared, *Qs = Ks + L * ROW;
    float *X = (float *)shared;                                    // T, once K and Q are done with

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15, g = lane >> 4;
    const int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int group = a.Hv / a.Hk, member = id % group, at = id / group;   // value heads that share keys are neighbours
    const int chunk = at % mem.chunks, kh = at / mem.chunks, b = kh / a.Hk, hk = kh - b * a.Hk, h = hk * group + member;
    const long long head = (long long)b * a.Hv + h;
    const bool first = member == 0;                                 // this workgroup writes the key head's blocks too
    const int len = sequence_length(a, b), t0 = chunk * L;
    if (t0 >= len) return;
    unsigned char *key = mem.key + ((long long)kh * mem.chunks + chunk) * mem.key_units * 1024;
    unsigned char *value = mem.value + (head * mem.chunks + chunk) * mem.value_units * 1024;

    const E *k = (const E *)a.k + (b * a.sk.batch + (long long)t0 * a.sk.token + hk * a.sk.head);
    const E *q = (const E *)a.q + (b * a.sq.batch + (long long)t0 * a.sq.token + hk * a.sq.head);
    // All loads of a chunk are on their way before the first is waited for: one after the other they were 15 of 32 thousand cycles (heads of 64).
    const bool live = wave == 0 && lane < L && t0 + lane < len;
    float be = 0.0f, log_decay = 0.0f;
    if (live) {
        be = a.beta[b * a.sbeta.batch + (long long)(t0 + lane) * a.sbeta.token + h * a.sbeta.head];
        if (a.g) log_decay = a.g[b * a.sg.batch + (long long)(t0 + lane) * a.sg.token + h * a.sg.head];
    }
    constexpr int LOADS = L * DKP / 8 / (64 * NT), QUADS = 8 * sizeof(E) / 16;
    if (vec.k && vec.q && a.Dk % 8 == 0) {
        uint4 kx[LOADS][QUADS], qx[LOADS][QUADS];
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int s = tid + x * 64 * NT, row = s / (DKP / 8), d = s % (DKP / 8) * 8;
            const bool there = t0 + row < len && d < a.Dk;         // the chunk's first token in place of what does not count
            const uint4 *kp = (const uint4 *)(k + (there ? row * a.sk.token + d : 0)), *qp = (const uint4 *)(q + (there ? row * a.sq.token + d : 0));
#pragma unroll
            for (int w = 0; w < QUADS; ++w) kx[x][w] = kp[w], qx[x][w] = qp[w];
        }
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int s = tid + x * 64 * NT, row = s / (DKP / 8), d = s % (DKP / 8) * 8;
            const bool there = t0 + row < len && d < a.Dk;
#pragma unroll
            for (int w = 0; w < QUADS; ++w) {
                ((uint4 *)(Ks + row * ROW + d))[w] = there ? kx[x][w] : uint4{0, 0, 0, 0};
                ((uint4 *)(Qs + row * ROW + d))[w] = there ? qx[x][w] : uint4{0, 0, 0, 0};
            }
        }
    } else {
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int s = tid + x * 64 * NT, row = s / (DKP / 8), d = s % (DKP / 8) * 8, n = t0 + row < len ? a.Dk - d : 0;
            row_to_lds(k + row * a.sk.token + d, n, vec.k, Ks + row * ROW + d);
            row_to_lds(q + row * a.sq.token + d, n, vec.q, Qs + row * ROW + d);
        }
    }
    if (wave == 0) {
        // running sums of g in 64 bits; what is below any exponent counts as -1e5 each, so that differences past a reset stay exact
        double s = log_decay < -1e5f ? -1e5 : (double)log_decay;
        for (int step = 1; step < L; step <<= 1) {
            const double u = __shfl_up(s, step, 64);
            if (lane >= step) s += u;
        }
        s *= 1.4426950408889634;
        const double all = __shfl(s, L - 1, 64);
        if (lane < L) {
            const float h0 = (float)s, l0 = (float)(s - (double)h0);
            hi[lane] = h0, lo[lane] = l0;
            beta[lane] = be;
            DeltaGates<L> *gates = (DeltaGates<L> *)value;
            gates->decay[lane] = __builtin_amdgcn_exp2f((float)s);
            gates->beta[lane] = be;
            gates->left[lane] = __builtin_amdgcn_exp2f((float)(all - s));
            if (lane == 0) gates->whole = __builtin_amdgcn_exp2f((float)all);
            if (lane == 0 && !TAPE) *(uint4 *)(value + DELTA_ZEROS) = uint4{0, 0, 0, 0};
            if (TAPE) {
                float *logs = mem.logs + (head * mem.chunks + chunk) * 2 * L;
                logs[lane] = h0, logs[L + lane] = l0;
            }
        }
    }
    __syncthreads();

    {
        const int w = wave, own = tile_index(w, m);                 // the lane's token
        floatx4 kk[NT], qk[NT], kq[NT];                             // k_row.k_own, q_row.k_own and k_row.q_own
#pragma unroll
        for (int i = 0; i < NT; ++i) kk[i] = qk[i] = kq[i] = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const Frag<PI> kf = row_frag<PI>(Ks + own * ROW + 32 * kb + 8 * g), qf = row_frag<PI>(Qs + own * ROW + 32 * kb + 8 * g);
            if (first && (TAPE || !mem.rows)) {
                store_frag<PI>(key + (U::K + (w * KB + kb) * PI) * 1024, lane, kf);
                store_frag<PI>(key + (U::Q + (w * KB + kb) * PI) * 1024, lane, qf);
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {            // all tiles, the unused ones too: no branches between the products
                const int at = tile_index(i, m) * ROW + 32 * kb + 8 * g;
                const Frag<PI> other = row_frag<PI>(Ks + at);
                kk[i] = mm<3>(other, kf, kk[i]);
                kq[i] = mm<3>(other, qf, kq[i]);
                if (TAPE) qk[i] = mm<3>(row_frag<PI>(Qs + at), kf, qk[i]);
            }
        }
        // Results are read here, in the line of their products, and not behind the branches that follow: this kernel once gave a wrong inverse where products and the reads of their
        // results had uniform branches between them, for a cause that was not found (the compiler leaves as many wait states there as in a line).
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            asm volatile("" : "+v"(kk[i]), "+v"(kq[i]));
            if (TAPE) asm volatile("" : "+v"(qk[i]));
        }
        const float hi_own = hi[own], lo_own = lo[own], beta_own = beta[own];
#pragma unroll
        for (int s = 0; s < LB; ++s) {
            float h8[8], l8[8], u[8];
            load_gates(hi + 32 * s + 8 * g, h8);
            load_gates(lo + 32 * s + 8 * g, l8);
            if (s >= w / 2) {           // the lane's token is the column: N, and with a tape P'
                float n[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int row = 32 * s + 8 * g + e;
                    const float decay = decay_between(h8[e], l8[e], hi_own, lo_own);
                    n[e] = own < row ? decay * kk[2 * s + (e >> 2)][e & 3] * beta_own : 0.0f;
                    u[e] = own <= row ? decay * qk[2 * s + (e >> 2)][e & 3] : 0.0f;
                }
                store8(N + own * COL + 32 * s + 8 * g, 8, true, n);
                if (TAPE) store_frag<PM>(value + (U::PT + U::upper(w, s) * PM) * 1024, lane, make_frag<PM>(u));
            }
            if (s <= w / 2) {           // the lane's token is the row: P
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    u[e] = 32 * s + 8 * g + e <= own ? decay_between(hi_own, lo_own, h8[e], l8[e]) * kq[2 * s + (e >> 2)][e & 3] : 0.0f;
                store_frag<PM>(value + (U::P + U::lower(w, s) * PM) * 1024, lane, make_frag<PM>(u));
            }
        }
        if (first)         // K' and Q': tiles of Dk rows, blocks of 32 tokens
#pragma unroll
            for (int x = 0; x < DT * LB / NT; ++x) {
                const int y = w + x * NT, t = y / LB, kb = y % LB, from = (32 * kb + 8 * g) * ROW + tile_index(t, m);
                store_frag<PI>(key + (U::KT + y * PI) * 1024, lane, column_frag<PI>(Ks + from, ROW));
                if (TAPE) store_frag<PI>(key + (U::QT + y * PI) * 1024, lane, column_frag<PI>(Qs + from, ROW));
            }
    }
    __syncthreads();

    // the diagonal block of a wave: lane m has its column m, and takes row after row off the ones below it
    const int J = wave;
    floatx4 col[NT];
    {
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = i == m ? 1.0f : 0.0f;
#pragma unroll
        for (int j = 0; j < 15; ++j) {
            float n[16];
#pragma unroll
            for (int i = (j + 1) & ~3; i < 16; i += 4) {
                const float4 u = *reinterpret_cast<const float4 *>(N + (16 * J + j) * COL + 16 * J + i);
                n[i] = u.x, n[i + 1] = u.y, n[i + 2] = u.z, n[i + 3] = u.w;
            }
#pragma unroll
            for (int i = j + 1; i < 16; ++i) x[i] = fmaf(-n[i], x[j], x[i]);
        }
        if (g == 0) {
#pragma unroll
            for (int i = 0; i < 16; ++i) X[(16 * J + i) * COL + 16 * J + m] = x[i];
        } else if (g == 1 && (J & 1)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) X[(16 * (J - 1) + i) * COL + 16 * J + m] = 0.0f;     // right of the pair's first diagonal block
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) col[0][r] = g == 0 ? x[r] : g == 1 ? x[4 + r] : g == 2 ? x[8 + r] : x[12 + r];
    }
    __syncthreads();
#pragma unroll
    for (int step = 1; step < NT; ++step) {
        const int I = J + step;
        if (I >= NT) break;
        floatx4 sum = {0, 0, 0, 0}, out = {0, 0, 0, 0};
#pragma unroll
        for (int M = 0; M < step; ++M)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                sum = __builtin_amdgcn_mfma_f32_16x16x4f32(N[(16 * (J + M) + 4 * g + r) * COL + 16 * I + m], col[M][r], sum, 0, 0, 0);
        const float4 diagonal = *reinterpret_cast<const float4 *>(X + (16 * I + m) * COL + 16 * I + 4 * g);
        const float d[4] = {diagonal.x, diagonal.y, diagonal.z, diagonal.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) out = __builtin_amdgcn_mfma_f32_16x16x4f32(d[r], sum[r], out, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            col[step][r] = -out[r];
            X[(16 * I + 4 * g + r) * COL + 16 * J + m] = -out[r];
        }
    }
    __syncthreads();
    {
        const int i = wave, row = tile_index(i, m);
#pragma unroll
        for (int kb = 0; kb < LB; ++kb) {
            if (kb <= i / 2) store_frag<PM>(value + (U::T + U::lower(i, kb) * PM) * 1024, lane, row_frag<PM>(X + row * COL + 32 * kb + 8 * g));
            if (TAPE && kb >= i / 2) store_frag<PM>(value + (U::TT + U::upper(i, kb) * PM) * 1024, lane, column_frag<PM>(X + (32 * kb + 8 * g) * COL + row, COL));
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// An address that is the same for all lanes, in scalar registers.
template <class T>
__device__ __forceinline__ T *uniform(T *p)
{
    const uintptr_t u = (uintptr_t)p;
    return (T *)((uintptr_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)u));
}
// The element `bytes` behind a uniform address: 32 bits a lane, so that the address stays scalar.
template <class E>
__device__ __forceinline__ const E *behind(const E *p, unsigned bytes) { return (const E *)((const char *)p + bytes); }
template <class E>
__device__ __forceinline__ E *behind(E *p, unsigned bytes) { return (E *)((char *)p + bytes); }

// 16 bytes of each lane from global memory to LDS, 1024 bytes from `to` on, which is the same for all lanes.
__device__ __forceinline__ void lanes_to_lds(const void *from, const unsigned char *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
// Units of 1024 bytes from global memory to LDS by one wave; they are there for the others after its wait for its loads (s_waitcnt 0) and a barrier.
// The wave reads no LDS itself: before that the compiler would wait for all of them.
__device__ __forceinline__ void units_to_lds(const unsigned char *from, const unsigned char *to, int units, int lane)
{
    const unsigned at = lane * 16;          // a uniform address and 32 bits a lane
    from = uniform(from);
    for (int u = 0; u < units; ++u, to += 1024, from += 1024) lanes_to_lds(behind(from, at), to);
}

// A wave's column of one chunk, eight consecutive tokens for each pair of tiles, from a tensor [token, column] whose first token counts.  `at`
// is the lane's offset in bytes (8 g tokens and its column, or column 0 past the last one); distances of tokens are uniform.  In a chunk that ends early, the
// first token is read in place of those that do not count: loads without branches between them.
template <class E, int LB>
__device__ __forceinline__ void load_columns(const E *p, long long token, unsigned at, int g, int count, E (&u)[LB][8])
{
    if (count >= 32 * LB) {
        asm("" : "+v"(at));          // its extension to 64 bits belongs to the loads' addresses and not in front of the loop
        const E *q = uniform(p);
#pragma unroll
        for (int s = 0; s < LB; ++s, q += 24 * token)
#pragma unroll
            for (int e = 0; e < 8; ++e, q += token) u[s][e] = *behind(q, at);
    } else {
        p = behind(p, at) - 8 * g * token;
        int first = 8 * g;
        asm volatile("" : "+v"(first));        // its products with the distance belong here and not into registers that the loop's products need
#pragma unroll
        for (int s = 0; s < LB; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) u[s][e] = p[32 * s + first + e < count ? (32 * s + first + e) * token : 0];
    }
}
// Zeros in place of what does not count.
template <class E, int LB>
__device__ __forceinline__ void mask_columns(E (&u)[LB][8], bool all_columns, bool column, int g, int count)
{
    if (all_columns && count >= 32 * LB) return;
#pragma unroll
    for (int s = 0; s < LB; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) u[s][e] = column && 32 * s + 8 * g + e < count ? u[s][e] : E{};
}

// A wave's state: element r of tile t is row tile_index(t, 4 g + r), column `col`.
template <int DT>
__device__ __forceinline__ void load_state(const float *p, int Dk, int Dv, int col, int g, floatx4 (&S)[DT])
{
#pragma unroll
    for (int t = 0; t < DT; ++t) S[t] = floatx4{0, 0, 0, 0};
    if (!p) return;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = tile_index(t, 4 * g + r);
            S[t][r] = p[d < Dk && col < Dv ? d * Dv + col : 0];
        }
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (tile_index(t, 4 * g + r) >= Dk || col >= Dv) S[t][r] = 0.0f;
}
template <int DT>
__device__ __forceinline__ void store_state(float *p, int Dk, int Dv, int col, int g, const floatx4 (&S)[DT])
{
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = tile_index(t, 4 * g + r);
            if (d < Dk && col < Dv) p[d * Dv + col] = S[t][r];
        }
}
// A 4 x 4 transposition in each group of four lanes: element r of lane j becomes element j of lane r.
template <int CONTROL>
__device__ __forceinline__ float quad_move(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}
__device__ __forceinline__ floatx4 quad_transpose(const floatx4 &x, int lane)
{
    const bool odd = lane & 1, high = lane & 2;
    const float s0 = quad_move<0xB1>(odd ? x[0] : x[1]), s1 = quad_move<0xB1>(odd ? x[2] : x[3]);      // from the lane next to it
    const float a0 = odd ? s0 : x[0], a1 = odd ? x[1] : s0, a2 = odd ? s1 : x[2], a3 = odd ? x[3] : s1;
    const float u0 = quad_move<0x4E>(high ? a0 : a2), u1 = quad_move<0x4E>(high ? a1 : a3);            // from the other pair
    return floatx4{high ? u0 : a0, high ? u1 : a1, high ? a2 : u0, high ? a3 : u1};
}

// Tiles of rows tile_index(t, 4 g + r) and columns m of a matrix of `stride` columns in the memory between the kernels, 16 bytes a lane: after the
// transposition a lane has four columns of row j = lane % 4.  `at` = 8 g + j rows and the first of those columns, in bytes.  (One dword a row and
// lane took four times the instructions: a chunk's states and errors were 8000 of the 23000 cycles of a training scan.)
template <int N>
__device__ __forceinline__ void store_tiles(float *p, int stride, unsigned at, int lane, const floatx4 (&x)[N])
{
#pragma unroll
    for (int t = 0; t < N; ++t) *behind((floatx4 *)(p + (32 * (t >> 1) + 4 * (t & 1)) * stride), at) = quad_transpose(x[t], lane);
}
// The lane's offset for store_tiles.
__device__ __forceinline__ unsigned tiles_at(int stride, int col0, int lane)
{
    return ((8 * (lane >> 4) + (lane & 3)) * stride + col0 + (lane & 12)) * 4;
}

// LDS of a scan, in units: what a chunk needs first (FIRST) for two chunks, what its last products need (LAST) for two where that fits into 160,
// else for one.
template <int FIRST_, int LAST_>
struct ScanLds {
    static constexpr int FIRST = FIRST_, LAST = LAST_;
    static constexpr bool DOUBLE = 2 * (FIRST + LAST) <= 160;
    static constexpr int BYTES = (2 * FIRST + (DOUBLE ? 2 : 1) * LAST) * 1024;
    static __device__ __forceinline__ unsigned char *first(unsigned char *lds, int parity) { return lds + parity * FIRST * 1024; }
    static __device__ __forceinline__ unsigned char *last(unsigned char *lds, int parity) { return lds + (2 * FIRST + (DOUBLE ? parity * LAST : 0)) * 1024; }
};

// What a walk is for: outputs; outputs and a tape; the effect of each segment on the state alone.
enum { SCAN_OUTPUTS, SCAN_TAPE, SCAN_EFFECTS };
// K, Q, gates, T, P | K'; for effects without Q and P
template <class E, int KB, int MODE>
struct ForwardLds : ScanLds<(MODE == SCAN_EFFECTS ? DeltaUnits<E, KB>::Q + DeltaUnits<E, KB>::P : DeltaUnits<E, KB>::KT + DeltaUnits<E, KB>::VALUE_FORWARD),
                            DeltaUnits<E, KB>::QT - DeltaUnits<E, KB>::KT> {};

constexpr int SCAN_WAVES = 4, SCAN_THREADS = 64 * (SCAN_WAVES + 1);       // waves that compute, at most, and one that loads

// A workgroup walks through the chunks of one head, or of one segment of it, with 16 columns of its state a wave, which stay in the wave's registers.
// One more wave does nothing but bring the next chunk's blocks to LDS (75 cycles of issue each, 85 of them for heads of 128: a wave that
// computes would lose 3000 cycles to a half of them); K', where two chunks' do not fit (heads over 64), comes while the chunk's first products run.  Blocks are read from LDS
// one group ahead of their products, a group has several accumulators, and the splits stand between the products: 216 of them are 3500 cycles or 1.5 us,
// a chunk takes 4.6 us (B 1, T 16384, 8 heads of 128 in 16 segments: 73 us for the outputs; 86 for the effects) and 6.0 with a tape (B 4, T 2048, 16 heads of 128:
// 192 us), bound by one wave's issue; with many heads (256 x 1024 tokens, 2 heads of 64) it moves 77 KiB a chunk, in one piece in 167 us, 3.9 TB/s, in two, whose
// blocks come from the last-level cache, in 63 us each, 5.1 TB/s.  256 registers a wave, none of them accumulation registers, whose copies would cost as
// much as the splits.  Effects: columns of B start from zeros, columns of A from the identity, without values.
template <class E, int KB, int MODE>
__global__ __launch_bounds__(SCAN_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_delta_scan(DeltaArgs a, DeltaMemory mem, int blocks_per_head, int segments)
{
    typedef DeltaUnits<E, KB> U;
    constexpr int L = U::L, NT = U::NT, LB = U::LB, DT = U::DT, PI = U::PI, PM = DELTA_PM;
    constexpr bool TAPE = MODE == SCAN_TAPE, EFFECTS = MODE == SCAN_EFFECTS;
    typedef ForwardLds<E, KB, MODE> Lds;
    constexpr int A_UNITS = EFFECTS ? U::Q : U::KT, VALUE_UNITS = EFFECTS ? U::P : U::VALUE_FORWARD;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = (blockDim.x >> 6) - 1;      // and one that loads
    const int m = lane & 15, g = lane >> 4;
    const int id = xcd_contiguous(blockIdx.x, gridDim.x);       // the blocks of a head, and heads that share keys, on one XCD
    const int block = id % blocks_per_head, part = id / blocks_per_head, segment = part % segments, head = part / segments;
    const long long at = (long long)head * mem.segments + segment;
    const int b = head / a.Hv, h = head - b * a.Hv, hk = h / (a.Hv / a.Hk);
    const int len = sequence_length(a, b), all = (len + L - 1) / L;
    const int begin = segment * mem.segment_chunks, n = all < begin + mem.segment_chunks ? all : begin + mem.segment_chunks;   // chunks begin .. n - 1
    const unsigned char *key = mem.key + (long long)(b * a.Hk + hk) * mem.chunks * mem.key_units * 1024;
    const unsigned char *value = mem.value + (long long)head * mem.chunks * mem.value_units * 1024;
    const int col0 = (block * waves + wave) * 16, col = col0 + m;
    const bool all_columns = a.Dv % 32 == 0;

    floatx4 S[DT];
    if constexpr (EFFECTS) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = tile_index(t, 4 * g + r) == col - mem.dvp ? 1.0f : 0.0f;
    } else if (mem.segments > 1) load_state<DT>(mem.segment_states + at * U::DKP * mem.dvp, U::DKP, mem.dvp, col, g, S);
    else load_state<DT>(a.initial ? a.initial + (long long)head * a.Dk * a.Dv : nullptr, a.Dk, a.Dv, col, g, S);
    const E *v = (const E *)a.v + (b * a.sv.batch + h * a.sv.head);
    E *o = (E *)a.o + (b * a.so.batch + h * a.so.head);
    const unsigned at_v = (8 * g * (unsigned)a.sv.token + (col < a.Dv ? col : 0)) * sizeof(E);
    const unsigned at_tape = tiles_at(mem.dvp, col0, lane);
    const int lane_token = 8 * (m >> 2) + (m & 3);              // where tokens are columns: token lane_token of a tile, columns col0 + 4 g ..
    const unsigned at_o = (lane_token * (unsigned)a.so.token + 4 * g) * sizeof(E);

    // Blocks of a tensor of BF16 are its rows as they are, 16 bytes a lane; lanes past its end read zeros.
    auto rows_to_lds = [&](const void *x, const Strides &s, int chunk, unsigned char *to) {
        const E *p = (const E *)x + (b * s.batch + hk * s.head + (long long)(chunk * L + 8 * (m >> 2) + (m & 3)) * s.token + 8 * g);
        const void *zeros = value + (long long)chunk * mem.value_units * 1024 + DELTA_ZEROS;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const E *row = p + tile_index(i, 0) * s.token;
            const bool there = chunk * L + tile_index(i, m) < len;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb, to += 1024) lanes_to_lds(there && 32 * kb + 8 * g < a.Dk ? (const void *)(row + 32 * kb) : zeros, to);
        }
    };
    auto load_first = [&](int chunk, int parity) {
        unsigned char *to = Lds::first(lds, parity);
        if (PI == 1 && !TAPE && mem.rows) {
            rows_to_lds(a.k, a.sk, chunk, to);
            if (!EFFECTS) rows_to_lds(a.q, a.sq, chunk, to + U::Q * 1024);
        } else {
            units_to_lds(key + ((long long)chunk * mem.key_units + U::K) * 1024, to, A_UNITS, lane);
        }
        units_to_lds(value + (long long)chunk * mem.value_units * 1024, to + A_UNITS * 1024, VALUE_UNITS, lane);
    };
    auto load_last = [&](int chunk, int parity) {
        units_to_lds(key + ((long long)chunk * mem.key_units + U::KT) * 1024, Lds::last(lds, parity), Lds::LAST, lane);
    };
    E next[LB][8] = {};
    auto load_v = [&](int chunk) {
        if (EFFECTS && col0 >= mem.dvp) return;
        load_columns<E, LB>(v + (long long)chunk * L * a.sv.token, a.sv.token, at_v, g, len - chunk * L, next);
    };
    auto load_next = [&](int chunk) {
        if (!Lds::DOUBLE) load_last(chunk, chunk & 1);
        if (chunk + 1 < n) {
            load_first(chunk + 1, (chunk + 1) & 1);
            if (Lds::DOUBLE) load_last(chunk + 1, (chunk + 1) & 1);
        }
    };
    if (wave == waves) {
        if (n > begin) {
            load_first(begin, begin & 1);
            if (Lds::DOUBLE) load_last(begin, begin & 1);
        }
        for (int chunk = begin; chunk < n; ++chunk) {
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
    if (n > begin) load_v(begin);
    Frag<PM> Sf[KB];            // the state as operand
    auto split_s = [&](int kb) {
        float u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = S[2 * kb + (e >> 2)][e & 3];
        Sf[kb] = make_frag<PM>(u);
    };
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) split_s(kb);
    __builtin_amdgcn_s_waitcnt(0);
    for (int chunk = begin; chunk < n; ++chunk) {
        const int t0 = chunk * L, parity = chunk & 1;
        const unsigned char *ldsA = Lds::first(lds, parity), *ldsB = ldsA + A_UNITS * 1024, *ldsKT = Lds::last(lds, parity);
        const DeltaGates<L> *gates = (const DeltaGates<L> *)ldsB;
        __syncthreads();
        mask_columns<E, LB>(next, all_columns, col < a.Dv, g, len - t0);
        const int after = chunk + 1 < n ? chunk + 1 : chunk;
        if (TAPE && col0 < mem.dvp) store_tiles<DT>(mem.states + ((long long)head * mem.chunks + chunk) * U::DKP * mem.dvp, mem.dvp, at_tape, lane, S);
        region_end();

        // K S, tokens in rows; then (Q S)', tokens in columns, and meanwhile R = V - e^G K S as operand (effects: R alone)
        floatx4 KS[NT], QS[NT];
        Frag<PM> R[LB];
        {
            Frag<PI> kf[2][NT];
            auto read = [&](int unit, int kb, int to) {
#pragma unroll
                for (int i = 0; i < NT; ++i) kf[to][i] = load_frag<PI>(ldsA + (unit + (i * KB + kb) * PI) * 1024, lane);
            };
            floatx4 *ks[NT], *qs[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) KS[i] = QS[i] = floatx4{0, 0, 0, 0}, ks[i] = &KS[i], qs[i] = &QS[i];
            read(U::K, 0, 0);
            float decay[LB][8];
#pragma unroll
            for (int s = 0; s < LB; ++s) load_gates(gates->decay + 32 * s + 8 * g, decay[s]);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                if (kb + 1 < KB) read(U::K, kb + 1, (kb + 1) & 1);
                else if (!EFFECTS) read(U::Q, 0, (kb + 1) & 1);
                region_end();
                mm_many<3, false>(kf[kb & 1], Sf[kb], ks, NoWeave());
                region_end();
            }
            constexpr int MFMA = KB * NT * products(PI, PM, 3);
            auto pieces = weave<at_least_1(MFMA / (2 * LB)), 2 * LB>([&](int k) {
                const int s = k >> 1, e = k & 1;
                float u[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) u[r] = fmaf(-decay[s][4 * e + r], KS[2 * s + e][r], to_float(next[s][4 * e + r]));
                set_four<PM>(R[s], e, u);
            });
            if constexpr (!EFFECTS)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    if (kb + 1 < KB) read(U::Q, kb + 1, (KB + kb + 1) & 1);
                    region_end();
                    mm_many<3, true>(kf[(KB + kb) & 1], Sf[kb], qs, pieces);
                    region_end();
                }
            pieces.rest();
#pragma unroll
            for (int s = 0; s < LB; ++s) hold(R[s]);
        }
        load_v(after);

        // E = T R, the tokens of one pair of tiles after the other, and U = beta E as operand, for the outputs and times e^(GL-G) for the state, while
        // the products of the next pair run; then the outputs' P U and the first part of S <- e^GL S + K' (e^(GL-G) U) while the last pair is split
        floatx4 Ee[NT];
        Frag<PM> W[LB];
        Frag<PM> Uf[LB];
        float be[LB][8], left[LB][8], decay_o[NT];
        Frag<PM> tf[2][2];
        auto read_t = [&](int s, int kb, int to) {
#pragma unroll
            for (int p = 0; p < 2; ++p) tf[to][p] = load_frag<PM>(ldsB + (U::T + U::lower(2 * s + p, kb) * PM) * 1024, lane);
        };
        read_t(0, 0, 0);
#pragma unroll
        for (int i = 0; i < NT; ++i) decay_o[i] = EFFECTS ? 0.0f : gates->decay[tile_index(i, m)], Ee[i] = floatx4{0, 0, 0, 0};
        const float whole = gates->whole;
        auto split_u = [&](int s, int e) {
            float u[4], w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                u[r] = be[s][4 * e + r] * Ee[2 * s + e][r];
                w[r] = left[s][4 * e + r] * u[r];
            }
            if (!EFFECTS) set_four<PM>(Uf[s], e, u);
            set_four<PM>(W[s], e, w);
        };
        Frag<PM> pf[2][2];
        auto read_p = [&](int s, int kb, int to) {
#pragma unroll
            for (int p = 0; p < 2; ++p) pf[to][p] = load_frag<PM>(ldsB + (U::P + U::lower(2 * s + p, kb) * PM) * 1024, lane);
        };
        {
            floatx4 *to[2] = {&Ee[0], &Ee[1]};
            if (LB > 1) read_t(1, 0, 1);
            load_gates(gates->beta + 8 * g, be[0]);
            load_gates(gates->left + 8 * g, left[0]);
            region_end();
            auto pieces = weave<1, NT + DT>([&](int k) {
                if (k >= DT) QS[k - DT] *= decay_o[k - DT];
                else S[k] *= whole;
            });
            mm_many<3, false>(tf[0], R[0], to, pieces);
            if (LB > 1) read_t(1, 1, 0);
            if (!EFFECTS) read_p(0, 0, 0);
            pieces.rest();
        }
        if constexpr (LB > 1) {
            floatx4 *to[2] = {&Ee[2], &Ee[3]};
            auto pieces = weave<8, 2>([&](int e) { split_u(0, e); });
            mm_many<3, false>(tf[1], R[0], to, pieces);
            load_gates(gates->beta + 32 * (LB - 1) + 8 * g, be[LB - 1]);
            load_gates(gates->left + 32 * (LB - 1) + 8 * g, left[LB - 1]);
            mm_many<3, false>(tf[0], R[LB - 1], to, pieces);
            pieces.rest();
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) split_u(0, e);
        }
        if (TAPE && col0 < mem.dvp) store_tiles<NT>(mem.errors + ((long long)head * mem.chunks + chunk) * L * mem.dvp, mem.dvp, at_tape, lane, Ee);
        if (!Lds::DOUBLE) {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
        }
        // the updates of the state's pairs of tiles, first with tokens 0 .. 31, then with the others: blocks are read two updates ahead
        Frag<PI> kf[2][2];
        auto read_k = [&](int update) {
            if (update >= LB * KB) return;
#pragma unroll
            for (int p = 0; p < 2; ++p) kf[update & 1][p] = load_frag<PI>(ldsKT + ((2 * (update % KB) + p) * LB + update / KB) * PI * 1024, lane);
        };
        floatx4 *o0[2] = {&QS[0], &QS[1]};
        read_k(0);
        read_k(1);
        if constexpr (LB > 1) {
            constexpr int MFMA = (EFFECTS ? 0 : 4 * products(PM, PM, 3)) + KB * 2 * products(PI, PM, 3);
            floatx4 *o1[2] = {&QS[2], &QS[3]};
            auto pieces = weave<MFMA / 3, 2>([&](int e) { split_u(1, e); });
            if constexpr (!EFFECTS) {
                read_p(1, 0, 1);
                region_end();
                mm_many<3, true>(pf[0], Uf[0], o0, pieces);
                read_p(1, 1, 0);
                region_end();
                mm_many<3, true>(pf[1], Uf[0], o1, pieces);
            }
#pragma unroll
            for (int pair = 0; pair < KB; ++pair) {
                floatx4 *to[2] = {&S[2 * pair], &S[2 * pair + 1]};
                mm_many<3, false>(kf[pair & 1], W[0], to, pieces);
                read_k(pair + 2);
                region_end();
            }
            pieces.rest();
        }
        // the last tokens' products; a pair of tiles of the state is split for the next chunk while those of the next pair run, then of the outputs
        {
            constexpr int LAST = (LB - 1) * KB;
            auto split_s = [&](int pair, int e) {
                const floatx4 &x = S[2 * pair + e];
                set_four<PM>(Sf[pair], e, {x[0], x[1], x[2], x[3]});
            };
#pragma unroll
            for (int pair = 0; pair < KB; ++pair) {
                floatx4 *to[2] = {&S[2 * pair], &S[2 * pair + 1]};
                auto pieces = weave<2, 2>([&](int e) {
                    if (pair > 0) split_s(pair - 1, e);
                });
                mm_many<3, false>(kf[(LAST + pair) & 1], W[LB - 1], to, pieces);
                read_k(LAST + pair + 2);
                region_end();
            }
            auto pieces = weave<2, 2>([&](int e) { split_s(KB - 1, e); });
            floatx4 *to[2] = {&QS[NT - 2], &QS[NT - 1]};
            if constexpr (!EFFECTS) mm_many<3, true>(pf[0], Uf[LB - 1], to, pieces);
            pieces.rest();
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) hold(Sf[kb]);
            region_end();
        }
        // what the next chunk needs is there; the outputs are stored behind that wait and have the next chunk's time
        if (Lds::DOUBLE) __builtin_amdgcn_s_waitcnt(0);
        if (EFFECTS) continue;
        const bool plain = mem.vec_o && t0 + L <= a.T && (all_columns || col0 + 16 <= a.Dv);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int tile_token = t0 + 32 * (i >> 1) + 4 * (i & 1);
            E *to = o + tile_token * a.so.token + col0;
            float u[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) u[r] = tile_token + lane_token < len ? a.scale * QS[i][r] : 0.0f;       // past the end zeros beside a NaN too
            if (plain) {
                if (col0 < a.Dv) store4(behind(to, at_o), u);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (tile_token + lane_token < a.T && col0 + 4 * g + r < a.Dv) store_element(behind(to, at_o) + r, u[r]);
            }
        }
    }
    if (EFFECTS) {
        const int width = mem.dvp + U::DKP;
        if (col0 < width) store_tiles<DT>(mem.effects + at * U::DKP * width, width, tiles_at(width, col0, lane), lane, S);
        return;
    }
    // past the sequence's end
    const int last = min((begin + mem.segment_chunks) * L, a.T);
    for (int t = (n > begin ? n : begin) * L + g; t < last; t += 4)
        if (col < a.Dv) store_element(o + t * a.so.token + col, 0.0f);
    if (a.final_state && segment + 1 == mem.segments) store_state<DT>(a.final_state + (long long)head * a.Dk * a.Dv, a.Dk, a.Dv, col, g, S);
}

// The states before the segments, one after the other: S <- A S + B.  BACK: the gradients of the states after them, from the last one:
// dS <- A' dS + b.  A workgroup takes four tiles of columns of a head, two waves a tile, each with half of the state's rows: the waves split A
// and their part of the state for all of them in LDS, and fetch the next segment's A and B meanwhile.  Each segment waits for the one before: 16 segments of 8 heads of
// 128 take 73 us (with one wave a tile and nothing fetched ahead the whole call took 157 us more).
constexpr int JOIN_TILES = 4, JOIN_THREADS = 512;
template <int KB>
struct JoinLds { static constexpr int DT = 2 * KB, A = DT * KB * DELTA_PM, BYTES = (A + JOIN_TILES * KB * DELTA_PM) * 1024; };

template <int KB, bool BACK>
__global__ __launch_bounds__(JOIN_THREADS) void k_delta_join(DeltaArgs a, DeltaMemory mem, int blocks_per_head)
{
    constexpr int DT = 2 * KB, DKP = 32 * KB, PM = DELTA_PM, WAVES = JOIN_THREADS / 64, OWN = KB, FRAGS = (DT * KB + WAVES - 1) / WAVES;
    extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
    unsigned char *As = lds, *Ss = lds + JoinLds<KB>::A * 1024;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, g = lane >> 4, block = blockIdx.x % blocks_per_head, head = blockIdx.x / blocks_per_head;
    const int tile = wave >> 1, half = wave & 1;                   // row tiles half * KB .. + KB - 1 of the state: pairs where KB is even
    const int width = mem.dvp + DKP, col0 = (block * JOIN_TILES + tile) * 16, col = col0 + m;
    const bool live = col0 < mem.dvp;
    const float *from = BACK ? a.d_final : a.initial;
    floatx4 S[OWN], next_b[OWN] = {};
    float next_a[FRAGS][8];
    // an element of the wave's rows
    auto at_row = [&](int t, int r) { return tile_index(half * KB + t, 4 * g + r); };
    auto load_own = [&](const float *p, int rows, int columns, int stride, floatx4 (&x)[OWN]) {
#pragma unroll
        for (int t = 0; t < OWN; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) x[t][r] = p[at_row(t, r) < rows && col < columns ? at_row(t, r) * stride + col : 0];
#pragma unroll
        for (int t = 0; t < OWN; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (at_row(t, r) >= rows || col >= columns) x[t][r] = 0.0f;
    };
    auto load_next = [&](int segment) {
        const long long at = (long long)head * mem.segments + segment;
        const float *A = mem.effects + at * DKP * width + mem.dvp;
        const int stride = BACK ? mem.dvp : width;
        if (live) {
            const float *b = uniform((BACK ? mem.back_effects : mem.effects) + at * DKP * stride);
            unsigned off = (8 * g * stride + col) * 4;
            asm("" : "+v"(off));
#pragma unroll
            for (int t = 0; t < OWN; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) next_b[t][r] = *behind(b + (tile_index(half * KB + t, 0) + r) * stride, off);
        }
#pragma unroll
        for (int x = 0; x < FRAGS; ++x) {
            const int f = wave + x * WAVES;
            if (f < DT * KB) {
                // row tile_index(f / KB, m), columns 32 (f % KB) + 8 g ..; of A' if BACK
                const int row = tile_index(f / KB, 0), k = 32 * (f % KB), lane_row = 8 * (m >> 2) + (m & 3);
                const float *p = uniform(BACK ? A + k * width + row : A + row * width + k);
                unsigned off = (BACK ? 8 * g * width + lane_row : lane_row * width + 8 * g) * 4;
                asm("" : "+v"(off));
                if (BACK) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) next_a[x][e] = *behind(p + e * width, off);
                } else {
                    load8(behind(p, off), 8, true, next_a[x]);
                }
            }
        }
    };
#pragma unroll
    for (int t = 0; t < OWN; ++t) S[t] = floatx4{0, 0, 0, 0};
    if (from) load_own(from + (long long)head * a.Dk * a.Dv, a.Dk, a.Dv, a.Dv, S);
    load_next(BACK ? mem.segments - 1 : 0);
    for (int step = 0; step < mem.segments; ++step) {
        const int segment = BACK ? mem.segments - 1 - step : step;
        const long long at = (long long)head * mem.segments + segment;
        if (live) {
            float *to = (BACK ? mem.segment_d_states : mem.segment_states) + at * DKP * mem.dvp;
#pragma unroll
            for (int t = 0; t < OWN; ++t) {
                const int tt = half * KB + t;
                *behind((floatx4 *)(to + (32 * (tt >> 1) + 4 * (tt & 1)) * mem.dvp), tiles_at(mem.dvp, col0, lane)) = quad_transpose(S[t], lane);
            }
        }
        if (step + 1 == mem.segments) break;
#pragma unroll
        for (int x = 0; x < FRAGS; ++x)
            if (wave + x * WAVES < DT * KB) store_frag<PM>(As + (wave + x * WAVES) * PM * 1024, lane, make_frag<PM>(next_a[x]));
        // the state as operand blocks: four of a lane's eight values are a tile's
#pragma unroll
        for (int t = 0; t < OWN; ++t) {
            const int tt = half * KB + t;
            Frag<PM> f{};
            set_four<PM>(f, 0, {S[t][0], S[t][1], S[t][2], S[t][3]});
#pragma unroll
            for (int p = 0; p < PM; ++p)
                *reinterpret_cast<uint2 *>(Ss + ((tile * KB + (tt >> 1)) * PM + p) * 1024 + lane * 16 + (tt & 1) * 8) = make_uint2(f.w[p][0], f.w[p][1]);
        }
        floatx4 sum[OWN];
#pragma unroll
        for (int t = 0; t < OWN; ++t) sum[t] = next_b[t];
        if (step + 2 < mem.segments) load_next(BACK ? segment - 1 : segment + 1);
        __syncthreads();
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const Frag<PM> sf = load_frag<PM>(Ss + (tile * KB + kb) * PM * 1024, lane);
            Frag<PM> f[OWN];
            floatx4 *to[OWN];
#pragma unroll
            for (int t = 0; t < OWN; ++t) f[t] = load_frag<PM>(As + ((half * KB + t) * KB + kb) * PM * 1024, lane), to[t] = &sum[t];
            mm_many<3, false>(f, sf, to, NoWeave());
        }
#pragma unroll
        for (int t = 0; t < OWN; ++t) S[t] = sum[t];
        __syncthreads();
    }
}

}  // namespace tfno
