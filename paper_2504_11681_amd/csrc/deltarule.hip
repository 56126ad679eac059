// Launches of the gated delta rule over sequences.
#include "deltagrad_kernel.h"

#include <algorithm>

namespace tfno {

namespace {

constexpr int SEGMENT_MAX_WAVES = 256, SEGMENT_WAVES = 1024, SEGMENT_MIN_CHUNKS = 4;

size_t pad(size_t n) { return (n + 255) / 256 * 256; }

// Segments of a head's chunks that are walked through at once.  They cost: the effect of each is walked through beforehand with Dk more columns, and the
// states between them are joined one after the other.  So they are for few heads, whose columns leave most of the chip idle, and many chunks.  Measured in
// us, in segments and in one walk, BF16 unless stated (B, T, heads, Dk = Dv; waves: 16 columns each): forward 1, 16384, 8, 128 (64 waves) 244 and 907, its training 830
// and 2423; 4, 4096, 8, 64 (128 waves) 100 and 191; 2, 1024, 4, 64 38 and 51; 8, 8192, 8, 64 (256 waves) 352 and 480; with 512 waves about the same, 4, 2048, 16, 128 155 and 154,
// 16, 2048, 8, 64 151 and 156.  More segments than 1024 waves lose, fewer too (the first one: 329 with 2048, 316 with 512).  Below some chunks they do: 1, 512, 8, 128
// 48 and 40, float32 8, 1000, 8, 64 82 and 79.  In chunks, two walks, slower where more than two waves a CU share it, and the joins make the estimate below.
int segments_of(const DeltaArgs &a, int chunks)
{
    const long long waves = (long long)a.B * a.Hv * ((a.Dv + 31) / 32 * 2);
    if (waves == 0 || waves > SEGMENT_MAX_WAVES) return 1;
    const long long n = std::min<long long>(SEGMENT_WAVES / waves, chunks / SEGMENT_MIN_CHUNKS);
    if (n < 2 || 2.0 * chunks / n * (waves * n > 512 ? 1.75 : 1.0) + 3.0 + 0.5 * n >= chunks) return 1;
    const int each = (int)((chunks + n - 1) / n);
    return (chunks + each - 1) / each;           // none without chunks
}

// Layout of the tape, or of the workspace of a forward pass without one; `base` may be NULL for its size alone.
template <class E, int KB>
size_t forward_memory(const DeltaArgs &a, unsigned char *base, bool tape, DeltaMemory *m)
{
    typedef DeltaUnits<E, KB> U;
    m->chunks = (a.T + U::L - 1) / U::L;
    m->dvp = (a.Dv + 31) / 32 * 32;
    m->key_units = tape ? U::KEY_TAPE : U::KEY_FORWARD;
    m->value_units = tape ? U::VALUE_TAPE : U::VALUE_FORWARD;
    m->segments = segments_of(a, m->chunks);
    m->segment_chunks = (m->chunks + m->segments - 1) / m->segments;
    const size_t keys = (size_t)a.B * a.Hk * m->chunks, values = (size_t)a.B * a.Hv * m->chunks, parts = (size_t)a.B * a.Hv * m->segments;
    size_t at = 0;
    m->key = base + at, at += keys * m->key_units * 1024;
    m->value = base + at, at += values * m->value_units * 1024;
    if (tape) {
        m->logs = (float *)(base + at), at += pad(values * 2 * U::L * sizeof(float));
        m->states = (float *)(base + at), at += values * U::DKP * m->dvp * sizeof(float);
        m->errors = (float *)(base + at), at += values * U::L * m->dvp * sizeof(float);
    }
    if (m->segments > 1) {
        m->effects = (float *)(base + at), at += parts * U::DKP * (m->dvp + U::DKP) * sizeof(float);
        m->segment_states = (float *)(base + at), at += parts * U::DKP * m->dvp * sizeof(float);
    }
    return at;
}
template <class E, int KB>
size_t backward_memory(const DeltaArgs &a, unsigned char *base, DeltaMemory *m)
{
    typedef DeltaUnits<E, KB> U;
    const int chunks = (a.T + U::L - 1) / U::L, segments = segments_of(a, chunks);
    const size_t values = (size_t)a.B * a.Hv * chunks, dvp = (a.Dv + 31) / 32 * 32, parts = (size_t)a.B * a.Hv * segments;
    size_t at = 0;
    m->d_states = (float *)(base + at), at += values * U::DKP * dvp * sizeof(float);
    m->d_values = (float *)(base + at), at += values * U::L * dvp * sizeof(float);
    if (a.Hv > a.Hk) m->sums = (float *)(base + at), at += (size_t)a.B * a.Hk * chunks * 2 * U::L * U::DKP * sizeof(float);
    if (segments > 1) {
        m->back_effects = (float *)(base + at), at += parts * U::DKP * dvp * sizeof(float);
        m->segment_d_states = (float *)(base + at), at += parts * U::DKP * dvp * sizeof(float);
    }
    return at;
}

// Rows whose elements may be read or written eight at a time.
bool rows_of_8(const void *p, const Strides &s, bool bf16)
{
    const long long unit = bf16 ? 8 : 4;
    return ((uintptr_t)p & 15) == 0 && s.batch % unit == 0 && s.token % unit == 0 && s.head % unit == 0;
}

// Rows that are written four elements at a time.
bool rows_of_4(const void *p, const Strides &s, int columns, bool bf16)
{
    return columns % 4 == 0 && ((uintptr_t)p & (bf16 ? 7 : 15)) == 0 && s.batch % 4 == 0 && s.token % 4 == 0 && s.head % 4 == 0;
}

// Waves of a scan's workgroup that compute, one for 16 columns: as many as share a chunk's blocks, down to two where there are few.
struct ScanShape { int waves, blocks; };
ScanShape scan_shape(long long walks, int tiles)
{
    ScanShape s{SCAN_WAVES, 0};
    while (s.waves > 2 && (walks * tiles < 256LL * s.waves || s.waves > tiles)) s.waves >>= 1;
    s.blocks = (tiles + s.waves - 1) / s.waves;
    return s;
}

template <class... Kernels>
hipError_t allow_lds(LdsLimitOnce &limit, int bytes, Kernels... k) { return limit.set({(const void *)k...}, bytes); }

template <class E, int KB, int MODE>
hipError_t scan_one(const DeltaArgs &a, const DeltaMemory &m, int segments, int tiles, hipStream_t s)
{
    constexpr int bytes = ForwardLds<E, KB, MODE>::BYTES;
    static LdsLimitOnce limit;
    if (hipError_t e = allow_lds(limit, bytes, k_delta_scan<E, KB, MODE>); e != hipSuccess) return e;
    const long long walks = (long long)a.B * a.Hv * segments;
    const ScanShape sh = scan_shape(walks, tiles);
    k_delta_scan<E, KB, MODE><<<(unsigned)(walks * sh.blocks), 64 * (sh.waves + 1), bytes, s>>>(a, m, sh.blocks, segments);
    return hipGetLastError();
}
template <int KB, bool BACK>
hipError_t join(const DeltaArgs &a, const DeltaMemory &m, hipStream_t s)
{
    static LdsLimitOnce limit;
    if (hipError_t e = allow_lds(limit, JoinLds<KB>::BYTES, k_delta_join<KB, BACK>); e != hipSuccess) return e;
    const int blocks = (m.dvp / 16 + JOIN_TILES - 1) / JOIN_TILES;
    k_delta_join<KB, BACK><<<(unsigned)(a.B * a.Hv * blocks), JOIN_THREADS, JoinLds<KB>::BYTES, s>>>(a, m, blocks);
    return hipGetLastError();
}
template <class E, int KB, bool TAPE>
hipError_t scan(const DeltaArgs &a, const DeltaMemory &m, hipStream_t s)
{
    if (m.segments > 1) {
        // the last segment's effect is of use to the backward pass alone
        if (hipError_t e = scan_one<E, KB, SCAN_EFFECTS>(a, m, TAPE ? m.segments : m.segments - 1, m.dvp / 16 + 2 * KB, s); e != hipSuccess) return e;
        if (hipError_t e = join<KB, false>(a, m, s); e != hipSuccess) return e;
    }
    return scan_one<E, KB, TAPE ? SCAN_TAPE : SCAN_OUTPUTS>(a, m, m.segments, m.dvp / 16, s);
}
template <class E, int KB>
hipError_t scan_back(const DeltaArgs &a, const DeltaMemory &m, hipStream_t s)
{
    constexpr int bytes = BackwardLds<E, KB>::BYTES;
    static LdsLimitOnce limit;
    if (hipError_t e = allow_lds(limit, bytes, k_delta_scan_back<E, KB, false>, k_delta_scan_back<E, KB, true>); e != hipSuccess) return e;
    const long long heads = (long long)a.B * a.Hv;
    if (m.segments > 1) {
        const ScanShape sh = scan_shape(heads * (m.segments - 1), m.dvp / 16);
        k_delta_scan_back<E, KB, true><<<(unsigned)(heads * (m.segments - 1) * sh.blocks), 64 * (sh.waves + 1), bytes, s>>>(a, m, sh.blocks);
        if (hipError_t e = join<KB, true>(a, m, s); e != hipSuccess) return e;
    }
    const ScanShape sh = scan_shape(heads * m.segments, m.dvp / 16);
    k_delta_scan_back<E, KB, false><<<(unsigned)(heads * m.segments * sh.blocks), 64 * (sh.waves + 1), bytes, s>>>(a, m, sh.blocks);
    return hipGetLastError();
}

// Threads of the largest launch for a batch of B sequences: preparation, walk, gradients.  A launch takes less than 2^32.
template <class E, int KB>
long long launch_threads(const DeltaArgs &a, int B, bool tape)
{
    typedef DeltaUnits<E, KB> U;
    const long long chunks = (a.T + U::L - 1) / U::L, heads = (long long)B * a.Hv;
    const ScanShape sh = scan_shape(heads, (a.Dv + 31) / 32 * 2);
    const long long walk = heads * sh.blocks * 64 * (sh.waves + 1), prepare = heads * chunks * 64 * U::NT;
    return std::max({walk, prepare, tape ? (long long)B * a.Hk * chunks * 128 * U::NT : 0});
}
constexpr long long MOST_THREADS = (1LL << 32) - 1;

// Sequences of a batch that go through preparation and walk before the next ones do, without a tape: what the one leaves for the other then stays in the
// last-level cache (256 MB), in memory that the next ones use again, instead of passing through HBM.  Whole rounds of workgroups, one a CU, of up to 192 MB; not where
// one round is more than the cache.  In us, in one piece and in such ones (B, T, heads, Dk = Dv): BF16 256, 1024, 2, 64 262 and 226, 512, 512, 4, 32 421 and 373, float32
// 64, 512, 8, 64 237 and 198; rounds over 256 MB gain nothing or lose, BF16 32, 2048, 16, 64 504 and 503, float32 100, 777, 6, 48 412 and 448.  Heads over 64 are bound by the
// walk's instructions and gain nothing: BF16 64, 512, 16, 128 471 and 477, 48, 512, 16, 128 350 and 358.
template <class E, int KB>
int batch_piece(const DeltaArgs &a)
{
    typedef DeltaUnits<E, KB> U;
    const int chunks = (a.T + U::L - 1) / U::L;
    if (a.B < 2 || segments_of(a, chunks) > 1) return a.B;
    int most = a.B;               // that launches take, and half of it more (next_piece)
    while (most > 1 && launch_threads<E, KB>(a, most, false) > MOST_THREADS / 2) most = (most + 1) / 2;
    if (KB > 2 || chunks == 0) return most;
    const long long key_units = U::PI == 1 ? U::QT - U::KT : U::KEY_FORWARD;
    const long long bytes = chunks * (a.Hk * key_units + a.Hv * (long long)U::VALUE_FORWARD) * 1024;
    const long long workgroups = a.Hv * (((a.Dv + 31) / 32 * 2 + SCAN_WAVES - 1) / SCAN_WAVES);
    const long long round = std::max<long long>(1, 256 / workgroups), fit = (192LL << 20) / bytes;
    if (round * bytes > 256LL << 20) return most;
    return (int)std::min<long long>(most, std::max(round, fit / round * round));
}
// How many of `left` sequences are next: what is less than half a piece goes with the last whole one.
int next_piece(int left, int piece) { return left < piece + (piece + 1) / 2 ? left : piece; }

template <class E, int KB>
hipError_t forward_piece(const DeltaArgs &a, hipStream_t s)
{
    typedef DeltaUnits<E, KB> U;
    DeltaMemory m{};
    const bool tape = a.tape != nullptr;
    forward_memory<E, KB>(a, tape ? a.tape : a.workspace, tape, &m);
    DeltaVec vec{};
    vec.q = rows_of_8(a.q, a.sq, a.bf16), vec.k = rows_of_8(a.k, a.sk, a.bf16);
    m.vec_o = rows_of_4(a.o, a.so, a.Dv, a.bf16);
    // Without a tape nothing else needs blocks of K and Q, and in BF16 they are the rows that the caller has.
    m.rows = !tape && a.bf16 && vec.q && vec.k && a.Dk % 8 == 0;
    const unsigned grid = (unsigned)(a.B * a.Hv * m.chunks);
    if (grid && tape) k_delta_prepare<E, KB, true><<<grid, 64 * U::NT, 0, s>>>(a, m, vec);
    else if (grid) k_delta_prepare<E, KB, false><<<grid, 64 * U::NT, 0, s>>>(a, m, vec);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    return tape ? scan<E, KB, true>(a, m, s) : scan<E, KB, false>(a, m, s);
}
template <class E, int KB>
hipError_t forward(const DeltaArgs &a, hipStream_t s)
{
    if (a.tape) return forward_piece<E, KB>(a, s);
    const int piece = batch_piece<E, KB>(a);
    const long long states = (long long)a.Hv * a.Dk * a.Dv;
    for (int b = 0; b < a.B;) {
        DeltaArgs p = a;
        p.B = next_piece(a.B - b, piece);
        p.q = (const E *)a.q + b * a.sq.batch, p.k = (const E *)a.k + b * a.sk.batch, p.v = (const E *)a.v + b * a.sv.batch;
        p.o = (E *)a.o + b * a.so.batch, p.beta = a.beta + b * a.sbeta.batch;
        if (a.g) p.g = a.g + b * a.sg.batch;
        if (a.lengths) p.lengths = a.lengths + b;
        if (a.initial) p.initial = a.initial + b * states;
        if (a.final_state) p.final_state = a.final_state + b * states;
        if (hipError_t e = forward_piece<E, KB>(p, s); e != hipSuccess) return e;
        b += p.B;
    }
    return hipSuccess;
}

template <class E, int KB>
hipError_t backward(const DeltaArgs &a, hipStream_t s)
{
    typedef DeltaUnits<E, KB> U;
    DeltaMemory m{};
    forward_memory<E, KB>(a, a.tape, true, &m);
    backward_memory<E, KB>(a, a.workspace, &m);
    DeltaVec vec{};
    vec.d_o = rows_of_8(a.d_o, a.sdo, a.bf16), vec.dq = rows_of_8(a.dq, a.sdq, a.bf16), vec.dk = rows_of_8(a.dk, a.sdk, a.bf16);
    m.vec_dv = rows_of_4(a.dv, a.sdv, a.Dv, a.bf16);
    if (hipError_t e = scan_back<E, KB>(a, m, s); e != hipSuccess) return e;
    if (m.chunks == 0) return hipSuccess;
    constexpr int bytes = GradientLds<E, KB>::BYTES;
    static LdsLimitOnce limit;
    if (hipError_t e = allow_lds(limit, bytes, k_delta_gradients<E, KB>); e != hipSuccess) return e;
    k_delta_gradients<E, KB><<<(unsigned)(a.B * a.Hk * m.chunks), 128 * U::NT, bytes, s>>>(a, m, vec);
    return hipGetLastError();
}

template <class E, class F>
auto by_size(const DeltaArgs &a, F f)
{
    return a.Dk <= 32 ? f.template operator()<E, 1>() : a.Dk <= 64 ? f.template operator()<E, 2>() : f.template operator()<E, 4>();
}
struct Forward { const DeltaArgs &a; hipStream_t s; template <class E, int KB> hipError_t operator()() const { return forward<E, KB>(a, s); } };
struct Backward { const DeltaArgs &a; hipStream_t s; template <class E, int KB> hipError_t operator()() const { return backward<E, KB>(a, s); } };
struct ForwardBytes {
    const DeltaArgs &a; bool tape;
    template <class E, int KB> size_t operator()() const
    {
        DeltaMemory m{};
        if (tape) return forward_memory<E, KB>(a, nullptr, true, &m);
        const int piece = batch_piece<E, KB>(a);
        size_t most = 0;
        DeltaArgs p = a;
        for (int b = 0; b < a.B; b += p.B) {
            p.B = next_piece(a.B - b, piece);
            most = std::max(most, forward_memory<E, KB>(p, nullptr, false, &m));
        }
        return most;
    }
};
struct Launches {
    const DeltaArgs &a; bool whole;
    template <class E, int KB> bool operator()() const { return launch_threads<E, KB>(a, whole ? a.B : 1, whole) <= MOST_THREADS; }
};
struct BackwardBytes {
    const DeltaArgs &a;
    template <class E, int KB> size_t operator()() const { DeltaMemory m{}; return backward_memory<E, KB>(a, nullptr, &m); }
};
template <class F>
auto by_kind(const DeltaArgs &a, F f) { return a.bf16 ? by_size<bf16>(a, f) : by_size<float>(a, f); }

}  // namespace

size_t delta_tape_bytes(const DeltaArgs &a) { return by_kind(a, ForwardBytes{a, true}); }
size_t delta_workspace_bytes(const DeltaArgs &a, bool backward) { return backward ? by_kind(a, BackwardBytes{a}) : by_kind(a, ForwardBytes{a, false}); }
bool delta_launches(const DeltaArgs &a, bool whole) { return by_kind(a, Launches{a, whole}); }
hipError_t delta_forward_launch(const DeltaArgs &a, hipStream_t s) { return by_kind(a, Forward{a, s}); }
hipError_t delta_backward_launch(const DeltaArgs &a, hipStream_t s) { return by_kind(a, Backward{a, s}); }

}  // namespace tfno
