// Launches of the norm of heads with rotation.
#include "headnorm_kernel.h"

namespace tfno {

namespace {

bool multiple_of_4(const Strides &s) { return ((s.batch | s.token | s.head) & 3) == 0; }

// Four pairs a lane: all of them turned or none, and every address a multiple of four elements.
bool vectors(const HeadNormArgs &a, bool backward)
{
    if (a.interleaved ? (a.R % 8 || a.D % 8) : (a.R % 8 || (a.D - a.R) % 8)) return false;
    const uintptr_t mask = a.bf16 ? 7 : 15;
    uintptr_t p = (uintptr_t)a.q | (uintptr_t)a.k;
    bool strides = multiple_of_4(a.sq) && multiple_of_4(a.sk) && multiple_of_4(a.sq_out) && multiple_of_4(a.sk_out);
    if (backward) {
        p |= (uintptr_t)a.dq_out | (uintptr_t)a.dk_out | (uintptr_t)a.dq | (uintptr_t)a.dk;
        strides = strides && multiple_of_4(a.sdq) && multiple_of_4(a.sdk);
    } else {
        p |= (uintptr_t)a.q_out | (uintptr_t)a.k_out;
    }
    return (p & mask) == 0 && strides && (((uintptr_t)a.cos | (uintptr_t)a.sin) & 15) == 0;
}

template <class E, int VEC, int ITER, int NH, bool INTER, bool BACKWARD>
hipError_t launch(const HeadNormArgs &a, int lpr, hipStream_t s)
{
    HeadNormShape g;
    g.lpr = lpr;
    const unsigned tokens = (unsigned)a.B * (unsigned)a.T, groups = HEAD_NORM_THREADS / lpr;
    const int heads[2] = {a.Hq, a.Hk};
    unsigned blocks[2];
    for (int i = 0; i < 2; ++i) {
        g.chunks[i] = heads[i] > 0 ? (heads[i] + NH - 1) / NH : 1;
        g.items[i] = heads[i] > 0 ? tokens * g.chunks[i] : 0;
        blocks[i] = (g.items[i] + groups - 1) / groups;
    }
    const unsigned long long all = (unsigned long long)blocks[0] + blocks[1];
    const unsigned most = BACKWARD ? HEAD_NORM_BLOCKS : HEAD_NORM_LAUNCH;
    if (all > most)      // shared out as the work is, each kind that has work its own
        for (int i = 0; i < 2; ++i)
            if (blocks[i]) blocks[i] = 1 + (unsigned)((unsigned long long)blocks[i] * (most - 2) / all);
    g.blocks_q = blocks[0];
    const unsigned grid = blocks[0] + blocks[1];
    if (grid) k_head_norm<E, VEC, ITER, NH, INTER, BACKWARD><<<grid, HEAD_NORM_THREADS, 0, s>>>(a, g);
    if (BACKWARD && (a.dwq || a.dwk))
        k_head_norm_weights<<<dim3((a.D + 15) / 16, 2), 1024, 0, s>>>(a.partial, blocks[0], grid, a.D, a.dwq, a.dwk);
    return hipGetLastError();
}

template <class E, bool INTER, bool BACKWARD>
hipError_t choose(const HeadNormArgs &a, hipStream_t s)
{
    const int slots = a.R / 2 + (a.D - a.R + 1) / 2;
    const bool vec = vectors(a, BACKWARD);
    int lpr = 1;
    while (lpr < 64 && lpr * (vec ? 4 : 1) < slots) lpr <<= 1;
    // Four heads a group where that still leaves waves enough for the chip: the forward pass of 393 thousand heads of 128 in BF16 43 us, with two 51, with one 65.
    const long long heads = (long long)a.B * a.T * (a.Hq + a.Hk);
    const bool many = heads * lpr >= 64LL * 4 * 4096;
    if (vec) return many ? launch<E, 4, 1, 4, INTER, BACKWARD>(a, lpr, s) : launch<E, 4, 1, 1, INTER, BACKWARD>(a, lpr, s);
    if (slots <= 64) return many ? launch<E, 1, 1, 4, INTER, BACKWARD>(a, lpr, s) : launch<E, 1, 1, 1, INTER, BACKWARD>(a, lpr, s);
    return launch<E, 1, 4, 1, INTER, BACKWARD>(a, lpr, s);
}

template <bool BACKWARD>
hipError_t typed(const HeadNormArgs &a, hipStream_t s)
{
    if (a.bf16) return a.interleaved ? choose<bf16, true, BACKWARD>(a, s) : choose<bf16, false, BACKWARD>(a, s);
    return a.interleaved ? choose<float, true, BACKWARD>(a, s) : choose<float, false, BACKWARD>(a, s);
}

}  // namespace

hipError_t head_norm_launch(const HeadNormArgs &a, hipStream_t s) { return typed<false>(a, s); }
hipError_t head_norm_backward_launch(const HeadNormArgs &a, hipStream_t s) { return typed<true>(a, s); }
size_t head_norm_workspace_bytes(int D) { return sizeof(float) * (size_t)HEAD_NORM_BLOCKS * D; }

}  // namespace tfno
