// norm = sqrt(sum over all tensors of x^2),   x <- x limit / norm where norm > limit.
//
// Bound by bytes: all tensors are read once for the norm, and read and written where there is something to clip.  Squares are added up in float64, so
// that no value over- or underflows and no order matters beyond a float32's last bit.  A launch takes a table of tensors, cut into pieces that its
// workgroups take by turns, all of them close together in memory (each its own stretch: 85 -> 87 us for 511 MB); the second launch adds up what the workgroups of the
// first left, each the same way, and goes through the pieces from the end.
#include "gradclip.h"

#include <algorithm>

namespace tfno {

namespace {

constexpr int CLIP_THREADS = 256, CLIP_TENSORS = 128, CLIP_BLOCKS = 2048;
constexpr int CLIP_ROUND = CLIP_THREADS * 4;        // vectors of 16 bytes in a piece

typedef unsigned Vector __attribute__((ext_vector_type(4)));

// Tensors of more bytes than this are loaded and stored past the caches (PAST): more than those hold, so the second pass finds little of them, and whoever wrote them and reads them next
// neither.  Fewer are kept.  A step that writes gradients, clips and reads them, kept and past: 1 MB 119 and 130 us, 64 MB 191 and 213, 192 MB 407 and 418, 288 MB 615 and 622, 320 MB
// 666 and 662, 512 MB 1000 and 961; clipping by itself, again and again: 64 MB 39 and 43, 288 MB 148 and 161, 352 MB 186 and 194, 512 MB 294 and 274.
constexpr unsigned long long CLIP_KEPT = 300ull << 20;

struct ClipTable {
    void *p[CLIP_TENSORS];
    long long n[CLIP_TENSORS];                      // elements
    unsigned first[CLIP_TENSORS + 1];               // pieces of each tensor begin here
    unsigned bf16_mask[CLIP_TENSORS / 32];
    int count;
};

// A workgroup looks for its first piece's tensor and then goes on from there, in either direction.
struct Piece {
    int tensor;
    Vector *p;                                      // the tensor, down to a multiple of 16 bytes, from the piece on
    long long from, to;                             // elements from p on that are the tensor's
    int per;                                        // elements of a vector
    bool bf16, whole;
    __device__ __forceinline__ Piece(const ClipTable &t, unsigned piece)
    {
        int hi = t.count - 1;
        tensor = 0;
        while (tensor < hi) {
            const int mid = (tensor + hi + 1) >> 1;
            if (t.first[mid] <= piece) tensor = mid;
            else hi = mid - 1;
        }
        set(t, piece);
    }
    __device__ __forceinline__ void go(const ClipTable &t, unsigned piece)
    {
        while (t.first[tensor] > piece) --tensor;
        while (t.first[tensor + 1] <= piece) ++tensor;
        set(t, piece);
    }
    __device__ __forceinline__ void set(const ClipTable &t, unsigned piece)
    {
        bf16 = t.bf16_mask[tensor >> 5] >> (tensor & 31) & 1;
        per = bf16 ? 8 : 4;
        const uintptr_t at = (uintptr_t)t.p[tensor];
        const long long vector = (long long)(piece - t.first[tensor]) * CLIP_ROUND, skip = (long long)(at & 15) / (bf16 ? 2 : 4);
        p = (Vector *)(at & ~(uintptr_t)15) + vector;
        from = max(skip - vector * per, 0ll);
        to = min(skip + t.n[tensor] - vector * per, (long long)CLIP_ROUND * per);
        whole = from == 0 && to == (long long)CLIP_ROUND * per;
    }
    template <bool PAST>
    __device__ __forceinline__ void load(Vector (&in)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Vector *at = p + threadIdx.x + i * CLIP_THREADS;
            in[i] = PAST ? __builtin_nontemporal_load(at) : *at;
        }
    }
};

unsigned pieces_of(const tfno_tensor &t)
{
    const int elem = t.dtype == TFNO_BF16 ? 2 : 4;
    const unsigned long long bytes = ((uintptr_t)t.data & 15) + (unsigned long long)t.elements * elem;
    return (unsigned)((bytes + 16 * CLIP_ROUND - 1) / (16 * CLIP_ROUND));
}

__device__ __forceinline__ double square(float x) { return (double)x * (double)x; }
__device__ __forceinline__ double squares(Vector v, bool bf16)
{
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (bf16) sum += square(__uint_as_float(w[i] << 16)) + square(__uint_as_float(w[i] & 0xffff0000u));
        else sum += square(__uint_as_float(w[i]));
    }
    return sum;
}

__device__ __forceinline__ double block_sum(double v, double (&meet)[CLIP_THREADS / 64])
{
    for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s, 64);
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = v;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < CLIP_THREADS / 64; ++w) all += meet[w];
    return all;
}

template <bool PAST>
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_squares(ClipTable t, double *partial)
{
    __shared__ double meet[CLIP_THREADS / 64];
    double sum = 0.0;
    const unsigned end = t.first[t.count];
    unsigned piece = blockIdx.x;
    Piece at(t, piece);
    Vector next[4];
    if (at.whole) at.template load<PAST>(next);
    while (piece < end) {
        const Piece now = at;
        Vector in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i] = next[i];
        if ((piece += gridDim.x) < end) {
            at.go(t, piece);
            if (at.whole) at.template load<PAST>(next);
        }
        if (now.whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += squares(in[i], now.bf16);
        } else {
            for (long long i = now.from + threadIdx.x; i < now.to; i += CLIP_THREADS)
                sum += square(now.bf16 ? to_float(((const bf16 *)now.p)[i]) : ((const float *)now.p)[i]);
        }
    }
    sum = block_sum(sum, meet);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__device__ __forceinline__ float scaled(float x, double scale) { return (float)((double)x * scale); }

template <bool PAST>
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_scale(ClipTable t, const double *partial, int partials, double limit, float *norm)
{
    __shared__ double meet[CLIP_THREADS / 64];
    double sum = 0.0;
    for (int i = threadIdx.x; i < partials; i += CLIP_THREADS) sum += partial[i];
    const double all = sqrt(block_sum(sum, meet));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)all;
    if (!(all > limit) || isinf(all)) return;      // nothing to clip, or nothing to clip it by
    const double scale = limit / all;
    const unsigned pieces = t.first[t.count];
    if (blockIdx.x >= pieces) return;
    unsigned piece = pieces - 1 - blockIdx.x;
    Piece at(t, piece);
    Vector next[4];
    if (at.whole) at.template load<PAST>(next);
    for (;;) {
        const Piece now = at;
        Vector in[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) in[k] = next[k];
        const bool more = piece >= gridDim.x;
        if (more) {
            at.go(t, piece -= gridDim.x);
            if (at.whole) at.template load<PAST>(next);
        }
        if (now.whole) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                unsigned w[4] = {in[k].x, in[k].y, in[k].z, in[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (now.bf16) w[e] = bf16_pair(scaled(__uint_as_float(w[e] << 16), scale), scaled(__uint_as_float(w[e] & 0xffff0000u), scale));
                    else w[e] = __float_as_uint(scaled(__uint_as_float(w[e]), scale));
                }
                Vector *to = now.p + threadIdx.x + k * CLIP_THREADS;
                if (PAST) __builtin_nontemporal_store(Vector{w[0], w[1], w[2], w[3]}, to);
                else *to = Vector{w[0], w[1], w[2], w[3]};
            }
        } else {
            for (long long k = now.from + threadIdx.x; k < now.to; k += CLIP_THREADS) {
                if (now.bf16) store_element((bf16 *)now.p + k, scaled(to_float(((const bf16 *)now.p)[k]), scale));
                else ((float *)now.p)[k] = scaled(((const float *)now.p)[k], scale);
            }
        }
        if (!more) return;
    }
}

// The tensors from `from` on that one table takes.
int fill(ClipTable &t, const tfno_tensor *tensors, int from, int count)
{
    t.count = 0;
    t.first[0] = 0;
    for (unsigned &m : t.bf16_mask) m = 0;
    for (; from < count && t.count < CLIP_TENSORS; ++from) {
        const unsigned pieces = pieces_of(tensors[from]);
        if (tensors[from].elements == 0) continue;
        if (t.count > 0 && (unsigned long long)t.first[t.count] + pieces > 0x7fffffffu) break;
        t.p[t.count] = tensors[from].data, t.n[t.count] = tensors[from].elements;
        if (tensors[from].dtype == TFNO_BF16) t.bf16_mask[t.count >> 5] |= 1u << (t.count & 31);
        t.first[t.count + 1] = t.first[t.count] + pieces;
        ++t.count;
    }
    return from;
}
unsigned blocks_of(const ClipTable &t) { return std::min(t.first[t.count], (unsigned)CLIP_BLOCKS); }

template <bool PAST>
hipError_t clip(const tfno_tensor *tensors, int count, double limit, float *norm, double *partial, hipStream_t s)
{
    ClipTable t;
    int partials = 0;
    for (int from = 0; from < count;) {
        from = fill(t, tensors, from, count);
        if (const unsigned grid = blocks_of(t)) {
            k_clip_squares<PAST><<<grid, CLIP_THREADS, 0, s>>>(t, partial + partials);
            partials += grid;
        }
    }
    bool wrote = false;
    for (int from = 0; from < count;) {
        from = fill(t, tensors, from, count);
        if (const unsigned grid = blocks_of(t)) {
            k_clip_scale<PAST><<<std::isinf(limit) ? 1 : grid, CLIP_THREADS, 0, s>>>(t, partial, partials, limit, wrote ? nullptr : norm);
            if (wrote = true; std::isinf(limit)) break;
        }
    }
    if (!wrote) {       // no element at all
        t.count = 0, t.first[0] = 0;
        k_clip_scale<PAST><<<1, CLIP_THREADS, 0, s>>>(t, partial, 0, limit, norm);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t clip_launch(const tfno_tensor *tensors, int count, double limit, float *norm, double *partial, hipStream_t s)
{
    unsigned long long bytes = 0;
    for (int i = 0; i < count; ++i) bytes += (unsigned long long)tensors[i].elements * (tensors[i].dtype == TFNO_BF16 ? 2 : 4);
    return bytes > CLIP_KEPT ? clip<true>(tensors, count, limit, norm, partial, s) : clip<false>(tensors, count, limit, norm, partial, s);
}

size_t clip_workspace_bytes(int count) { return sizeof(double) * CLIP_BLOCKS * (size_t)(count / CLIP_TENSORS + 1); }

}  // namespace tfno
