// norm = sqrt(sum over all tensors of x^2),   x <- x limit / norm where norm > limit.
//
// Bound by bytes: all tensors are read once for the norm, and read and written where there is something to clip.  Squares are added up in float64, so
// that no value over- or underflows and no order matters beyond a float32's last bit.  A launch takes a table of tensors, cut into pieces that its
// workgroups take by turns; the second launch adds up what the workgroups of the first left, each the same way, and goes through the pieces from the end: the
// last ones read are still in the last-level cache.
#include "gradclip.h"

#include <algorithm>

namespace tfno {

namespace {

constexpr int CLIP_THREADS = 256, CLIP_TENSORS = 128, CLIP_BLOCKS = 2048;
constexpr int CLIP_ROUND = CLIP_THREADS * 4;        // vectors of 16 bytes in a piece

struct ClipTable {
    void *p[CLIP_TENSORS];
    long long n[CLIP_TENSORS];                      // elements
    unsigned first[CLIP_TENSORS + 1];               // pieces of each tensor begin here
    unsigned bf16_mask[CLIP_TENSORS / 32];
    int count;
};

struct Piece {
    void *p;                                        // of the tensor, down to a multiple of 16 bytes
    long long skip, end;                            // elements from there on that are the tensor's: skip .. end - 1
    long long vector;                               // the first vector of the piece
    bool bf16;
    __device__ __forceinline__ Piece(const ClipTable &t, unsigned piece)
    {
        int lo = 0, hi = t.count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (t.first[mid] <= piece) lo = mid;
            else hi = mid - 1;
        }
        bf16 = t.bf16_mask[lo >> 5] >> (lo & 31) & 1;
        const uintptr_t at = (uintptr_t)t.p[lo];
        p = (void *)(at & ~(uintptr_t)15);
        skip = (long long)(at & 15) / (bf16 ? 2 : 4);
        end = skip + t.n[lo];
        vector = (long long)(piece - t.first[lo]) * CLIP_ROUND;
    }
};

unsigned pieces_of(const tfno_tensor &t)
{
    const int elem = t.dtype == TFNO_BF16 ? 2 : 4;
    const unsigned long long bytes = ((uintptr_t)t.data & 15) + (unsigned long long)t.elements * elem;
    return (unsigned)((bytes + 16 * CLIP_ROUND - 1) / (16 * CLIP_ROUND));
}

__device__ __forceinline__ double square(float x) { return (double)x * (double)x; }
__device__ __forceinline__ double squares(uint4 v, bool bf16)
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

__global__ __launch_bounds__(CLIP_THREADS) void k_clip_squares(ClipTable t, double *partial)
{
    __shared__ double meet[CLIP_THREADS / 64];
    double sum = 0.0;
    for (unsigned piece = blockIdx.x; piece < t.first[t.count]; piece += gridDim.x) {
        const Piece at(t, piece);
        const int per = at.bf16 ? 8 : 4;
        if (at.vector * per >= at.skip && (at.vector + CLIP_ROUND) * per <= at.end) {
            const uint4 *v = (const uint4 *)at.p + at.vector + threadIdx.x;
            uint4 in[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) in[i] = v[i * CLIP_THREADS];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += squares(in[i], at.bf16);
        } else {
            const long long from = max(at.vector * per, at.skip), to = min((at.vector + CLIP_ROUND) * per, at.end);
            for (long long i = from + threadIdx.x; i < to; i += CLIP_THREADS)
                sum += square(at.bf16 ? to_float(((const bf16 *)at.p)[i]) : ((const float *)at.p)[i]);
        }
    }
    sum = block_sum(sum, meet);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__device__ __forceinline__ float scaled(float x, double scale) { return (float)((double)x * scale); }

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
    for (unsigned i = blockIdx.x; i < pieces; i += gridDim.x) {
        const Piece at(t, pieces - 1 - i);
        const int per = at.bf16 ? 8 : 4;
        if (at.vector * per >= at.skip && (at.vector + CLIP_ROUND) * per <= at.end) {
            uint4 *v = (uint4 *)at.p + at.vector + threadIdx.x;
            uint4 in[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) in[k] = v[k * CLIP_THREADS];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                unsigned w[4] = {in[k].x, in[k].y, in[k].z, in[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at.bf16) w[e] = bf16_pair(scaled(__uint_as_float(w[e] << 16), scale), scaled(__uint_as_float(w[e] & 0xffff0000u), scale));
                    else w[e] = __float_as_uint(scaled(__uint_as_float(w[e]), scale));
                }
                v[k * CLIP_THREADS] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
            const long long from = max(at.vector * per, at.skip), to = min((at.vector + CLIP_ROUND) * per, at.end);
            for (long long k = from + threadIdx.x; k < to; k += CLIP_THREADS) {
                if (at.bf16) store_element((bf16 *)at.p + k, scaled(to_float(((const bf16 *)at.p)[k]), scale));
                else ((float *)at.p)[k] = scaled(((const float *)at.p)[k], scale);
            }
        }
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

}  // namespace

hipError_t clip_launch(const tfno_tensor *tensors, int count, double limit, float *norm, double *partial, hipStream_t s)
{
    ClipTable t;
    int partials = 0;
    for (int from = 0; from < count;) {
        from = fill(t, tensors, from, count);
        if (const unsigned grid = blocks_of(t)) {
            k_clip_squares<<<grid, CLIP_THREADS, 0, s>>>(t, partial + partials);
            partials += grid;
        }
    }
    bool wrote = false;
    for (int from = 0; from < count;) {
        from = fill(t, tensors, from, count);
        if (const unsigned grid = blocks_of(t)) {
            k_clip_scale<<<std::isinf(limit) ? 1 : grid, CLIP_THREADS, 0, s>>>(t, partial, partials, limit, wrote ? nullptr : norm);
            if (wrote = true; std::isinf(limit)) break;
        }
    }
    if (!wrote) {       // no element at all
        t.count = 0, t.first[0] = 0;
        k_clip_scale<<<1, CLIP_THREADS, 0, s>>>(t, partial, 0, limit, norm);
    }
    return hipGetLastError();
}

size_t clip_workspace_bytes(int count) { return sizeof(double) * CLIP_BLOCKS * (size_t)(count / CLIP_TENSORS + 1); }

}  // namespace tfno
