// One token of the gated delta rule for many sequences:
//
//   Sb = exp(g) S,   u = beta (v - Sb' k),   S <- Sb + k u',   o = scale S' q = scale (Sb' q + (k.q) u).
//
// Bound by the bytes of the state, which is read and written once: the two products with Sb are taken in one pass over it while it
// lies in registers, so the workgroup meets once, for the sums over the rows.  A workgroup takes `cols` columns of one head's state:
// a thread four neighbouring columns (one, where Dv or an address is no multiple of four) of ROWS rows.  256 sequences of 16 heads of 128 out of a larger pool: 89 us
// for 537 MB of states, 6.0 TB/s (a part of them stays in the last-level cache from step to step; a copy reaches 5.1).
#include "deltarule.h"

#include <algorithm>

namespace tfno {

namespace {

constexpr int STEP_THREADS = 256, STEP_BLOCKS = 1 << 23;      // a launch takes less than 2^32 threads

template <class E, int VEC, int ROWS>
__global__ __launch_bounds__(STEP_THREADS) void k_delta_step(DeltaStepArgs a, int lanes, int blocks_per_head)
{
    __shared__ float qs[128], ks[128];
    __shared__ float sums[2][STEP_THREADS / 64][128];
    __shared__ float qk_part[2];
    const int tid = threadIdx.x, wave = tid >> 6, groups = STEP_THREADS / lanes, cl = tid & (lanes - 1), rg = tid / lanes;
    const int block = blockIdx.x % blocks_per_head, head = a.first + blockIdx.x / blocks_per_head;
    const int b = head / a.Hv, h = head - b * a.Hv, hk = h / (a.Hv / a.Hk);
    const int c = (block * lanes + cl) * VEC;
    const bool live = c < a.Dv;
    E *o = (E *)a.o + (b * a.so.batch + h * a.so.head) + c;
    const int slot = a.slots ? a.slots[b] : b;
    if ((unsigned)slot >= (unsigned)a.pool) {            // no sequence here (zeros), or one that the pool does not hold (NaN)
        if (rg == 0 && live)
            for (int e = 0; e < VEC; ++e) store_element(o + e, slot < 0 ? 0.0f : __uint_as_float(0x7fc00000u));
        return;
    }
    float *S = a.state + ((long long)slot * a.Hv + h) * a.Dk * a.Dv + c;
    float s[ROWS][VEC];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = rg + i * groups;
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[i][e] = 0.0f;
        if (r < a.Dk && live) {
            if constexpr (VEC == 4) load4(S + (long long)r * a.Dv, s[i]);
            else s[i][0] = S[(long long)r * a.Dv];
        }
    }
    if (tid < 128) {
        float qv = 0.0f, kv = 0.0f;
        if (tid < a.Dk) {
            qv = to_float(((const E *)a.q)[b * a.sq.batch + hk * a.sq.head + tid]);
            kv = to_float(((const E *)a.k)[b * a.sk.batch + hk * a.sk.head + tid]);
        }
        qs[tid] = qv, ks[tid] = kv;
        const float p = group_sum(qv * kv, 64);
        if ((tid & 63) == 0) qk_part[wave] = p;
    }
    const float decay = a.g ? expf(a.g[b * a.sg.batch + h * a.sg.head]) : 1.0f;
    const float beta = a.beta[b * a.sbeta.batch + h * a.sbeta.head];
    float v[VEC] = {};
    if (live)
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = to_float(((const E *)a.v)[b * a.sv.batch + h * a.sv.head + c + e]);
    __syncthreads();
    float sk[VEC] = {}, sq[VEC] = {};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = rg + i * groups;
        const float kr = r < 128 ? ks[r] : 0.0f, qr = r < 128 ? qs[r] : 0.0f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            s[i][e] = decay == 0.0f ? 0.0f : s[i][e] * decay;          // forgotten whatever it was: a place of the pool that nobody wrote may hold NaN
            sk[e] = fmaf(kr, s[i][e], sk[e]);
            sq[e] = fmaf(qr, s[i][e], sq[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        for (int step = lanes; step < 64; step <<= 1) {
            sk[e] += __shfl_xor(sk[e], step, 64);
            sq[e] += __shfl_xor(sq[e], step, 64);
        }
        if ((tid & 63) < lanes) {
            sums[0][wave][cl * VEC + e] = sk[e];
            sums[1][wave][cl * VEC + e] = sq[e];
        }
    }
    __syncthreads();
    const float qk = qk_part[0] + qk_part[1];
    float u[VEC], out[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const int at = cl * VEC + e;
        const float kS = (sums[0][0][at] + sums[0][1][at]) + (sums[0][2][at] + sums[0][3][at]);
        const float qS = (sums[1][0][at] + sums[1][1][at]) + (sums[1][2][at] + sums[1][3][at]);
        u[e] = beta * (v[e] - kS);
        out[e] = a.scale * fmaf(qk, u[e], qS);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = rg + i * groups;
        if (r < a.Dk && live) {
            const float kr = ks[r];
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[i][e] = fmaf(kr, u[e], s[i][e]);
            if constexpr (VEC == 4) store4(S + (long long)r * a.Dv, s[i]);
            else S[(long long)r * a.Dv] = s[i][0];
        }
    }
    if (rg == 0 && live)
#pragma unroll
        for (int e = 0; e < VEC; ++e) store_element(o + e, out[e]);
}

template <class E, int VEC>
hipError_t launch(const DeltaStepArgs &a, hipStream_t s)
{
    // whole heads a workgroup where there are heads enough, down to 16 lanes of columns where there are few; at most 32 lanes
    // of columns, and at least as many groups of rows as keep a thread's rows at 16
    const long long heads = (long long)a.B * a.Hv;
    int lanes = 1;
    while (lanes < 32 && lanes * VEC < a.Dv) lanes <<= 1;
    while (lanes > 4 && heads * ((a.Dv + lanes * VEC - 1) / (lanes * VEC)) < 512) lanes >>= 1;
    const int per_head = (a.Dv + lanes * VEC - 1) / (lanes * VEC), groups = STEP_THREADS / lanes;
    const int rows = (a.Dk + groups - 1) / groups, most = STEP_BLOCKS / per_head;
    for (long long first = 0; first < heads; first += most) {
        DeltaStepArgs p = a;
        p.first = (int)first;
        const unsigned grid = (unsigned)(std::min<long long>(heads - first, most) * per_head);
        if (rows <= 1) k_delta_step<E, VEC, 1><<<grid, STEP_THREADS, 0, s>>>(p, lanes, per_head);
        else if (rows <= 2) k_delta_step<E, VEC, 2><<<grid, STEP_THREADS, 0, s>>>(p, lanes, per_head);
        else if (rows <= 4) k_delta_step<E, VEC, 4><<<grid, STEP_THREADS, 0, s>>>(p, lanes, per_head);
        else if (rows <= 8) k_delta_step<E, VEC, 8><<<grid, STEP_THREADS, 0, s>>>(p, lanes, per_head);
        else k_delta_step<E, VEC, 16><<<grid, STEP_THREADS, 0, s>>>(p, lanes, per_head);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t delta_step_launch(const DeltaStepArgs &a, hipStream_t s)
{
    const bool vec = a.Dv % 4 == 0 && ((uintptr_t)a.state & 15) == 0;
    if (a.bf16) return vec ? launch<bf16, 4>(a, s) : launch<bf16, 1>(a, s);
    return vec ? launch<float, 4>(a, s) : launch<float, 1>(a, s);
}

}  // namespace tfno
