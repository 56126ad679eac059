// Norm of queries and keys for each head with the rotation by position: what the C ABI hands to the kernels.
#pragma once
#include "elements.h"

namespace tfno {

struct HeadNormArgs {
    const void *q, *k;                  // [B, T, Hq, D], [B, T, Hk, D]
    void *q_out, *k_out;                // forward: results
    const void *dq_out, *dk_out;        // backward: gradients of the results, and
    void *dq, *dk;                      // of q and k
    const float *wq, *wk;               // [D] or NULL (ones)
    const float *cos, *sin;             // [P, R / 2]
    const int *positions;               // [B, T] or NULL (the token's index)
    float *dwq, *dwk;                   // [D] or NULL
    float *partial;                     // workspace of the weights' gradients, [blocks][D], or NULL where neither is asked for
    Strides sq, sk, sq_out, sk_out, sdq, sdk;
    long long positions_batch;
    int B, T, Hq, Hk, D, R, P;
    float eps;
    bool bf16, interleaved;
};

hipError_t head_norm_launch(const HeadNormArgs &a, hipStream_t s);
hipError_t head_norm_backward_launch(const HeadNormArgs &a, hipStream_t s);
size_t head_norm_workspace_bytes(int D);

}  // namespace tfno
