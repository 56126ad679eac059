// Norms after one block and before the next, with the gate and the residual between them: what the C ABI hands to the kernels.
#pragma once
#include "elements.h"

namespace tfno {

struct BlockNormArgs {
    const void *y, *r, *gate;           // [B, T, C]; r may be NULL, gate as gate_kind says
    const float *w_after, *w_before;    // [C] or NULL (ones)
    const int *lengths;                 // [B] or NULL
    void *r_out, *n_out;                // forward: either may be NULL
    const void *d_r_out, *d_n_out;      // backward: either may be NULL (zeros)
    void *dy, *dr, *dgate;              // dr, dgate may be NULL
    float *dw_after, *dw_before;        // [C] or NULL
    float *workspace;
    Strides sy, sr, sgate, sr_out, sn_out, sdy, sdr, sdgate;
    int B, T, C, gate_kind, activation; // tfno_gate, tfno_activation
    float residual_scale, eps;
    bool bf16, residual_bf16, norm_after;
};

hipError_t block_norm_launch(const BlockNormArgs &a, hipStream_t s);
hipError_t block_norm_backward_launch(const BlockNormArgs &a, hipStream_t s);
size_t block_norm_workspace_bytes(int B, int T, int C, int gate_kind);

}  // namespace tfno
