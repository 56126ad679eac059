// Gated delta rule: what the C ABI hands to the kernels.
#pragma once
#include "elements.h"

namespace tfno {

struct DeltaArgs {
    const void *q, *k;                  // [B, T, Hk, Dk]
    const void *v;                      // [B, T, Hv, Dv]
    const float *g, *beta;              // [B, T, Hv]; g NULL: no decay
    const int *lengths;                 // [B] or NULL: tokens of each sequence that count
    const float *initial;               // [B, Hv, Dk, Dv] or NULL (zeros)
    void *o;                            // [B, T, Hv, Dv]
    float *final_state;                 // [B, Hv, Dk, Dv] or NULL
    // backward
    const void *d_o;
    const float *d_final;               // or NULL (zeros)
    void *dq, *dk, *dv;
    float *dg, *dbeta, *d_initial;      // dg and d_initial or NULL
    Strides sq, sk, sv, so, sg, sbeta, sdo, sdq, sdk, sdv, sdg, sdbeta;
    int B, T, Hk, Hv, Dk, Dv;
    float scale;
    bool bf16;
    // memory of the caller: the workspace of the forward pass without a tape and of the backward pass, the tape of the two
    unsigned char *workspace, *tape;
};

struct DeltaStepArgs {
    const void *q, *k, *v;              // [B, Hk, Dk], [B, Hv, Dv]
    const float *g, *beta;              // [B, Hv]; g NULL: no decay
    const int *slots;                   // [B] or NULL (the sequence's index)
    float *state;                       // [pool, Hv, Dk, Dv]
    void *o;                            // [B, Hv, Dv]
    Strides sq, sk, sv, so, sg, sbeta;  // the token's stride is not used
    int B, Hk, Hv, Dk, Dv, pool;
    int first;                          // of a launch's heads [B Hv]: more than one launch takes go in several
    float scale;
    bool bf16;
};

size_t delta_tape_bytes(const DeltaArgs &a);
size_t delta_workspace_bytes(const DeltaArgs &a, bool backward);
bool delta_launches(const DeltaArgs &a, bool whole);       // whether launches take the call: a batch `whole` (with a tape), or at least one sequence
hipError_t delta_forward_launch(const DeltaArgs &a, hipStream_t s);
hipError_t delta_backward_launch(const DeltaArgs &a, hipStream_t s);
hipError_t delta_step_launch(const DeltaStepArgs &a, hipStream_t s);

}  // namespace tfno
