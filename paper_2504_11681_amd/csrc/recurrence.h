// Gated linear recurrence: what the C ABI hands to the kernels.
#pragma once
#include "elements.h"

namespace tfno {

struct RecurrenceArgs {
    const void *x, *gate, *input_gate;  // [B, T, C]; input_gate may be NULL (open)
    const float *rate;                  // [C], or NULL: gate is the logarithm of the decay itself
    const int *lengths;                 // [B] or NULL
    const float *initial;               // [B, C] or NULL
    void *y;                            // forward
    float *final_state;                 // [B, C] or NULL
    float *tape;                        // [B, ceil(T / 2^tape_log2), C]: the state before every so many tokens; NULL: none is kept
    const void *dy;                     // backward
    const float *d_final;               // [B, C] or NULL
    void *dx, *dgate, *dinput_gate;
    float *drate, *d_initial;
    float *states;                      // step: [pool, C]
    const int *slots;
    float *effects;                     // workspace: what each segment does to the state, three numbers each
    float *partial;                     // workspace: each workgroup's part of drate
    Strides sx, sgate, sinput, sy, sdx, sdgate, sdinput;      // sy: y, or dy
    int B, T, C, pool, tape_log2;
    bool bf16, normalise;
};

hipError_t recurrence_launch(const RecurrenceArgs &a, hipStream_t s);
hipError_t recurrence_backward_launch(const RecurrenceArgs &a, hipStream_t s);
hipError_t recurrence_step_launch(const RecurrenceArgs &a, hipStream_t s);
size_t recurrence_tape_bytes(int B, int T, int C, bool bf16);
size_t recurrence_workspace_bytes(int B, int T, int C, bool bf16, bool backward);

}  // namespace tfno
