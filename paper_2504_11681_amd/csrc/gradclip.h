// The norm over many tensors and the clipping to it: what the C ABI hands to the kernels.
#pragma once
#include "../../include/tfno.h"
#include "elements.h"

namespace tfno {

hipError_t clip_launch(const tfno_tensor *tensors, int count, double limit, float *norm, double *partial, hipStream_t s);
size_t clip_workspace_bytes(int count);

}  // namespace tfno
