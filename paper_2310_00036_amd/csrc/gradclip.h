// Internal interface of the clip over many gradient tensors (gradclip.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/cleanba_learner.h"

namespace cb {

size_t grad_clip_ws_bytes(const grad_tensor_t* t, int n);
hipError_t grad_clip_run(const grad_tensor_t* t, int n, float max_norm, float* stats, void* ws, hipStream_t s);

}  // namespace cb
