// The step that follows a gradient: what the C entry points (step.cpp) hand to
// the kernels' launchers (k_step.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/reno_step.h"

namespace reno {

// sets the calling thread's message of reno_last_error(NULL) (api.cpp)
reno_status fail_thread(reno_status s, const char* msg);

// partial sums of reno_grad_norm (doubles)
int64_t norm_parts(const reno_gradient* g, int64_t count);
hipError_t launch_norm(const reno_gradient* g, int64_t count, double scale, float* norm, double* parts, hipStream_t st);
hipError_t launch_clip(const reno_gradient* g, int64_t count, const float* norm, double scale, double max_norm,
                       hipStream_t st);
hipError_t launch_adamw(const reno_parameter* p, int64_t count, const reno_adamw& how, hipStream_t st);

}  // namespace reno
