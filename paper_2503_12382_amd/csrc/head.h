// The head's training operators: what the C entry points (head.cpp) hand to
// the kernels' launchers (k_head.hip, k_top.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/reno_head.h"

namespace reno {

// sets the calling thread's message of reno_last_error(NULL) (api.cpp)
reno_status fail_thread(reno_status s, const char* msg);

struct HeadCall {
  reno_head p{};
  reno_head_data d{};
  int k = 1;                        // entries a row
  const int32_t* index = nullptr;   // [N][k]
  const float* logit = nullptr;     // [N][k] (distillation), or null: code length
  float temperature = 1.0f;
  bool grad = false;
  char* ws = nullptr;
};

int64_t head_workspace(const reno_head& p, int k, bool grad);
hipError_t launch_head(const HeadCall& c, hipStream_t stream);
hipError_t launch_top(const void* logits, int type, int64_t rows, int symbols, int64_t stride, int k, int32_t* index,
                      float* value, float* lse, hipStream_t stream);

}  // namespace reno
