// The head's training operators: what the C entry points (head.cpp) hand to
// the kernels' launchers (k_head.hip, k_top.hip, k_sample.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/reno_head.h"

namespace reno {

// sets the calling thread's message of reno_last_error(NULL) (api.cpp)
reno_status fail_thread(reno_status s, const char* msg);

// rows of a launch that gives a row up to 256 threads: a grid has less than 2^32
constexpr int64_t LAUNCH_ROWS = int64_t(1) << 23;

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

// Targets of the rows: as given (code length: one symbol a row, the rest null),
// or a distillation's entries with those of one index joined.
struct HeadTargets {
  const int32_t* index;   // [N][k], -1: none
  const float* q;         // [N][k]
  const float* ent;       // [N] sum q log2 q
  const uint8_t* flag;    // [N] 0: left out, 1: taken, 2: an index outside the alphabet
};

// fp32 heads that one kernel takes whole (k_head_narrow.hip)
bool head_is_narrow(const reno_head& p);
int64_t head_narrow_bytes(const reno_head& p, bool grad);
// gpart: partial maxima of the rows' weights, over which dz is carried, or null
hipError_t launch_head_narrow(const HeadCall& c, const HeadTargets& t, const float* gpart, char* ws, hipStream_t stream);

int64_t head_workspace(const reno_head& p, int k, bool grad);
hipError_t launch_head(const HeadCall& c, hipStream_t stream);
hipError_t launch_top(const void* logits, int type, int64_t rows, int symbols, int64_t stride, int k, int32_t* index,
                      float* value, float* lse, hipStream_t stream);
hipError_t launch_sample(const reno_sample& p, const void* logits, const float* u, int32_t* symbol, float* bits,
                         hipStream_t stream);

}  // namespace reno
