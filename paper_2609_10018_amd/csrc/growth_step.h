// The growth step with a loss of the caller's (growth.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include "layout.h"

namespace elasto {

// The student's logits (fp32, row stride ld) and where the loss goes: its
// gradient with respect to them, of the mean over the batch (bf16, row stride
// ldg), and the loss of each row.
struct GrowthLogits {
  const float* logits;
  int64_t ld;
  void* dlogits;
  int64_t ldg;
  float* rowloss;
  int classes, batch;
};
struct GrowthLoss {
  const char* name;
  hipError_t (*launch)(const void* args, const GrowthLogits& z, hipStream_t s);
  const void* args;
};

elasto_status_t growth_step(elasto_growth_t g, int32_t mode, const void* images, int32_t batch,
                            float lr, float clip_norm, float* stats, void* hip_stream,
                            const GrowthLoss& loss);

}  // namespace elasto
