// The distillation loss (host-side declarations).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace elasto {

constexpr int kMaxTop = 256;  // teacher entries of a row: one a thread

struct DistillArgs {
  int dtype = 0, grad_dtype = 0;
  const void* logits = nullptr;
  int64_t ld = 0, rows = 0;
  int classes = 0, top = 0;
  const float* values = nullptr;      // [rows][top]
  const int32_t* indices = nullptr;   // [rows][top]
  const int32_t* labels = nullptr;    // [rows] or NULL
  const float* row_weight = nullptr;  // [rows] or NULL
  float temperature = 1.0f, alpha = 1.0f, scale = 1.0f;
  float* loss = nullptr;              // [rows]
  void* dlogits = nullptr;            // NULL: the loss alone
  int64_t ldg = 0;
};

// False, with the thread's error message set, where the arguments are refused.
bool check_distill(const DistillArgs& a);
hipError_t launch_distill(const DistillArgs& a, hipStream_t s);

}  // namespace elasto
