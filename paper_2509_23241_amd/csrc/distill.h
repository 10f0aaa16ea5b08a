// Distillation loss and its gradient (see kernels_distill.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tp {

struct DistillArgs {
  int rows, classes, k;
  const void* logits;       // [rows x classes] in elt
  const float* teacher;     // [rows x k]
  const int32_t* ids;       // [rows x k], negative: no entry
  const int32_t* labels;    // [rows], or null where label_weight is 0
  float temperature, label_weight;
  float teacher_weight;     // 1 - the labels' weight, taken before either is rounded to 32 bits: next to 1 that rounding is much of what is left
  void* dlogits;            // [rows x classes] in elt
  float* row_loss;          // scratch, [rows]
  uint32_t* counter;        // zero before the launch and after it
  float* loss;
  int first_row = 0;        // of this launch
};
hipError_t launch_distill(hipStream_t s, int elt, const DistillArgs& a);

}  // namespace tp
